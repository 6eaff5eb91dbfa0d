"""The training command's losses and optimizers, looked at before anything else is done."""
import pytest

from paper_2307_16273_amd import train_quantized


@pytest.mark.parametrize("how", [dict(loss="cross"), dict(optimizer="adam"), dict(state_bits=16), dict(limit=0.0), dict(limit=-1.0), dict(limit=float("nan")),
                                 dict(loss="preference", batch=1)], ids=str)
def test_what_is_not_known_is_refused(monkeypatch, capsys, how):
    name = "batch" if "batch" in how else next(iter(how))
    with pytest.raises(ValueError, match=name):
        train_quantized.run(**how, say=lambda s: None)
    monkeypatch.setattr("sys.argv", ["train_quantized"] + [x for k, v in how.items() for x in (f"--{k.replace('_', '-')}", str(v))])
    with pytest.raises(SystemExit) as e:
        train_quantized.main()
    assert e.value.code == 2 and name in capsys.readouterr().err
