"""The training command's arguments, looked at before anything else is done."""
import pytest

from paper_2307_16273_amd import train_quantized


@pytest.mark.parametrize("name,value", [("steps", 0), ("steps", -1), ("layers", 0), ("layers", 3), ("width", 1000), ("batch", 48), ("batch", -2)])
def test_sizes_that_cannot_be_proved_are_refused(monkeypatch, capsys, name, value):
    with pytest.raises(ValueError, match=name):
        train_quantized.run(**{name: value}, say=lambda s: None)
    monkeypatch.setattr("sys.argv", ["train_quantized", f"--{name}", str(value)])
    with pytest.raises(SystemExit) as e:
        train_quantized.main()
    assert e.value.code == 2 and name in capsys.readouterr().err
