"""Losses, norm and update together, as a training program uses them: a layer in 8-bit integers, the policy's loss on its output, the gradient of its
weights by 8-bit products, its norm and limit, AdamW in 8 bits.  Each part is compared with its definition in 64 bits on what the part in front gave."""
import math

import pytest
import torch

from test_gpu_losses import Row64, gen, policy64
from test_gpu_update import HOW, adam64, bits16, check_params, decode, encode

pytestmark = pytest.mark.gpu


def test_a_layer_as_a_policy(lib, ctx):
    g = gen(21)
    T, width, V = 96, 256, 1000
    w = (torch.randn(width, V, generator=g) * width ** -0.5 * 3).cuda()
    gain = torch.ones(width).cuda()
    x = torch.randn(T, width, generator=g).to(torch.bfloat16).cuda()
    params = [w, gain]
    state = lib.adamw_state(params, bits=8)
    y = torch.randint(0, V, (T,), generator=g).cuda()
    y[::8] = -1
    adv = torch.randn(T, generator=g).cuda()
    old = ref = None
    for k in (1, 2):
        n = lib.rmsnorm_i8(ctx, x, gain)
        wq = lib.quantize_i8(ctx, w, axis=-2)
        logits = lib.matmul_i8(ctx, n["q"], wq["q"], n["scale"], wq["scale"], dtype=torch.bfloat16)
        row = Row64(logits, y, 1.0)
        if k == 1:
            lp = lib.token_logprobs(ctx, logits, y)
            row.check(lp)
            old, ref = lp["logp"] - 0.05, lp["logp"] + 0.1
        got = lib.policy_loss(ctx, logits, y, old, adv, ref_logp=ref, kl=0.5, clip_low=0.999, clip_high=1e6)
        every = torch.full((T,), 1 / T)
        sums, errs, dlogp, derr = policy64(row, old, adv, ref, every, 0.999, 1e6, 0.5)
        assert abs(got["loss"].item() - sums[0].item()) <= errs[0].item()
        row.check_slope(got["dlogits"], dlogp, derr + 2.0 ** -24 * dlogp.abs(), torch.bfloat16)
        back = lib.matmul_i8_backward(ctx, got["dlogits"], n["q"], n["scale"], wq["q"], wq["scale"])
        norm = lib.rmsnorm_i8_backward(ctx, back["da"], x, gain, n["rstd"])
        grads = [back["dw"], norm["dweight"]]
        size = lib.gradient_norm(ctx, grads, limit=0.01)
        want = math.sqrt(sum(float(d.double().square().sum()) for d in grads))
        assert abs(size["norm"].item() - want) <= 1.01 * 2.0 ** -24 * want
        factor = size["factor"].item()
        assert abs(factor - min(1.0, 0.01 / want)) <= 1.01 * 2.0 ** -24
        before = [[t.cpu().clone() for t in l] for l in (params, grads, state["m"], state["v"], state["m_scale"], state["v_scale"])]
        lib.adamw_step(ctx, params, grads, state, k, factor=size["factor"], seed=5, **HOW)
        for i in range(2):
            p, d, cm, cv, em, ev = (l[i] for l in before)
            to, move, m, v = adam64(p, d, decode(cm, em, 4), decode(cv, ev, 5), k, factor=factor, **HOW)
            check_params(params[i], to, move, p)
            for name, z, log, b in zip(("m", "v"), (m, v), (4, 5), bits16(p.numel(), 5, k, i)):
                code, scale = encode(z, log, b)
                assert torch.equal(state[name][i].cpu(), code) and torch.equal(state[name + "_scale"][i].cpu(), scale)


@pytest.mark.parametrize("how", [dict(loss="policy", optimizer="adamw", state_bits=8, limit=1.0), dict(loss="preference", optimizer="adamw"),
                                 dict(loss="policy", limit=0.5), dict(loss="squares", optimizer="adamw", state_bits=8), dict(loss="preference", batch=2)], ids=str)
def test_the_command_trains_answers_and_proves(lib, how):
    from paper_2307_16273_amd import train_quantized
    losses, rows_equal, holds = train_quantized.run(**{**dict(layers=2, width=64, batch=16, steps=3, say=lambda s: None), **how})
    assert len(losses) == 3 and all(math.isfinite(x) for x in losses) and rows_equal and holds


def test_the_commands_gradients_are_the_losses_slopes(lib, ctx):
    """An objective's gradient against central differences of its loss: h = 2^-5 along unit directions of outputs of size 1, weights 1 / rows, third
    derivatives below 4 (beta 0.5, kl 0.01): off by less than h^2 4 / 6 < 7e-4 and the losses' own roundings, 2e-6 / h < 7e-5."""
    from paper_2307_16273_amd import train_quantized as tq
    g = gen(2)
    teacher, before, out = (torch.randn(16, 64, generator=g).cuda() for _ in range(3))
    for make in (lambda: tq.squares(lib, ctx, teacher), lambda: tq.policy(torch, lib, ctx, teacher, before), lambda: tq.preference(torch, lib, ctx, teacher, before)):
        objective = make()
        objective(out)                       # (the policy draws its choices here, and uses them in the next step)
        slope = objective(out)[1]
        for _ in range(3):
            v = torch.randn(16, 64, generator=g).cuda()
            v /= v.norm()
            ends = []
            for s in (1, -1):
                again = make()
                again(out)
                ends.append(again(out + s * 2.0 ** -5 * v)[0].double().item())
            # of the squares the mean over the columns is left to the learning rate
            scale = 64 if again.__qualname__.startswith("squares") else 1
            assert abs(scale * (ends[0] - ends[1]) / 2.0 ** -4 - (slope.double() * v.double()).sum().item()) <= scale * 7.7e-4


@pytest.mark.parametrize("optimizer", ["sgd", "adamw"])
def test_a_gradient_without_end_leaves_the_step_out(lib, ctx, optimizer):
    """With a limit on the norm one infinite or NaN entry of one layer leaves all weights as they are, bit for bit; the next step is an ordinary one."""
    from paper_2307_16273_amd import train_quantized as tq
    g = gen(7)
    tensors = lambda: ([torch.randn(8, 8, generator=g).cuda() for _ in range(3)], [torch.randn(8, generator=g).cuda() for _ in range(3)])
    net = dict(zip(("w", "gain"), tensors()))
    net["w"][0][0, 0] = -0.0
    update = tq.sgd(torch, lib, ctx, net, 0.5, 1.0) if optimizer == "sgd" else tq.adamw(lib, ctx, net, 0.5, 1.0, 32)
    before = [t.clone() for l in net.values() for t in l]
    for bad in (math.inf, -math.inf, math.nan):
        dw, dgain = tensors()
        dw[1][3, 4] = bad
        update(dw, dgain)
        assert all(torch.equal(t.view(torch.int32), b.view(torch.int32)) for t, b in zip((t for l in net.values() for t in l), before))
    dw, dgain = tensors()
    update(dw, dgain)
    after = [t for l in net.values() for t in l]
    assert all(torch.isfinite(t).all() and not torch.equal(t, b) for t, b in zip(after, before))
    if optimizer == "sgd":
        # limit 1: norm rounded once, the factor once, and product, rate and difference in 32 bits
        norm = math.sqrt(sum(float(d.double().square().sum()) for d in dw + dgain))
        for t, b, d in zip(after, before, dw + dgain):
            step = 0.5 * min(1.0, 1 / norm) * d.double()
            assert torch.all((t.double() - (b.double() - step)).abs() <= 2.0 ** -24 * (4 * step.abs() + b.double().abs() + step.abs()))
