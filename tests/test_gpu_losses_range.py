"""The losses where 32 bits would not do: shares of rows that are rounded once, ratios and divergences beyond the range of 32 bits.  U = 2^-24 is the unit
roundoff of 32-bit floats; a sum of a few thousand numbers in 64 bits and the functions that go into them are off by less than a hundredth of it."""
import math

import pytest
import torch

from test_gpu_losses import Row64, TYPES, U, gen, inputs, policy64

pytestmark = pytest.mark.gpu

# rows of a few lanes, of a wave, of a block, of a block with a part in LDS, and in parts
PATHS = [(64, 40), (70, 900), (70, 9000), (192, 50000), (5, 90000)]


@pytest.mark.parametrize("T,n", [(64, 5), (64, 10), (64, 15), (192, 16), (8, 17)])
def test_a_rows_share_of_the_policy_loss_is_rounded_once(lib, ctx, T, n):
    """Rows of 2^n equals: the sum of exponentials is exact and logp is -n log 2 in 64 bits.  All rows are alike, so roundings do not cancel: a row's share and the
    sum are rounded once each, 2 U; dlogp once and the gradient's product once more (the token's own entry twice), where p comes from log_sum as
    well, log_sum and its product with log2(e) are off by 2 U n log 2 more."""
    logp, x, y = -n * math.log(2), torch.zeros(T, 2 ** n, device="cuda"), torch.arange(T, device="cuda") % 2 ** n
    ones = torch.ones(T, device="cuda")
    for k in range(16):
        old, ref = (torch.tensor(logp + s, dtype=torch.float32).item() for s in (0.013 - 0.04 * (k - 8), 0.29 - 0.05 * k))
        got = lib.policy_loss(ctx, x, y, old * ones, 1.1 * ones, ref_logp=ref * ones, weight=ones * 2.0 ** -9, clip_low=1.0, clip_high=1e30, kl=0.375)
        a, r, d = torch.tensor(1.1).item(), math.exp(logp - old), ref - logp
        div, w = math.expm1(d) - d, 2.0 ** -9
        for name, each in (("loss", w * (0.375 * div - r * a)), ("divergence", w * div)):
            # (expm1(d) - d cancels in 64 bits as well: 2^-52 of d)
            assert abs(got[name].item() - T * each) <= 2.02 * U * T * abs(each) + T * w * abs(d) * 2.0 ** -50, (name, k)
        dlogp = w * (-a * r - 0.375 * math.expm1(d))
        want = torch.full((T, 2 ** n), -dlogp / 2 ** n, dtype=torch.float64, device="cuda")
        want[torch.arange(T, device="cuda"), y] += dlogp
        off = (got["dlogits"].double() - want).abs()
        assert torch.all(off <= (3.03 + (0 if n < 17 else 4 * n * math.log(2))) * U * want.abs())


@pytest.mark.parametrize("shape", PATHS, ids=str)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_ratios_and_divergences_beyond_32_bits(lib, ctx, shape, dtype):
    """exp(92) and exp(95) are no 32-bit numbers; with weights of 1e-4 and 1e-6 the loss and the gradient are."""
    T, V = shape
    g = gen(T + V)
    x, y = inputs(g, T, V, dtype, ignore=False, scale=1.0)
    row = Row64(x, y, 1.0)
    logp = row.logp.cpu()
    old, ref, adv, w = (logp - 0.125).float(), (logp + 0.25).float(), torch.randn(T, generator=g), torch.full((T,), 1.0 / T)
    ref[0], w[0] = (logp[0] + 92).float(), 1e-4
    old[1], adv[1], w[1] = (logp[1] - 95).float(), -1.0, 1e-6
    dev = [t.cuda() for t in (x, y, old, adv)]
    for rows in (slice(0, T), slice(1, T)):         # (with the first row, and without what is larger than all the rest)
        ws = w.clone()
        ws[:rows.start] = 0
        got = lib.policy_loss(ctx, *dev, ref_logp=ref.cuda(), weight=ws.cuda(), clip_low=0.2, clip_high=0.3, kl=0.125)
        sums, errs, dlogp, derr = policy64(row, old, adv, ref, ws, 0.2, 0.3, 0.125)
        for k, s, e in zip(("loss", "divergence", "clipped"), sums, errs):
            assert abs(got[k].item() - s.item()) <= e.item(), k
        row.check_slope(got["dlogits"], dlogp, derr, TYPES[dtype])


@pytest.mark.parametrize("shape", PATHS, ids=str)
def test_a_divergence_without_end(lib, ctx, shape):
    """A token that cannot be, to a reference that gives it a chance: the divergence is infinite, and the loss if it has a part in it."""
    T, V = shape
    x, y = inputs(gen(V), T, V, "f32", ignore=False)
    x[2, y[2]] = -math.inf
    x, y, f = x.cuda(), y.cuda(), torch.full((T,), -3.0).cuda()
    for kl, want in ((0.5, math.inf), (-0.5, -math.inf)):
        got = lib.policy_loss(ctx, x, y, f, f, ref_logp=f, kl=kl, gradient=False)
        assert got["loss"].item() == want and got["divergence"].item() == math.inf
    got = lib.policy_loss(ctx, x, y, f, f, ref_logp=f)
    alone = lib.policy_loss(ctx, x, y, f, f)
    assert got["divergence"].item() == math.inf and torch.equal(got["loss"], alone["loss"]) and torch.isfinite(got["loss"])
