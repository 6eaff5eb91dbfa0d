"""The losses where 32 bits would not do: shares of rows that are rounded once, ratios and divergences beyond the range of 32 bits.  U = 2^-24 is the unit
roundoff of 32-bit floats; a sum of a few thousand numbers in 64 bits and the functions that go into them are off by less than a hundredth of it."""
import math

import pytest
import torch

from test_gpu_losses import Row64, TYPES, U, gen, inputs, policy64, preference64

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


LARGE = {"f32": (-1e4, -65504.0, -1e9, torch.finfo(torch.float32).min, 3e37), "f16": (-1e4, -65504.0, 6e4), "bf16": (-1e4, -1e9, torch.finfo(torch.bfloat16).min, 3e37)}


@pytest.mark.parametrize("shape", PATHS, ids=str)
@pytest.mark.parametrize("dtype", list(TYPES))
def test_rows_of_equals_of_any_size_away_from_temperature_1(lib, ctx, shape, dtype):
    """Every row holds one value, far from zero: p is 1 / V whatever the value is.  The sum is exact; log_sum and its product with log2(e) are rounded, 3 U log V
    in p with the exponential's ulp, a ratio has the rounding of logp, U log V, and the rest is products: 8 U."""
    T, V = shape
    t = TYPES[dtype]
    value = torch.tensor(LARGE[dtype]).repeat(T)[:T]
    x, y = value[:, None].expand(T, V).to(t).cuda(), torch.arange(T).cuda() % V
    g = gen(V)
    dlogp, off = torch.randn(T, generator=g), [0, 1, 3, T // 2, T] if T > 6 else [0, 2, T]
    hot = torch.nn.functional.one_hot(y, V).double()
    for tau in (0.7, 1.3):
        tau32 = torch.tensor(tau).item()
        lp = lib.token_logprobs(ctx, x, y, temperature=tau)
        assert torch.all((lp["logp"] + math.log(V)).abs() <= 2 * U * math.log(V))

        def check(got, d):
            c = d.double().cuda()[:, None] / tau32
            want = c * (hot - 1 / V)
            err = c.abs() * ((math.log(V) + 8) * U * hot + (4 * math.log(V) + 8) * U / V + 2.0 ** -126)
            half = torch.finfo(t).eps / 2
            assert torch.all((got.double() - want).abs() <= err + half * (want.abs() + err) + torch.finfo(t).smallest_normal * half)

        check(lib.token_logprobs_backward(ctx, dlogp.cuda(), x, y, lp["top"], lp["log_sum"], temperature=tau), dlogp)
        # ratios of 1, but for the rounding of logp: dlogp is -weight advantage
        got = lib.policy_loss(ctx, x, y, lp["logp"], dlogp.cuda(), weight=torch.ones(T).cuda(), clip_low=1.0, clip_high=1e30, temperature=tau)
        check(got["dlogits"], -dlogp)
        # margins of whole multiples of log V
        got = lib.preference_loss(ctx, x, y, torch.tensor(off).cuda(), beta=0.125, form="square", temperature=tau, ref_logp=torch.zeros(T).cuda())
        d = torch.zeros(T, dtype=torch.float64)
        for i in range(len(off) // 2):
            a, b, c = off[2 * i:2 * i + 3]
            m = -0.125 * math.log(V) * ((b - a) - (c - b))
            d[a:b], d[b:c] = 2 * m * 0.125 / (len(off) // 2), -2 * m * 0.125 / (len(off) // 2)
        check(got["dlogits"], d)


@pytest.mark.parametrize("shape", PATHS, ids=str)
def test_gradients_of_logits_far_from_zero(lib, ctx, shape):
    """Logits around 4000 at a temperature of 0.7, where one step of 32 bits is 2^-12: what stays in the library has no rounding of that size.  A
    thread adds at most 8 (32 + 1) terms of its own."""
    T, V = shape
    x, y = inputs(gen(T * V), T, V, "f32", ignore=False, scale=1.0)
    x = x + 4000
    row = Row64(x, y, torch.tensor(0.7).item())
    row.sum_err = (2 * math.log(V) + 22 + 264 + 3 * math.log(V)) * U
    row.log_sum_err = row.sum_err + 4 * U * row.log_sum.abs()
    row.logp_err = 3 * U * (row.logp + row.log_sum).abs() + row.log_sum_err + 2 * U * row.logp.abs()
    old, adv, w = row.logp.float().cpu() - 0.125, torch.randn(T, generator=gen(1)), torch.full((T,), 1 / T)
    x, y = x.cuda(), y.cuda()
    got = lib.policy_loss(ctx, x, y, old.cuda(), adv.cuda(), weight=w.cuda(), clip_low=0.2, clip_high=0.3, temperature=0.7)
    _, _, dlogp, derr = policy64(row, old, adv, None, w, 0.2, 0.3, 0.0)
    row.check_slope(got["dlogits"], dlogp, derr, torch.float32)
    off = [0, 1, 3, T // 2, T] if T > 6 else [0, 2, T]
    pairs = torch.full((len(off) // 2,), 0.5)
    got = lib.preference_loss(ctx, x, y, torch.tensor(off).cuda(), weight=pairs.cuda(), beta=0.03125, temperature=0.7)
    margins, merr, _, _, dlogp, derr, _ = preference64(row, off, None, pairs, 0.03125, 0.0, 0.0, "logistic", False)
    assert torch.all((got["margin"].cpu().double() - margins).abs() <= merr)
    row.check_slope(got["dlogits"], dlogp, derr, torch.float32)


@pytest.mark.parametrize("T,n", [(64, 5), (70, 10), (70, 13), (5, 17)])
def test_a_margin_is_rounded_once(lib, ctx, T, n):
    """Rows of 2^n equals, whose logp is -n log 2 in 64 bits, against a reference of the same rounded to 32: what is left of a sequence is that rounding times its
    rows.  The margin is one rounding off, and 2^-50 of what cancels."""
    ref = torch.tensor(-n * math.log(2), dtype=torch.float32)
    delta = -n * math.log(2) - ref.double().item()
    assert abs(delta) > 1e-9
    x, y = torch.ones(T, 2 ** n, device="cuda"), torch.arange(T, device="cuda") % 2 ** n
    y[-1] = -1
    first = T - 2
    off = torch.tensor([0, first, T], device="cuda")        # one row that counts in the second sequence
    for average in (False, True):
        got = lib.preference_loss(ctx, x, y, off, ref_logp=ref.cuda().expand(T).contiguous(), beta=2.0 ** 20, form="square", average=average)
        want = 2.0 ** 20 * (delta * (1 if average else first) - delta)
        noise = 2.0 ** 20 * T * n * 2.0 ** -50
        assert abs(got["margin"].item() - want) <= 1.01 * U * abs(want) + noise
        assert abs(got["loss"].item() - want ** 2) <= 1.01 * 2 * U * want ** 2 + (2 * abs(want) + noise) * noise
        assert torch.all(got["logp"][:-1] == ref.item()) and got["logp"][-1] == 0


@pytest.mark.parametrize("shape", PATHS + [(1030, 3500), (192, 131072)], ids=str)
@pytest.mark.parametrize("dtype", list(TYPES))
def test_log_probabilities_of_logits_far_from_zero(lib, ctx, shape, dtype):
    """logp is the token's distance from the row's largest entry less log_sum, with no rounding of either's size.  A thread adds at most 8 (32 + 1) terms;
    1 / temperature is rounded where it is in 32 bits, and logp once."""
    T, V = shape
    g = torch.Generator(device="cuda").manual_seed(V)
    x = (3000 + torch.randn((T, V), generator=g, device="cuda") * (64 if dtype == "bf16" else 4)).to(TYPES[dtype])
    y = torch.randint(0, V, (T,), generator=g, device="cuda")
    for tau in (0.7, 1.3):
        row = Row64(x, y, torch.tensor(tau).item())
        row.sum_err = (2 * math.log(V) + 22 + 264) * U
        row.log_sum_err = row.sum_err + U * row.log_sum.abs()
        row.logp_err = row.sum_err + U * row.logp.abs()
        for got in (lib.token_logprobs(ctx, x, y, temperature=tau), lib.policy_loss(ctx, x, y, row.logp.float(), row.logp.float(), temperature=tau)):
            row.check({k: got[k] for k in ("logp", "log_sum") if k in got})


@pytest.mark.parametrize("shape", PATHS, ids=str)
def test_temperatures_from_one_end_to_the_other(lib, ctx, shape):
    """Logits a few temperatures apart, and among them the largest and the lowest, whose distance is no 32-bit number.  Beyond 2^120 such a distance would count
    for something: refused."""
    T, V = shape
    g = gen(T * V + 1)
    for tau in (2.0 ** -126, 2.0 ** -124 / 3, 1e-20, 1e20, 1e35, 2.0 ** 120):
        tau = torch.tensor(tau).item()
        x, y = (2 * tau * torch.randn((T, V), generator=g).double()).float(), torch.randint(0, V, (T,), generator=g)
        x[1, 0], x[1, V // 2], x[2, 3] = torch.finfo(torch.float32).max, torch.finfo(torch.float32).min, torch.finfo(torch.float32).min
        row = Row64(x, y, tau)
        row.sum_err = (2 * math.log(V) + 22 + 264) * U
        row.log_sum_err = row.sum_err + U * row.log_sum.abs()
        row.logp_err = row.sum_err + U * row.logp.abs() * 4
        got = lib.token_logprobs(ctx, x.cuda(), y.cuda(), temperature=tau)
        finite = row.logp.abs() < 3e38      # (a distance of more temperatures than 32 bits hold is infinite)
        assert torch.all(((got["logp"].double() - row.logp).abs() <= row.logp_err) | ~finite) and torch.all(got["logp"][~finite] == -math.inf)
        assert torch.all((got["log_sum"].double() - row.log_sum).abs() <= row.log_sum_err)
    for tau in (2.0 ** 120 * (1 + 2.0 ** -23), 8e37, 2.0 ** -125 / 3, 2.0 ** -127):
        for call in (lambda: lib.token_logprobs(ctx, x.cuda(), y.cuda(), temperature=tau),
                     lambda: lib.preference_loss(ctx, x.cuda(), y.cuda(), torch.tensor([0, 1, T]).cuda(), temperature=tau)):
            with pytest.raises(lib.ZkdlError):
                call()
