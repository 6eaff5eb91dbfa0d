"""The losses of tokens against their definitions in 64 bits.

u = 2^-24 is the unit roundoff of 32-bit floats.  With c the row's largest logit and d_j = (x_j - c) / temperature, a term exp(d_j) of a row's sum
is off by (2 |d_j| + 4) u (the factor log2(e) / temperature, the fused product's rounding, the exponential's 1 ulp), the mean of |d_j| over the
softmax is at most log V + 1 (the entropy), and one thread adds at most t = 128 terms before trees of 16 levels: the sum is off by
(2 log V + 2 + 4 + t + 16) u, and its logarithm by as much and three roundings of its own."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF_ULP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -126, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -126}


def gen(seed):
    return torch.Generator().manual_seed(seed)


def inputs(g, T, V, dtype, masked=False, ignore=True, scale=3.0):
    x = torch.randn((T, V), generator=g) * scale
    y = torch.randint(0, V, (T,), generator=g)
    x[torch.arange(T), y] += 4 * torch.rand(T, generator=g)
    if masked and V > 3:
        x[:, 1::3] = float("-inf")
        y = torch.where(y % 3 == 1, y - 1, y)
    if ignore and T > 2:
        y[1::3] = -1 - y[1::3] // 2
    return x.to(TYPES[dtype]), y


def spread(t, pad_cols=5, offset=3):
    """The same matrix on the GPU in a larger buffer: odd row stride, odd address."""
    rows, cols = t.shape
    buf = torch.empty(rows * (cols + pad_cols) + offset + 16, dtype=t.dtype, device="cuda")
    v = buf[offset:offset + rows * (cols + pad_cols)].view(rows, cols + pad_cols)[:, :cols]
    v.copy_(t)
    return v


class Row64:
    """Statistics of every row that counts in 64 bits, and by how much 32-bit ones may differ."""

    def __init__(self, x, y, tau):
        x, y = x.cuda(), y.cuda()
        self.live = y >= 0
        u = x.double() / tau
        self.d = u - u.amax(1, keepdim=True)
        self.u, self.tau, self.y = u, tau, y
        self.top = torch.where(self.live, u.amax(1), 0.0)
        self.log_sum = torch.where(self.live, self.d.exp().sum(1).log(), 0.0)
        mine = self.d.gather(1, y.clamp(min=0)[:, None])[:, 0]
        self.logp = torch.where(self.live, mine - self.log_sum, 0.0)
        V = x.shape[1]
        self.sum_err = (2 * math.log(V) + 22 + 128) * U
        self.log_sum_err = self.sum_err + 4 * U * self.log_sum.abs()
        self.top_err = 2 * U * self.top.abs()
        self.logp_err = torch.where(self.live, 3 * U * mine.abs() + self.top_err + self.log_sum_err + 2 * U * self.logp.abs(), 0.0)

    def check(self, got):
        for k, err in (("logp", self.logp_err), ("top", self.top_err), ("log_sum", self.log_sum_err)):
            if k in got:
                v = got[k].double()
                assert torch.all((v - getattr(self, k)).abs() <= err), (k, (v - getattr(self, k)).abs().max())
                assert torch.all(v[~self.live] == 0)

    def check_slope(self, got, dlogp, dlogp_err, dtype):
        """The gradient of the logits, dlogp being known up to dlogp_err."""
        c, ce = (dlogp.cuda() / self.tau)[:, None], (dlogp_err.cuda() / self.tau)[:, None]
        p = torch.where(self.live[:, None], (self.d - self.log_sum[:, None]).exp(), 0.0)
        hot = torch.zeros_like(p)
        hot[torch.arange(len(self.y), device="cuda"), self.y.clamp(min=0)] = self.live.double()
        want = c * (hot - p)
        far = torch.where(p > 0, self.d.abs(), 0.0)
        err = ce * (hot + p) + c.abs() * (p * (2 * far * U + self.sum_err + 10 * U) + hot * 3 * U + 2.0 ** -126)
        err = err + HALF_ULP[dtype] * (want.abs() + err) + TINY[dtype]
        off = (got.double() - want).abs()
        assert torch.all(off <= err), ((off - err).max(), (off / err).max())
        assert torch.all(got[~self.live] == 0)


# both sides of every bound between kernels
SHAPES = [(1, 1), (3, 1), (2, 7), (5, 8), (70, 7), (70, 8), (70, 9), (4, 71), (65, 511), (65, 512), (65, 513), (70, 1024), (70, 1025), (66, 2047),
          (66, 2048), (66, 2049), (1, 4096), (64, 4097), (3, 8192), (64, 8193), (63, 8200), (64, 16384), (65, 16385), (2, 16385), (64, 32768), (64, 32769),
          (64, 65536), (64, 65537), (1, 131072), (64, 131072), (64, 131073), (1, 200001), (300, 33), (1000, 7), (40, 63), (41, 64), (39, 65), (20, 127), (17, 128), (19, 129), (9, 255), (7, 256), (11, 257)]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("dtype", list(TYPES))
def test_token_logprobs(lib, ctx, shape, dtype):
    g = gen(shape[0] * 7 + shape[1])
    x, y = inputs(g, *shape, dtype, masked=shape[1] % 2 == 1)
    for tau, where, wide in ((1.0, lambda t: t.cuda(), torch.int64), (0.6, spread, torch.int32)):
        want = Row64(x, y, np.float32(tau).item())
        want.check(lib.token_logprobs(ctx, where(x), y.to(wide).cuda(), temperature=tau))


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("dtype", list(TYPES))
def test_token_logprobs_backward(lib, ctx, shape, dtype):
    g = gen(shape[0] * 11 + shape[1])
    x, y = inputs(g, *shape, dtype, masked=shape[1] % 2 == 1)
    dlogp = torch.randn(shape[0], generator=g)
    if shape[0] > 4:
        dlogp[2] = 0
    for tau, where, wide in ((1.0, lambda t: t.cuda(), torch.int64), (0.6, spread, torch.int32)):
        tau = np.float32(tau).item()
        want = Row64(x, y, tau)
        top, log_sum = want.top.float(), want.log_sum.float()
        got = lib.token_logprobs_backward(ctx, dlogp.cuda(), where(x), y.to(wide).cuda(), top, log_sum, temperature=tau)
        # the statistics are rounded: the logits' own roundings (1 / temperature, the product) count as they stand
        want.sum_err = (3 * want.u.abs().nan_to_num(0, 0, 0).amax().item() + 3 * want.log_sum.amax().item() + 3 * want.top.abs().amax().item() + 10) * U
        assert got.dtype == TYPES[dtype] and got.shape == x.shape
        want.check_slope(got, dlogp.double(), torch.zeros(shape[0]).double(), TYPES[dtype])


def test_a_mask_of_the_lowest_value(lib, ctx):
    """Masked entries of the type's lowest finite value: nothing of them is left, and a row of nothing else is a row of equals."""
    for dtype, t in TYPES.items():
        for T, V in ((66, 40), (3, 20000), (70, 9000)):
            x, y = inputs(gen(V), T, V, dtype, ignore=False)
            x[:, 2::5] = torch.finfo(t).min
            y = torch.where(y % 5 == 2, y - 1, y)
            x[0] = torch.finfo(t).min
            x[1, 0] = torch.finfo(t).max
            got = lib.token_logprobs(ctx, x.cuda(), y.cuda())
            want = Row64(x, y, 1.0)
            want.check(got)
            back = lib.token_logprobs_backward(ctx, torch.ones(T).cuda(), x.cuda(), y.cuda(), got["top"], got["log_sum"])
            want.sum_err = (3 * want.log_sum.amax().item() + 3 * want.u[2:].abs().nan_to_num(0, 0, 0).clamp(max=100).amax().item() + 160) * U
            want.check_slope(back, torch.ones(T).double(), torch.zeros(T).double(), t)


@pytest.mark.parametrize("shape", [(66, 40), (5, 250), (70, 9000), (3, 20000), (4, 140001)], ids=str)
@pytest.mark.parametrize("dtype", list(TYPES))
def test_a_mask_of_the_lowest_value_below_temperature_1(lib, ctx, shape, dtype):
    """logits / temperature leave the range of 32 bits where nothing but the mask, or nothing but the largest value, is left: a row of equals all the same."""
    T, V = shape
    x, y = inputs(gen(V + 1), T, V, dtype, ignore=False)
    t = TYPES[dtype]
    x[:, 2::5] = torch.finfo(t).min
    y = torch.where(y % 5 == 2, y - 1, y)
    x[0], x[1] = torch.finfo(t).min, torch.finfo(t).max
    row = Row64(x, y, 0.5)
    # log-probabilities are (logit - the largest) / temperature - log_sum: of the largest itself they have no rounding
    row.logp_err = 3 * U * (row.logp + row.log_sum).abs() + row.log_sum_err + 2 * U * row.logp.abs()
    x, y = x.cuda(), y.cuda()
    got = lib.token_logprobs(ctx, x, y, temperature=0.5)
    row.check({k: got[k] for k in ("logp", "log_sum")})
    if dtype != "f16":
        assert got["top"][0] == -math.inf and got["top"][1] == math.inf
    ones, none = torch.ones(T), torch.zeros(T).double()
    old, ref, w = row.logp.float().cpu(), row.logp.float().cpu() - 0.25, torch.full((T,), 1 / T)
    policy = lib.policy_loss(ctx, x, y, old.cuda(), ones.cuda(), ref_logp=ref.cuda(), weight=w.cuda(), clip_low=0.2, clip_high=0.3, kl=0.125, temperature=0.5)
    off = [0, 1, 2, T // 2 + 1, T] if T > 4 else [0, 1, T]
    pairs = torch.full((len(off) // 2,), 0.5)
    preference = lib.preference_loss(ctx, x, y, torch.tensor(off).cuda(), weight=pairs.cuda(), beta=0.25, temperature=0.5)
    back = lib.token_logprobs_backward(ctx, ones.cuda(), x, y, got["top"], got["log_sum"], temperature=0.5)
    sums, errs, dlogp, derr = policy64(row, old, ones, ref, w, 0.2, 0.3, 0.125)
    for k, s, e in zip(("loss", "divergence", "clipped"), sums, errs):
        assert abs(policy[k].item() - s.item()) <= e.item(), k
    margins, merr, loss, lerr, dpref, dpref_err, seen = preference64(row, off, None, pairs, 0.25, 0.0, 0.0, "logistic", False)
    assert seen.all() and torch.all((preference["margin"].cpu().double() - margins).abs() <= merr) and abs(preference["loss"].item() - loss) <= lerr
    # what comes from top and log_sum has their roundings, as in the test of that pass
    row.sum_err += (3 * row.u[2:].amax().item() + 3 * row.log_sum.amax().item() + 3 * row.top[2:].abs().amax().item() + 10) * U
    row.check_slope(policy["dlogits"], dlogp, derr, t)
    row.check_slope(preference["dlogits"], dpref, dpref_err, t)
    row.check_slope(back, ones.double(), none, t)


@pytest.mark.parametrize("n", range(18))
def test_rows_of_equals_are_rounded_once(lib, ctx, n):
    """Terms are 1 and their sums exact: log_sum and logp are n log 2 rounded to 32 bits, whatever the temperature."""
    want = torch.tensor(n * math.log(2), dtype=torch.float64).float().cuda()
    for T in (3, 70):
        for t in TYPES.values():
            x, y = torch.full((T, 2 ** n), 1.5, dtype=t).cuda(), torch.arange(T).cuda() % 2 ** n
            for tau in (1.0, 0.7):
                got = lib.token_logprobs(ctx, x, y, temperature=tau)
                assert torch.all(got["log_sum"] == want) and torch.all(got["logp"] == -want)


def policy64(row, old, adv, ref, w, lo, hi, kl):
    """Loss, divergence, clipped, dlogp and by how much they may differ."""
    E = row.logp_err
    old, adv, ref, w = (None if t is None else t.cuda() for t in (old, adv, ref, w))
    lo, hi = 1 - np.float32(lo).item(), 1 + np.float32(hi).item()
    w = torch.where(row.live, w.double(), 0.0)
    a, r = adv.double(), (row.logp - old.double()).exp()
    assert torch.all((r - lo).abs() > 1e-4) and torch.all((r - hi).abs() > 1e-4)
    Er = r * (E + 3 * U + U * (row.logp - old.double()).abs())
    gain = torch.minimum(r * a, r.clamp(lo, hi) * a)
    flat = ((a > 0) & (r > hi)) | ((a < 0) & (r < lo))
    dlogp, k = torch.where(flat, 0.0, -r * a), torch.zeros_like(r)
    derr, kerr = a.abs() * (Er + 2 * U * r), torch.zeros_like(r)
    if ref is not None:
        d = ref.double() - row.logp
        Ed = E + U * d.abs()
        em = torch.expm1(d)
        k = em - d
        kerr = em.abs() * Ed + 4 * U * (em.abs() + d.abs())
        dlogp = dlogp - kl * em
        derr = derr + abs(kl) * (d.exp() * Ed + 4 * U * em.abs())
    terr = a.abs() * (Er + 2 * U * r) + abs(kl) * (kerr + U * k) + U * (gain.abs() + abs(kl) * k)
    each = kl * k - gain
    sums = [(w * t).sum() for t in (each, k, flat.double())]
    errs = [(w.abs() * e).sum() + 2 * U * (w * t).abs().sum() + U * s.abs() + 2.0 ** -149
            for e, t, s in zip((terr, kerr, torch.zeros_like(r)), (each, k, flat.double()), sums)]
    return sums, errs, w * dlogp, w.abs() * derr + 3 * U * (w * dlogp).abs()


def policy_inputs(g, row, T):
    """Ratios on both sides of the clipping, none at its edges."""
    moved = 0.4 * torch.randn(T, generator=g)
    for edge in (math.log(0.8), math.log(1.3)):
        moved = torch.where((moved - edge).abs() < 1e-2, torch.full_like(moved, edge + 2e-2), moved)
    logp = row.logp.cpu()
    old = (logp - moved.double()).float()
    ref = (logp + 0.5 * torch.randn(T, generator=g).double()).float()
    ref[::4] = (logp[::4] + 1e-3 * torch.randn(len(ref[::4]), generator=g).double()).float()
    return old, torch.randn(T, generator=g), ref, torch.rand(T, generator=g) / T


@pytest.mark.parametrize("shape", SHAPES + [(700, 260), (20000, 16)], ids=str)
@pytest.mark.parametrize("dtype", list(TYPES))
def test_policy_loss(lib, ctx, shape, dtype):
    T, V = shape
    g = gen(T * 13 + V)
    x, y = inputs(g, T, V, dtype, masked=V % 2 == 1)
    for tau, where, with_ref, wide in ((1.0, lambda t: t.cuda(), True, torch.int64), (0.6, spread, False, torch.int32)):
        tau = np.float32(tau).item()
        row = Row64(x, y, tau)
        old, adv, ref, w = policy_inputs(g, row, T)
        if T > 5:
            adv[3] = 0
        if not with_ref:
            ref, w = None, None
        kl = 0.125 if with_ref else 0.0
        dev = lambda t: None if t is None else t.cuda()
        got = lib.policy_loss(ctx, where(x), y.to(wide).cuda(), dev(old), dev(adv), ref_logp=dev(ref), weight=dev(w), clip_low=0.2, clip_high=0.3, kl=kl, temperature=tau)
        row.check({"logp": got["logp"]})
        ws = w if w is not None else torch.full((T,), float(np.float32(1) / np.float32(T)))
        sums, errs, dlogp, derr = policy64(row, old, adv, ref, ws, 0.2, 0.3, kl)
        for k, s, e in zip(("loss", "divergence", "clipped"), sums, errs):
            assert got[k].shape == () and abs(got[k].item() - s.item()) <= e.item(), (k, got[k].item(), s.item(), e.item())
        row.check_slope(got["dlogits"], dlogp, derr, TYPES[dtype])
        alone = lib.policy_loss(ctx, where(x), y.to(wide).cuda(), dev(old), dev(adv), ref_logp=dev(ref), weight=dev(w), clip_low=0.2, clip_high=0.3, kl=kl, temperature=tau, gradient=False)
        assert alone["dlogits"] is None and all(torch.equal(alone[k], got[k]) for k in ("loss", "divergence", "clipped", "logp"))


# a length for each number of whole vectors a thread has, for a wave, a block of 256 and one of 512 threads a row (from 1024 rows on fewer threads
# have a row), and for rows of which a part lies in LDS (from 192 rows on)
LENGTHS = ([(5, 512 * w + 77) for w in range(4)] + [(1030, 512 * w + 509) for w in range(8)] + [(9, 2048 * w + 3) for w in range(1, 4)] +
           [(1024, 2048 * w + 1021) for w in range(2, 17)] + [(11, 4096 * w + 4089) for w in range(2, 17)])
LONG = [(192, 4096 * w + 1365) for w in range(9, 32)] + [(192, 131072), (193, 65536), (200, 131071), (191, 131072)]


@pytest.mark.parametrize("shape", LENGTHS + LONG, ids=str)
@pytest.mark.parametrize("dtype", list(TYPES))
def test_every_length(lib, ctx, shape, dtype):
    """Log-probabilities and the policy's gradient; inputs made on the device."""
    T, V = shape
    g = torch.Generator(device="cuda").manual_seed(V)
    x = (torch.randn((T, V), generator=g, device="cuda") * 2).to(TYPES[dtype])
    y = torch.randint(0, V, (T,), generator=g, device="cuda")
    y[0], y[1], y[2] = V - 1, V // 8 * 8 - 1, -1
    row = Row64(x, y, 1.0)
    row.check(lib.token_logprobs(ctx, x, y))
    old, adv, ref, w = policy_inputs(gen(V), row, T)
    got = lib.policy_loss(ctx, x, y, old.cuda(), adv.cuda(), ref_logp=ref.cuda(), weight=w.cuda(), clip_low=0.2, clip_high=0.3, kl=0.125)
    sums, errs, dlogp, derr = policy64(row, old, adv, ref, w, 0.2, 0.3, 0.125)
    for k, s, e in zip(("loss", "divergence", "clipped"), sums, errs):
        assert abs(got[k].item() - s.item()) <= e.item(), k
    row.check_slope(got["dlogits"], dlogp, derr, TYPES[dtype])


def preference64(row, off, ref, w, beta, target, smoothing, form, average):
    P, T = len(off) // 2, len(row.y)
    alive, logp, logp_err = row.live.cpu(), row.logp.cpu(), row.logp_err.cpu()
    dlogp, derr, margins, merr, loss, lerr = torch.zeros(T).double(), torch.zeros(T).double(), [], [], 0.0, 0.0
    seen = torch.zeros(T, dtype=torch.bool)
    for i in range(P):
        h, e, n = [], [], []
        for q in (2 * i, 2 * i + 1):
            s = slice(off[q], off[q + 1])
            live = alive[s]
            seen[s] = True
            n.append(max(1, int(live.sum())) if average else 1)
            h.append(float(((logp[s] - (ref[s].double() if ref is not None else 0)) * live).sum()) / n[-1])
            e.append(float((logp_err[s] * live).sum()) / n[-1])
        z = beta * (h[0] - h[1])
        m, me = z - target, abs(beta) * (e[0] + e[1])
        if form == "logistic":
            sig = 1 / (1 + math.exp(-m))
            each = (1 - smoothing) * (max(-m, 0) + math.log1p(math.exp(-abs(m)))) + smoothing * (max(m, 0) + math.log1p(math.exp(-abs(m))))
            slope, bend = sig - 1 + smoothing, .25
        elif form == "hinge":
            each, slope, bend = max(0.0, -m), -1.0 if m < 0 else 0.0, 0.0
            assert abs(m) > me or m == 0
        else:
            each, slope, bend = m * m, 2 * m, 2.0
        wi = float(w[i])
        margins.append(z)
        merr.append(me + U * abs(z) + 2.0 ** -149)
        loss += wi * each
        lerr += abs(wi) * (abs(slope) + bend * me) * me + 2 * U * abs(wi * each)
        for q, sign in ((0, 1.0), (1, -1.0)):
            s = slice(off[2 * i + q], off[2 * i + q + 1])
            dlogp[s] = sign * wi * slope * beta / n[q] * alive[s]
            derr[s] = abs(wi * beta) * bend * me / n[q] + U * dlogp[s].abs() + 2.0 ** -149
    return torch.tensor(margins).double(), torch.tensor(merr).double(), loss, lerr + U * abs(loss) + 2.0 ** -149, dlogp, derr, seen


@pytest.mark.parametrize("shape,off", [((12, 5), [0, 3, 6, 6, 9]), ((70, 700), [2, 20, 33, 50, 65]), ((64, 3000), [0, 1, 2, 32, 64]), ((3, 40000), [0, 1, 3]),
                                       ((90, 8200), [5, 5, 5, 40, 40, 41, 88]), ((2, 1), [0, 1, 2]), ((5, 9), [5, 5, 5]), ((600, 100), [0, 299, 600]),
                                       ((4, 16), [4]), ((64, 70000), [0, 10, 20, 21, 60]), ((5000, 12), [0, 2100, 5000]), ((2500, 300), [3, 7, 2499])], ids=str)
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("form", ["logistic", "hinge", "square"])
def test_preference_loss(lib, ctx, shape, off, dtype, form):
    T, V = shape
    g = gen(T * 17 + V)
    x, y = inputs(g, T, V, dtype, masked=V % 2 == 1)
    P = len(off) // 2
    for tau, where, average, wide in ((1.0, lambda t: t.cuda(), False, torch.int64), (0.6, spread, True, torch.int32)):
        tau = np.float32(tau).item()
        row = Row64(x, y, tau)
        ref = (row.logp.cpu() + 0.4 * torch.randn(T, generator=g).double()).float() if average or V > 100 else None
        w = torch.rand(P, generator=g) if average else None
        beta, target, smoothing = 0.25, 0.5 if form != "logistic" else 0.0, 0.125 if form == "logistic" and average else 0.0
        dev = lambda t: None if t is None else t.cuda()
        kw = dict(ref_logp=dev(ref), weight=dev(w), beta=beta, target=target, smoothing=smoothing, form=form, average=average, temperature=tau)
        got = lib.preference_loss(ctx, where(x), y.to(wide).cuda(), torch.tensor(off, dtype=wide).cuda(), **kw)
        ws = w if w is not None else torch.full((P,), float(np.float32(1) / np.float32(max(P, 1))))
        margins, merr, loss, lerr, dlogp, derr, seen = preference64(row, off, ref, ws, beta, target, smoothing, form, average)
        assert torch.all((got["margin"].cpu().double() - margins).abs() <= merr)
        assert abs(got["loss"].item() - loss) <= lerr and got["loss"].shape == ()
        row.live = row.live & seen.cuda()
        for k in ("logp", "logp_err"):
            setattr(row, k, torch.where(row.live, getattr(row, k), 0.0))
        row.check({"logp": got["logp"]})
        row.check_slope(got["dlogits"], dlogp, derr, TYPES[dtype])
        alone = lib.preference_loss(ctx, where(x), y.to(wide).cuda(), torch.tensor(off, dtype=wide).cuda(), gradient=False, **kw)
        assert alone["dlogits"] is None and all(torch.equal(alone[k], got[k]) for k in ("loss", "margin", "logp"))


@pytest.mark.parametrize("shape", [(5, 33), (70, 1000), (70, 8200), (3, 20000)], ids=str)
def test_rows_of_infinities_and_nan(lib, ctx, shape):
    """Row 0: nothing but -infinity; 1: a NaN; 2: +infinity; 3, 4 (where there are as many): a token of V, an ordinary row with one -infinity at its token."""
    T, V = shape
    x, y = inputs(gen(V), T, V, "f32", ignore=False)
    x[0] = float("-inf")
    x[1, V // 2] = float("nan")
    x[2, V - 1] = float("inf")
    bad = [0, 1, 2]
    if T > 4:
        y[3] = V
        bad.append(3)
        x[4, y[4]] = float("-inf")
    one = torch.ones(T).cuda()
    lp = lib.token_logprobs(ctx, x.cuda(), y.cuda())
    assert torch.all(torch.isnan(lp["logp"][bad]))
    assert torch.all(torch.isnan(lp["top"][:3])) and torch.all(torch.isnan(lp["log_sum"][:3]))
    got = lib.policy_loss(ctx, x.cuda(), y.cuda(), -one, one)
    assert torch.isnan(got["loss"]) and torch.all(torch.isnan(got["dlogits"][bad]))
    back = lib.token_logprobs_backward(ctx, one, x.cuda(), y.cuda(), lp["top"], lp["log_sum"])
    assert torch.all(torch.isnan(back[bad]))
    rest = [t for t in range(T) if t not in bad and t != 4]
    if T > 4:
        assert lp["logp"][4] == float("-inf") and torch.isfinite(lp["log_sum"][4])
        assert torch.all(torch.isfinite(back[4])) and torch.all(got["dlogits"][4] == 0)       # a ratio of 0 moves nothing
    assert torch.all(torch.isfinite(back[rest])) and torch.all(torch.isfinite(got["dlogits"][rest]))
    # rows that count for nothing are not looked at
    y[bad] = -1
    got = lib.policy_loss(ctx, x.cuda(), y.cuda(), -one, one, ref_logp=-one, kl=0.0)
    assert torch.all(got["dlogits"][bad] == 0) and torch.all(got["logp"][bad] == 0)
    if T == 3:
        assert got["loss"].item() == 0


@pytest.mark.parametrize("V", [40, 3000, 40000])
def test_a_nan_among_masked_entries(lib, ctx, V):
    """A NaN whose whole neighbourhood is -infinity is not lost, in rows of any number of parts."""
    x, y = inputs(gen(V), 5, V, "f32", ignore=False)
    x[:, V // 2:] = float("-inf")
    y %= V // 2
    x[1:3, V - 3] = float("nan")
    got = lib.token_logprobs(ctx, x.cuda(), y.cuda())
    assert torch.isnan(got["logp"]).tolist() == [False, True, True, False, False]
    x = x.repeat(1, 1 if V < 40000 else 4)      # a row in parts
    got = lib.token_logprobs(ctx, x.cuda(), y.cuda())
    assert torch.isnan(got["logp"]).tolist() == [False, True, True, False, False]
    assert torch.isnan(got["top"]).tolist() == torch.isnan(got["log_sum"]).tolist() == [False, True, True, False, False]


@pytest.mark.parametrize("shape", [(70, 300), (5, 90000)], ids=str)
def test_rows_of_weight_0(lib, ctx, shape):
    """Nothing that such a row holds reaches the loss, nor a divergence that has no part in it."""
    T, V = shape
    x, y = inputs(gen(6), T, V, "f32", ignore=False)
    old, adv, ref, w = torch.full((T,), -3.0), torch.ones(T), torch.full((T,), -3.0), torch.full((T,), 1.0 / T)
    w[1] = w[3] = 0
    clean = lib.policy_loss(ctx, x.cuda(), y.cuda(), old.cuda(), adv.cuda(), weight=w.cuda(), clip_high=1e30)
    old[1], adv[1], ref[1], x[3] = -math.inf, -math.nan, math.nan, math.nan
    ref[0] = 1e30
    got = lib.policy_loss(ctx, x.cuda(), y.cuda(), old.cuda(), adv.cuda(), ref_logp=ref.cuda(), weight=w.cuda(), clip_high=1e30)
    assert torch.equal(got["loss"], clean["loss"]) and torch.equal(got["dlogits"], clean["dlogits"]) and not got["dlogits"][[1, 3]].any()
    off = torch.tensor([0, 1, 2, 4, 5]).cuda()
    pref = lib.preference_loss(ctx, x.cuda(), y.cuda(), off, weight=torch.tensor([1.0, 0.0]).cuda())
    assert torch.isfinite(pref["loss"]) and torch.isnan(pref["margin"][1]) and not pref["dlogits"][2:].any() and pref["dlogits"][0].any()


def test_margins_without_end(lib, ctx):
    """A pair whose other answer holds an entry that cannot be: nothing is lost by it and nothing to be learnt; the other way round the loss has no end."""
    x = torch.zeros(2, 10)
    x[1, 3] = -math.inf
    y, off = torch.tensor([3, 3]).cuda(), torch.tensor([0, 1, 2]).cuda()
    for form in ("logistic", "hinge"):
        got = lib.preference_loss(ctx, x.cuda(), y, off, form=form)
        assert got["margin"].item() == math.inf and got["loss"].item() == 0 and not got["dlogits"].any()
        got = lib.preference_loss(ctx, x.flip(0).cuda(), y, off, form=form)
        assert got["margin"].item() == -math.inf and got["loss"].item() == math.inf
    assert lib.preference_loss(ctx, x.cuda(), y, off, smoothing=1.0)["loss"].item() == math.inf


def test_logits_of_any_size(lib, ctx):
    """Logits far from zero and far apart, and the largest of their type."""
    x = torch.tensor([[1e4, 1e4 - 1, 0.0], [-1e30, -1e30, -1e30], [3e38, -3e38, 3e38], [88.0, 0.0, -88.0], [0.0, -200.0, -1e9]])
    y = torch.tensor([1, 2, 0, 2, 0])
    got = lib.token_logprobs(ctx, x.cuda(), y.cuda())
    Row64(x, y, 1.0).check(got)
    p = lib.token_logprobs_backward(ctx, torch.ones(5).cuda(), x.cuda(), y.cuda(), got["top"], got["log_sum"]).cpu().double()
    want = torch.nn.functional.one_hot(y, 3) - torch.softmax(x.double(), 1)
    assert torch.all((p - want).abs() <= 20 * U)


@pytest.mark.parametrize("form", ["policy", "logistic", "square"])
def test_gradients_are_the_slopes_of_the_losses(lib, ctx, form):
    """Central differences along random directions.  With |x| <= 8 and steps h = 2^-5 along a unit direction the third derivative of these losses
    (weights 1 / T) is below 4, so the difference is off by h^2 4 / 6 < 7e-4 and by the losses' own roundings (2e-6 each) / 2 h = 4e-5."""
    T, V, h = 70, 64, 2.0 ** -5
    g = gen(5)
    x, y = inputs(g, T, V, "f32", scale=1.0)
    row = Row64(x, y, 1.0)
    old, adv, ref, _ = policy_inputs(g, row, T)
    off = torch.tensor([0, 20, 35, 50, 70]).cuda()

    def loss(x):
        if form == "policy":
            return lib.policy_loss(ctx, x, y.cuda(), old.cuda(), adv.cuda(), ref_logp=ref.cuda(), kl=0.5, clip_low=0.99, clip_high=50.0)
        return lib.preference_loss(ctx, x, y.cuda(), off, ref_logp=ref.cuda(), beta=0.1, form=form)

    grad = loss(x.cuda())["dlogits"].cpu().double()
    for _ in range(5):
        v = torch.randn((T, V), generator=g)
        v /= v.norm()
        up, down = (loss((x + s * h * v).cuda())["loss"].double().item() for s in (1, -1))
        assert abs((up - down) / (2 * h) - (grad * v.double()).sum().item()) <= 7.5e-4


def test_same_results_every_time(lib, ctx):
    g = gen(8)
    x, y = inputs(g, 900, 3001, "bf16")
    old = torch.zeros(900).cuda() - 3
    adv = torch.randn(900, generator=g).cuda()
    off = torch.arange(0, 901, 90).cuda()
    a, b = (lib.policy_loss(ctx, x.cuda(), y.cuda(), old, adv, ref_logp=old, kl=0.1) for _ in range(2))
    assert all(torch.equal(a[k], b[k]) for k in a)
    a, b = (lib.preference_loss(ctx, x.cuda(), y.cuda(), off[:-1] if len(off) % 2 == 0 else off, ref_logp=old) for _ in range(2))
    assert all(torch.equal(a[k], b[k]) for k in a)


def test_broadcast_and_repeated_rows(lib, ctx):
    """A row of logits that stands for all rows, without being copied: every row has its own gradient."""
    g = gen(3)
    x, y = inputs(g, 1, 300, "f32")
    y = torch.randint(0, 300, (66,), generator=g)
    wide = x.cuda().expand(66, 300)
    got = lib.token_logprobs(ctx, wide, y.cuda())
    Row64(x.expand(66, 300), y, 1.0).check(got)
    back = lib.token_logprobs_backward(ctx, torch.ones(66).cuda(), wide, y.cuda(), got["top"], got["log_sum"])
    assert back.shape == (66, 300) and back.is_contiguous()


def test_offsets_beyond_32_bits(lib, ctx):
    """More than 2^32 logits: the last rows are the ones that a 32-bit offset would miss."""
    T, V = 40000, 110000
    x = torch.zeros((T, V), dtype=torch.bfloat16, device="cuda")
    g = gen(9)
    tail, y = inputs(g, 3, V, "bf16", ignore=False)
    x[-3:] = tail.cuda()
    tokens = torch.full((T,), -1, dtype=torch.int64)
    tokens[-3:] = y
    tokens[0] = 5
    row = Row64(tail, y, 1.0)
    got = lib.policy_loss(ctx, x, tokens.cuda(), torch.full((T,), -3.0).cuda(), torch.ones(T).cuda(), weight=torch.ones(T).cuda(), clip_high=1e30)
    assert torch.all((got["logp"][-3:].double() - row.logp).abs() <= row.logp_err)
    dlogp = -(row.logp + 3).exp()
    row.check_slope(got["dlogits"][-3:], dlogp, dlogp.abs() * (row.logp_err + U * (row.logp + 3).abs() + 8 * U), torch.bfloat16)
    assert not got["dlogits"][1:-3].any()
    back = lib.token_logprobs_backward(ctx, torch.ones(T).cuda(), x, tokens.cuda(), torch.zeros(T).cuda(), torch.full((T,), math.log(V)).cuda())
    assert not back[1:-3].any() and back[-3:].any() and back[0, 5] > 0.99


@pytest.mark.parametrize("shape", [(1100, 65541), (600, 120001), (520, 131072)], ids=str)
def test_large_gradients(lib, ctx, shape):
    """Gradients of more than 128 MiB go past the cache; a few of their rows against the definition, rows that count for nothing among them."""
    T, V = shape
    g = torch.Generator(device="cuda").manual_seed(V)
    x = (torch.randn((T, V), generator=g, device="cuda") * 2).to(torch.bfloat16)
    y = torch.randint(0, V, (T,), generator=g, device="cuda")
    y[1::50] = -1
    rows = torch.tensor([0, 1, 2, 63, T // 2, T - 2, T - 1], device="cuda")
    row = Row64(x[rows], y[rows], 1.0)
    lp = lib.token_logprobs(ctx, x, y)
    row.check({k: v[rows] for k, v in lp.items()})
    adv = torch.randn(T, generator=g, device="cuda")
    got = lib.policy_loss(ctx, x, y, lp["logp"], adv, weight=torch.ones(T, device="cuda"), clip_low=1.0, clip_high=1e30)
    dlogp = -adv[rows].double() * row.live
    row.check_slope(got["dlogits"][rows], dlogp, dlogp.abs() * (2 * row.logp_err + 8 * U), torch.bfloat16)
    back = lib.token_logprobs_backward(ctx, adv, x, y, lp["top"], lp["log_sum"])
    sum_err = row.sum_err
    row.sum_err = (3 * 40 + 3 * 20 + 200) * U + 2 * sum_err        # |logits| below 40, log_sum below 20, both statistics as they came out of the forward pass
    row.check_slope(back[rows], adv[rows].double() * row.live, torch.zeros(len(rows)).double(), torch.bfloat16)
    off = torch.tensor([0, T // 3, T], device="cuda")
    pref = lib.preference_loss(ctx, x, y, off, beta=0.01)
    m = pref["margin"].double().item()
    sign = torch.where(rows < T // 3, 1.0, -1.0).double()
    dlogp = sign * 0.01 * (1 / (1 + math.exp(-m)) - 1) * row.live
    # the margin is a sum over all rows and comes back rounded to 32 bits: |m| below 300 (T rows of at most 30 each), slope 1/4
    row.check_slope(pref["dlogits"][rows], dlogp, 0.01 * 0.25 * 300 * U + 4 * U * dlogp.abs(), torch.bfloat16)


def calls(lib, c, x, y, old, adv, off):
    lp = lib.token_logprobs(c, x, y)
    back = lib.token_logprobs_backward(c, adv, x, y, lp["top"], lp["log_sum"])
    pol = lib.policy_loss(c, x, y, old, adv, ref_logp=old, kl=0.1)
    pref = lib.preference_loss(c, x, y, off, ref_logp=old)
    return [lp["logp"], back, pol["loss"], pol["dlogits"], pref["loss"], pref["margin"], pref["dlogits"]]


@pytest.mark.parametrize("shape", [(70, 900), (5, 30000), (20000, 64)], ids=str)
def test_in_a_graph(lib, shape):
    """Captured once and replayed on new inputs, with other calls of the same context in between; every replay as the call without a graph."""
    T, V = shape
    g = gen(4)
    side = torch.cuda.Stream()
    own = lib.Context(0, stream=side.cuda_stream)
    x, y = (t.cuda() for t in inputs(g, T, V, "bf16"))
    old, adv, off = torch.zeros(T).cuda() - 3, torch.randn(T, generator=g).cuda(), torch.tensor([0, T // 3, T]).cuda()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        calls(lib, own, x, y, old, adv, off)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = calls(lib, own, x, y, old, adv, off)
    for k in range(4):
        torch.cuda.synchronize()
        nx, ny = inputs(g, T, V, "bf16", scale=1.0 + k)
        x.copy_(nx)
        y.copy_(ny)
        off[1] = T // (k + 2)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        with torch.cuda.stream(side):
            eager = calls(lib, own, x, y, old, adv, off)
        torch.cuda.synchronize()
        for p, q in zip(got, eager):
            assert torch.equal(p, q)
    del graph
    own.close()


def test_on_another_stream(lib, ctx):
    g = gen(2)
    x0, y = inputs(g, 300, 5000, "f32")
    old, adv, off = torch.zeros(300).cuda() - 3, torch.randn(300, generator=g).cuda(), torch.tensor([0, 100, 300]).cuda()
    x0, y = x0.cuda(), y.cuda()
    want = calls(lib, ctx, x0, y, old, adv, off)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    own = lib.Context(0, stream=side.cuda_stream)
    for c, on in ((ctx, side), (own, torch.cuda.default_stream()), (own, side)):
        with torch.cuda.stream(on):
            big = torch.randn(4096, 4096, device="cuda")
            for _ in range(3):
                big = big @ big                     # keeps the stream busy while the host goes on
            x = x0.clone()
            got = [t.clone() for t in calls(lib, c, x, y, old, adv, off)]
            del x
            torch.zeros(300, 5000, device="cuda")
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want))
    own.close()


def test_refusals(lib, ctx):
    x, y = torch.zeros(4, 8, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    f = torch.zeros(4, device="cuda")
    off = torch.tensor([0, 2, 4], device="cuda")
    for bad in (x.cpu(), x.double(), x[0], x.t(), x[None]):
        with pytest.raises(ValueError):
            lib.token_logprobs(ctx, bad, y)
    with pytest.raises(lib.ZkdlError):
        lib.token_logprobs(ctx, x.to(torch.int8), y)
    with pytest.raises(lib.ZkdlError):
        lib.token_logprobs(ctx, x[:, :0], y)
    for bad in (y.cpu(), y.float(), y[:3], y[:, None], y.to(torch.int16), torch.zeros(8, dtype=torch.int64, device="cuda")[::2]):
        with pytest.raises(ValueError):
            lib.token_logprobs(ctx, x, bad)
    for tau in (0.0, -1.0, float("nan"), float("inf"), 1e-42, 1e39, 1e-39):
        with pytest.raises(lib.ZkdlError):
            lib.token_logprobs(ctx, x, y, temperature=tau)
    for bad in (None, f[:3], f.half(), f.cpu()):
        with pytest.raises(ValueError):
            lib.token_logprobs_backward(ctx, bad, x, y, f, f)
        with pytest.raises(ValueError):
            lib.token_logprobs_backward(ctx, f, x, y, bad, f)
        with pytest.raises(ValueError):
            lib.policy_loss(ctx, x, y, bad, f)
        with pytest.raises(ValueError):
            lib.policy_loss(ctx, x, y, f, bad)
    for kw in (dict(clip_low=-0.1), dict(clip_low=1.5), dict(clip_high=-0.1), dict(clip_high=float("inf")), dict(clip_low=float("nan")), dict(kl=0.1),
               dict(kl=float("nan"), ref_logp=f), dict(temperature=0.0)):
        with pytest.raises(lib.ZkdlError):
            lib.policy_loss(ctx, x, y, f, f, **kw)
    for bad in (off[:2], off.float(), off.cpu(), off[:0]):
        with pytest.raises(ValueError):
            lib.preference_loss(ctx, x, y, bad)
    with pytest.raises(ValueError):
        lib.preference_loss(ctx, x, y, off, weight=f)          # one for each pair
    for kw in (dict(beta=float("inf")), dict(target=float("nan")), dict(smoothing=-0.1), dict(smoothing=1.1), dict(smoothing=0.1, form="hinge"), dict(temperature=-1.0)):
        with pytest.raises(lib.ZkdlError):
            lib.preference_loss(ctx, x, y, off, **kw)
    # and after all that the context serves the next call
    assert torch.all((lib.token_logprobs(ctx, x, y)["logp"] + math.log(8)).abs() <= 4 * U)


def test_no_rows(lib, ctx):
    x, y, f = torch.zeros(0, 8, device="cuda"), torch.zeros(0, dtype=torch.int64, device="cuda"), torch.zeros(0, device="cuda")
    got = lib.token_logprobs(ctx, x, y)
    assert all(got[k].shape == (0,) for k in got)
    assert lib.token_logprobs_backward(ctx, f, x, y, f, f).shape == (0, 8)
    got = lib.policy_loss(ctx, x, y, f, f)
    assert got["loss"].item() == 0 and got["clipped"].item() == 0 and got["dlogits"].shape == (0, 8)
    got = lib.preference_loss(ctx, x, y, torch.zeros(3, dtype=torch.int32, device="cuda"), beta=1.0)
    assert abs(got["loss"].item() - math.log(2)) <= 2 * U and got["margin"].tolist() == [0.0]
    got = lib.preference_loss(ctx, torch.zeros(4, 8, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda"))
    assert got["loss"].item() == 0 and got["margin"].shape == (0,) and not got["dlogits"].any()


def test_offsets_out_of_order_stay_in_bounds(lib, ctx):
    """Offsets are device data: what does not fit gives numbers without meaning, for the rows of this call alone."""
    x, y = (t.cuda() for t in inputs(gen(1), 8, 100, "f32"))
    for off in ([0, 100, 8], [-5, 3, 2 ** 40], [6, 2, 4], [8, 8, 0]):
        got = lib.preference_loss(ctx, x, y, torch.tensor(off, device="cuda"))
        assert got["dlogits"].shape == (8, 100)
    want = Row64(x.cpu(), y.cpu(), 1.0)
    want.check(lib.token_logprobs(ctx, x, y))
