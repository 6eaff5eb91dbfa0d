"""The gradient norm and AdamW against their definitions in 64 bits.  u = 2^-24 is the unit roundoff of 32-bit floats."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF_ULP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -133}
M32 = 0xFFFFFFFF


def gen(seed):
    return torch.Generator().manual_seed(seed)


def shifted(t, offset):
    """The same contiguous tensor on the GPU at an odd address."""
    buf = torch.empty(t.numel() + offset + 8, dtype=t.dtype, device="cuda")
    v = buf[offset:offset + t.numel()].view(t.shape)
    v.copy_(t)
    return v


# ---- norm ----------------------------------------------------------------------------------------------------------------

LISTS = [[(1,)], [(7,)], [(8191,)], [(8192,)], [(8193,)], [(3, 5), (0,), (1,), (100, 83)], [(17,)] * 161, [(2048, 1025), (5,)], [()], [(300, 8192)] * 3]


@pytest.mark.parametrize("shapes", LISTS, ids=lambda s: f"{len(s)}x{s[0]}")
@pytest.mark.parametrize("dtype", list(TYPES) + ["mixed"])
def test_gradient_norm(lib, ctx, shapes, dtype):
    """Squares of 32-bit numbers and their sums have 53 bits: what is left is the rounding to 32."""
    g = gen(len(shapes) + sum(shapes[0]) if shapes[0] else 1)
    ts = [torch.randn(s, generator=g).to(TYPES[dtype if dtype != "mixed" else ("f32", "bf16", "f16")[i % 3]]) for i, s in enumerate(shapes)]
    want = math.sqrt(sum(float(t.double().square().sum()) for t in ts))
    for where in (lambda t: t.cuda(), lambda t: shifted(t, 3)):
        dev = [where(t) for t in ts]
        got = lib.gradient_norm(ctx, dev, limit=want / 2)
        assert abs(got["norm"].item() - want) <= 1.01 * U * want and abs(got["factor"].item() - .5) <= 1.01 * U
        assert lib.gradient_norm(ctx, tuple(dev), limit=want * 2)["factor"].item() == 1
        assert lib.gradient_norm(ctx, dev)["factor"].item() == 1


def test_gradient_norm_of_any_size(lib, ctx):
    """Squares that 32 bits do not hold, infinities and NaN."""
    for x in (1e30, 3e38, 1e-30, 2.0 ** -149):
        t = torch.full((300,), x)
        want = math.sqrt(300) * float(t[0].double())
        got = lib.gradient_norm(ctx, [t.cuda()], limit=1.0)
        if want < 3.4e38:
            assert abs(got["norm"].item() - want) <= U * want + 2.0 ** -149
            assert abs(got["factor"].item() - min(1.0, 1 / want)) <= U * min(1.0, 1 / want) + 2.0 ** -149
        else:       # the norm itself is beyond 32 bits
            assert got["norm"].item() == math.inf and math.isnan(got["factor"].item())
    for bad in (math.inf, -math.inf, math.nan):
        t = torch.ones(9000)
        t[8999] = bad
        got = lib.gradient_norm(ctx, [torch.ones(5).cuda(), t.cuda()], limit=1.0)
        assert not math.isfinite(got["norm"].item()) and math.isnan(got["factor"].item())
    got = lib.gradient_norm(ctx, [], limit=1.0)
    assert got["norm"].item() == 0 and got["factor"].item() == 1


# ---- AdamW -----------------------------------------------------------------------------------------------------------------

def adam64(p, g, m, v, step, lr, beta1, beta2, eps, decay, factor):
    d = g.double() * factor
    m = beta1 * m.double() + (1 - beta1) * d
    v = beta2 * v.double() + (1 - beta2) * d * d
    m32, v32 = m.float().double(), v.float().double()
    move = lr / (1 - beta1 ** step) * m32 / (v32.sqrt() / math.sqrt(1 - beta2 ** step) + eps)
    return p.double() * (1 - lr * decay) - move, move, m, v


def check_params(got, want, move, before):
    """1 - lr decay and its product are rounded, and the move is a quotient of factors with a rounding or an ulp each, ten in all."""
    t = got.dtype
    err = 2 * U * before.double().abs() + 12 * U * move.abs() + 2.0 ** -149
    err = err + U * want.abs() + HALF_ULP[t] * (want.abs() + err) + TINY[t]
    assert torch.all((got.cpu().double() - want).abs() <= err), ((got.cpu().double() - want).abs() / err).max()


SHAPES = [[(1,)], [(7,), (8,), (9,)], [(256,), (255,), (257,)], [(4095,), (4096,), (4097,)], [(3, 0), (130, 70), ()], [(33,)] * 41, [(33,)] * 81, [(1000, 1003), (5,)]]
HOW = dict(lr=0.01, beta1=0.9, beta2=0.99, eps=1e-6, decay=0.1)


@pytest.mark.parametrize("shapes", SHAPES, ids=lambda s: f"{len(s)}x{s[0]}")
@pytest.mark.parametrize("ptype", list(TYPES))
@pytest.mark.parametrize("gtype", list(TYPES))
def test_adamw_32(lib, ctx, shapes, ptype, gtype):
    """Two steps behind each other, tensors at odd addresses; states are the 64-bit ones rounded once."""
    g = gen(len(shapes))
    for offset in (0, 3):
        params = [shifted(torch.randn(s, generator=g).to(TYPES[ptype]), offset) for s in shapes]
        state = lib.adamw_state(params)
        for k in ("m", "v"):
            state[k] = [shifted(t.cpu(), offset) for t in state[k]]
        for step in (1, 2):
            grads = [shifted((torch.randn(s, generator=g) * 10.0 ** (i % 4 - 2)).to(TYPES[gtype]), offset) for i, s in enumerate(shapes)]
            factor = torch.tensor(0.75, device="cuda") if step == 2 else None
            old = [[t.cpu().clone() for t in l] for l in (params, grads, state["m"], state["v"])]
            assert lib.adamw_step(ctx, params, grads, state, step, factor=factor, **HOW) == dict(m=None, v=None)
            for i in range(len(shapes)):
                p, d, m, v = (l[i] for l in old)
                # of the 64-bit sums b m + (1 - b) d each side has a rounding in either product (two in the second) and one of the sum: where the
                # two cancel (16-bit gradients of opposite sign do so to the last bit) what is left is off by that, whatever its own size
                slack = [2.0 ** -50 * (x.double().abs() + y) for x, y in ((m, d.double().abs()), (v, d.double() ** 2))]
                want, move, m, v = adam64(p, d, m, v, step, factor=0.75 if step == 2 else 1.0, **HOW)
                for got, x, more in ((state["m"][i], m, slack[0]), (state["v"][i], v, slack[1])):
                    assert torch.all((got.cpu().double() - x).abs() <= U * (1 + 2.0 ** -20) * x.abs() + more + 2.0 ** -149)
                check_params(params[i], want, move, p)


@pytest.mark.parametrize("eps", [1e-8, 1e-20, 1e-30, 1e-37])
def test_second_moments_below_the_normal_numbers(lib, ctx, eps):
    """Gradients from 1 down to 1e-23 and 0: v goes down to 0 through the subnormal numbers, and its root with it."""
    g = gen(31)
    n = 3000
    d = torch.randn(n, generator=g) * 10.0 ** (-(torch.arange(n) % 24).float())
    d[::50] = 0
    p, m, v = torch.randn(n, generator=g) * 1e-3, torch.zeros(n), torch.zeros(n)
    how = dict(lr=0.01, beta1=0.9, beta2=0.999, eps=eps, decay=0.0)
    want, move, m64, v64 = adam64(p, d, m, v, 1, factor=1.0, **how)
    assert ((v64.float() > 0) & (v64.float() < 2.0 ** -126)).sum() > 100
    for bits in (32, 8):
        w, state = p.cuda(), lib.adamw_state([p.cuda()], bits)
        lib.adamw_step(ctx, [w], [d.cuda()], state, 1, **how)
        # the 64-bit moments of either side may round to neighbouring numbers of 32 bits, of which subnormal ones are far apart
        (near, far) = (adam64(p, d * s, m, v, 1, factor=1.0, **how)[1] for s in (1 - 2.0 ** -50, 1 + 2.0 ** -50))
        slack = torch.maximum((near - move).abs(), (far - move).abs())
        err = 2 * U * p.double().abs() + 12 * U * move.abs() + U * want.abs() + 2.0 ** -148 + slack
        assert torch.all((w.cpu().double() - want).abs() <= err)


@pytest.mark.parametrize("eps", [1e15, 1e25, 1e38, 3e38])
def test_an_eps_as_large_as_numbers_go(lib, ctx, eps):
    """A step is as long as the definition's, from numbers of the host and of the device.  (v stays in the range of 32 bits.)"""
    n = 300
    for d, lr in ((torch.full((n,), 1e18), 1.0), (torch.linspace(1e16, 5e18, n), 1e6)):
        zero = torch.zeros(n)
        how = dict(beta1=0.9, beta2=0.999, eps=eps, decay=0.0)
        want, move, _, _ = adam64(zero, d, zero, zero, 1, factor=1.0, lr=lr, **how)
        for at in (1, torch.tensor(1, device="cuda")):
            w, state = torch.zeros(n, device="cuda"), lib.adamw_state([zero.cuda()])
            lib.adamw_step(ctx, [w], [d.cuda()], state, at, lr, **how)
            assert torch.all((w.cpu().double() - want).abs() <= 13 * U * move.abs() + 2.0 ** -149)


def mix(x):
    x = x ^ x >> 16
    x = x * 0x9E3779B1 & M32
    x = x ^ x >> 15
    x = x * 0x85A308D3 & M32
    return x ^ x >> 16


def bits16(n, seed, step, number):
    """(of m, of v) for each entry."""
    key = 0
    for w in (seed & M32, seed >> 32, step, number):
        key = int(mix(torch.tensor(key ^ w)))
    i = torch.arange(n)
    r = mix(mix(key ^ i // 256) + i % 256 * 0x9E3779B1 & M32)
    return r >> 16, r & 0xFFFF


def decode(code, scale, log):
    """The values of codes, by the format's definition."""
    c = code.reshape(-1).long()
    e = scale.long().clamp(min=40).repeat_interleave(256)[:c.numel()]
    sign = torch.where(c > 127, -1.0, 1.0).double() if log == 4 else torch.ones(c.shape).double()
    if log == 4:
        c = c & 127
    exp, f = c >> 3, c & 7
    value = sign * torch.where(exp > 0, f + 8, f).double() * torch.exp2((e - 127 - (2 ** log - 1) + exp.clamp(min=1) - 3).double())
    return torch.where(e == 255, torch.full_like(value, math.nan), value).view(code.shape)


def encode(x, log, b):
    """(codes, scales) of 32-bit numbers, by the format's definition: b are 16 random bits."""
    flat, n, last = x.reshape(-1).float(), x.numel(), 2 ** log - 1
    mag = flat.abs().double()
    top = torch.nn.functional.pad(mag, (0, -n % 256)).view(-1, 256).amax(1)
    frac, power = torch.frexp(top.nan_to_num(0, 0, 0))
    e = torch.where(top > 0, (power - 1 + (frac > 15 / 16).int() + 127).long(), torch.zeros(len(top), dtype=torch.long)).clamp(min=40)
    e = torch.where(~torch.isfinite(top) | (e > 254), torch.full_like(e, 255), e)
    ee = e.repeat_interleave(256)[:n]
    _, own = torch.frexp(mag.nan_to_num(0, 0, 0))
    exp = (torch.where(mag > 0, own.long() - 1 + 127, torch.zeros(n, dtype=torch.long)) - ee + last).clamp(min=0)
    unit = torch.exp2((ee - 127 - last + exp.clamp(min=1) - 3).double())
    place = mag.nan_to_num(0, 0, 0) / unit
    # 16 random bits decide between neighbours
    up = place - place.floor() + (b.double() + .5) / 65536 >= 1
    whole = place.floor() + up.double()
    code = torch.where(exp > 0, exp * 8 + whole.long() - 8, whole.long())
    if log == 5:
        code = torch.where(mag > 0, code.clamp(min=1), code)
    else:
        code = torch.where(torch.signbit(flat), code | 128, code)
    return torch.where(ee == 255, torch.zeros_like(code), code).to(torch.uint8).view(x.shape), e.to(torch.uint8)


@pytest.mark.parametrize("shapes", SHAPES, ids=lambda s: f"{len(s)}x{s[0]}")
@pytest.mark.parametrize("ptype,gtype", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("f16", "f32")])
def test_adamw_8(lib, ctx, shapes, ptype, gtype):
    """Three steps behind each other: codes, exponents and values are those of the definition, entry by entry."""
    g = gen(len(shapes) + 50)
    seed = 0x123456789ABCDEF
    for offset in (0, 3):
        params = [shifted(torch.randn(s, generator=g).to(TYPES[ptype]), offset) for s in shapes]
        state = lib.adamw_state(params, bits=8)
        for k in ("m", "v"):
            state[k] = [shifted(t.cpu(), offset) for t in state[k]]
        for step in (1, 2, 3):
            grads = [shifted((torch.randn(s, generator=g) * torch.exp(3 * torch.randn(s, generator=g))).to(TYPES[gtype]), offset) for s in shapes]
            old = [[t.cpu().clone() for t in l] for l in (params, grads, state["m"], state["v"], state["m_scale"], state["v_scale"])]
            got = lib.adamw_step(ctx, params, grads, state, step, seed=seed, values=step != 2, **HOW)
            for i in range(len(shapes)):
                p, d, cm, cv, em, ev = (l[i] for l in old)
                want, move, m, v = adam64(p, d, decode(cm, em, 4), decode(cv, ev, 5), step, factor=1.0, **HOW)
                check_params(params[i], want, move, p)
                for name, x, log, b in zip(("m", "v"), (m, v), (4, 5), bits16(p.numel(), seed, step, i)):
                    code, scale = encode(x, log, b)
                    assert torch.equal(state[name][i].cpu(), code) and torch.equal(state[name + "_scale"][i].cpu(), scale)
                    if step != 2:
                        assert torch.equal(got[name][i].cpu().double(), decode(code, scale, log))


def test_8_bit_states_of_any_size(lib, ctx):
    """Blocks of the smallest and largest numbers, of zeros, with infinities and NaN: others are not touched by their neighbours' size."""
    p = torch.zeros(8 * 256 + 3)
    d = torch.zeros_like(p)
    d[:256] = torch.linspace(-1, 1, 256)
    d[256:512] = 2.0 ** -149
    d[512:768] = 1e19                        # squares up to 1e38
    d[768:1024] = 1e25                       # squares beyond 32 bits
    d[1024 + 7] = math.inf
    d[1280 + 7] = math.nan
    d[1536:1792] = 2.0 ** torch.arange(-128, 128).clamp(max=60).float()
    d[-1] = 3.0
    params, grads = [p.cuda()], [d.cuda()]
    state = lib.adamw_state(params, bits=8)
    got = lib.adamw_step(ctx, params, grads, state, 1, values=True, **HOW)
    want, move, m, v = adam64(p, d, torch.zeros_like(p), torch.zeros_like(p), 1, factor=1.0, **HOW)
    for name, x, log, b in zip(("m", "v"), (m, v), (4, 5), bits16(p.numel(), 0, 1, 0)):
        code, scale = encode(x, log, b)
        assert torch.equal(state[name][0].cpu(), code) and torch.equal(state[name + "_scale"][0].cpu(), scale)
        assert torch.equal(got[name][0].cpu().double().nan_to_num(7), decode(code, scale, log).nan_to_num(7))
    fine = torch.ones(len(p), dtype=torch.bool)
    fine[768:1536] = False
    assert torch.all(torch.isfinite(params[0].cpu()[fine]))
    assert torch.all((got["v"][0] > 0).cpu()[fine] == (v.float() > 0)[fine])         # no second moment vanishes


def test_8_bit_states_are_right_on_average(lib, ctx):
    """256 seeds on the same numbers.  Between two codes the mean of the results' distances to the true value, in codes' distances, has a standard
    deviation of at most 1/2 / sqrt(256 n); six of them are allowed, and the random bits' own 2^-17 of a distance."""
    n, seeds = 2048, 256
    g = gen(1)
    p, d = torch.zeros(n), torch.randn(n, generator=g)
    m0, v0, total = None, None, [torch.zeros(n).double(), torch.zeros(n).double()]
    for seed in range(seeds):
        params = [p.cuda()]
        state = lib.adamw_state(params, bits=8)
        got = lib.adamw_step(ctx, params, [d.cuda()], state, 1, seed=seed, values=True, **HOW)
        for k, name in enumerate(("m", "v")):
            total[k] += got[name][0].cpu().double()
    _, _, m, v = adam64(p, d, torch.zeros(n), torch.zeros(n), 1, factor=1.0, **HOW)
    for x, s, log in ((m, total[0], 4), (v, total[1], 5)):
        x = x.float().double()
        top = x.abs().view(-1, 256).amax(1)
        _, e = torch.frexp(top)
        lowest = (e - 1 - (2 ** log - 1) + 1).repeat_interleave(256)        # at least: a block that is rounded up has one more
        own = torch.frexp(x)[1] - 1
        unit = torch.exp2((torch.maximum(own, lowest) - 3).double())
        keep = x.abs() > 16 * torch.exp2((lowest - 3).double())             # those whose distance does not depend on the block's exponent
        off = ((s / seeds - x) / unit)[keep]
        assert abs(off.mean().item()) <= 6 * .5 / math.sqrt(seeds * int(keep.sum())) + 2.0 ** -17
        assert off.abs().max().item() <= 6 * .5 / math.sqrt(seeds) + 2.0 ** -17


def test_8_bit_states_follow_small_changes(lib, ctx):
    """A step of beta2 = 0.999 moves v by less than a code's distance.  300 steps of gradients of 1 and -1: the mean over 4096 entries of v is
    1 - 0.999^300 = 0.259; each rounding has a variance of at most (v / 8)^2 / 4 and is kept by 0.999 a step, so the mean's standard deviation
    is at most sqrt(300) (0.26 / 16) / sqrt(4096) = 0.0044.  Five of them are allowed."""
    n = 4096
    params = [torch.zeros(n, device="cuda")]
    state = lib.adamw_state(params, bits=8)
    sign = torch.where(torch.arange(n) % 3 == 0, -1.0, 1.0).cuda()
    for step in range(1, 301):
        got = lib.adamw_step(ctx, params, [sign], state, step, 1e-3, beta2=0.999, values=step == 300)
    assert abs(got["v"][0].mean().item() - (1 - 0.999 ** 300)) <= 5 * 0.0044
    assert abs((got["m"][0] * sign).mean().item() - 1) <= 0.01


@pytest.mark.parametrize("bits", [32, 8])
def test_steps_that_are_left_out(lib, ctx, bits):
    g = gen(3)
    params = [torch.randn(5000, generator=g).cuda(), torch.randn(3, generator=g).cuda()]
    grads = [torch.randn(5000, generator=g).cuda(), torch.randn(3, generator=g).cuda()]
    state = lib.adamw_state(params, bits=bits)
    first = lib.adamw_step(ctx, params, grads, state, 1, 0.1, values=bits == 8)
    kept = [t.clone() for l in (params, state["m"], state["v"], state["m_scale"], state["v_scale"]) for t in l]
    same = lambda: all(torch.equal(a, b) for a, b in zip(kept, [t for l in (params, state["m"], state["v"], state["m_scale"], state["v_scale"]) for t in l]))
    for factor in (math.nan, math.inf, -math.inf):
        got = lib.adamw_step(ctx, params, grads, state, 2, 0.1, factor=torch.tensor(factor, device="cuda"), values=bits == 8)
        assert same()
        if bits == 8:
            assert all(torch.equal(a, b) for k in ("m", "v") for a, b in zip(got[k], first[k]))
    grads[1][0] = math.inf
    n = lib.gradient_norm(ctx, grads, limit=1.0)
    lib.adamw_step(ctx, params, grads, state, 2, 0.1, factor=n["factor"])
    assert same()
    for step in (0, -3, 2 ** 31, 2 ** 40):      # a number on the device that is no step's
        lib.adamw_step(ctx, params, [torch.ones_like(p) for p in params], state, torch.tensor(step, device="cuda"), 0.1)
        assert same()
    lib.adamw_step(ctx, params, [torch.ones_like(p) for p in params], state, 2, 0.1)
    assert not same()


@pytest.mark.parametrize("bits", [32, 8])
def test_step_and_rate_from_the_device(lib, ctx, bits):
    """The same bits as with numbers from the host; lr is a number that 32 bits hold."""
    g = gen(7)
    for step in (1, 2, 1000, 2 ** 31 - 1):
        p = torch.randn(9001, generator=g)
        d = torch.randn(9001, generator=g).cuda()
        outs = []
        for s, lr in ((step, 0.125), (torch.tensor(step, device="cuda"), torch.tensor([0.125], device="cuda")), (step, torch.tensor(0.125, device="cuda"))):
            params = [p.cuda()]
            state = lib.adamw_state(params, bits=bits)
            lib.adamw_step(ctx, params, [d], state, s, lr, seed=-1)
            outs.append((params[0], state["m"][0], state["v"][0]))
        for o in outs[1:]:
            assert all(torch.equal(a, b) for a, b in zip(o, outs[0]))


@pytest.mark.parametrize("bits", [32, 8])
def test_many_types_in_one_call(lib, ctx, bits):
    """A list of mixed types and sizes gives what each tensor gives alone at the same place."""
    g = gen(11)
    kinds = [(p, d) for p in TYPES.values() for d in TYPES.values()] * 6
    ps = [torch.randn(100 + 37 * i, generator=g).to(p).cuda() for i, (p, _) in enumerate(kinds)]
    ds = [torch.randn(100 + 37 * i, generator=g).to(d).cuda() for i, (_, d) in enumerate(kinds)]
    together = [p.clone() for p in ps]
    state = lib.adamw_state(together, bits=bits)
    lib.adamw_step(ctx, together, ds, state, 3, 0.01)
    for i, (p, d) in enumerate(zip(ps, ds)):
        if bits == 8 and i:
            continue                # the random bits are the place's: the others are compared by parameters, which do not depend on them
        alone = [p.clone()]
        one = lib.adamw_state(alone, bits=bits)
        lib.adamw_step(ctx, alone, [d], one, 3, 0.01)
        assert torch.equal(one["m"][0], state["m"][i]) and torch.equal(one["v"][0], state["v"][i])
    for i, (p, d) in enumerate(zip(ps, ds)):
        alone = [p.clone()]
        lib.adamw_step(ctx, alone, [d], lib.adamw_state(alone, bits=bits), 3, 0.01)
        assert torch.equal(alone[0], together[i])


def test_norm_and_step_in_a_graph(lib):
    """Norm, factor and update captured once, the step's number and the rate in device memory, replayed against calls without a graph."""
    g = gen(4)
    side = torch.cuda.Stream()
    own = lib.Context(0, stream=side.cuda_stream)
    for bits in (32, 8):
        params = [torch.randn(s, generator=g).cuda() for s in ((300, 70), (5,))]
        other = [p.clone() for p in params]
        grads = [torch.zeros_like(p) for p in params]
        state, mirror = lib.adamw_state(params, bits=bits), lib.adamw_state(params, bits=bits)
        step, lr = torch.zeros((), dtype=torch.int64, device="cuda"), torch.tensor(0.01, device="cuda")

        def update(p, s):
            n = lib.gradient_norm(own, grads, limit=1.0)
            lib.adamw_step(own, p, grads, s, step, lr, factor=n["factor"])
            return n["norm"]

        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            update(other, mirror)           # a step numbered 0 changes nothing
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(params, other))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            norm = update(params, state)
        for k in range(4):
            torch.cuda.synchronize()
            step += 1
            lr *= 0.5
            for d in grads:
                d.copy_(torch.randn(d.shape, generator=g) * 10 ** (k - 2))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            with torch.cuda.stream(side):
                want = update(other, mirror)
            torch.cuda.synchronize()
            assert torch.equal(norm, want)
            for a, b in zip(params + state["m"] + state["v"] + state["v_scale"], other + mirror["m"] + mirror["v"] + mirror["v_scale"]):
                assert torch.equal(a, b)
        del graph
    own.close()


def test_on_another_stream(lib, ctx):
    g = gen(2)
    p0, d0 = torch.randn(300, 500, generator=g).cuda(), torch.randn(300, 500, generator=g).cuda()
    side = torch.cuda.Stream()
    own = lib.Context(0, stream=side.cuda_stream)

    def update(c, p, d):
        state = lib.adamw_state([p], bits=8)
        n = lib.gradient_norm(c, [d], limit=2.0)
        lib.adamw_step(c, [p], [d], state, 1, 0.1, factor=n["factor"])
        return [p, state["m"][0], state["v"][0], n["norm"]]

    want = update(ctx, p0.clone(), d0)
    torch.cuda.synchronize()
    for c, on in ((ctx, side), (own, torch.cuda.default_stream()), (own, side)):
        with torch.cuda.stream(on):
            big = torch.randn(4096, 4096, device="cuda")
            for _ in range(3):
                big = big @ big                     # keeps the stream busy while the host goes on
            d = d0.clone()
            got = [t.clone() for t in update(c, p0.clone(), d)]
            del d
            torch.zeros(300, 500, device="cuda")
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    own.close()


def test_autograd_is_told_of_the_update(lib, ctx):
    """A backward pass that would read a parameter of before the update is refused by autograd, as after any operation in place."""
    w = torch.randn(4, 4, device="cuda", requires_grad=True)
    x = torch.randn(4, 4, device="cuda", requires_grad=True)
    y = (w * x).sum()
    lib.adamw_step(ctx, [w], [torch.ones(4, 4, device="cuda")], lib.adamw_state([w]), 1, 0.1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


@pytest.mark.parametrize("bits", [32, 8])
def test_a_refused_update_leaves_autograd_alone(lib, ctx, bits):
    """Tensors that overlap, a rate that is no number: nothing is written, and what autograd keeps of the tensors is still theirs."""
    w = torch.randn(4, 4, device="cuda", requires_grad=True)
    x = torch.randn(4, 4, device="cuda", requires_grad=True)
    y = (w * x).sum()
    d, state = torch.ones(4, 4, device="cuda"), lib.adamw_state([w], bits)
    tensors = [w, *state["m"], *state["v"], *state["m_scale"], *state["v_scale"]]
    versions = [t._version for t in tensors]
    for grads, kw in (([w], {}), ([d], dict(lr=math.nan)), ([d], dict(beta1=1.0)), ([d], dict(eps=0.0)), ([d], dict(step=0))):
        with pytest.raises(lib.ZkdlError):
            lib.adamw_step(ctx, [w], grads, state, **{**dict(step=1, lr=0.1), **kw})
    assert [t._version for t in tensors] == versions
    y.backward()
    assert torch.equal(x.grad, w.detach())
    lib.adamw_step(ctx, [w], [d], state, 1, 0.1)
    assert all(t._version > v for t, v in zip(tensors, versions))


def test_tensors_of_inference_mode(lib, ctx):
    """Updated inside of it; refused outside, with nothing written."""
    with torch.inference_mode():
        w = [torch.ones(300, device="cuda")]
        d, state = [torch.ones(300, device="cuda")], lib.adamw_state(w)
        lib.adamw_step(ctx, w, d, state, 1, 0.25, decay=0.0)
    kept = w[0].cpu()
    assert torch.all((kept - 0.75).abs() < 1e-6)
    with pytest.raises(RuntimeError, match="nference"):
        lib.adamw_step(ctx, w, d, state, 2, 0.25)
    assert torch.equal(w[0].cpu(), kept)


def test_lists_of_any_kind(lib, ctx):
    """Tuples, generators and a stack of parameters, on the context's stream and on another."""
    stack, d = torch.zeros(3, 50, device="cuda"), torch.ones(3, 50, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for k, on in enumerate((torch.cuda.default_stream(), side)):
        with torch.cuda.stream(on):
            assert abs(lib.gradient_norm(ctx, (x for x in d))["norm"].item() - math.sqrt(150)) <= 1e-6
            state = lib.adamw_state(stack)
            lib.adamw_step(ctx, stack, (x for x in d), state, 1, 0.5, decay=0.0)
            lib.adamw_step(ctx, (x for x in stack), tuple(d), state, 2, 0.5, decay=0.0)
            assert torch.all(stack < -0.9 * (k + 1)) and torch.all(stack > -1.1 * (k + 1))
        torch.cuda.synchronize()


def test_refusals(lib, ctx):
    p, d = [torch.zeros(10, device="cuda")], [torch.ones(10, device="cuda")]
    s, s8 = lib.adamw_state(p), lib.adamw_state(p, bits=8)
    for bad in ([torch.zeros(10)], [torch.zeros(10, device="cuda").double()], [torch.zeros(20, device="cuda")[::2]], [None], 3):
        with pytest.raises(ValueError):
            lib.gradient_norm(ctx, bad)
        with pytest.raises(ValueError):
            lib.adamw_step(ctx, bad, d, s, 1, 0.1)
        with pytest.raises(ValueError):
            lib.adamw_step(ctx, p, bad, s, 1, 0.1)
    for limit in (0.0, -1.0, math.nan):
        with pytest.raises(lib.ZkdlError):
            lib.gradient_norm(ctx, d, limit=limit)
    with pytest.raises(ValueError):
        lib.adamw_step(ctx, p + p, d, s, 1, 0.1)
    with pytest.raises(ValueError):
        lib.adamw_step(ctx, p, [torch.ones(2, 5, device="cuda")], s, 1, 0.1)
    with pytest.raises(ValueError):
        lib.adamw_step(ctx, p, d, dict(s, m=[torch.zeros(11, device="cuda")]), 1, 0.1)
    with pytest.raises(ValueError):
        lib.adamw_step(ctx, p, d, dict(s, v=s8["v"]), 1, 0.1)
    with pytest.raises(ValueError):
        lib.adamw_step(ctx, p, d, dict(s8, v_scale=[torch.zeros(2, dtype=torch.uint8, device="cuda")]), 1, 0.1)
    with pytest.raises(ValueError):
        lib.adamw_step(ctx, p, d, s, 1, 0.1, values=True)
    with pytest.raises(ValueError):
        lib.adamw_step(ctx, p, d, s, 1, 0.1, factor=torch.ones(2, device="cuda"))
    with pytest.raises(ValueError):
        lib.adamw_step(ctx, p, d, s, torch.tensor(1, dtype=torch.int32, device="cuda"), 0.1)
    with pytest.raises(ValueError):
        lib.adamw_step(ctx, p, d, s, 1, torch.tensor(0.1, dtype=torch.float64, device="cuda"))
    for kw in (dict(step=0), dict(step=2 ** 31), dict(lr=math.nan), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=math.nan), dict(eps=0.0),
               dict(eps=1e-42), dict(eps=math.inf), dict(decay=math.inf)):
        with pytest.raises(lib.ZkdlError):
            lib.adamw_step(ctx, p, d, s, **{**dict(step=1, lr=0.1), **kw})
    with pytest.raises(lib.ZkdlError):
        lib.adamw_step(ctx, p, d, dict(s, bits=16), 1, 0.1)
    # the same memory twice: two tensors of the list, a gradient that is a parameter, a state for two, parts that overlap
    flat = torch.zeros(30, device="cuda")
    two = lib.adamw_state([flat[:10], flat[:10]])
    for ps, ds, st in (([flat[:10]] * 2, d + d, two), ([flat[:10], flat[9:19]], d + d, two), ([flat[:10]], [flat[5:15]], s),
                       ([flat[:10], flat[10:20]], d + d, dict(two, m=[two["m"][0]] * 2)), ([flat[:10], flat[10:20]], d + d, dict(two, v=two["m"])),
                       ([flat[:10]], d, dict(s, m=[flat[9:19]]))):
        with pytest.raises(lib.ZkdlError):
            lib.adamw_step(ctx, ps, ds, st, 1, 0.1)
    assert not flat.any() and not p[0].any() and not s["m"][0].any()
    # one gradient for two parameters is read twice, and neighbours do not overlap
    lib.adamw_step(ctx, [flat[:10], flat[10:20]], d + d, two, 1, 0.1)
    assert torch.equal(flat[:10], flat[10:20]) and flat[0] != 0 and not flat[20:].any()
    lib.adamw_step(ctx, [], [], lib.adamw_state([]), 1, 0.1)
