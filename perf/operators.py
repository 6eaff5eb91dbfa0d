"""Performance cases of the 8-bit layer operators: norm, quantisation and integer products, forward and backward.

A case is a dict of plain values.  `prepare` makes what a program holds before the call, `run` is one call.  Where `own` is false `run`
computes the operator from elementary torch operations in 32 bits, else it calls the library.

Kinds
  norm        rmsnorm_i8: residual added, RMS norm, 8-bit output with a scale for each token
  norm_bwd    rmsnorm_i8_backward: gradients of the summed stream and of the norm's weight
  quant       quantize_i8: a scale for each row (axis -1) or column (axis -2), for one matrix or a stack
  mm          matmul_i8: op(A) op(B) of 8-bit integers, int32 accumulators or scaled for each token and channel
  mm_bwd      matmul_i8_backward: gradients of a layer's input and weights through two 8-bit products

8-bit results are returned as the values they stand for (the operators' `values` output, in the input's type).
"""
import functools

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "i32": torch.int32}
EPS = 1e-6


def listed():
    return [
        # serving, one token through the norm in front of a 4096-wide layer: latency
        dict(name="norm_1x4096", kind="norm", M=1, N=4096, dtype="bf16", residual=True),
        # an evaluation batch of odd sizes without a residual: rows whose addresses are not aligned
        dict(name="norm_509x1001", kind="norm", M=509, N=1001, dtype="f16", residual=False),
        # a training batch of 8192 tokens, width 4096
        dict(name="norm_8192x4096", kind="norm", M=8192, N=4096, dtype="bf16", residual=True),
        # the headline network's batch (64 rows of 1024), master precision
        dict(name="norm_bwd_64x1024", kind="norm_bwd", M=64, N=1024, dtype="f32", residual=True),
        # the training batch's backward pass
        dict(name="norm_bwd_8192x4096", kind="norm_bwd", M=8192, N=4096, dtype="bf16", residual=True),
        # the weights of the headline network (8 layers of 1024 x 1024): a scale for each output channel
        dict(name="quant_w_8x1024x1024", kind="quant", S=8, M=1024, N=1024, axis=-2, dtype="f32", mult=False),
        # gradients of 4096 tokens times their channels' scales: a scale for each token
        dict(name="quant_g_4096x4096", kind="quant", S=1, M=4096, N=4096, axis=-1, dtype="bf16", mult=True),
        # serving, one token through a 4096 x 4096 layer whose weights are stored output channel first
        dict(name="mm_1x4096x4096", kind="mm", S=1, M=1, K=4096, N=4096, ta=False, tb=True, out="bf16"),
        # the forward products of the headline network, exact accumulators: the stack that is proved
        dict(name="mm_8x64x1024x1024_i32", kind="mm", S=8, M=64, K=1024, N=1024, ta=False, tb=False, out="i32"),
        # the training batch through a 4096 x 4096 layer: bound by the matrix cores
        dict(name="mm_8192x4096x4096", kind="mm", S=1, M=8192, K=4096, N=4096, ta=False, tb=True, out="bf16"),
        # a small layer of odd sizes, backward: nothing aligned, all three layouts
        dict(name="mm_bwd_333x1000x517", kind="mm_bwd", M=333, K=1000, N=517, tw=False, dtype="f16"),
        # 4096 tokens through a 4096 x 4096 layer, weights stored input first as the proofs have them
        dict(name="mm_bwd_4096x4096x4096", kind="mm_bwd", M=4096, K=4096, N=4096, tw=False, dtype="bf16"),
    ]


def _size(rng, lo, hi):
    """Log-uniform; half of the sizes are multiples of 64 (or powers of two below), the others whatever comes."""
    n = int(round(lo * (hi / lo) ** rng.random()))
    if rng.random() < 0.5:
        n = max(lo, n // 64 * 64 if n >= 64 else 1 << (n.bit_length() - 1))
    return n - 1 if n == 3072 else n      # no configuration here has that width


def draw(rng):
    kind = rng.choice(["norm", "norm_bwd", "quant", "mm", "mm_bwd"])
    dtype = rng.choice(["bf16", "f16", "f32"])
    size = 4 if dtype == "f32" else 2
    while True:
        M, N, K = _size(rng, 1, 8192), _size(rng, 16, 8192), _size(rng, 16, 8192)
        if kind in ("norm", "norm_bwd"):
            c = dict(kind=kind, M=M, N=N, dtype=dtype, residual=rng.random() < 0.6)
            if M * N * size <= 2 * 8192 * 4096:
                return c
        elif kind == "quant":
            c = dict(kind=kind, S=rng.choice([1, 1, 2, 4, 8]), M=M, N=N, axis=rng.choice([-1, -2]), dtype=dtype, mult=rng.random() < 0.5)
            if c["S"] * M * N * size <= 2 * 8192 * 4096:
                return c
        elif kind == "mm":
            ta, tb = rng.choice([(False, False), (False, True), (True, False), (False, True)])
            c = dict(kind=kind, S=rng.choice([1, 1, 1, 2, 8]), M=M, K=K, N=N, ta=ta, tb=tb, out=rng.choice(["i32", "bf16", "f16", "f32"]))
            if c["S"] * M * K * N <= 8192 * 4096 * 4096 and c["S"] * (K * N + M * K + 4 * M * N) <= 1 << 28:
                return c
        else:
            c = dict(kind=kind, M=M, K=K, N=N, tw=rng.random() < 0.5, dtype=dtype)
            if M * K * N <= 4096 * 4096 * 4096:
                return c


# ---- inputs -------------------------------------------------------------------------------------------------------------

def _activations(g, shape, dtype):
    """Normal, a few channels an order of magnitude larger, every 61st row a padded token of zeros."""
    x = torch.randn(shape, generator=g, device="cuda")
    x *= 1 + 15 * (torch.rand(shape[-1], generator=g, device="cuda") < 0.01)
    if shape[-2] > 60:
        x[..., 60::61, :] = 0
    return x.to(dtype)


def _gradients(g, shape, dtype):
    """What comes back through a ReLU: half of the entries are zero."""
    return (torch.randn(shape, generator=g, device="cuda") * 0.1 * (torch.rand(shape, generator=g, device="cuda") < 0.5)).to(dtype)


def _codes(g, shape, scale_shape):
    """8-bit integers as quantisation leaves them (|q| <= 127, about normal) and their scales."""
    q = (torch.randn(shape, generator=g, device="cuda") * 36).round_().clamp_(-127, 127).to(torch.int8)
    return q, 0.001 + 0.01 * torch.rand(scale_shape, generator=g, device="cuda")


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda").manual_seed(seed)
    if c["kind"] in ("norm", "norm_bwd"):
        t, shape = TYPES[c["dtype"]], (c["M"], c["N"])
        c["x"] = _activations(g, shape, t)
        c["weight"] = (1 + 0.2 * torch.randn(c["N"], generator=g, device="cuda")).to(t)
        c["r"] = None
        if c["kind"] == "norm":
            if c["residual"]:
                c["r"] = _activations(g, shape, t)
        else:
            c["dy"] = _gradients(g, shape, t)
            if c["residual"]:
                c["r"] = _gradients(g, shape, t)
            c["rstd"] = torch.rsqrt(c["x"].float().square().mean(-1) + EPS)
    elif c["kind"] == "quant":
        shape = (c["S"], c["M"], c["N"]) if c["S"] > 1 else (c["M"], c["N"])
        c["x"] = (_gradients if c["mult"] else _activations)(g, shape, TYPES[c["dtype"]])
        c["m"] = 0.001 + 0.01 * torch.rand(shape[:-2] + (shape[c["axis"]],), generator=g, device="cuda") if c["mult"] else None
    elif c["kind"] == "mm":
        lead = (c["S"],) if c["S"] > 1 else ()
        c["a"], sa = _codes(g, lead + ((c["K"], c["M"]) if c["ta"] else (c["M"], c["K"])), lead + (c["M"],))
        c["b"], sb = _codes(g, lead + ((c["N"], c["K"]) if c["tb"] else (c["K"], c["N"])), lead + (c["N"],))
        c["sa"], c["sb"] = (None, None) if c["out"] == "i32" else (sa, sb)
    else:
        c["a"], c["sa"] = _codes(g, (c["M"], c["K"]), (c["M"],))
        c["w"], c["sw"] = _codes(g, (c["N"], c["K"]) if c["tw"] else (c["K"], c["N"]), (c["N"],))
        c["dy"] = _gradients(g, (c["M"], c["N"]), TYPES[c["dtype"]])
    return c


# ---- the plain forms: elementary operations in 32 bits --------------------------------------------------------------------

def _quantise(v, dim):
    top = v.abs().amax(dim, keepdim=True)
    q = torch.round(v * torch.where(top > 0, torch.full_like(top, 127.0) / top, torch.zeros_like(top)))
    return q, top / 127.0


def _product(a, b):
    """[.., M, K] x [.., K, N] of 8-bit integers, as int32.  A sum of 1024 products of magnitude 127^2 is below 2^24, so 32-bit
    floats hold it exactly; longer sums are added as integers."""
    k, step = a.shape[-1], 1024
    n = -(-k // step)
    a = torch.nn.functional.pad(a.float(), (0, n * step - k)) if n > 1 else a.float()
    b = torch.nn.functional.pad(b.float(), (0, 0, 0, n * step - k)) if n > 1 else b.float()
    if n == 1:
        return torch.matmul(a, b).to(torch.int32)
    a = a.unflatten(-1, (n, step)).movedim(-2, 0).contiguous()
    b = b.unflatten(-2, (n, step)).movedim(-3, 0).contiguous()
    return torch.matmul(a, b).to(torch.int32).sum(0, dtype=torch.int32)


def _plain(s):
    kind = s["kind"]
    if kind == "norm":
        t = s["x"].dtype
        h = s["x"].float() if s["r"] is None else s["x"].float() + s["r"].float()
        rstd = 1.0 / torch.sqrt(h.square().mean(-1, keepdim=True) + EPS)
        # one factor for a whole row leaves the rounded quotients as they are: it goes into the scale alone
        q, scale = _quantise(h * s["weight"].float(), -1)
        scale = scale * rstd
        out = {"values": (q * scale).to(t), "scale": scale[:, 0], "rstd": rstd[:, 0]}
        if s["r"] is not None:
            out["total"] = h.to(t)
        return out
    if kind == "norm_bwd":
        t = s["x"].dtype
        rstd, dy = s["rstd"][:, None], s["dy"].float()
        n = s["x"].float() * rstd
        g = dy * s["weight"].float()
        dx = rstd * (g - n * (g * n).mean(-1, keepdim=True))
        if s["r"] is not None:
            dx = dx + s["r"].float()
        return {"dx": dx.to(t), "dweight": (dy * n).sum(0)}
    if kind == "quant":
        v = s["x"].float()
        if s["m"] is not None:
            v = v * s["m"].unsqueeze(-1 if s["axis"] == -2 else -2)
        q, scale = _quantise(v, s["axis"])
        return {"values": (q * scale).to(s["x"].dtype), "scale": scale.squeeze(s["axis"])}
    if kind == "mm":
        acc = _product(s["a"].transpose(-1, -2) if s["ta"] else s["a"], s["b"].transpose(-1, -2) if s["tb"] else s["b"])
        if s["sa"] is None:
            return acc
        return (acc.float() * s["sa"].unsqueeze(-1) * s["sb"].unsqueeze(-2)).to(TYPES[s["out"]])
    dy, w = s["dy"].float(), s["w"]
    q, t = _quantise(dy * s["sw"][None, :], -1)
    p, u = _quantise(dy * s["sa"][:, None], -2)
    da = (_product(q, w if s["tw"] else w.t()).float() * t).to(s["dy"].dtype)
    dw = _product(s["a"].t(), p).float() * u
    return {"da": da, "dw": dw.t().contiguous() if s["tw"] else dw}


# ---- the library's operators --------------------------------------------------------------------------------------------

@functools.lru_cache(maxsize=1)
def _library():
    import paper_2307_16273_amd as zk
    return zk, zk.Context(0)


def _call(s):
    zk, ctx = _library()
    kind = s["kind"]
    if kind == "norm":
        got = zk.rmsnorm_i8(ctx, s["x"], s["weight"], residual=s["r"], eps=EPS, values=True)
        return {k: got[k] for k in ("values", "scale", "rstd") + (("total",) if s["r"] is not None else ())}
    if kind == "norm_bwd":
        return zk.rmsnorm_i8_backward(ctx, s["dy"], s["x"], s["weight"], s["rstd"], dtotal=s["r"])
    if kind == "quant":
        got = zk.quantize_i8(ctx, s["x"], axis=s["axis"], mult=s["m"], values=True)
        return {k: got[k] for k in ("values", "scale")}
    if kind == "mm":
        return zk.matmul_i8(ctx, s["a"], s["b"], s["sa"], s["sb"], trans_a=s["ta"], trans_b=s["tb"], dtype=TYPES[s["out"]])
    return zk.matmul_i8_backward(ctx, s["dy"], s["a"], s["sa"], s["w"], s["sw"], trans_w=s["tw"])


def run(state):
    return _call(state) if own else _plain(state)


# ---- what a pass cannot do without --------------------------------------------------------------------------------------

def work(case):
    c, kind = case, case["kind"]
    size = {"f32": 4, "i32": 4}.get(c.get("dtype", c.get("out")), 2)
    if kind == "norm":
        n = c["M"] * c["N"]
        return {"bytes": n * (size + 1 + size + (2 * size if c["residual"] else 0)) + 8 * c["M"] + size * c["N"], "flops": 8 * n}
    if kind == "norm_bwd":
        n = c["M"] * c["N"]
        return {"bytes": n * size * (4 if c["residual"] else 3) + 4 * c["M"] + (size + 4) * c["N"], "flops": 10 * n}
    if kind == "quant":
        n = c["S"] * c["M"] * c["N"]
        rows = c["S"] * (c["N"] if c["axis"] == -2 else c["M"])
        return {"bytes": n * (2 * size + 1) + 4 * rows + (4 * n // max(1, rows) * c["S"] if c["mult"] else 0), "flops": 4 * n}
    m, k, n = c["M"], c["K"], c["N"]
    if kind == "mm":
        scales = 0 if c["out"] == "i32" else 4 * (m + n)
        return {"bytes": c["S"] * (m * k + k * n + m * n * size + scales), "flops": 2 * c["S"] * m * k * n}
    return {"bytes": m * n * size + m * k + k * n + m * k * size + 4 * k * n + 4 * (m + n), "flops": 4 * m * k * n + 8 * m * n}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    d = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor)}

    def codes(y, axis):
        """Nearest integers of 127 y / max|y| along the axis, and max|y| / 127."""
        peak = torch.linalg.vector_norm(y, ord=float("inf"), dim=axis, keepdim=True)
        safe = torch.where(peak == 0, torch.ones_like(peak), peak)
        return torch.round(y * 127.0 / safe), peak / 127.0

    if s["kind"] == "norm":
        h = d["x"] + d["r"] if "r" in d else d["x"]
        rstd = (torch.sum(h * h, 1) / h.shape[1] + EPS) ** -0.5
        y = rstd[:, None] * h * d["weight"]
        q, scale = codes(y, 1)
        out = {"values": q * scale, "scale": scale[:, 0], "rstd": rstd}
        if "r" in d:
            out["total"] = h
        return out
    if s["kind"] == "norm_bwd":
        # y_j = w_j x_j rstd,  d rstd / d x_i = - rstd^3 x_i / N
        x, r, gw = d["x"], d["rstd"][:, None], d["dy"] * d["weight"]
        dx = gw * r - x * r ** 3 * torch.sum(gw * x, 1, keepdim=True) / x.shape[1]
        return {"dx": dx + d["r"] if "r" in d else dx, "dweight": torch.sum(d["dy"] * x * r, 0)}
    if s["kind"] == "quant":
        y = d["x"]
        if "m" in d:
            y = y * (d["m"][..., :, None] if s["axis"] == -2 else d["m"][..., None, :])
        q, scale = codes(y, s["axis"])
        return {"values": q * scale, "scale": scale.squeeze(s["axis"])}
    if s["kind"] == "mm":
        a = d["a"].mT.contiguous() if s["ta"] else d["a"]
        b = d["b"].mT.contiguous() if s["tb"] else d["b"]
        y = a @ b
        return y.round().to(torch.int32) if s["out"] == "i32" else y * d["sa"][..., :, None] * d["sb"][..., None, :]
    w = d["w"].T.contiguous() if s["tw"] else d["w"]          # [K, N]
    q, t = codes(d["dy"] * d["sw"], 1)
    p, u = codes(d["sa"][:, None] * d["dy"], 0)
    dw = (d["a"].T.contiguous() @ p) * u
    return {"da": (q @ w.T.contiguous()) * t, "dw": dw.T.contiguous() if s["tw"] else dw}
