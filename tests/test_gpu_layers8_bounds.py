"""8-bit layers where one kernel or one way of the work gives way to the next: sizes on both sides of each bound, and memory that a graph keeps.

u = 2^-24 is the unit roundoff of 32-bit floats."""
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def gen(seed):
    return torch.Generator().manual_seed(seed)


def codes(g, shape):
    return torch.randint(-128, 128, shape, generator=g, dtype=torch.int32).to(torch.int8)


def codes32(v, axis):
    """The operator's quantisation in its own 32-bit steps."""
    top = v.abs().amax(axis, keepdim=True)
    inv = torch.where(top > 0, torch.full_like(top, 127.0) / top, torch.zeros_like(top))
    return torch.round(v * inv), top.double() / 127


# rows x in x out.  The gradient's preparation: 1024 | 1025 and 2048 | 2049 rows, 512, 1024, 2048, 4096 columns | one more, 8192 | 8193, and
# 5 * 2^19 entries | more (1025 x 2557 | 2558, 1279 x 2049, 1280 x 2048 | 2049); the two quantisations in one pass: the same widths to 16384 | 16385.
PREPARED = [(1025, 40, 2557), (1025, 40, 2558), (1088, 64, 2304), (1100, 33, 2300), (1152, 48, 2112), (1279, 33, 2049), (1279, 17, 2050), (1280, 33, 2048),
            (1281, 40, 2047), (1280, 16, 2049), (1024, 40, 2560), (1024, 40, 2561), (1024, 24, 2049), (1025, 24, 512), (1025, 24, 513), (1024, 24, 1024),
            (1025, 24, 1025), (2048, 24, 1025), (2048, 24, 1280), (2049, 24, 1281), (640, 24, 4096), (639, 24, 4097), (320, 24, 8192), (319, 24, 8193),
            (4096, 17, 4097), (4096, 17, 8193), (4096, 16, 16384), (4096, 16, 16385)]


@pytest.mark.parametrize("shape", PREPARED, ids=str)
@pytest.mark.parametrize("trans_w", [False, True])
def test_gradients_on_both_sides_of_each_bound(lib, ctx, shape, trans_w):
    """The largest magnitudes of half of the rows stand in the last columns: one that is not looked at changes its row's scale."""
    m, k, n = shape
    g = gen(sum(shape))
    a, w = codes(g, (m, k)), codes(g, (k, n))
    sa, sw = torch.rand(m, generator=g) + 0.1, torch.rand(n, generator=g) + 0.1
    dy = torch.randn((m, n), generator=g) * 0.1
    dy[::2, -1] = 3.0
    dy[::4, -2] = -5.0
    q, tq = codes32(dy * sw, 1)
    p, u = codes32(dy * sa[:, None], 0)
    da, dw = (q.double() @ w.double().t()) * tq, (a.double().t() @ p.double()) * u
    dev = dy.cuda(), a.cuda(), sa.cuda(), (w.t().contiguous() if trans_w else w).cuda(), sw.cuda()
    got = lib.matmul_i8_backward(ctx, *dev, trans_w=trans_w)
    gw = got["dw"].cpu().double()
    assert torch.all((got["da"].cpu().double() - da).abs() <= 6 * U * da.abs())
    assert torch.all(((gw.t() if trans_w else gw) - dw).abs() <= 6 * U * dw.abs())
    # either gradient alone is made by other kernels, of the same codes
    assert torch.equal(lib.matmul_i8_backward(ctx, *dev, trans_w=trans_w, need_dw=False)["da"], got["da"])
    assert torch.equal(lib.matmul_i8_backward(ctx, *dev, trans_w=trans_w, need_da=False)["dw"], got["dw"])


@pytest.mark.parametrize("cols", [7, 300, 16400])
def test_norm_with_a_large_eps(lib, ctx, cols):
    """eps as large as the mean square of rows whose squares, or whose mean square with eps, leave the range of 32 bits."""
    g = gen(cols)
    x = torch.randn((4, cols), generator=g)
    for size, eps in ((1e19, 3e38), (2.5e19, 1e38), (1.4e19, 2.5e38), (1e19, 1e-6), (1.0, 3e38)):
        h = x * size
        got = lib.rmsnorm_i8(ctx, h.cuda(), torch.ones(cols, device="cuda"), eps=eps)
        eps32 = float(torch.tensor(eps, dtype=torch.float32))
        rstd = (h.double().square().mean(1) + eps32) ** -0.5
        top = h.double().abs().amax(1)
        # a thread adds at most 8 ceil(16400 / 512) = 264 squares, then 12 levels; half of that error is left by the root
        err = (264 + 20) * U
        assert torch.all((got["rstd"].cpu().double() - rstd).abs() <= err * rstd), (size, eps)
        assert torch.all((got["scale"].cpu().double() - top * rstd / 127).abs() <= (err + 4 * U) * top * rstd / 127), (size, eps)


@pytest.mark.parametrize("n", [3, 17, 64])
def test_products_of_very_wide_operands(lib, ctx, n):
    """Operands of 2^23 columns and more that do not run along k and do not start at multiples of 16 bytes: a product, and both gradients.
    32-bit floats hold these sums exactly (16 products of magnitude 2^14)."""
    wide, k = 2 ** 23 + 17, 16
    g = torch.Generator(device="cuda").manual_seed(n)

    def rand(shape):
        return torch.randint(-128, 128, shape, generator=g, dtype=torch.int8, device="cuda")

    a, b = rand((k, wide)), rand((k, n))
    got = lib.matmul_i8(ctx, a, b, trans_a=True)
    for lo in range(0, wide, 1 << 21):
        part = slice(lo, lo + (1 << 21))
        assert torch.equal(got[part].float(), a[:, part].float().t().contiguous() @ b.float())
    del got
    got = lib.matmul_i8(ctx, b, a, trans_a=True)
    for lo in range(0, wide, 1 << 21):
        part = slice(lo, lo + (1 << 21))
        assert torch.equal(got[:, part].float(), b.float().t().contiguous() @ a[:, part].float())
    del got
    # gradients of x [n, wide] by w stored [k, wide]; dy of powers of two whose maxima are 127: the codes are dy itself
    x, w = rand((n, wide)), a
    dy = (torch.randint(-60, 61, (n, k), generator=g, device="cuda")).float()
    dy.fill_diagonal_(127.0)
    dy[:, 0], dy[0, :] = 127.0, 127.0
    one = torch.ones(max(n, k), device="cuda")
    got = lib.matmul_i8_backward(ctx, dy, x, one[:n], w, one[:k], trans_w=True)
    for lo in range(0, wide, 1 << 21):
        part = slice(lo, lo + (1 << 21))
        da, dw = dy @ w[:, part].float(), dy.t().contiguous() @ x[:, part].float()
        assert torch.equal(got["da"][:, part], da) and torch.equal(got["dw"][:, part], dw)


def test_a_graph_keeps_its_scratch(lib):
    """What a captured call works in is not given to tensors of the context made later, and goes on to work when the context is trimmed."""
    g = gen(6)
    side = torch.cuda.Stream()
    own = lib.Context(0, stream=side.cuda_stream)
    a, w = codes(g, (70, 500)).cuda(), codes(g, (500, 384)).cuda()
    sa, sw = torch.rand(70, generator=g).cuda(), torch.rand(384, generator=g).cuda()
    dy = torch.randn((70, 384), generator=g).cuda()

    def call():
        got = lib.matmul_i8_backward(own, dy, a, sa, w, sw)
        return got["da"], got["dw"]

    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = call()
    raws = [bytes(range(1, 9)) * (4 << k) for k in range(8, 13)]          # 32 bytes an entry
    tabs = [lib.fr_tensor_upload(own, r, (1 << k,)) for k, r in zip(range(8, 13), raws)]
    before = [t.download() for t in tabs]
    for k in range(3):
        torch.cuda.synchronize()
        dy.copy_(torch.randn((70, 384), generator=g))
        if k == 1:
            own.trim()
            junk = [torch.full((1 << 16,), 7, dtype=torch.uint8, device="cuda") for _ in range(64)]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        assert all(t.download() == b for t, b in zip(tabs, before))
        with torch.cuda.stream(side):
            eager = call()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, eager))
    assert all(torch.all(t == 7) for t in junk)
    del graph, tabs
    own.close()
