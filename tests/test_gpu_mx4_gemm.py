"""Products and layers in microscaled 4-bit floats against 64 bits.

Where the scales of an operand span four binades, every product and partial sum is a whole number of units of 2^-8 (0.25 under the smallest scales, 2^-3 each)
below 2^24 of them, so sums of fp32 are exact in any order: results are compared bit for bit.  Elsewhere a sum of K products is off by at most K steps
of 2^-23 (a cut addition) of the sum of their magnitudes, and the result by its type's rounding."""
import numpy as np
import pytest

from tests import mx4_ref as ref
from tests.gpu_util import dev, host, say

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


@pytest.fixture(scope="module")
def fxp():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: there is no CPU path in libfxp")
    from paper_2207_08822_amd import fxp as binding
    binding.lib()
    return binding


def random_mx4(fxp, rng, rows, cols, low=124, high=128):
    """A mapped matrix of random codes and scales, and its values."""
    codes, scales = rng.integers(0, 16, (rows, cols)), rng.integers(low, high, (rows, -(-cols // 32)))
    return pack(fxp, codes, scales), ref.values(codes, scales)


def pack(fxp, codes, scales):
    rows, cols = codes.shape
    panels = -(-cols // 256)
    c, s = np.zeros((rows, panels * 256), np.uint8), np.zeros((rows, panels * 8), np.uint8)
    c[:, :cols], s[:, :scales.shape[1]] = codes, scales
    c = c.reshape(rows, panels, 128, 2).transpose(1, 0, 2, 3)
    s = s.reshape(rows, panels, 8).transpose(1, 0, 2)[:, :, ref.ORDER]
    return fxp.Mx4.of(dev((c[..., 0] | c[..., 1] << 4).astype(np.uint8)), dev(s.astype(np.uint8)), rows, cols)


# M, N, K: few rows, tiles, ends of tiles and panels, parts of the contraction, and lengths whose sums stay below 2^24 units of 2^-8: 36 * 2^8 K < 2^24
SIZES = [(1, 1, 1), (1, 16, 32), (1, 700, 256), (2, 33, 257), (7, 100, 1800), (16, 2000, 64), (17, 50, 500), (33, 129, 1300), (48, 65, 900), (64, 64, 1024), (65, 64, 96),
         (65, 1, 300), (128, 128, 128), (129, 257, 700), (200, 300, 1820), (1000, 70, 33), (70, 1000, 290), (300, 300, 1800), (1100, 2300, 300), (2100, 2050, 600)]


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("M,N,K", SIZES)
def test_exact_sums(fxp, M, N, K, kind):
    say("mx4_gemm", M, N, K, kind)
    rng = np.random.default_rng(M + 7 * N + 31 * K)
    A, a = random_mx4(fxp, rng, M, K)
    B, b = random_mx4(fxp, rng, N, K)
    want = torch.tensor(a @ b.T).float().to(TYPES[kind])
    room = torch.full((M, N + 5), 7.0, dtype=TYPES[kind], device="cuda")
    for out in (None, room[:, 2:N + 2]):
        got = fxp.mx4_gemm(A, B, TYPES[kind], out=out)
        assert torch.equal(got.cpu(), want)
    assert bool((room[:, :2] == 7).all()) and bool((room[:, N + 2:] == 7).all())


@pytest.mark.parametrize("M,N,K", [(1, 40, 9000), (3, 600, 12000), (40, 100, 5000), (90, 80, 11000), (300, 200, 4096), (600, 500, 700)])
def test_scales_of_all_sizes(fxp, M, N, K):
    say("mx4_gemm, wide scales", M, N, K)
    rng = np.random.default_rng(K)
    A, a = random_mx4(fxp, rng, M, K, 100, 140)
    B, b = random_mx4(fxp, rng, N, K, 110, 150)
    got = host(fxp.mx4_gemm(A, B).double())
    assert np.all(np.abs(got - a @ b.T) <= np.abs(a) @ np.abs(b).T * (K * 2.0 ** -23) + 2.0 ** -149)


def test_the_ends_of_the_scales(fxp):
    """The smallest scale (a sub-normal factor), the largest, and the one that makes its block NaN, in each block of a panel."""
    for M in (16, 80):
        for block in range(8):
            codes = np.zeros((M, 256), int)
            codes[:, 32 * block:32 * block + 32] = 2                                   # ones
            a, b = np.full((M, 8), 127), np.full((M, 8), 127)
            a[0, block], a[1, block], a[2, block], a[3, block], b[5, block] = 0, 1, 254, 255, 255
            b[6, block], b[7, block] = 253, 20
            got = host(fxp.mx4_gemm(pack(fxp, codes, a), pack(fxp, codes, b)))
            with np.errstate(over="ignore"):
                want = (32 * 2.0 ** (a[:, block] - 127.0)[:, None] * 2.0 ** (b[:, block] - 127.0)).astype(np.float32)
            want[3], want[:, 5] = np.nan, np.nan
            # a product under the smallest normal number may be flushed
            assert np.array_equal(np.where(want < 2.0 ** -126, 0, want), np.where(got < 2.0 ** -126, 0, got), equal_nan=True), (M, block)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("M,K,N", [(1, 100, 64), (1, 3000, 77), (2, 255, 40), (3, 2500, 33), (4, 1030, 50), (5, 256, 300), (31, 1000, 77), (130, 520, 260), (700, 64, 300)])
def test_linear(fxp, M, K, N, kind):
    say("mx4_linear", M, K, N, kind)
    rng = np.random.default_rng(M * K + N)
    x = torch.tensor(rng.standard_normal((M, K)).astype(np.float32) * 2.0 ** rng.integers(-2, 3, (1, K)).astype(np.float32)).to(TYPES[kind])
    W = torch.randn((K, N), device="cuda") * 0.1
    w = fxp.mx4_map(W, rounding=fxp.NEAREST, want_q=False, want_qT=True)[1]
    a, b = ref.values(*ref.encode(x.double().numpy())), ref.values(*ref.encode(W.double().cpu().numpy().T))
    want, size = a @ b.T, np.abs(a) @ np.abs(b).T
    wide = torch.zeros((M, K + 9), dtype=x.dtype, device="cuda")
    wide[:, 4:K + 4] = x.cuda()
    room = torch.full((M, N + 3), 7.0, dtype=x.dtype, device="cuda")
    first = fxp.mx4_linear(x.cuda(), w)
    second = fxp.mx4_linear(wide[:, 4:K + 4], w, out=room[:, 1:N + 1])
    assert first.dtype == x.dtype and torch.equal(first, second) and bool((room[:, 0] == 7).all()) and bool((room[:, N + 1:] == 7).all())
    got = host(first.double())
    assert np.all(np.abs(got - want) <= size * (K * 2.0 ** -23) + np.abs(want) * torch.finfo(x.dtype).eps / 2 * 1.01 + 2.0 ** -25)


@pytest.mark.parametrize("stochastic", [False, True])
@pytest.mark.parametrize("M,K,N,kind", [(1, 1, 1, "fp32"), (40, 70, 33, "fp32"), (197, 96, 130, "bf16"), (300, 260, 64, "fp16"), (2000, 64, 96, "fp32"), (520, 515, 258, "fp32")])
def test_layer(fxp, M, K, N, kind, stochastic):
    say("mx4 layer", M, K, N, kind, stochastic)
    rng = np.random.default_rng(M + K + N)
    make = lambda shape, size: torch.tensor((rng.standard_normal(shape) * size).astype(np.float32)).to(TYPES[kind])  # noqa: E731
    X, W, dY = make((M, K), 1.0), make((K, N), 0.25), make((M, N), 0.5)
    buf = fxp.Mx4LayerBuffers(M, K, N, TYPES[kind])
    how = dict(seed=77, step=3, rounding=fxp.STOCHASTIC if stochastic else fxp.NEAREST)
    Y = fxp.mx4_linear_fwd(X.cuda(), W.cuda(), buf, **how)
    dX, dW = fxp.mx4_linear_bwd(dY.cuda(), buf, **how)
    four = {}
    for tag, (name, t) in enumerate((("X", X), ("W", W), ("dY", dY))):
        t = t.double().numpy()
        word = ref.words(*t.shape, 77, (3 << 8) | tag) if stochastic else None
        four[name] = ref.values(*ref.encode(t, word))
        four[name + "T"] = ref.values(*ref.encode(t.T, word.T if stochastic else None)).T
    eps = torch.finfo(TYPES[kind]).eps
    for got, a, b in ((Y, four["X"], four["WT"]), (dX, four["dY"], four["W"].T), (dW, four["XT"].T, four["dYT"])):
        want, size, n = a @ b, np.abs(a) @ np.abs(b), a.shape[1]
        assert np.all(np.abs(host(got.double()) - want) <= size * (n * 2.0 ** -23) + np.abs(want) * eps / 2 * 1.01 + 2.0 ** -25)
    # one gradient at a time
    one, other = fxp.Mx4LayerBuffers(M, K, N, TYPES[kind]), fxp.Mx4LayerBuffers(M, K, N, TYPES[kind])
    fxp.mx4_linear_fwd(X.cuda(), W.cuda(), one, **how)
    fxp.mx4_linear_fwd(X.cuda(), W.cuda(), other, **how)
    a, none = fxp.mx4_linear_bwd(dY.cuda(), one, need_dW=False, **how)
    none2, b = fxp.mx4_linear_bwd(dY.cuda(), other, need_dX=False, **how)
    assert none is None and none2 is None and torch.equal(a, dX) and torch.equal(b, dW)


def test_layer_against_differences(fxp):
    """Operands that 4 bits hold along both axes (every block has a 6): the layer is linear then, and a step of one element from 6 to 4 moves the sum of Y * dY by
    the gradient times it, exactly."""
    rng = np.random.default_rng(8)
    M, K, N = 96, 64, 96
    X, W, dY = (torch.tensor(rng.choice([0.0, 0.5, -1.0, 1.5, -2.0, 3.0, 4.0, 6.0, -6.0], s), dtype=torch.float32, device="cuda") for s in ((M, K), (K, N), (M, N)))
    for t in (X, W, dY):
        i = torch.arange(max(t.shape), device="cuda")
        t[i[:t.shape[0]], i[:t.shape[0]] % t.shape[1]] = 6.0
        t[i[:t.shape[1]] % t.shape[0], i[:t.shape[1]]] = 6.0
        t[(i[:t.shape[0]]), (i[:t.shape[0]] + 32) % t.shape[1]] = -6.0
        t[(i[:t.shape[0]]), (i[:t.shape[0]] + 64) % t.shape[1]] = 6.0
    buf = fxp.Mx4LayerBuffers(M, K, N)
    total = lambda a, b: (fxp.mx4_linear_fwd(a, b, buf).double() * dY.double()).sum().item()  # noqa: E731
    base = total(X, W)
    dX, dW = (g.double().clone() for g in fxp.mx4_linear_bwd(dY, buf))
    for t, grad, which in ((X, dX, 0), (W, dW, 1)):
        for r, c in ((0, 5), (33, 63), (50, 20)):
            if abs(t[r, c].item()) == 6:
                c = (c + 1) % t.shape[1]
            moved = t.clone()
            moved[r, c] = 4.0 if t[r, c].item() != 4.0 else 3.0
            d = total(*((moved, W) if which == 0 else (X, moved))) - base
            assert d == grad[r, c].item() * (moved[r, c] - t[r, c]).item()


def test_empty(fxp):
    e = lambda r, c: fxp.mx4_map(torch.zeros((r, c), device="cuda"))[0]  # noqa: E731
    assert fxp.mx4_gemm(e(0, 40), e(5, 40)).shape == (0, 5) and fxp.mx4_gemm(e(5, 40), e(0, 40)).shape == (5, 0)
    for M in (3, 100):
        out = torch.full((M, 7), 7.0, device="cuda")
        assert not fxp.mx4_gemm(e(M, 0), e(7, 0), out=out).any()                     # sums of nothing
        out.fill_(7)
        assert not fxp.mx4_linear(torch.zeros((M, 0), device="cuda"), e(7, 0), out=out).any()
    buf = fxp.Mx4LayerBuffers(0, 20, 30)
    buf.dw.fill_(7)
    assert fxp.mx4_linear_fwd(torch.zeros((0, 20), device="cuda"), torch.zeros((20, 30), device="cuda"), buf).shape == (0, 30)
    dX, dW = fxp.mx4_linear_bwd(torch.zeros((0, 30), device="cuda"), buf)
    assert dX.shape == (0, 20) and not dW.any()


def test_refused(fxp):
    x = torch.randn((40, 64), device="cuda")
    q, r = fxp.mx4_map(x)[0], fxp.mx4_map(x[:30, :32])[0]
    buf = fxp.Mx4LayerBuffers(40, 64, 30)
    W = torch.randn((64, 30), device="cuda")
    room = torch.empty((40, 104), device="cuda")
    bad = [lambda: fxp.mx4_gemm(q, r), lambda: fxp.mx4_gemm(q, q, torch.float64), lambda: fxp.mx4_gemm(q, q, out=room[:, :39]), lambda: fxp.mx4_gemm(q, q, out=room[:1, :40].expand(40, 40)),
           lambda: fxp.mx4_linear(x[:, :63], q), lambda: fxp.mx4_linear(x, q, out=x.half()), lambda: fxp.mx4_linear(room[:, :64], q, out=room[:, 50:90]),
           lambda: fxp.mx4_linear(x, q, ws=torch.empty(8, dtype=torch.uint8, device="cuda")), lambda: fxp.mx4_linear(x.double(), q), lambda: fxp.mx4_linear_fwd(x.half(), W, buf),
           lambda: fxp.mx4_linear_fwd(x[:, :32], W, buf), lambda: fxp.mx4_linear_fwd(x, W, buf, rounding=5), lambda: fxp.mx4_linear_bwd(x, buf), lambda: fxp.mx4_linear_fwd(x, W.cpu(), buf),
           lambda: fxp.Mx4LayerBuffers(4, 4, 4, torch.float64)]
    for i, f in enumerate(bad):
        with pytest.raises(fxp.FxpError):
            f()
            pytest.fail(str(i))
    assert fxp.mx4_linear(room[:, :64].copy_(x), q, out=room[:, 64:]).shape == (40, 40)          # beside x in one buffer


def test_replayed(fxp):
    """A step and a single token's product from a graph, each replay against the eager call."""
    M, K, N = 90, 2100, 70
    buf, eager = fxp.Mx4LayerBuffers(M, K, N), fxp.Mx4LayerBuffers(M, K, N)
    X, W, dY, x = torch.zeros((M, K), device="cuda"), torch.zeros((K, N), device="cuda"), torch.zeros((M, N), device="cuda"), torch.zeros((1, K), device="cuda", dtype=torch.bfloat16)
    w = fxp.mx4_map(torch.randn((N, K), device="cuda"))[0]
    y = torch.empty((1, N), device="cuda", dtype=torch.bfloat16)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")

    def step(b, y):
        fxp.mx4_linear_fwd(X, W, b, seed=5)
        fxp.mx4_linear_bwd(dY, b, seed=5)
        return fxp.mx4_linear(x, w, out=y, ws=ws)

    step(eager, y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(buf, y)
    for i in range(4):
        for t in (X, W, dY, x):
            t.copy_(torch.randn(t.shape, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        want = step(eager, torch.empty_like(y))
        assert torch.equal(y, want) and torch.equal(buf.y, eager.y) and torch.equal(buf.dx, eager.dx) and torch.equal(buf.dw, eager.dw) and buf.dw.any()


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("M", [1, 3, 4, 9, 80])
def test_rows_that_are_not_finite(fxp, M, kind):
    """Inf or NaN in a row of x makes that row of y NaN and leaves the others; in a row of the weights, that column."""
    say("mx4_linear, not finite", M, kind)
    K, N = 700, 90
    x, W = torch.randn((M, K), device="cuda").to(TYPES[kind]), torch.randn((N, K), device="cuda")
    w = fxp.mx4_map(W, rounding=fxp.NEAREST)[0]
    want = fxp.mx4_linear(x, w)
    assert bool(want.isfinite().all())
    x[0, 699] = float("nan")
    x[M // 2, 3] = float("-inf")
    W[17, 300] = float("inf")
    got = fxp.mx4_linear(x, fxp.mx4_map(W, rounding=fxp.NEAREST)[0])
    want[0], want[M // 2], want[:, 17] = float("nan"), float("nan"), float("nan")
    assert torch.equal(got.nan_to_num(1e4), want.nan_to_num(1e4)) and torch.equal(got.isnan(), want.isnan())


def test_large_tiles_with_the_sum_of_a_split_product(fxp):
    """A layer whose weight gradient is split over its rows and added up beside the input gradient's tiles."""
    M, K, N = 12608, 768, 128
    say("mx4 layer", M, K, N)
    X, W, dY = (torch.randn(s, device="cuda", dtype=torch.bfloat16) for s in ((M, K), (K, N), (M, N)))
    buf = fxp.Mx4LayerBuffers(M, K, N, torch.bfloat16)
    Y = fxp.mx4_linear_fwd(X, W, buf)
    dX, dW = fxp.mx4_linear_bwd(dY, buf)
    value = lambda q: fxp.mx4_unmap(q).double()  # noqa: E731
    for got, a, b in ((Y, buf.X, buf.WT), (dX, buf.dY, buf.W), (dW, buf.XT, buf.dYT)):
        a, b = value(a), value(b).T.contiguous()
        want, bound = a @ b, a.abs() @ b.abs() * (a.shape[1] * 2.0 ** -23)
        assert bool(((got.double() - want).abs() <= bound + want.abs() * 2.0 ** -8 * 1.01 + 2.0 ** -25).all())
    first = dX.clone(), dW.clone()
    fxp.mx4_linear_bwd(dY, buf, need_dX=False)
    assert torch.equal(buf.dw, first[1])
    fxp.mx4_linear_bwd(buf.y.copy_(dY), buf)                                             # a gradient written over the output
    assert torch.equal(buf.dx, first[0]) and torch.equal(buf.dw, first[1])


def test_elements_past_32_bits(fxp):
    """A matrix, and a product, of more than 2^31 elements: their last rows and columns are those of a small one."""
    rows, cols = 70016, 32800
    say("mx4 past 32 bits", rows, cols)
    x = torch.randn((rows, cols), device="cuda", dtype=torch.bfloat16)
    q, qT = fxp.mx4_map(x, rounding=fxp.NEAREST, want_qT=True)
    alone = fxp.mx4_map(x, rounding=fxp.NEAREST)[0]
    assert torch.equal(alone.data, q.data) and torch.equal(alone.scales, q.scales)
    part, partT = fxp.mx4_map(x[-64:], rounding=fxp.NEAREST)[0], fxp.mx4_map(x[:, -64:], rounding=fxp.NEAREST, want_q=False, want_qT=True)[1]
    for whole, end in ((q, part), (qT, partT)):
        assert torch.equal(whole.data[:, -64:], end.data) and torch.equal(whole.scales[:, -64:], end.scales)
    x.zero_()
    assert torch.equal(fxp.mx4_unmap(q, out=x)[-64:], fxp.mx4_unmap(part, torch.bfloat16))
    del q, qT, alone
    rng = np.random.default_rng(6)
    (A, _), (B, b) = random_mx4(fxp, rng, rows, 64), random_mx4(fxp, rng, cols, 64)
    a = fxp.mx4_unmap(A)[-64:].double().cpu().numpy()
    got = fxp.mx4_gemm(A, B, out=x)[-64:]
    assert torch.equal(got.cpu(), torch.tensor(a @ b.T).float().bfloat16())              # exact sums, rounded once
