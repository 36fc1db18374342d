"""Products in 4-bit floats along every way they are cut: tiles of each size over many panels, several panels of a wave in flight and more than one turn of
them, parts of long contractions, and layers whose sums ride or wait.

Where an operand's rows have one scale each, every product of a row and a column is a whole number of units of a quarter of both scales, 144 at most, so sums
of fp32 are exact in any order as long as 144 K < 2^24 (K < 116508): results are compared bit for bit with 64 bits at any such length.  A dropped, repeated or
misplaced panel, block or scale changes them."""
import pytest

from tests.gpu_util import say

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
ORDER = [0, 2, 4, 6, 1, 3, 5, 7]                # blocks of a panel in the order of their scales


@pytest.fixture(scope="module")
def fxp():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: there is no CPU path in libfxp")
    from paper_2207_08822_amd import fxp as binding
    binding.lib()
    return binding


def grid():
    return torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64, device="cuda")


def power(n):
    """2^n of whole numbers from -200 to 200, exactly: the device's own function is off in the last place for some."""
    return torch.tensor([2.0 ** i for i in range(-200, 201)], dtype=torch.float64, device="cuda")[n.long() + 200]


def random_mx4(fxp, g, rows, cols, low, high):
    """A mapped matrix of random codes, a random scale from low to high - 1 a row, and its values in 64 bits."""
    panels = -(-cols // 256)
    codes = torch.randint(0, 16, (rows, panels * 256), generator=g, device="cuda", dtype=torch.uint8)
    codes[:, cols:] = 0
    scale = torch.randint(low, high, (rows,), generator=g, device="cuda", dtype=torch.uint8)
    blocks = torch.zeros((rows, panels * 8), device="cuda", dtype=torch.uint8)
    blocks[:, :-(-cols // 32)] = scale[:, None]
    pairs = codes.view(rows, panels, 128, 2).transpose(0, 1)
    data = (pairs[..., 0] | pairs[..., 1] << 4).contiguous()
    scales = blocks.view(rows, panels, 8).transpose(0, 1)[..., ORDER].contiguous()
    return fxp.Mx4.of(data, scales, rows, cols), grid()[codes[:, :cols].long()] * power(scale.long() - 127)[:, None]


def on_grid(g, rows, cols, dtype, low=-3, high=4):
    """A matrix that 4 bits hold exactly, each block of 32 along its rows with a 6 in it, and a power of two of its own for each row."""
    x = grid()[torch.randint(0, 16, (rows, cols), generator=g, device="cuda")]
    x[:, ::32] = 6.0
    if cols % 32 and cols > 32:
        x[:, -1] = -6.0
    x *= power(torch.randint(low, high, (rows, 1), generator=g, device="cuda"))
    assert torch.equal(x.to(dtype).double(), x)
    return x.to(dtype)


def rounded(x, kind):
    return x.float().to(TYPES[kind])


# M, N that go by tiles of 256 x 256 (one round of them, where 128 x 128 take two), of 128 x 128 and of 64 x 64, whole and with ends; panels: 1 to 34
LARGE = [(4096, 4096), (4095, 4090), (12608, 768), (3841, 3843)]


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("M,N,K", [(M, N, K) for M, N in LARGE for K in (290, 600, 1700)] + [(4095, 4090, 256), (4095, 4090, 8453), (3841, 3843, 1024)] +
                         [(2048, 2048, 512), (2050, 2047, 2000), (1700, 1300, 3000), (1000, 1030, 1100)])
def test_tiles(fxp, M, N, K, kind):
    say("mx4_gemm, tiles", M, N, K, kind)
    g = torch.Generator("cuda").manual_seed(M + 3 * N + 7 * K)
    (A, a), (B, b) = random_mx4(fxp, g, M, K, 122, 127), random_mx4(fxp, g, N, K, 120, 126)
    want = rounded(a @ b.T, kind)
    room = torch.full((M + 2, N + 5), 7.0, dtype=TYPES[kind], device="cuda")
    for out in (None, room[1:M + 1, 2:N + 2]):
        assert torch.equal(fxp.mx4_gemm(A, B, TYPES[kind], out=out), want)
    assert bool((room[:, :2] == 7).all() & (room[:, N + 2:] == 7).all() & (room[0] == 7).all() & (room[M + 1] == 7).all())


# rows, tiles whose contraction is split into parts, tiles of 256 x 256
@pytest.mark.parametrize("K", [5000, 9000, 12608, 40000])
@pytest.mark.parametrize("M,N", [(1, 40), (7, 100), (40, 100), (64, 33), (90, 80), (300, 200), (70, 1000), (4095, 4090)])
def test_long_contractions(fxp, M, N, K):
    say("mx4_gemm, long", M, N, K)
    g = torch.Generator("cuda").manual_seed(M * N + K)
    (A, a), (B, b) = random_mx4(fxp, g, M, K, 100, 150), random_mx4(fxp, g, N, K, 110, 140)
    want = a @ b.T
    assert torch.equal(fxp.mx4_gemm(A, B), want.float())
    assert torch.equal(fxp.mx4_gemm(A, B, torch.bfloat16), rounded(want, "bf16"))


# K: panels of a wave in flight (4 for one row, 3 for two to four, 2 up to 32, eight waves; one of four waves beyond), one turn of them and several; ends of panels
@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("M", [1, 2, 3, 4, 5, 9, 16, 20, 32, 40, 48, 50, 64])
@pytest.mark.parametrize("K", [256, 1000, 1500, 2500, 4096, 4100, 5000, 6145, 8192, 8500, 17000])
def test_few_rows(fxp, M, K, kind):
    say("mx4_linear, few rows", M, K, kind)
    g = torch.Generator("cuda").manual_seed(1000 * M + K)
    N = 77
    x = on_grid(g, M, K, TYPES[kind])
    w, b = random_mx4(fxp, g, N, K, 118, 124)
    want = rounded(x.double() @ b.T, kind)
    assert bool(want.isfinite().all())
    wide = torch.zeros((M, K + 9), dtype=x.dtype, device="cuda")                     # off the vector's addresses
    wide[:, 1:K + 1] = x
    room = torch.full((M, N + 3), 7.0, dtype=x.dtype, device="cuda")
    assert torch.equal(fxp.mx4_linear(x, w), want)
    assert torch.equal(fxp.mx4_linear(wide[:, 1:K + 1], w, out=room[:, 1:N + 1]), want) and bool((room[:, 0] == 7).all() & (room[:, N + 1:] == 7).all())
    if M > 4:
        assert torch.equal(fxp.mx4_gemm(fxp.mx4_map(x, rounding=fxp.NEAREST)[0], w, TYPES[kind]), want)


def layer(fxp, M, K, N, kind):
    """A layer's step against 64 bits: Y, dX and dW from the operands as they were mapped."""
    say("mx4 layer", M, K, N, kind)
    g = torch.Generator("cuda").manual_seed(M + K + N)
    X, W, dY = (torch.randn(s, generator=g, device="cuda").to(TYPES[kind]) for s in ((M, K), (K, N), (M, N)))
    buf = fxp.Mx4LayerBuffers(M, K, N, TYPES[kind])
    how = dict(seed=3, step=5)
    Y = fxp.mx4_linear_fwd(X, W, buf, **how)
    dX, dW = fxp.mx4_linear_bwd(dY, buf, **how)
    value = lambda q: fxp.mx4_unmap(q).double()  # noqa: E731
    half = torch.finfo(TYPES[kind]).eps / 2
    for got, a, b in ((Y, buf.X, buf.WT), (dX, buf.dY, buf.W), (dW, buf.XT, buf.dYT)):
        a, b = value(a), value(b).T.contiguous()
        # a sum of n products: n - 1 additions of at most 2^-23 (cut) of the sum of the magnitudes
        want, bound = a @ b, a.abs() @ b.abs() * (a.shape[1] * 2.0 ** -23)
        assert bool(((got.double() - want).abs() <= bound + want.abs() * half * 1.01 + 2.0 ** -25).all())
    first = [t.clone() for t in (Y, dX, dW)]
    # bit for bit the products of the mapped operands alone, and one gradient at a time
    for got, a, b in zip(first, (buf.X, buf.dY, buf.XT), (buf.WT, buf.W, buf.dYT)):
        assert torch.equal(fxp.mx4_gemm(a, b, TYPES[kind]), got)
    for t in (buf.dx, buf.dw):
        t.fill_(7)
    assert torch.equal(fxp.mx4_linear_bwd(dY, buf, need_dW=False, **how)[0], first[1]) and bool((buf.dw == 7).all())
    buf.dx.fill_(7)
    assert torch.equal(fxp.mx4_linear_bwd(dY, buf, need_dX=False, **how)[1], first[2]) and bool((buf.dx == 7).all())


@pytest.mark.parametrize("kind", list(TYPES))
def test_sum_beside_large_tiles(fxp, kind):
    """The weight gradient is split over its rows and added up in the input gradient's launch, of 256 x 256 tiles with three panels."""
    assert fxp.lib().fxp_mx4_gemm_workspace_bytes(768, 768, 12608) > 0 and fxp.lib().fxp_mx4_gemm_workspace_bytes(12608, 768, 768) == 0
    layer(fxp, 12608, 768, 768, kind)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("M,K,N", [(2100, 128, 2100), (2500, 70, 3001)])
def test_both_gradients_are_split(fxp, M, K, N, kind):
    """Both want the workspace: one after the other."""
    assert fxp.lib().fxp_mx4_gemm_workspace_bytes(K, N, M) > 0 and fxp.lib().fxp_mx4_gemm_workspace_bytes(M, K, N) > 0
    layer(fxp, M, K, N, kind)


@pytest.mark.parametrize("M,K,N", [(2048, 2048, 100), (2050, 2047, 130), (3000, 900, 700), (2049, 70, 64)])
def test_sum_beside_smaller_tiles(fxp, M, K, N):
    """The same beside tiles of 128 x 128 and of 64 x 64."""
    assert fxp.lib().fxp_mx4_gemm_workspace_bytes(K, N, M) > 0 and fxp.lib().fxp_mx4_gemm_workspace_bytes(M, K, N) == 0
    layer(fxp, M, K, N, "fp32")
