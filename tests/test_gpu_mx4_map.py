"""Mapping to microscaled 4-bit numbers and back, bit for bit against the definition: sizes, types, both copies, both roundings, values at the edges."""
import numpy as np
import pytest

from tests import mx4_ref as ref
from tests.gpu_util import host, say

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


def check(q, x, word=None):
    """The layout's codes (a zero's sign apart) and scales, and zeros up to the panel's end."""
    codes, scales = ref.unpack(host(q.data), host(q.scales), q.cols)
    want_codes, want_scales = ref.encode(x, word)
    blocks = want_scales.shape[1]
    assert np.array_equal(scales[:, :blocks], want_scales)
    good = np.repeat(want_scales, 32, 1)[:, :q.cols] != 255            # codes under the scale that is none mean nothing
    assert np.array_equal(np.where(good, codes[:, :q.cols], 0), np.where(good, want_codes, 0))
    tail = codes[:, q.cols:blocks * 32]
    assert not tail[np.repeat(want_scales[:, -1:] != 255, tail.shape[1], 1)].any() and not codes[:, blocks * 32:].any() and not scales[:, blocks:].any()
    return ref.values(want_codes, want_scales)


def matrix(rows, cols, kind, seed=0):
    """Sizes over many binades, values on the grid and half way between its points among them."""
    rng = np.random.default_rng(rows * 7919 + cols + seed)
    x = rng.standard_normal((rows, cols)) * 2.0 ** rng.integers(-4, 5, (rows, 1)) * 2.0 ** rng.integers(-4, 5, (1, cols))
    x[:, ::5] = rng.choice([0, 0.25, 0.5, 0.75, 1.25, 1.5, 1.75, 2.5, 3, 3.5, 5, 6, -0.25, -2.5, -5], x[:, ::5].shape)
    x[rng.random(x.shape) < 0.05] = 0
    return torch.tensor(x.astype(np.float32)).to(TYPES[kind])


SIZES = [(1, 1), (1, 32), (3, 31), (5, 33), (32, 32), (1, 256), (2, 257), (64, 64), (65, 300), (129, 130), (256, 96), (300, 517), (33, 1000), (700, 1)]


CASES = [(r, c, kind, stochastic) for r, c in SIZES for kind in TYPES for stochastic in (False, True)]
CASES += [(r, c, kind, kind != "fp16") for r, c in ((2112, 2052), (2049, 2050)) for kind in TYPES]           # of large tiles


@pytest.mark.parametrize("rows,cols,kind,stochastic", CASES)
def test_map(fxp, rows, cols, kind, stochastic):
    say("mx4_map", rows, cols, kind, stochastic)
    x = matrix(rows, cols, kind)
    seed, stream = (3 << 40) + 11, (1 << 50) + 5
    how = dict(seed=seed, stream_id=stream, rounding=fxp.STOCHASTIC if stochastic else fxp.NEAREST)
    word = ref.words(rows, cols, seed, stream) if stochastic else None
    a = x.double().numpy()
    q, qT = fxp.mx4_map(x.cuda(), want_qT=True, **how)
    v = check(q, a, word)
    vT = check(qT, a.T, word.T if stochastic else None)
    for t, want in ((q, v), (qT, vT)):
        for dtype in TYPES.values():
            assert torch.equal(fxp.mx4_unmap(t, dtype).cpu(), torch.tensor(want).float().to(dtype))
    # one copy at a time, of rows with room between them, not on the grid of vector loads
    wide = torch.full((rows, cols + 3), float("nan"), dtype=x.dtype, device="cuda")
    wide[:, 1:cols + 1] = x.cuda()
    for want_q, whole in ((True, q), (False, qT)):
        one = fxp.mx4_map(wide[:, 1:cols + 1], want_q=want_q, want_qT=not want_q, **how)
        assert one[want_q] is None
        one = one[not want_q]
        assert torch.equal(one.data, whole.data) and torch.equal(one.scales, whole.scales)


@pytest.mark.parametrize("stochastic", [False, True])
def test_edges(fxp, stochastic):
    """The largest and the smallest numbers, halves with a last bit more or less, Inf and NaN: one block a row."""
    big, tiny = np.float32(3.4028235e38), np.float32(1e-45)
    rows = [[0, -0.0, 0], [big, -big, 1.0], [tiny, 0, -tiny], [2.0 ** -126, 2.0 ** -127, tiny * 7], [6 * 2.0 ** -127, 0.25 * 2.0 ** -127, 0.75 * 2.0 ** -127],
            [np.float32(1.5) * 2.0 ** -124, 2.0 ** -126, 0], [np.inf, 1, 2], [1, np.nan, 2], [-np.inf, 0, 0], [6, 0.25, np.nextafter(np.float32(0.25), np.float32(1))],
            [6, np.nextafter(np.float32(0.25), np.float32(0)), 5], [np.nextafter(np.float32(6), np.float32(9)), 5, 0.5], [6, np.float32(0.25) + 2.0 ** -26, 2.0 ** -24],
            [3, 1e-30, -1e-38], [1.5, 1.25, -0.375]]
    x = np.zeros((len(rows), 32), np.float32)
    for i, r in enumerate(rows):
        x[i, 7:10] = r
    with np.errstate(all="ignore"):
        word = ref.words(*x.shape, 9, 2) if stochastic else None
        q, qT = fxp.mx4_map(torch.tensor(x).cuda(), seed=9, stream_id=2, rounding=fxp.STOCHASTIC if stochastic else fxp.NEAREST, want_qT=True)
        want = check(q, x.astype(np.float64), word)
        check(qT, x.T.astype(np.float64), word.T if stochastic else None)
    got = fxp.mx4_unmap(q).cpu().numpy()
    with np.errstate(over="ignore"):
        assert np.array_equal(got, want.astype(np.float32), equal_nan=True) and np.isnan(got[6:9]).all()


def test_stochastic_rounding_is_unbiased(fxp):
    """Mean of 2^20 roundings of one value: each is a coin of two neighbours, so the mean is within 6 of its deviations of the value (odds below 1e-8)."""
    n = 1 << 20
    for v in (0.1, 0.6, 1.3, 2.25, 3.9, 5.0, -4.5):
        x = torch.full((n // 32, 32), v, device="cuda")
        x[:, 0] = 6.0                                       # the scale
        y = fxp.mx4_unmap(fxp.mx4_map(x, seed=4)[0])[:, 1:].double()
        below = max(g for g in ref.GRID if g <= abs(v))
        gap = min(g for g in ref.GRID if g > abs(v)) - below
        p = (abs(v) - below) / gap
        assert abs(y.mean().item() - v) < 6 * gap * (p * (1 - p) / y.numel()) ** 0.5


def test_out_and_refusals(fxp):
    x = torch.randn((40, 70), device="cuda")
    q, qT = fxp.Mx4(40, 70), fxp.Mx4(70, 40)
    a, b = fxp.mx4_map(x, rounding=fxp.NEAREST, out=(q, qT))
    assert a is q and b is qT
    c, d = fxp.mx4_map(x, rounding=fxp.NEAREST, want_qT=True)
    assert torch.equal(c.data, q.data) and torch.equal(d.data, qT.data) and torch.equal(c.scales, q.scales) and torch.equal(d.scales, qT.scales)
    room = torch.full((40, 80), 7.0, device="cuda")
    y = fxp.mx4_unmap(q, out=room[:, 3:73])
    assert torch.equal(y, fxp.mx4_unmap(q)) and bool((room[:, :3] == 7).all()) and bool((room[:, 73:] == 7).all())
    for rows, cols in ((0, 5), (5, 0), (0, 0)):
        e, f = fxp.mx4_map(torch.zeros((rows, cols), device="cuda"), want_qT=True)
        assert fxp.mx4_unmap(e).shape == (rows, cols) and fxp.mx4_unmap(f).shape == (cols, rows)
    bad = [lambda: fxp.mx4_map(x, out=(qT, None)), lambda: fxp.mx4_map(x, want_q=False), lambda: fxp.mx4_map(x.double()), lambda: fxp.mx4_map(x.t()),
           lambda: fxp.mx4_map(x.cpu()), lambda: fxp.mx4_map(x, rounding=2), lambda: fxp.mx4_map(x[:1].expand(4, 70)), lambda: fxp.mx4_unmap(q, torch.float64),
           lambda: fxp.mx4_unmap(q, out=room[:, :69]), lambda: fxp.Mx4.of(q.data, q.scales, 41, 70), lambda: fxp.Mx4.of(q.data, qT.scales, 40, 70),
           lambda: fxp.Mx4(1 << 24, 4), lambda: fxp.Mx4(-1, 4), lambda: fxp.Mx4(4, 4, device="cpu")]
    for i, f in enumerate(bad):
        with pytest.raises(fxp.FxpError):
            f()
            pytest.fail(str(i))


def test_two_copies_in_one_place_are_refused(fxp):
    x = torch.randn((64, 64), device="cuda")
    q = fxp.Mx4(64, 64)
    for other in (q, fxp.Mx4.of(q.data, torch.zeros_like(q.scales), 64, 64), fxp.Mx4.of(torch.zeros_like(q.data), q.scales, 64, 64)):
        with pytest.raises(fxp.FxpError):
            fxp.mx4_map(x, out=(q, other))
