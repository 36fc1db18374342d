"""Products with 4-bit weights: the packing bit for bit, the products against 64-bit sums within bounds that follow from the arithmetic."""
import numpy as np
import pytest

from tests import serve_ref as ref
from tests.gpu_util import dev, host, say

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
TYPES = {"fp32": (torch.float32, 23, 2.0 ** -24), "bf16": (torch.bfloat16, 15, 2.0 ** -8), "fp16": (torch.float16, 15, 2.0 ** -11)}


@pytest.fixture(scope="module")
def fxp():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: there is no CPU path in libfxp")
    from paper_2207_08822_amd import fxp as binding
    binding.lib()
    return binding


def groups_of(a, group):
    """[K, ...] cut into [groups, group, ...], zero behind K."""
    pad = np.zeros((-(-a.shape[0] // group) * group,) + a.shape[1:])
    pad[:a.shape[0]] = a
    return pad.reshape((-1, group) + a.shape[1:])


@pytest.mark.parametrize("K,N,group", [(1, 1, 64), (64, 16, 64), (130, 33, 32), (257, 100, 128), (1000, 48, 64), (128, 300, 32)])
@pytest.mark.parametrize("kind", list(TYPES))
def test_pack4(fxp, K, N, group, kind):
    say("w4_pack", (K, N, group, kind))
    rng = np.random.default_rng(K + N)
    W = rng.standard_normal((K, N)) * 2.0 ** rng.integers(-5, 3, (1, N))
    W[:, ::3] = np.round(W[:, ::3] * 8) / 8                       # halves among them
    if N > 4:
        W[:, 4] = 0
    W = torch.tensor(W.astype(np.float32)).to(TYPES[kind][0])
    wide = torch.zeros((K, N + 3), dtype=W.dtype, device="cuda")
    wide[:, 1:N + 1] = W.cuda()
    w = fxp.pack4(wide[:, 1:N + 1], group)
    q, unit = ref.unpack4(host(w.packed), host(w.scales), K, N, group)
    parts = groups_of(W.double().numpy(), group)
    e = np.array([[ref.exponent(parts[i, :, n]) for n in range(N)] for i in range(len(parts))])
    want = np.stack([ref.to_units(parts[i], e[i], 4) for i in range(len(parts))]).reshape(-1, N)[:K]
    assert np.array_equal(unit, np.repeat(2.0 ** (e - 129.0), group, 0)[:K])
    assert np.array_equal(q, want)
    # what lies behind K and N is zero
    kt, nt = -(-K // 128), -(-N // 16)
    q, _ = ref.unpack4(host(w.packed), host(w.scales), kt * 128, nt * 16, group)
    assert not q[K:].any() and not q[:, N:].any()


def weights(fxp, rng, K, N, group):
    """Packed weights with random mantissas (zero behind K and N) and scales, and their values."""
    W = torch.tensor((rng.standard_normal((K, N)) * 2.0 ** rng.integers(-3, 4, (1, N))).astype(np.float32))
    w = fxp.pack4(W.cuda(), group)
    q, unit = ref.unpack4(host(w.packed), host(w.scales), K, N, group)
    return w, q * unit


def bound(x, W, y, group, unit_bits, half):
    """x's groups are rounded to half a unit 2^(e - 126 - unit_bits), e the exponent of the group's largest element (one more within 2^-7
    of the next binade); a group's integer sum becomes fp32 once (three times with a third digit), is scaled twice and added in: five roundings
    of 2^-24 of the group's sum of magnitudes, and one of the whole sum for each group and each of the eight partial sums joined."""
    gx, gw = groups_of(x.T, group), groups_of(W, group)               # [G, group, M], [G, group, N]
    top = np.abs(gx).max(1) * (1 + 2.0 ** -6)
    e = np.maximum(np.frexp(top)[1] + 126, 1)
    unit = 2.0 ** (e - 126.0 - unit_bits) * (top > 0)
    mass = np.abs(x) @ np.abs(W)
    inner = unit.T / 2 @ np.abs(gw).sum(1) + 2.0 ** -24 * (5 + len(gx) + 40) * mass
    return half * (np.abs(y) + inner) + inner


SIZES = [(1, 1, 1), (1, 64, 16), (2, 130, 33), (16, 128, 48), (17, 1000, 100), (1, 4096, 20), (5, 768, 2304), (64, 300, 70), (65, 257, 17),
         (130, 640, 40), (3, 20000, 5), (4, 200, 4100), (20, 129, 8190), (6, 64, 8200), (18, 300, 12288), (3, 96, 12300), (31, 200, 12300), (35, 200, 12300)]


@pytest.mark.parametrize("M,K,N", SIZES)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("kind", list(TYPES))
def test_linear4(fxp, M, K, N, group, kind):
    say("w4_linear", (M, K, N, group, kind))
    rng = np.random.default_rng(M * 3 + K + N)
    w, W = weights(fxp, rng, K, N, group)
    dtype, unit_bits, half = TYPES[kind]
    x = rng.standard_normal((M, K)) * np.exp2(rng.standard_normal((1, K)) * 2)
    x[:, :K // 3] = 0 if M == 2 else x[:, :K // 3]                    # whole groups of zeros
    x = torch.tensor(x.astype(np.float32)).to(dtype)
    y = x.double().numpy() @ W
    got = fxp.linear4(x.cuda(), w).double().cpu().numpy()
    off = bound(x.double().numpy(), W, y, group, unit_bits, half)
    assert (np.abs(got - y) <= off).all(), np.max(np.abs(got - y) / np.maximum(off, 1e-300))


@pytest.mark.parametrize("kind", list(TYPES))
def test_linear4_of_whole_numbers_is_exact(fxp, kind):
    """x in -8..8 and scales of one power of two: every product and sum fits fp32, and the result is rounded once."""
    say("w4_linear of whole numbers", kind)
    rng = np.random.default_rng(4)
    x = torch.tensor(rng.integers(-8, 9, (7, 500)).astype(np.float32)).to(TYPES[kind][0])
    W = rng.integers(-7, 8, (500, 90)).astype(np.float32)
    W[::32] = 7                                                      # every group's scale is that of 7
    w = fxp.pack4(torch.tensor(W).cuda(), 64)
    want = torch.tensor(x.double().numpy() @ W.astype(np.float64)).to(x.dtype)
    assert torch.equal(fxp.linear4(x.cuda(), w).cpu(), want)


def test_linear4_strides_and_rows(fxp):
    say("w4_linear, strided x and out, row by row")
    rng = np.random.default_rng(6)
    w, W = weights(fxp, rng, 333, 50, 64)
    wide = torch.randn((20, 400), device="cuda").to(torch.bfloat16)
    x = wide[:, 7:340]
    out = torch.full((20, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    fxp.linear4(x, w, out=out[:, 5:55])
    assert (out[:, :5] == 3).all() and (out[:, 55:] == 3).all()
    assert torch.equal(out[:, 5:55], fxp.linear4(x.contiguous(), w))
    for m in (0, 17):                                                # a row does not depend on the rows beside it
        assert torch.equal(out[m, 5:55], fxp.linear4(x[m:m + 3], w)[0])
    assert fxp.linear4(x[:0], w).shape == (0, 50)
    with pytest.raises(fxp.FxpError):
        fxp.linear4(wide[:1, :333].expand(4, 333), w)


def test_linear4_of_values_that_are_not_finite_or_tiny(fxp):
    say("w4_linear, Inf, NaN, sub-normal")
    rng = np.random.default_rng(7)
    w, W = weights(fxp, rng, 256, 32, 64)
    x = torch.randn((4, 256), device="cuda")
    want = fxp.linear4(x, w)
    bad = x.clone()
    bad[1, 70], bad[2, 3] = float("inf"), float("nan")
    got = fxp.linear4(bad, w)
    assert torch.equal(got[0], want[0]) and torch.equal(got[3], want[3]) and not torch.isnan(got).any()
    tiny = torch.full((1, 256), 1e-40, device="cuda")
    assert (fxp.linear4(tiny, w).abs() < 1e-36).all()


def test_linear4_from_a_graph(fxp):
    say("w4_linear captured")
    rng = np.random.default_rng(8)
    w, W = weights(fxp, rng, 1024, 200, 64)
    x = torch.randn((3, 1024), device="cuda").to(torch.float16)
    fxp.linear4(x, w)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = fxp.linear4(x, w)
    for i in range(4):
        x.copy_(torch.randn((3, 1024), device="cuda"))
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, fxp.linear4(x, w))


@pytest.mark.parametrize("M", [1, 2, 5, 20, 40])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("kind", ["fp32", "bf16"])
def test_linear4_of_the_largest_and_smallest_numbers(fxp, M, group, kind):
    """Results that the type holds come out whatever the sizes of x and of the weights are apart: nothing between passes the largest or the
    smallest fp32 number.  2^-149 besides the bound: a sum among sub-normal numbers may be that far off for each group and part."""
    say("w4_linear of the largest and smallest numbers", (M, group, kind))
    rng = np.random.default_rng(M + group)
    dtype, unit_bits, half = TYPES[kind]
    for x_exp, w_exp in ((124, -20), (127, -100), (90, 20), (-118, 20), (-126, 120), (-120, 0)):
        W = torch.tensor((rng.standard_normal((300, 33)) * 2.0 ** w_exp).astype(np.float32))
        w = fxp.pack4(W.cuda(), group)
        q, unit = ref.unpack4(host(w.packed), host(w.scales), 300, 33, group)
        x = torch.tensor((rng.uniform(-1, 1, (M, 300)) * 2.0 ** x_exp).astype(np.float32)).to(dtype)
        y = x.double().numpy() @ (q * unit)
        assert np.abs(y).max() < 2.0 ** 127
        got = fxp.linear4(x.cuda(), w).double().cpu().numpy()
        off = bound(x.double().numpy(), q * unit, y, group, unit_bits, half) + 2.0 ** -149 * (300 // group + 12)
        if dtype == torch.bfloat16:
            off += 2.0 ** -134                                       # half a step of its own sub-normal numbers
        assert (np.abs(got - y) <= off).all(), (x_exp, w_exp, np.max(np.abs(got - y) / off))


@pytest.mark.parametrize("M", [1, 2, 3, 40])
@pytest.mark.parametrize("kind", list(TYPES))
def test_linear4_with_inf_in_several_groups(fxp, M, kind):
    """Inf is mapped to the largest magnitude of its group, 2^129 and a little less, under a unit that leaves nothing of the others: with weights
    below 2^-3 and of either sign the sums stay finite.  One step of the type and a few of fp32: 2^-10 of the magnitudes."""
    say("w4_linear, Inf in three groups of a row", (M, kind))
    rng = np.random.default_rng(9)
    w = fxp.pack4(torch.tensor((rng.uniform(-1, 1, (256, 40)) / 8).astype(np.float32)).cuda(), 64)
    q, unit = ref.unpack4(host(w.packed), host(w.scales), 256, 40, 64)
    dtype, unit_bits, half = TYPES[kind]
    x = torch.tensor(rng.standard_normal((M, 256)).astype(np.float32)).to(dtype)
    x[0, 3], x[0, 70], x[0, 200] = float("inf"), float("inf"), float("-inf")
    most = (32639 if unit_bits == 15 else 8355711) * 2.0 ** (129 - unit_bits)
    as_mapped = np.zeros(256)
    as_mapped[[3, 70, 200]] = most, most, -most
    as_mapped[128:192] = x.double().numpy()[0, 128:192]
    got = fxp.linear4(x.cuda(), w).double().cpu().numpy()
    assert not np.isnan(got).any() and np.isfinite(got[1:]).all()
    if kind != "fp16":                                               # 2^126 is Inf in fp16
        want, mass = as_mapped @ (q * unit), np.abs(as_mapped) @ np.abs(q * unit)
        assert (np.abs(got[0] - want) <= half * np.abs(want) + 2.0 ** -20 * mass).all()


def test_linear4_refuses_an_output_that_shares_elements_with_its_input(fxp):
    say("w4_linear, out over x")
    rng = np.random.default_rng(10)
    w, _ = weights(fxp, rng, 64, 64, 64)
    room = torch.randn((41, 200), device="cuda")
    for M in (1, 2, 4, 40):
        x = room[:M, 10:74]
        for out in (x, room[:M, 73:137], room[:M, :64], room[1:M + 1, 20:84] if M > 1 else x, room.view(-1)[5:5 + 64 * M].view(M, 64)):
            before = room.clone()
            with pytest.raises(fxp.FxpError, match="shares elements"):
                fxp.linear4(x, w, out=out)
            assert torch.equal(room, before)
        want = fxp.linear4(x, w)
        assert torch.equal(fxp.linear4(x, w, out=room[:M, 74:138]), want)            # beside x in the same rows
