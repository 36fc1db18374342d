"""Matrices in 4-bit floats refuse operands that share memory, on the host, before anything touches a device."""
import pytest
import torch

from paper_2207_08822_amd import fxp
from tests.test_abi import load
from tests.test_serve_abi import mx4, c

BIG = 1 << 20          # addresses that are never dereferenced: every call below is refused
FAR = 1 << 30
VALUE = -10


@pytest.fixture(scope="module")
def L():
    load()
    return fxp.lib()


def shares(rows, row_bytes, stride, at, n):
    """Whether n bytes from offset `at` of a matrix on meet one of its rows."""
    return any(at < row * stride + row_bytes and row * stride < at + n for row in range(rows))


# bytes of a mapped matrix of 5 x 70: 640 of codes, 40 of scales; of 70 x 5: 8960 and 560
@pytest.mark.parametrize("which", ["data", "scales"])
@pytest.mark.parametrize("dtype,ld", [(0, 70), (0, 1000), (1, 70), (2, 700)])
def test_map_and_unmap(L, dtype, ld, which):
    size, far = 2 if dtype else 4, dict(data=FAR, scales=FAR << 1)
    n, nT = {"data": (640, 8960), "scales": (40, 560)}[which]
    seen = {False: 0, True: 0}
    for at in range(-9216, 5 * ld * size + 64, 16):                            # codes and scales are aligned
        # nothing is launched where there is a device: calls that are not refused are made elsewhere
        for meets, shape, other in ((shares(5, 70 * size, ld * size, at, n), (5, 70), (70, 5)), (shares(5, 70 * size, ld * size, at, nT), (70, 5), (5, 70))):
            if not meets and (torch.cuda.is_available() or at % 640):
                continue
            here, there = mx4(**(far | {which: BIG + at}), rows=shape[0], cols=shape[1]), mx4(data=FAR << 2, scales=FAR << 3, rows=other[0], cols=other[1])
            both = (here, there) if shape == (5, 70) else (there, here)
            alone = (here, None) if shape == (5, 70) else (None, here)
            got = [L.fxp_mx4_map(dtype, BIG, ld, 5, 70, *pair, 0, 0, 0, None) for pair in (both, alone)]
            if shape == (5, 70):
                got.append(L.fxp_mx4_unmap(here, dtype, BIG, ld, None))
            assert all((rc == VALUE) == meets for rc in got), (at, meets, got)
            seen[meets] += 1
    assert seen[True] > 40 and (torch.cuda.is_available() or seen[False] > 5)


@pytest.mark.parametrize("which", ["data", "scales"])
def test_products(L, which):
    """C, or Y, in the codes or the scales of an operand; 4 to 70 rows of 9 outputs, rows 9 and 100 elements apart."""
    far = dict(data=FAR, scales=FAR << 1)
    n = {"data": 640, "scales": 40}[which]
    for ld in (9, 100):
        for C in (BIG, BIG + n - 4, BIG - 8 * 4, BIG - 3 * ld * 4):
            free, met = mx4(**far, rows=4), mx4(**(far | {which: BIG}), rows=5)
            B = mx4(data=FAR << 2, scales=FAR << 3, rows=9)
            assert L.fxp_mx4_gemm(met, B, 0, C, ld, None, 0, None) == VALUE
            assert L.fxp_mx4_gemm(free, mx4(**(far | {which: BIG}), rows=9), 0, C, ld, None, 0, None) == VALUE
            for M in (1, 4, 5, 70):
                if M > 3 or C > BIG - 3 * ld * 4:
                    assert L.fxp_mx4_linear(0, FAR << 4, 70, M, mx4(**(far | {which: BIG}), rows=9), C, ld, FAR << 5, 1 << 20, None) == VALUE, (M, C)


def test_layers(L):
    M, K, N = 4, 70, 9
    shapes = dict(X=(M, K), XT=(K, M), W=(K, N), WT=(N, K), dY=(M, N), dYT=(N, M))

    def layer(**over):
        make = lambda i, n, s: fxp._Mx4(*(over.get(n) or (FAR << i, FAR << (6 + i))), *s)  # noqa: E731
        return c.byref(fxp._Mx4Layer(*[make(i, n, s) for i, (n, s) in enumerate(shapes.items())]))

    def fwd(X=BIG << 1, W=BIG << 2, Y=BIG << 3, l=None):
        return L.fxp_mx4_linear_fwd(0, X, W, M, K, N, Y, l, 0, 0, 0, BIG << 6, 1 << 20, None)

    def bwd(dY=BIG << 1, dX=BIG << 2, dW=BIG << 3, l=None):
        return L.fxp_mx4_linear_bwd(0, dY, l, M, K, N, dX, dW, 0, 0, 0, BIG << 6, 1 << 20, None)

    for place in ((BIG, FAR << 20), (FAR << 20, BIG)):                            # codes, then scales
        for name in ("X", "XT", "W", "WT"):
            for dense in ("X", "W", "Y"):
                assert fwd(l=layer(**{name: place}), **{dense: BIG}) == VALUE, (name, dense)
        for name in ("dY", "W", "dYT", "XT"):
            for dense in ("dY", "dX", "dW"):
                if (name, dense) not in (("W", "dY"), ("XT", "dY")):
                    assert bwd(l=layer(**{name: place}), **{dense: BIG}) == VALUE, (name, dense)
        assert bwd(l=layer(dY=place), dX=BIG, dW=None) == VALUE and bwd(l=layer(XT=place), dW=BIG, dX=None) == VALUE
    assert bwd(dX=BIG, dW=BIG, l=layer()) == VALUE and bwd(dX=BIG, dW=BIG + 4 * M * K - 4, l=layer()) == VALUE
