"""Rows without a token in outputs that the rotation makes itself: zeros, so that a product over all rows, as follows a gradient, is that of the rows with one."""
import pytest

from tests import rotary_ref as ref
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


def leave_nan(shape, dtype):
    """Memory of a new tensor of this size holds NaN, most likely: the allocator hands a block that was freed to the next of its size."""
    torch.full(shape, float("nan"), dtype=dtype, device="cuda")


# whole heads and parts of them, elements that are not rotated, sizes off the vector's; heads inside and outside
@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("near", [False, True])
@pytest.mark.parametrize("heads, dim, rot", [(2, 64, 64), (3, 80, 32), (1, 13, 6), (5, 97, 96)])
def test_rows_without_a_token(fxp, kind, near, heads, dim, rot):
    say("rotary, rows without a token", kind, near, heads, dim, rot)
    rope = fxp.Rotary(rot, interleaved=near)
    positions = torch.tensor([[0, 3, -1, 7, -5], [-1, -1, 2, -2147483648, 9]], dtype=torch.int32, device="cuda")
    there = host(positions) >= 0
    for outside in (False, True):
        x = torch.randn((2, heads, 5, dim) if outside else (2, 5, heads, dim), device="cuda").to(TYPES[kind])
        x = x.transpose(1, 2) if outside else x
        for backward, f in ((False, fxp.rotary), (True, fxp.rotary_bwd)):
            leave_nan(x.shape, x.dtype)
            y = f(x, positions, rope)
            assert not y[positions < 0].any() and bool(y.isfinite().all())
            want = ref.turn(host(x.float()), host(positions), rope, backward)
            assert ref.within(host(y.double())[there], want[there], host(x.double())[there], rope, torch.finfo(x.dtype).eps)
            # without batches
            leave_nan(x[0].shape, x.dtype)
            assert torch.equal(f(x[0], positions[0], rope), y[0])
            # an output of the caller's keeps them
            out = torch.full_like(y, 7.0)
            assert f(x, positions, rope, out=out) is out
            assert bool((out[positions < 0] == 7).all()) and torch.equal(out[positions >= 0], y[positions >= 0])


def test_none_has_a_token(fxp):
    rope = fxp.Rotary(128)
    for B, T in ((1, 1), (3, 1), (2, 700)):
        x = torch.randn((B, T, 4, 128), device="cuda", dtype=torch.bfloat16)
        leave_nan(x.shape, x.dtype)
        assert not fxp.rotary_bwd(x, torch.full((B, T), -1, dtype=torch.int32, device="cuda"), rope).any()


def test_weight_gradient_over_a_padded_batch(fxp):
    """The gradient of a projection whose batch has rows without a token is that of the rows with one."""
    rope = fxp.Rotary(64)
    K = 96
    X, dy = torch.randn((2, 20, K), device="cuda"), torch.randn((2, 20, 1, 64), device="cuda")
    positions = torch.arange(20, dtype=torch.int32, device="cuda").repeat(2, 1)
    positions[0, 15:], positions[1, 3:] = -1, -1
    leave_nan(dy.shape, dy.dtype)
    dq = fxp.rotary_bwd(dy, positions, rope).flatten(2)
    there = positions >= 0
    got, want = X.flatten(0, 1).T @ dq.flatten(0, 1), X[there].T @ dq[there]
    bound = X[there].abs().T @ dq[there].abs() * (40 * 2.0 ** -23)
    assert bool(((got - want).abs() <= bound + 2.0 ** -60).all())


@pytest.mark.parametrize("outside", [False, True])
@pytest.mark.parametrize("B, T, heads, dim, rot, kind", [(2, 301, 4, 128, 128, "bf16"), (1, 3, 300, 20, 12, "fp32"), (3, 70, 40, 64, 32, "fp16"), (70, 1, 7, 258, 64, "bf16"), (1, 9, 2, 4000, 1024, "fp32")])
def test_many_rows_and_heads(fxp, B, T, heads, dim, rot, kind, outside):
    """Several workgroups along tokens and heads: rows with a token are those of a call whose rows all have one, the others zeros."""
    say("rotary, many rows", B, T, heads, dim, rot, kind, outside)
    rope = fxp.Rotary(rot)
    g = torch.Generator("cuda").manual_seed(T)
    x = torch.randn((B, heads, T, dim) if outside else (B, T, heads, dim), device="cuda", generator=g).to(TYPES[kind])
    x = x.transpose(1, 2) if outside else x
    positions = torch.randint(0, 5000, (B, T), dtype=torch.int32, device="cuda", generator=g)
    want = fxp.rotary_bwd(x, positions, rope)
    gone = torch.rand((B, T), device="cuda", generator=g) < 0.4
    want[gone] = 0
    x = torch.where(gone[:, :, None, None], float("nan"), x)                # what such a row holds is not looked at
    leave_nan(x.shape, x.dtype)
    assert torch.equal(fxp.rotary_bwd(x, torch.where(gone, -1 - positions, positions), rope), want)
