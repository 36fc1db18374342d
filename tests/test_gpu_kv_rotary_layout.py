"""The cache's writer over a projection whose heads hold query, key and value beside each other, its queries turned in place."""
import numpy as np
import pytest

from tests.gpu_util import dev, say

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def fxp():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: there is no CPU path in libfxp")
    from paper_2207_08822_amd import fxp as binding
    binding.lib()
    return binding


@pytest.mark.parametrize("heads_outside", [False, True])
@pytest.mark.parametrize("T", [1, 40])
def test_in_place_beside_keys(fxp, T, heads_outside):
    say("kv_append_rotary, interleaved heads", T, heads_outside)
    H, D = 4, 64
    rope = fxp.Rotary(D)
    qkv = torch.randn((H, T, 3, D) if heads_outside else (T, H, 3, D), device="cuda", dtype=torch.bfloat16)
    q, k, v = (qkv.transpose(0, 1) if heads_outside else qkv).unbind(2)
    dense = [t.contiguous() for t in (q, k, v)]
    caches, tables = [fxp.KvCache(2, H, D) for _ in range(2)], []
    for cache in caches:
        for t in (cache.kq, cache.vq):
            t.zero_()
        tab = fxp.KvTables(1, 2, T, 2)
        fxp.kv_tables(dev(np.array([T], np.int32)), tab)
        tables.append(tab)
    want = fxp.kv_append_rotary(dense[1], dense[2], caches[0], tables[0], rope, q=dense[0])
    assert fxp.kv_append_rotary(k, v, caches[1], tables[1], rope, q=q, out=q) is q
    assert torch.equal(q, want) and torch.equal(k, dense[1]) and torch.equal(v, dense[2])
    for name in ("kq", "vq", "ek", "ev"):
        assert torch.equal(getattr(caches[0], name), getattr(caches[1], name)), name
    # one element further, the queries' rows are written over the keys
    if T > 1 and not heads_outside:
        room = torch.zeros(T * H * 3 * D + 8, device="cuda", dtype=torch.bfloat16)
        over = room[8:].view(T, H, 3, D)
        with pytest.raises(fxp.FxpError):
            fxp.kv_append_rotary(over[:, :, 1], over[:, :, 2], caches[1], tables[1], rope, q=q, out=room.as_strided((T, H, D), over[:, :, 0].stride(), 9))
