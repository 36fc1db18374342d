"""The cache's writer that turns keys and queries, against 64 bits: what it stores exactly, the queries to their type's rounding."""
import numpy as np
import pytest

from tests import rotary_ref
from tests import serve_ref as ref
from tests.gpu_util import dev, host, say
from tests.test_gpu_kv import check_cache, random_cache, values_of

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def fxp():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: there is no CPU path in libfxp")
    from paper_2207_08822_amd import fxp as binding
    binding.lib()
    return binding


def step_of(fxp, rng, spans, pages, more=()):
    """Tables that hold runs (count, offset) on pages of their own at positions up to 10^5, and `more` runs that are to be skipped."""
    T = sum(n for n, _ in spans)
    at, t, runs, positions = rng.permutation(pages), 0, [], []
    for i, (count, off) in enumerate(spans):
        runs.append((t, count, int(at[i]), off))
        block = 0 if i == 0 else int(rng.integers(0, 1600))
        positions += [64 * block + off + j for j in range(count)]
        t += count
    tab = fxp.KvTables(max(1, len(spans) + len(more)), 1700, T, 1)
    rows = tab.runs.shape[0]
    listed = (list(runs) + list(more))[:rows]
    tab.runs[:len(listed)] = dev(np.array(listed, np.int32))
    tab.positions.copy_(dev(np.array(positions, np.int32)))
    return tab, runs, positions


# heads, query heads, dim, rot, type, bits, runs as (count, offset)
CASES = [(1, 1, 16, 16, "fp32", 8, [(1, 0)]), (8, 32, 128, 128, "bf16", 8, [(1, 5), (1, 63), (1, 0), (1, 17)]), (3, 21, 80, 40, "fp16", 8, [(64, 0), (3, 61), (33, 2)]),
         (2, 4, 256, 256, "fp32", 8, [(64, 0), (1, 1), (63, 1), (5, 30)]), (2, 0, 256, 64, "bf16", 5, [(1, 62), (1, 3)]), (4, 4, 64, 2, "fp16", 2, [(10, 0), (20, 9)]),
         (12, 12, 64, 46, "fp32", 7, [(1, i) for i in range(64)]), (2, 2, 48, 12, "bf16", 8, [(2, 2), (3, 1), (4, 4), (6, 0)]), (1, 16, 160, 30, "bf16", 8, [(64, 0), (40, 3)]), (2, 6, 96, 32, "fp16", 8, [(64, 0), (5, 3)]), (2, 2, 16, 16, "bf16", 8, [(7, 0), (30, 20)])]


@pytest.mark.parametrize("near", [False, True])
@pytest.mark.parametrize("H,QH,D,rot,kind,bits,spans", CASES)
@pytest.mark.parametrize("layout", ["dense", "fused", "odd", "heads_first", "in_place"])
def test_append(fxp, H, QH, D, rot, kind, bits, spans, layout, near):
    say("kv_append_rotary", (H, QH, D, rot, kind, bits, len(spans), layout, near))
    rng = np.random.default_rng(H * D + bits)
    pages = len(spans) + 2
    cache, k, v = random_cache(fxp, rng, pages, H, D, bits)
    T = sum(n for n, _ in spans)
    tab, runs, positions = step_of(fxp, rng, spans, pages, [(0, 0, -1, 0), (0, 2, -1, 0), (T, 1, pages - 1, 0), (0, 1, pages, 0), (0, 4, pages - 1, 61)])
    rope = fxp.Rotary(rot, interleaved=near, amplitude=1.25)
    x = [values_of(rng, T, h, D, kind) for h in (H, H, QH)]
    if layout == "odd":                   # no row begins on a multiple of four elements
        both = torch.zeros((T, max(H, QH), 3 * D + 3), dtype=x[0].dtype, device="cuda")
        dk, dv, dq = (both[:, :t.shape[1], i * (D + 1) + 1:][..., :D] for i, t in enumerate(x))
        for a, b in zip((dk, dv, dq), x):
            a.copy_(b)
    elif layout == "heads_first":
        dk, dv, dq = (t.transpose(0, 1).contiguous().cuda().transpose(0, 1) for t in x)
    elif layout == "dense":
        dk, dv, dq = (t.cuda() for t in x)
    else:
        dk, dv, dq = torch.cat(x, 1).cuda().split([H, H, QH], 1)
    turned = rotary_ref.turn(x[0].double().numpy(), np.array(positions), rope)
    k.append(turned, np.array(runs))
    v.append(x[1].double().numpy(), np.array(runs))
    out = None if QH == 0 else dq if layout == "in_place" else torch.full((T, QH, D), 7.0, dtype=dq.dtype, device="cuda")
    got = fxp.kv_append_rotary(dk, dv, cache, tab, rope, q=dq if QH else None, out=out)
    check_cache(cache, k, v, runs)
    assert torch.equal(dk.cpu(), x[0]) and torch.equal(dv.cpu(), x[1])
    if QH:
        assert got is out
        want = rotary_ref.turn(x[2].double().numpy(), np.array(positions), rope)
        assert rotary_ref.within(host(got.double()), want, x[2].double().numpy(), rope, torch.finfo(got.dtype).eps)
        assert torch.equal(got[..., rot:].cpu(), x[2][..., rot:])
    else:
        assert got is None


def test_rows_of_refused_requests_stay(fxp):
    tab = fxp.KvTables(3, 2, 5, 2)
    tab.lens.copy_(torch.tensor([63, 128, 0]))          # the second one's row is full
    tab.block_table[0, 0] = 1
    tab.n_free.fill_(1)
    fxp.kv_tables(dev(np.array([2, 1, 1], np.int32)), tab)
    assert tab.refused.tolist() == [0, 1, 1] and tab.positions.tolist() == [63, 64, 128, 0, -1]
    cache, rope = fxp.KvCache(2, 1, 16), fxp.Rotary(16)
    x = torch.randn((5, 3, 16), device="cuda")
    out = torch.full((5, 1, 16), 7.0, device="cuda")
    fxp.kv_append_rotary(x[:, :1], x[:, 1:2], cache, tab, rope, q=x[:, 2:], out=out)
    assert torch.equal(out[:2], fxp.rotary(x[:2, 2:], tab.positions[:2], rope)) and bool((out[2:] == 7).all())


def test_values_that_are_not_finite_or_tiny(fxp):
    say("kv_append_rotary of Inf, NaN, zeros and sub-normal values")
    x = torch.zeros((4, 1, 16))
    x[0, 0, [0, 8, 1]] = torch.tensor([float("nan"), 1.0, 2.0])
    x[1, 0, :3] = torch.tensor([1e-45, -1.1e-38, 2e-38])
    x[3, 0, :] = torch.finfo(torch.float32).max
    cache, tab = fxp.KvCache(4, 1, 16), fxp.KvTables(4, 1, 4, 4)
    tab.runs.copy_(torch.tensor([[i, 1, i, 0] for i in range(4)], dtype=torch.int32))
    tab.positions.copy_(torch.tensor([3, 0, 5, 1], dtype=torch.int32))
    fxp.kv_append_rotary(x.cuda(), x.cuda(), cache, tab, fxp.Rotary(16))
    # the third is all zeros; the fourth's pairs are turned past the largest number
    assert host(cache.ek)[:, 0].tolist() == [255, 1, 1, 255]
    q = host(cache.kq)[:, 0, 0]
    assert q[0, 0] == 0 and q[0, 8] == 0 and q[1, :3].tolist() == [0, -60, 109] and not q[2].any()


def test_a_cache_past_32_bits(fxp):
    say("kv_append_rotary behind 4 GiB of keys")
    pages, H, D = 34000, 8, 256
    cache, rope = fxp.KvCache(pages, H, D), fxp.Rotary(128)
    rng = np.random.default_rng(2)
    x = values_of(rng, 70, H, D, "bf16")
    tab = fxp.KvTables(2, 4, 70, 1)
    tab.runs[:2] = dev(np.array([[0, 64, pages - 1, 0], [64, 6, 32768, 0]], np.int32))
    tab.positions.copy_(torch.arange(70))
    cache.kq[0].fill_(3)
    fxp.kv_append_rotary(x.cuda(), x.cuda(), cache, tab, rope)
    want = ref.Cache(np.zeros((2, H, 64, D)), np.ones((2, H)), 8)
    want.append(rotary_ref.turn(x.double().numpy(), np.arange(70), rope), np.array([[0, 64, 0, 0], [64, 6, 1, 0]]))
    assert np.array_equal(host(cache.kq[pages - 1]), want.q[0]) and np.array_equal(host(cache.kq[32768])[:, :6], want.q[1][:, :6])
    assert np.array_equal(host(cache.ek)[[pages - 1, 32768]], want.e) and bool((cache.kq[0] == 3).all())


def test_without_positions_it_is_kv_append(fxp):
    """At position 0 nothing turns: the same bytes as kv_append, in a page of old tokens too."""
    rng = np.random.default_rng(5)
    for kind in ("fp32", "bf16", "fp16"):
        x = [values_of(rng, 90, 4, 96, kind).cuda() for _ in range(2)]
        a, _, _ = random_cache(fxp, np.random.default_rng(6), 3, 4, 96, 8)
        b, _, _ = random_cache(fxp, np.random.default_rng(6), 3, 4, 96, 8)
        tab = fxp.KvTables(3, 4, 90, 1)
        tab.runs[:3] = dev(np.array([[0, 64, 2, 0], [64, 6, 0, 11], [70, 20, 1, 44]], np.int32))
        tab.positions.zero_()
        fxp.kv_append(x[0], x[1], a, tab.runs)
        fxp.kv_append_rotary(x[0], x[1], b, tab, fxp.Rotary(64))
        for name in ("kq", "vq", "ek", "ev"):
            assert torch.equal(getattr(a, name), getattr(b, name)), (kind, name)


def test_refused(fxp):
    cache, rope, tab = fxp.KvCache(3, 2, 32), fxp.Rotary(32), fxp.KvTables(2, 2, 4, 3)
    qkv = torch.randn((4, 8, 32), device="cuda")
    q, k, v = qkv.split([4, 2, 2], 1)
    call = fxp.kv_append_rotary
    bad = [lambda: call(k, v.half(), cache, tab, rope), lambda: call(k[:3], v[:3], cache, tab, rope), lambda: call(k, v, cache, tab, fxp.Rotary(64)),
           lambda: call(k, v, cache, tab, rope, q=qkv[:, :3]), lambda: call(k, v, cache, tab, rope, q=q.half()), lambda: call(k, v, cache, tab, rope, out=q),
           lambda: call(k, v, cache, tab, rope, q=q, out=qkv[:, 1:5]), lambda: call(k, v, cache, tab, rope, q=q, out=qkv[:, 4:]),
           lambda: call(k, v, cache, tab, rope, q=q.clone(), out=qkv[:, 3:7]), lambda: call(k, v, cache, tab, rope, q=q, out=q[:1].expand(4, 4, 32)),
           lambda: call(k.cpu(), v, cache, tab, rope)]
    for i, f in enumerate(bad):
        with pytest.raises(fxp.FxpError):
            f()
            pytest.fail(str(i))
    assert call(k, v, cache, tab, rope, q=q, out=q) is q        # beside k and v in one buffer


def test_replayed_step(fxp):
    """Tables, writer and attention of a decode step from a graph, each replay against the same step run eagerly."""
    B, H, QH, D = 5, 2, 6, 64
    rope = fxp.Rotary(D)

    def fresh():
        tab = fxp.KvTables(B, 4, B, 40)
        return tab, fxp.KvCache(40, H, D)

    n_new = torch.ones(B, dtype=torch.int32, device="cuda")
    qkv = torch.zeros((B, QH + 2 * H, D), dtype=torch.bfloat16, device="cuda")
    out = torch.empty((B, QH, D), dtype=torch.bfloat16, device="cuda")
    (tab, cache), (tab2, cache2) = fresh(), fresh()
    buf = fxp.AttentionBuffers(B, B, QH, cache)

    def step(tab, cache, out):
        fxp.kv_tables(n_new, tab)
        q = fxp.kv_append_rotary(qkv[:, QH:QH + H], qkv[:, QH + H:], cache, tab, rope, q=qkv[:, :QH])
        return fxp.kv_attention(q, cache, tab, buf, out=out)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*fresh(), out)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(tab, cache, out)
    for i in range(70):                     # past a page
        qkv.copy_(torch.randn(qkv.shape, device="cuda"))
        graph.replay()
        want = step(tab2, cache2, torch.empty_like(out))
        assert torch.equal(out, want) and torch.equal(tab.lens, tab2.lens)
