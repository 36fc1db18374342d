"""The tables, the writer and the reader of the paged cache against their definitions, bit for bit."""
import numpy as np
import pytest

from tests import serve_ref as ref
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


def make_tables(fxp, rng, lens, n_new, blocks, n_free, tokens=None, in_place=False):
    """KvTables with these lengths on random pages, and the inputs as arrays."""
    B, T = len(lens), int(sum(n_new)) if tokens is None else tokens
    held = [-(-int(n) // 64) for n in lens]
    order = rng.permutation(sum(held) + max(n_free, 1)).astype(np.int32)
    table = np.full((B, blocks), -1, np.int32)
    at = 0
    for b, n in enumerate(held):
        table[b, :n] = order[at:at + n]
        at += n
    free = order[at:]
    tab = fxp.KvTables(B, blocks, T, len(free), in_place=in_place)
    for mine, theirs in ((tab.block_table, table), (tab.lens, lens), (tab.free, free), (tab.n_free, [n_free])):
        mine.copy_(torch.tensor(np.array(theirs, dtype=np.int32)))
    return tab, table, free


def check_tables(tab, want):
    for name, w in want.items():
        assert np.array_equal(host(getattr(tab, name)).astype(np.int64), w), name


# requests, longest, most new tokens, blocks, pages missing from the stack, tokens behind the last one
TABLES = [(1, 0, 1, 1, 0, 0), (1, 5000, 1, 80, 0, 0), (1, 63, 400, 8, 0, 3), (5, 200, 0, 4, 0, 7), (256, 3000, 1, 50, 0, 0), (300, 900, 90, 20, 0, 11),
          (1024, 100, 3, 4, 17, 0), (1025, 500, 30, 9, 100, 5), (2600, 300, 70, 4, 300, 64), (7, 100, 9000, 60, 2, 1)]


@pytest.mark.parametrize("B,longest,most,blocks,short,behind", TABLES)
@pytest.mark.parametrize("in_place", [False, True])
def test_tables(fxp, B, longest, most, blocks, short, behind, in_place):
    say("kv_tables", (B, longest, most, blocks, short, behind, in_place))
    rng = np.random.default_rng(B * 3 + most)
    lens = np.minimum(rng.integers(0, longest + 1, B), blocks * 64)
    n_new = rng.integers(0, most + 1, B) if most != 1 else np.ones(B, int)
    need = sum(max(0, -(-(a + n) // 64) - -(-a // 64)) for a, n in zip(lens, n_new) if a + n <= blocks * 64)
    tab, table, free = make_tables(fxp, rng, lens, n_new, blocks, max(0, need - short), int(n_new.sum()) + behind, in_place)
    want = ref.tables(lens, n_new, table, free, max(0, need - short), tab.tokens, len(tab.runs))
    fxp.kv_tables(dev(n_new.astype(np.int32)), tab)
    check_tables(tab, want)
    assert not host(tab.ws).any()
    if not in_place:                       # the inputs stay, and a second call gives the same again
        assert np.array_equal(host(tab.lens), lens)
        fxp.kv_tables(dev(n_new.astype(np.int32)), tab)
        check_tables(tab, want)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B,most,tokens", [(4, 50, 0), (5, 90, 100), (900, 3, 700), (900, 40, 9000), (6, 500, 70), (1, 40, 39)])
def test_tables_of_a_step_with_too_few_rows(fxp, B, most, tokens, in_place):
    """From the first request whose tokens pass the step's on, those that have any are refused and keep their lengths; others are served."""
    say("kv_tables, more new tokens than rows", (B, most, tokens, in_place))
    rng = np.random.default_rng(B + most)
    lens, n_new = rng.integers(0, 200, B), rng.integers(0, most + 1, B)
    n_new[-1] = most
    assert n_new.sum() > tokens
    tab, table, free = make_tables(fxp, rng, lens, n_new, 12, 9 * B, tokens, in_place)
    want = ref.tables(lens, n_new, table, free, 9 * B, tokens, len(tab.runs))
    fxp.kv_tables(dev(n_new.astype(np.int32)), tab)
    check_tables(tab, want)
    refused = host(tab.refused).astype(bool)
    assert refused.any() and (B < 900 or not refused.all()) and np.array_equal(host(tab.lens_after)[refused], lens[refused])


def test_tables_step_by_step_from_a_graph(fxp):
    say("kv_tables, ten replays of one captured step in place")
    rng = np.random.default_rng(5)
    B, blocks = 700, 5
    lens = rng.integers(0, 300, B)
    tab, table, free = make_tables(fxp, rng, lens, np.full(B, 40), blocks, 800, B * 40, in_place=True)
    n_new = torch.zeros(B, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    fxp.kv_tables(n_new, tab)              # adds nothing
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        fxp.kv_tables(n_new, tab)
    n_free = 800
    for step in range(10):
        n = rng.integers(0, 40, B)
        n_new.copy_(torch.tensor(n.astype(np.int32)))
        graph.replay()
        want = ref.tables(lens, n, table, free, n_free, tab.tokens, len(tab.runs))
        check_tables(tab, want)
        lens, table, n_free = want["lens_after"], want["block_table"], int(want["n_free_after"][0])
    assert want["refused"].any() and not want["refused"].all()


def test_tables_with_lengths_that_are_no_lengths(fxp):
    say("kv_tables, negative and huge lengths")
    B = 300
    tab = fxp.KvTables(B, 4, 100, 50, in_place=False)
    rng = np.random.default_rng(1)
    lens = rng.integers(-(2 ** 31), 2 ** 31, B).astype(np.int32)
    n_new = rng.integers(-(2 ** 31), 2 ** 31, B).astype(np.int32)
    tab.lens.copy_(torch.tensor(lens))
    tab.n_free.fill_(2 ** 31 - 1)
    fxp.kv_tables(dev(n_new), tab)
    assert 0 <= int(tab.n_free_after) <= 50
    table = host(tab.block_table)
    assert ((table >= -1) & (table < 50)).all()
    assert (host(tab.slots) < 50 * 64).all()


def random_cache(fxp, rng, pages, H, D, bits):
    top = 2 ** (bits - 1)
    kq = rng.integers(1 - top, top, (pages, H, 64, D)).astype(np.int8)
    vq = rng.integers(1 - top, top, (pages, H, 4, D, 16)).astype(np.int8)
    ek, ev = rng.integers(120, 131, (pages, H)).astype(np.int32), rng.integers(120, 131, (pages, H)).astype(np.int32)
    cache = fxp.KvCache.of(dev(kq), dev(vq), dev(ek), dev(ev), bits)
    return cache, ref.Cache(kq, ek, bits), ref.Cache(ref.rows_of(vq), ev, bits)


def check_cache(cache, k, v, runs):
    """Scales everywhere, mantissas of every block outside the runs and of the tokens up to the last new one inside."""
    assert np.array_equal(host(cache.ek), k.e) and np.array_equal(host(cache.ev), v.e)
    for q, want in ((host(cache.kq), k.q), (ref.rows_of(host(cache.vq)), v.q)):
        q, want = q.astype(np.float64), want.copy()
        for _, count, page, off in runs:
            if count > 0 and 0 <= page < len(want):
                q[page, :, off + count:] = want[page, :, off + count:] = 0
        assert np.array_equal(q, want)


def values_of(rng, T, H, D, kind):
    """Values with halves of a unit among them, of sizes that make some blocks grow and others not."""
    x = rng.standard_normal((T, H, D)) * 2.0 ** rng.integers(-6, 6, (T, 1, 1))
    x[:, :, ::7] = np.round(x[:, :, ::7] * 128) / 128
    return torch.tensor(x.astype(np.float32)).to(TYPES[kind])


# heads, dim, type, bits, runs as (count, offset)
APPEND = [(1, 16, "fp32", 8, [(1, 0)]), (8, 128, "bf16", 8, [(1, 5), (1, 63), (1, 0), (1, 17)]), (3, 80, "fp16", 8, [(64, 0), (3, 61), (33, 2)]),
          (2, 256, "fp32", 8, [(64, 0), (1, 1), (63, 1), (5, 30)]), (2, 256, "bf16", 5, [(1, 62), (1, 3)]), (4, 64, "fp16", 2, [(10, 0), (20, 9)]),
          (12, 64, "fp32", 7, [(1, i) for i in range(64)]), (2, 48, "bf16", 8, [(2, 2), (3, 1), (4, 4), (6, 0)])]


@pytest.mark.parametrize("H,D,kind,bits,spans", APPEND)
@pytest.mark.parametrize("layout", ["dense", "fused", "odd", "heads_first"])
def test_append_and_load(fxp, H, D, kind, bits, spans, layout):
    say("kv_append", (H, D, kind, bits, len(spans), layout))
    rng = np.random.default_rng(H * D + bits)
    pages = len(spans) + 2
    cache, k, v = random_cache(fxp, rng, pages, H, D, bits)
    at, T, runs = rng.permutation(pages), 0, []
    for i, (count, off) in enumerate(spans):
        runs.append((T, count, int(at[i]), off))
        T += count
    runs += [(0, 0, -1, 0), (0, 2, -1, 0), (T, 1, int(at[-1]), 0), (0, 1, pages, 0), (0, 4, int(at[-1]), 61), (-1, 1, int(at[-1]), 0)]
    xk, xv = values_of(rng, T, H, D, kind), values_of(rng, T, H, D, kind)
    if layout == "dense":
        dk, dv = xk.cuda(), xv.cuda()
    elif layout == "fused":
        both = torch.cat([xk.view(T, -1), xv.view(T, -1)], 1).cuda()
        dk, dv = both[:, :H * D].unflatten(1, (H, D)), both[:, H * D:].unflatten(1, (H, D))
    elif layout == "odd":                   # no row begins on a multiple of four elements
        both = torch.zeros((T, H, 2 * D + 3), dtype=xk.dtype, device="cuda")
        both[:, :, 1:D + 1], both[:, :, D + 2:2 * D + 2] = xk.cuda(), xv.cuda()
        dk, dv = both[:, :, 1:D + 1], both[:, :, D + 2:2 * D + 2]
    else:
        dk, dv = (x.transpose(0, 1).contiguous().cuda().transpose(0, 1) for x in (xk, xv))
    real = np.array(runs[:len(spans)])
    k.append(xk.double().numpy(), real)
    v.append(xv.double().numpy(), real)
    d_runs = dev(np.array(runs, dtype=np.int32))
    fxp.kv_append(dk, dv, cache, d_runs)
    check_cache(cache, k, v, runs[:len(spans)])
    fxp.kv_append(dk, dv, cache, d_runs)            # the same tokens again change nothing
    check_cache(cache, k, v, runs[:len(spans)])
    # back: exactly the values, rows of no run left alone
    for dtype in TYPES.values():
        out = [torch.full((T + 1, H, D), 7.0, dtype=dtype, device="cuda") for _ in range(2)]
        d_runs[len(spans) + 2, 0] = T + 1           # the bad runs of the append are bad here too
        fxp.kv_load(cache, d_runs, T + 1, out=out)
        for o, c in zip(out, (k, v)):
            want = np.concatenate([c.values()[p, :, off:off + n].transpose(1, 0, 2) for _, n, p, off in runs[:len(spans)]])
            assert torch.equal(o[:T].cpu(), torch.tensor(want).float().to(dtype))
            assert (o[T] == 7).all()
    d_runs[len(spans) + 2, 0] = T


def test_a_page_written_at_once_is_the_map_of_its_tensor(fxp):
    say("kv_append against fxp.scale_map")
    x = torch.randn((64, 1, 128), device="cuda") * 3
    cache = fxp.KvCache(2, 1, 128)
    fxp.kv_append(x, x, cache, dev(np.array([[0, 64, 1, 0]], np.int32)))
    e, q, qT = fxp.scale_map(x.view(64, 128), rounding=fxp.NEAREST, want_qT=True)
    assert int(cache.ek[1, 0]) == int(cache.ev[1, 0]) == int(e)
    assert torch.equal(cache.kq[1, 0], q)
    assert torch.equal(cache.vq[1, 0].permute(1, 0, 2).reshape(128, 64), qT)


def test_append_of_values_that_are_not_finite_or_tiny(fxp):
    say("kv_append of Inf, NaN, zeros and sub-normal values")
    x = torch.zeros((4, 1, 16))
    x[0, 0, :4] = torch.tensor([float("inf"), float("-inf"), float("nan"), 1.0])
    x[1, 0, :3] = torch.tensor([1e-45, -1.1e-38, 2e-38])
    x[3, 0, :] = torch.finfo(torch.float32).max
    cache = fxp.KvCache(4, 1, 16)
    runs = np.array([[i, 1, i, 0] for i in range(4)], np.int32)
    fxp.kv_append(x.cuda(), x.cuda(), cache, dev(runs))
    assert host(cache.ek)[:, 0].tolist() == [255, 1, 1, 254]
    q = host(cache.kq)[:, 0, 0]
    assert q[0, :4].tolist() == [127, -127, 0, 0] and q[1, :3].tolist() == [0, -60, 109] and not q[2].any() and (q[3] == 127).all()
    assert np.array_equal(host(cache.vq)[:, 0, 0, :, 0], q)


def test_a_cache_past_32_bits(fxp):
    say("kv_append and kv_load behind 4 GiB of keys")
    pages, H, D = 34000, 8, 256
    cache = fxp.KvCache(pages, H, D)
    rng = np.random.default_rng(2)
    x = values_of(rng, 70, H, D, "bf16")
    runs = dev(np.array([[0, 64, pages - 1, 0], [64, 6, 32768, 0]], np.int32))
    cache.kq[0].fill_(3)
    cache.vq[0].fill_(3)
    fxp.kv_append(x.cuda(), x.cuda(), cache, runs)
    k, v = fxp.kv_load(cache, runs, 70)
    want = ref.Cache(np.zeros((2, H, 64, D)), np.ones((2, H)), 8)
    want.append(x.double().numpy(), np.array([[0, 64, 0, 0], [64, 6, 1, 0]]))
    want = torch.tensor(np.concatenate([want.values()[0].transpose(1, 0, 2), want.values()[1][:, :6].transpose(1, 0, 2)])).float()
    assert torch.equal(k.cpu(), want) and torch.equal(v.cpu(), want)
    assert (cache.kq[0] == 3).all() and (cache.vq[0] == 3).all()


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("asked,many,tokens", [(1 << 20, 4096, 1 << 20), (1 << 16, 65536, 1 << 16), (2 ** 31 - 1, 4, 70)])
def test_tables_of_requests_whose_sums_pass_32_bits(fxp, asked, many, tokens, in_place):
    """`many` requests ask for more than their rows hold, 2^32 tokens together; those behind them, who ask for 5, must not be taken for the first."""
    say("kv_tables, sums past 32 bits", (asked, many, tokens, in_place))
    n_new = np.concatenate([np.full(many, asked, np.int64), np.full(5, 5), np.zeros(2, np.int64)])
    B = len(n_new)
    tab = fxp.KvTables(B, 3, tokens, 40, in_place=in_place)
    lens = np.full(B, 7, np.int32)
    lens[many:] = 62
    tab.lens.copy_(torch.tensor(lens))
    tab.refused.fill_(-1)
    fxp.kv_tables(dev(n_new.astype(np.int32)), tab)
    refused = np.ones(B)
    refused[-2:] = 0                                          # these ask for nothing
    assert np.array_equal(host(tab.refused), refused)
    assert np.array_equal(host(tab.lens_after), lens) and int(tab.n_free_after) == 40 and (host(tab.block_table) == -1).all()
    # of a request that asks for more than the step's rows, as many as those are counted
    sums = np.concatenate([[0], np.cumsum(np.minimum(n_new, tokens))])
    assert np.array_equal(host(tab.first), np.minimum(sums, 2 ** 31 - 1))
    assert (host(tab.slots) == -1).all()
    asked = min(asked, tokens)
    assert np.array_equal(host(tab.positions), 7 + np.arange(tokens) % asked)
    assert (host(tab.runs)[:, 2] == -1).all() and not host(tab.ws).any()


def test_load_refuses_outputs_that_share_elements(fxp):
    say("kv_load into one tensor twice")
    cache = fxp.KvCache(2, 3, 16)
    cache.kq.fill_(1)
    cache.vq.fill_(2)
    runs = dev(np.array([[0, 4, 1, 0]], np.int32))
    room = torch.zeros((9, 3, 16), device="cuda")
    for k, v in ((room[:4], room[:4]), (room[:4], room[3:7]), (room[4:8], room[1:5])):
        with pytest.raises(fxp.FxpError, match="share elements"):
            fxp.kv_load(cache, runs, 4, out=(k, v))
    assert not room.any()
    k, v = fxp.kv_load(cache, runs, 4, out=(room[:4], room[4:8]))
    assert (k * 2 == v).all() and k.any() and not room[8:].any()


@pytest.mark.parametrize("bits", [2, 8])
def test_load_under_every_scale(fxp, bits):
    """The smallest and the largest scales, and what is none: counted as 1 and 255."""
    say("kv_load under all scales", bits)
    H, D, top = 2, 16, 2 ** (bits - 1) - 1
    scales = np.array(list(range(1, 256)) + [0, -7, 256, 2 ** 31 - 1, -(2 ** 31)])
    rng = np.random.default_rng(3)
    q = rng.integers(-top, top + 1, (len(scales), H, 64, D)).astype(np.int8)
    cache = fxp.KvCache(len(scales), H, D, bits)
    cache.kq.copy_(torch.tensor(q))
    cache.vq.copy_(torch.tensor(q.reshape(len(scales), H, 4, 16, D).transpose(0, 1, 2, 4, 3).copy()))
    cache.ek.copy_(torch.tensor(scales.astype(np.int32))[:, None])
    cache.ev.copy_(torch.tensor(scales.astype(np.int32))[:, None])
    runs = np.array([[i * 6, 6, i, 3] for i in range(len(scales))], np.int32)
    want = q[:, :, 3:9].transpose(0, 2, 1, 3).reshape(-1, H, D) * np.repeat(2.0 ** (np.clip(scales, 1, 255) - 125.0 - bits), 6)[:, None, None]
    for dtype in TYPES.values():
        for got in fxp.kv_load(cache, dev(runs), len(want), dtype):
            assert torch.equal(got.cpu(), torch.tensor(want).float().to(dtype))
