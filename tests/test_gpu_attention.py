"""Attention over the paged 8-bit cache against its definition in 64 bits, within bounds that follow from the stated arithmetic."""
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


class Case:
    """A cache, tables and queries on the device and as arrays."""

    def __init__(self, fxp, lens, news, QH, H, D, kind, bits=8, seed=0, behind=0, missing=(), sharp=1.0, sink=False, spare=0):
        rng = np.random.default_rng(seed + 1000 * D + QH)
        self.lens, self.T = np.array(lens), int(sum(news)) + behind
        self.first = np.concatenate([[0], np.cumsum(news)])
        held = [-(-n // 64) for n in lens]
        self.blocks, pages = max(max(held), 1) + 1, sum(held) + 2 + spare
        order = (rng.permutation(pages - spare) + spare).astype(np.int32)
        self.table, at = np.full((len(lens), self.blocks), -1, np.int32), 0
        for b, n in enumerate(held):
            self.table[b, :n] = order[at:at + n]
            at += n
        for b, j, page in missing:
            self.table[b, j] = page
        top = 2 ** (bits - 1)
        bell = lambda shape: np.clip(np.round(rng.standard_normal(shape) * top / 3), 1 - top, top - 1).astype(np.int8)  # noqa: E731
        kq, vq = bell((pages - spare, H, 64, D)), bell((pages - spare, H, 4, D, 16))
        ek, ev = rng.integers(126, 129, (pages - spare, H)), rng.integers(120, 130, (pages - spare, H))
        if sink:                              # the first token of each request outweighs all others by far
            for b, n in enumerate(held):
                if n:
                    kq[self.table[b, 0] - spare, :, 0] = np.sign(kq[self.table[b, 0] - spare, :, 0]) * (top - 1)
        self.k, self.v = ref.Cache(kq, ek, bits), ref.Cache(ref.rows_of(vq), ev, bits)
        self.spare = spare
        if spare:
            self.cache = fxp.KvCache(pages, H, D, bits)
            for mine, theirs in ((self.cache.kq, kq), (self.cache.vq, vq), (self.cache.ek, ek), (self.cache.ev, ev)):
                mine[spare:].copy_(torch.tensor(theirs))
        else:
            self.cache = fxp.KvCache.of(dev(kq), dev(vq), dev(ek.astype(np.int32)), dev(ev.astype(np.int32)), bits)
        self.tab = fxp.KvTables(len(lens), self.blocks, self.T, 4, in_place=False)
        self.tab.block_table.copy_(torch.tensor(self.table))
        self.tab.lens_after.copy_(torch.tensor(self.lens.astype(np.int32)))
        self.tab.first.copy_(torch.tensor(self.first.astype(np.int32)))
        dtype, self.unit_bits, self.half = TYPES[kind]
        q = torch.tensor((rng.standard_normal((self.T, QH, D)) * sharp).astype(np.float32)).to(dtype)
        if sink:
            for b, n in enumerate(held):
                if n:
                    for h in range(QH):
                        row = torch.tensor(np.sign(kq[self.table[b, 0] - spare, h // (QH // H), 0]).astype(np.float32)).to(dtype)
                        q[self.first[b]:self.first[b + 1], h] += row * sharp
        self.q, self.dq = q, q.cuda()
        self.scale = float(np.float32(D ** -0.5))

    def want(self, window=0):
        table = np.where((self.table >= self.spare) & (self.table < self.spare + len(self.k.q)), self.table - self.spare, -1)
        return ref.attention(self.q.double().numpy(), self.k.values(), self.v.values(), self.first, self.lens, table, self.scale, window,
                             self.unit_bits, self.half)

    def check(self, out, lse=None, window=0, want=None):
        o, logs, off = want or self.want(window)
        rows = self.first[-1]
        got = out.double().cpu().numpy()
        far = np.abs(got - o)[:rows]
        assert (far <= off[:rows]).all(), f"off by {np.max(far / np.maximum(off[:rows], 1e-300))} of what it may be"
        if lse is not None:
            got = lse.double().cpu().numpy()[:rows]
            assert np.array_equal(np.isinf(got), np.isinf(logs[:rows]))
            m = np.isfinite(logs[:rows])
            # the weights' factor, plus fp32 roundings of the logarithm, its sum with the largest score and that score
            assert (np.abs(got[m] - logs[:rows][m]) <= 2e-3 * (self.unit_bits < 20) + 4e-6 * (1 + np.abs(logs[:rows][m]))).all()


# lengths, new tokens, query heads, heads, dim
CASES = [([1], [1], 1, 1, 16), ([64], [1], 4, 4, 64), ([65, 1, 200, 63], [1, 1, 1, 1], 8, 2, 128), ([300, 5, 0, 129], [5, 5, 0, 3], 14, 2, 80),
         ([257], [17], 6, 2, 48), ([1000, 640], [1, 2], 16, 1, 256), ([40, 700], [40, 33], 3, 3, 112), ([100, 0, 77], [1, 2, 9], 4, 2, 192),
         ([2, 3, 64, 128], [2, 3, 64, 70], 2, 1, 64), ([3000], [1], 32, 8, 128)]


@pytest.mark.parametrize("lens,news,QH,H,D", CASES)
@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("window", [0, 70])
def test_attention(fxp, lens, news, QH, H, D, kind, window):
    say("kv_attention", (lens, news, QH, H, D, kind, window))
    c = Case(fxp, lens, news, QH, H, D, kind, behind=2)
    out = torch.full((c.T, QH, D), 9.0, dtype=c.dq.dtype, device="cuda")
    lse = torch.full((c.T, QH), 9.0, device="cuda")
    got = fxp.kv_attention(c.dq, c.cache, c.tab, scale=c.scale, window=window, out=out, lse=lse)
    assert got is out
    c.check(out, lse, window)
    assert (out[c.first[-1]:] == 9).all() and (lse[c.first[-1]:] == 9).all()      # rows behind the last request


# requests whose rows fill 256 blocks of 64 together (heads x blocks): the kernel for many rows, short requests among them
MANY = [([520, 3, 200, 0, 64], [300, 1, 200, 0, 40], 28, 14, 64), ([257], [257], 64, 16, 16), ([90, 700, 33], [80, 301, 33], 32, 32, 80),
        ([300, 140], [150, 140], 48, 48, 128), ([130, 70], [65, 70], 130, 65, 192), ([150], [100], 128, 128, 256), ([10, 400], [100, 130], 66, 66, 112)]


@pytest.mark.parametrize("lens,news,QH,H,D", MANY)
@pytest.mark.parametrize("kind,window,bits", [("fp32", 0, 8), ("bf16", 90, 8), ("fp16", 0, 5)])
def test_attention_of_prompts(fxp, lens, news, QH, H, D, kind, window, bits):
    say("kv_attention of many rows", (lens, news, QH, H, D, kind, window, bits))
    c = Case(fxp, lens, news, QH, H, D, kind, bits=bits, behind=3, missing=[(0, 1, -1)] if len(lens) > 2 else ())
    out, lse = torch.full((c.T, QH, D), 9.0, dtype=c.dq.dtype, device="cuda"), torch.full((c.T, QH), 9.0, device="cuda")
    fxp.kv_attention(c.dq, c.cache, c.tab, scale=c.scale, window=window, out=out, lse=lse)
    c.check(out, lse, window)
    assert (out[c.first[-1]:] == 9).all() and (lse[c.first[-1]:] == 9).all()


@pytest.mark.parametrize("bits", [2, 4, 7])
def test_attention_over_other_widths(fxp, bits):
    say("kv_attention, bits", bits)
    c = Case(fxp, [500, 31], [2, 1], 8, 4, 64, "bf16", bits=bits)
    c.check(fxp.kv_attention(c.dq, c.cache, c.tab, scale=c.scale))


@pytest.mark.parametrize("kind", list(TYPES))
def test_attention_with_a_token_that_outweighs_thousands(fxp, kind):
    say("kv_attention, one large weight and a long tail", kind)
    c = Case(fxp, [4000], [1], 2, 1, 64, kind, sink=True, sharp=2.0)
    lse = torch.empty((1, 2), device="cuda")
    c.check(fxp.kv_attention(c.dq, c.cache, c.tab, scale=c.scale, lse=lse), lse)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("sharp", [30.0, 1000.0])
def test_attention_with_large_scores(fxp, kind, sharp):
    """Scores in the hundreds and tens of thousands: their fp32 roundings must not lift a weight above the largest digit."""
    say("kv_attention, large scores", kind, sharp)
    c = Case(fxp, [900, 64], [2, 1], 8, 4, 64, kind, sharp=sharp)
    c.check(fxp.kv_attention(c.dq, c.cache, c.tab, scale=c.scale))


@pytest.mark.parametrize("kind", list(TYPES))
def test_attention_is_the_value_where_all_values_are_one(fxp, kind):
    """Weights rounded to half a unit of 1/32639 of the page's largest: 64 of them are off by 64 * 0.5 / 32639 of it at most."""
    say("kv_attention over constant values", kind)
    c = Case(fxp, [1500, 3], [1, 1], 4, 2, 64, kind)
    c.cache.vq.fill_(64)
    c.cache.ev.fill_(127)                                     # 64 * 2^(127 - 133) = 1
    out = fxp.kv_attention(c.dq, c.cache, c.tab, scale=c.scale).double()
    most = 32639 if c.unit_bits == 15 else 8355711
    assert float((out - 1).abs().max()) <= 32 / most + c.half + 2.0 ** -20


@pytest.mark.parametrize("window", [0, 100])
def test_attention_with_pages_that_do_not_exist(fxp, window):
    say("kv_attention, bad pages")
    c = Case(fxp, [500, 64, 130], [3, 1, 1], 4, 2, 64, "bf16", missing=[(0, 2, -1), (0, 5, 10 ** 9), (1, 0, -(2 ** 31)), (2, 2, 17)])
    lse = torch.empty((c.T, 4), device="cuda")
    out = fxp.kv_attention(c.dq, c.cache, c.tab, scale=c.scale, window=window, lse=lse)
    c.check(out, lse, window)
    assert not out[3].any() and torch.isinf(lse[3]).all()     # the only page of the second request is missing


def test_attention_layouts_and_types_of_rows(fxp):
    say("kv_attention, strided q and out")
    c = Case(fxp, [200, 90], [3, 2], 6, 2, 80, "bf16")
    want = c.want()
    fused = torch.zeros((c.T, 6, 3 * 80 + 1), dtype=torch.bfloat16, device="cuda")
    fused[:, :, 1:81] = c.dq
    c.check(fxp.kv_attention(fused[:, :, 1:81], c.cache, c.tab, scale=c.scale, out=fused[:, :, 81:161]), want=want)
    assert not fused[:, :, 0].any() and not fused[:, :, 161:].any() and torch.equal(fused[:, :, 1:81], c.dq)
    first = c.dq.transpose(0, 1).contiguous().transpose(0, 1)
    c.check(fxp.kv_attention(first, c.cache, c.tab, scale=c.scale, out=torch.empty_like(first)), want=want)
    assert torch.equal(fxp.kv_attention(first, c.cache, c.tab, scale=c.scale), fxp.kv_attention(c.dq, c.cache, c.tab, scale=c.scale))


def test_attention_refuses_rows_of_out_that_share_elements(fxp):
    say("kv_attention, overlapping rows of out")
    c = Case(fxp, [20], [3], 4, 2, 16, "fp32")
    room = torch.zeros(400, device="cuda")
    for strides in ((16, 16), (0, 16), (48, 16), (16, 40), (64, 8), (0, 0)):
        with pytest.raises(fxp.FxpError, match="overlap"):
            fxp.kv_attention(c.dq, c.cache, c.tab, scale=c.scale, out=room.as_strided((3, 4, 16), strides + (1,)))
    want = c.want()
    for strides in ((64, 16), (16, 48), (80, 20), (70, 17)):
        c.check(fxp.kv_attention(c.dq, c.cache, c.tab, scale=c.scale, out=room.as_strided((3, 4, 16), strides + (1,))), want=want)


def test_attention_in_place(fxp):
    """out may be q: every row of q is read before its output is written, by whichever workgroups share it."""
    say("kv_attention into q")
    for lens, news, QH, H, D in (([4000, 70], [1, 2], 8, 2, 64), ([300, 140], [150, 140], 48, 48, 128)):
        c = Case(fxp, lens, news, QH, H, D, "bf16")
        want, q = fxp.kv_attention(c.dq, c.cache, c.tab, scale=c.scale), c.dq.clone()
        assert torch.equal(fxp.kv_attention(q, c.cache, c.tab, scale=c.scale, out=q), want)


def test_attention_many_requests(fxp):
    say("kv_attention, 600 requests, most of them short")
    rng = np.random.default_rng(3)
    lens = rng.integers(0, 40, 600)
    lens[::100] = 600
    c = Case(fxp, lens.tolist(), np.minimum(rng.integers(0, 3, 600), 2).tolist(), 2, 2, 16, "fp32")
    c.check(fxp.kv_attention(c.dq, c.cache, c.tab, scale=c.scale))


def test_attention_from_a_graph_and_on_another_stream(fxp):
    say("kv_attention captured, replayed with other lengths")
    c = Case(fxp, [700, 64, 5], [1, 1, 1], 8, 4, 128, "fp16")
    buf = fxp.AttentionBuffers(3, 3, 8, c.cache)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out = fxp.kv_attention(c.dq, c.cache, c.tab, buf, scale=c.scale)
    side.synchronize()
    c.check(out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = fxp.kv_attention(c.dq, c.cache, c.tab, buf, scale=c.scale)
    for lens in ([700, 64, 5], [1, 2, 3], [320, 0, 5], [700, 64, 5]):
        c.lens = np.array(lens)
        c.tab.lens_after.copy_(torch.tensor(lens, dtype=torch.int32))
        out.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        c.check(out)
        assert torch.equal(out, fxp.kv_attention(c.dq, c.cache, c.tab, scale=c.scale))


def test_attention_answers_alike_every_time(fxp):
    say("kv_attention, twenty calls")
    c = Case(fxp, [5000, 900], [1, 3], 16, 2, 128, "bf16")
    want = fxp.kv_attention(c.dq, c.cache, c.tab, scale=c.scale)
    for _ in range(20):
        assert torch.equal(fxp.kv_attention(c.dq, c.cache, c.tab, scale=c.scale), want)


def test_attention_calls_of_many_sizes_take_turns_with_one_workspace(fxp):
    """What one call left behind the tickets is no ticket of the next: other numbers of tiles, other dims, other types."""
    say("kv_attention, one workspace, many sizes")
    cases = [Case(fxp, [3000], [1], 2, 1, 256, "fp32"), Case(fxp, [2000, 900, 640], [3, 1, 2], 32, 4, 64, "bf16"), Case(fxp, [4000], [2], 2, 2, 16, "fp16"),
             Case(fxp, [700] * 20, [1] * 20, 16, 8, 128, "bf16"), Case(fxp, [1500], [40], 4, 4, 192, "fp32")]
    buf = fxp.AttentionBuffers(20, 40, 16, cases[0].cache)
    assert not buf.ws[:fxp.KV_TICKET_BYTES].any()
    buf.ws[fxp.KV_TICKET_BYTES:].fill_(0xff)
    for c in cases + cases[::-1]:
        c.check(fxp.kv_attention(c.dq, c.cache, c.tab, buf, scale=c.scale))
        assert not buf.ws[:fxp.KV_TICKET_BYTES].any()


@pytest.mark.parametrize("requests", [65, 200, 4200])
def test_attention_of_a_padded_batch(fxp, requests):
    """Most requests have no new tokens, some of them cached ones; one long request in front, one behind them all."""
    say("kv_attention, padded batch", requests)
    lens, news = np.zeros(requests, int), np.zeros(requests, int)
    lens[1], news[1], lens[-1], news[-1], lens[requests // 2], news[requests // 2], lens[3] = 2500, 2, 1300, 1, 64, 1, 200
    c = Case(fxp, lens.tolist(), news.tolist(), 8, 2, 64, "bf16", behind=3)
    out = torch.full((c.T, 8, 64), 9.0, dtype=c.dq.dtype, device="cuda")
    c.check(fxp.kv_attention(c.dq, c.cache, c.tab, scale=c.scale, out=out))
    assert (out[c.first[-1]:] == 9).all()


def test_attention_over_a_cache_past_32_bits(fxp):
    say("kv_attention behind 4 GiB of keys")
    c = Case(fxp, [130, 64], [1, 2], 16, 8, 256, "bf16", spare=33000)
    c.check(fxp.kv_attention(c.dq, c.cache, c.tab, scale=c.scale))


def test_attention_of_rows_that_are_not_finite(fxp):
    """As everywhere in the library: NaN maps to 0, Inf to the largest magnitude; other rows are not touched by it."""
    say("kv_attention, Inf and NaN in q, the largest scales in the cache")
    c = Case(fxp, [100, 100], [1, 1], 2, 2, 64, "fp32")
    want = fxp.kv_attention(c.dq, c.cache, c.tab, scale=c.scale)
    q = c.dq.clone()
    q[0, 0, 3], q[0, 1, :] = float("inf"), float("nan")
    out = fxp.kv_attention(q, c.cache, c.tab, scale=c.scale)
    assert torch.equal(out[1], want[1]) and torch.isfinite(out).all()
    c.cache.ek.fill_(255)
    assert torch.isfinite(fxp.kv_attention(c.dq * 1e30, c.cache, c.tab, scale=c.scale)).all()


def one_large_weight(fxp, c, above):
    """Every row of c scores `above` at the first token of each request and 0 at the others; all values are 1."""
    c.cache.kq.zero_()
    c.cache.ek.fill_(127)                                     # 64 * 2^(127 - 133) = 1
    c.cache.kq[torch.tensor(c.table[:, 0]).long(), :, 0, 0] = 64
    c.cache.vq.fill_(64)
    c.cache.ev.fill_(127)
    c.dq.zero_()
    c.dq[:, :, 0] = 1
    return float(torch.tensor(above, dtype=torch.float32))


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("lens,news,QH,H,D", [([64], [1], 2, 1, 64), ([1500, 3], [1, 1], 4, 2, 64), ([900], [2], 4, 1, 160), ([257], [257], 64, 16, 16),
                                              ([300, 140], [150, 140], 48, 48, 128)])
def test_attention_to_values_of_one_is_one(fxp, kind, lens, news, QH, H, D):
    """Outputs are divided by the sum of the weights they were made with, as rounded.  An output and that sum then differ by the fp32 roundings
    of either: a page's product (three with a third digit) and its place in the sum, for up to 24 pages, the joins of eight parts and the quotient:
    fewer than 2 * (24 * 4 + 40) of 2^-24, below 2^-15.  Rounded to 8 or 11 bits, 1 less 2^-15 is 1.  `above`: 63 weights of 1.5e-5, under half
    a unit of 1/32639, so that none of them reaches the output, and of 4.6e-5, which are rounded up."""
    say("kv_attention over values of one", kind, (lens, news, QH, H, D))
    c = Case(fxp, lens, news, QH, H, D, kind)
    c.check(fxp.kv_attention(c.dq, c.cache, c.tab, scale=c.scale))
    for above in (11.1, 10.0, 0.5):
        scale = one_large_weight(fxp, c, above)
        lse = torch.empty((c.T, QH), device="cuda")
        out = fxp.kv_attention(c.dq, c.cache, c.tab, scale=scale, lse=lse).double()
        if kind == "fp32":
            assert float((out - 1).abs().max()) <= 2.0 ** -15
        else:
            assert (out == 1).all(), float((out - 1).abs().max())
        # the logarithm's sum has the weights as they are: fp32 roundings of as many terms
        seen = np.concatenate([n_all - n + 1 + np.arange(n) for n_all, n in zip(lens, news)])
        want = above + np.log1p((seen - 1) * np.exp(-above))
        assert np.abs(lse.double().cpu().numpy() - want[:, None]).max() <= 2.0 ** -15 + 2.0 ** -21 * above


def test_attention_refuses_an_output_that_is_q_in_part(fxp):
    say("kv_attention, out over a part of q")
    c = Case(fxp, [700, 20], [2, 1], 4, 2, 64, "bf16")
    room = torch.zeros((4, 4, 200), dtype=torch.bfloat16, device="cuda")
    q = room[:3, :, :64]
    q.copy_(c.dq)
    flat = room.view(-1)
    for out in (room[1:, :, :64], room[:3, :, 1:65], room[:3, :, 63:127], flat[64:64 + 3 * 256].view(3, 4, 64), flat.as_strided((3, 4, 64), (64, 192, 1)),
                q.transpose(0, 1)[:3].as_strided((3, 4, 64), (200, 800, 1))):
        with pytest.raises(fxp.FxpError):
            fxp.kv_attention(q, c.cache, c.tab, scale=c.scale, out=out)
    assert torch.equal(q, c.dq)
    want = fxp.kv_attention(q, c.cache, c.tab, scale=c.scale)
    assert torch.equal(fxp.kv_attention(q, c.cache, c.tab, scale=c.scale, out=room[:3, :, 64:128]), want)
    assert torch.equal(fxp.kv_attention(q, c.cache, c.tab, scale=c.scale, out=q), want)


# requests of many rows, some of them too long for their number of rows beside the others; lengths, new tokens, query heads, heads, dim, rows behind, window
LONG = [([6000, 3, 200, 300, 64], [40, 1, 200, 200, 40], 28, 14, 64, 0, 0), ([5000], [40], 16, 8, 64, 1001, 0), ([2500, 2600, 300], [50, 1, 300], 64, 16, 16, 0, 0),
        ([4000, 4000, 1100], [60, 33, 600], 16, 16, 80, 5, 3000), ([200, 5000, 40], [200, 40, 40], 96, 24, 128, 0, 0), ([3000, 90], [70, 90], 66, 66, 160, 0, 0)]


@pytest.mark.parametrize("lens,news,QH,H,D,behind,window", LONG)
@pytest.mark.parametrize("kind", list(TYPES))
def test_attention_of_prompts_beside_long_contexts(fxp, lens, news, QH, H, D, behind, window, kind):
    say("kv_attention of many rows, long contexts among them", (lens, news, QH, H, D, behind, window, kind))
    c = Case(fxp, lens, news, QH, H, D, kind, behind=behind)
    out, lse = torch.full((c.T, QH, D), 9.0, dtype=c.dq.dtype, device="cuda"), torch.full((c.T, QH), 9.0, device="cuda")
    buf = fxp.AttentionBuffers(len(lens), c.T, QH, c.cache)
    for _ in range(2):
        fxp.kv_attention(c.dq, c.cache, c.tab, buf, scale=c.scale, window=window, out=out, lse=lse)
    c.check(out, lse, window)
    assert (out[c.first[-1]:] == 9).all() and (lse[c.first[-1]:] == 9).all() and not buf.ws[:fxp.KV_TICKET_BYTES].any()


def test_attention_to_one_long_context_is_spread_out_whatever_else_is_in_the_step(fxp):
    """22 requests of 40 rows, 131000 tokens in one of them: one page after the other, eight workgroups take 25 times as long as all for it and for the
    rest apart; 4 times is the limit here."""
    say("kv_attention, a long context among short ones, timed")
    H, QH, D, long_, short = 8, 64, 64, 131000, 500
    rng = np.random.default_rng(0)
    i8 = lambda *shape: dev(rng.integers(-100, 101, shape).astype(np.int8))  # noqa: E731
    ones = lambda: torch.full((100, H), 127, dtype=torch.int32, device="cuda")  # noqa: E731
    cache = fxp.KvCache.of(i8(100, H, 64, D), i8(100, H, 4, D, 16), ones(), ones())

    def time_of(lens):
        tab = fxp.KvTables(len(lens), -(-max(lens) // 64), 5 * len(lens), 100, in_place=False)
        tab.block_table.copy_(torch.tensor(rng.integers(0, 100, tab.block_table.shape)))
        tab.lens_after.copy_(torch.tensor(lens))
        tab.first.copy_(torch.arange(0, 5 * len(lens) + 1, 5))
        q = torch.randn((tab.tokens, QH, D), device="cuda").bfloat16()
        buf, out, best = fxp.AttentionBuffers(len(lens), tab.tokens, QH, cache), torch.empty_like(q), float("inf")
        for _ in range(6):
            begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            begin.record()
            for _ in range(3):
                fxp.kv_attention(q, cache, tab, buf, out=out)
            end.record()
            end.synchronize()
            best = min(best, begin.elapsed_time(end))
        return best

    apart = time_of([long_]) + time_of([short] * 21)
    together = time_of([short] * 9 + [long_] + [short] * 12)
    assert together < 4 * apart, (together, apart)


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
def test_attention_of_more_than_64_pages_a_wave(fxp, kind):
    """32 heads of 5000 pages: a workgroup's share is 313 pages, 79 of them one wave's, whose numbers it loads 64 at a time."""
    say("kv_attention over 320000 tokens", kind)
    c, rng = Case(fxp, [640], [1], 32, 32, 16, kind), np.random.default_rng(2)
    c.lens, c.table = np.array([5000 * 64 - 5]), rng.integers(0, 10, (1, 5000)).astype(np.int32)
    c.table[0, rng.integers(0, 5000, 40)] = -1
    c.tab = fxp.KvTables(1, 5000, 1, 4, in_place=False)
    for mine, theirs in ((c.tab.block_table, c.table), (c.tab.lens_after, c.lens), (c.tab.first, c.first)):
        mine.copy_(torch.tensor(theirs.astype(np.int32)))
    lse = torch.empty((1, 32), device="cuda")
    c.check(fxp.kv_attention(c.dq, c.cache, c.tab, scale=c.scale, lse=lse), lse)


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
@pytest.mark.parametrize("lens,news,QH,H,D", [([1500], [1], 4, 2, 64), ([257], [257], 64, 16, 16)])
def test_attention_to_the_largest_values(fxp, kind, lens, news, QH, H, D):
    """Values times the tokens seen up to 2^119: outputs before the division hold up to 2^8 of them, the lag of the scores' reference."""
    say("kv_attention to values near 2^108", kind, (lens, news, QH, H, D))
    c = Case(fxp, lens, news, QH, H, D, kind, sharp=20.0)
    ev = np.full(c.v.e.shape, 108 + 126)                      # below 2^108, times 1500
    c.v.e, c.cache.ev[:] = ev, 108 + 126
    out = fxp.kv_attention(c.dq, c.cache, c.tab, scale=c.scale)
    assert torch.isfinite(out).all()
    c.check(out)
