"""The serving operators together, as a decoder uses them: prompts, then single tokens, through two layers that share the tables,
a projection in 4 bits before and after the attention; against the same steps in 64 bits on the values the calls themselves stored."""
import numpy as np
import pytest

from tests import serve_ref as ref
from tests.gpu_util import host, say

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
WIDTH, QH, H, D, LAYERS = 96, 6, 2, 32, 2


@pytest.fixture(scope="module")
def fxp():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: there is no CPU path in libfxp")
    from paper_2207_08822_amd import fxp as binding
    binding.lib()
    return binding


class Model:
    def __init__(self, fxp, requests, blocks, pages):
        torch.manual_seed(0)
        self.fxp, self.tab_of = fxp, {}
        self.caches = [fxp.KvCache(pages, H, D) for _ in range(LAYERS)]
        self.into = [fxp.pack4(torch.randn((WIDTH, (QH + 2 * H) * D), device="cuda") * WIDTH ** -0.5) for _ in range(LAYERS)]
        self.out = [fxp.pack4(torch.randn((QH * D, WIDTH), device="cuda") * (QH * D) ** -0.5, 32) for _ in range(LAYERS)]

    def step(self, x, n_new, tab, seen=None):
        """One pass over the rows x; `seen` receives what each layer computed."""
        fxp = self.fxp
        fxp.kv_tables(n_new, tab)
        for cache, into, out in zip(self.caches, self.into, self.out):
            qkv = fxp.linear4(x, into).unflatten(1, (QH + 2 * H, D))
            fxp.kv_append(qkv[:, QH:QH + H], qkv[:, QH + H:], cache, tab.runs)
            o = fxp.kv_attention(qkv[:, :QH], cache, tab)
            y = fxp.linear4(o.flatten(1), out)
            if seen is not None:
                seen.append((x, qkv, o, y))
            x = x + y
        return x


def check_step(model, tab, seen, caches):
    """Attention of each layer within its bound, on the cache that its own tokens make in 64 bits."""
    runs, rows = host(tab.runs), int(tab.first[-1])
    for layer, (x, qkv, o, y) in enumerate(seen):
        k, v = caches[layer]
        k.append(qkv[:, QH:QH + H].double().cpu().numpy(), runs)
        v.append(qkv[:, QH + H:].double().cpu().numpy(), runs)
        assert np.array_equal(host(model.caches[layer].ek), k.e)
        want, _, off = ref.attention(qkv[:, :QH].double().cpu().numpy(), k.values(), v.values(), host(tab.first), host(tab.lens_after),
                                     host(tab.block_table), float(np.float32(D ** -0.5)), 0, 15, 2.0 ** -8)
        assert (np.abs(o.double().cpu().numpy() - want)[:rows] <= off[:rows]).all()
        for a, w, b in ((x, model.into[layer], qkv.flatten(1)), (o.flatten(1), model.out[layer], y)):
            q, unit = ref.unpack4(host(w.packed), host(w.scales), w.K, w.N, w.group)
            a, b = a.double().cpu().numpy()[:rows], b.double().cpu().numpy()[:rows]
            mass = np.abs(a) @ np.abs(q * unit)
            # a group's elements are off by at most 2^-15 of the group's largest, and so by that of the row's
            inner = 2.0 ** -15 * np.abs(a).max(1, keepdims=True) * np.abs(q * unit).sum(0) + 2.0 ** -20 * mass
            assert (np.abs(b - a @ (q * unit)) <= 2.0 ** -8 * (np.abs(a @ (q * unit)) + inner) + inner).all()


def test_prompts_then_tokens(fxp):
    say("prompts of 5 requests, 12 single tokens each, one request refused on the way")
    B, blocks, pages = 5, 4, 12
    model = Model(fxp, B, blocks, pages)
    rng = np.random.default_rng(0)
    lens, news = torch.zeros(B, dtype=torch.int32, device="cuda"), np.array([130, 0, 63, 1, 70])
    prompt = fxp.KvTables(B, blocks, int(news.sum()), pages)
    for t in prompt.block_table, prompt.lens:
        assert t.is_cuda
    fresh = lambda: [(ref.Cache(np.zeros((pages, H, 64, D)), np.ones((pages, H)), 8), ref.Cache(np.zeros((pages, H, 64, D)), np.ones((pages, H)), 8))  # noqa: E731
                     for _ in range(LAYERS)]
    caches, seen = fresh(), []
    x = torch.randn((prompt.tokens, WIDTH), device="cuda").bfloat16()
    model.step(x, torch.tensor(news, dtype=torch.int32, device="cuda"), prompt, seen)
    check_step(model, prompt, seen, caches)
    assert host(prompt.lens).tolist() == news.tolist() and int(prompt.n_free) == pages - 7

    decode = fxp.KvTables(B, blocks, B, pages)
    for name in ("block_table", "lens", "free", "n_free"):
        getattr(decode, name).copy_(getattr(prompt, name))
    one = torch.ones(B, dtype=torch.int32, device="cuda")
    for step in range(3):
        seen = []
        model.step(torch.randn((B, WIDTH), device="cuda").bfloat16(), one, decode, seen)
        check_step(model, decode, seen, caches)
    assert not host(decode.refused).any()

    # the same step from a graph, replayed with new tokens; eager work and a synchronization between the replays
    x, graph, seen = torch.zeros((B, WIDTH), device="cuda").bfloat16(), torch.cuda.CUDAGraph(), []
    with torch.cuda.graph(graph):
        y = model.step(x, one, decode, seen)
    for step in range(6):
        x.copy_(torch.randn((B, WIDTH), device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        check_step(model, decode, seen, caches)
        assert host(decode.lens).tolist() == (news + 4 + step).tolist()
    # no pages left: the request that needs one is refused and the others go on
    decode.n_free.zero_()
    decode.lens.copy_(torch.tensor([128, 9, 72, 10, 79], dtype=torch.int32))
    graph.replay()
    assert host(decode.refused).tolist() == [1, 0, 0, 0, 0] and host(decode.lens).tolist() == [128, 10, 73, 11, 80]
    assert torch.isfinite(y).all()


def test_the_same_answer_in_one_prompt_and_token_by_token(fxp):
    """A prompt's last row sees the cache as it is after the whole prompt; token by token the last row sees the same tokens, mapped
    under scales that grew step by step: the two differ by roundings of 8-bit mantissas, half a unit (2^-7 of the block's binade) each time."""
    say("a prompt at once and token by token, values of one binade")
    n, H1, D1 = 70, 2, 32
    torch.manual_seed(3)
    k, v, q = ((torch.rand((n, H1, D1), device="cuda") + 1) * torch.randint(0, 2, (n, H1, D1), device="cuda").mul(2).sub(1) for _ in range(3))
    at_once, in_steps = fxp.KvCache(4, H1, D1), fxp.KvCache(4, H1, D1)
    tab = fxp.KvTables(1, 2, n, 4)
    fxp.kv_tables(torch.tensor([n], dtype=torch.int32, device="cuda"), tab)
    fxp.kv_append(k, v, at_once, tab.runs)
    whole = fxp.kv_attention(q, at_once, tab)
    tab = fxp.KvTables(1, 2, 1, 4)
    one = torch.ones(1, dtype=torch.int32, device="cuda")
    for i in range(n):
        fxp.kv_tables(one, tab)
        fxp.kv_append(k[i:i + 1], v[i:i + 1], in_steps, tab.runs)
        row = fxp.kv_attention(q[i:i + 1], in_steps, tab)
        # all magnitudes lie in [1, 2): every block has the same scale from its first token on, and both sides are within
        # 64 * 0.5 / 8355711 of a largest value of 2
        assert float((row - whole[i]).abs().max()) <= 2.0 ** -16
    k1, v1 = fxp.kv_load(at_once, torch.tensor([[0, 64, 0, 0], [64, 6, 1, 0]], dtype=torch.int32, device="cuda"), n)
    k2, v2 = fxp.kv_load(in_steps, torch.tensor([[0, 64, 0, 0], [64, 6, 1, 0]], dtype=torch.int32, device="cuda"), n)
    assert torch.equal(k1, k2) and torch.equal(v1, v2)


def test_what_lies_on_another_device_is_refused(fxp):
    """Pointers of another device than the current one, whose stream the calls use, must not reach a kernel."""
    say("caches, tables, buffers and weights marked as another device's")
    cache, tab, w = fxp.KvCache(4, H, D), fxp.KvTables(2, 2, 2, 4), fxp.pack4(torch.randn((D, 16), device="cuda"))
    buf, q, n_new = fxp.AttentionBuffers(2, 2, QH, cache), torch.zeros((2, QH, D), device="cuda"), torch.ones(2, dtype=torch.int32, device="cuda")
    calls = [(tab, lambda: fxp.kv_tables(n_new, tab)), (cache, lambda: fxp.kv_append(q[:, :H], q[:, :H], cache, tab.runs)),
             (cache, lambda: fxp.kv_load(cache, tab.runs, 2)), (w, lambda: fxp.linear4(q[:, 0], w))]
    calls += [(x, lambda: fxp.kv_attention(q, cache, tab, buf)) for x in (cache, tab, buf)]
    for owner, call in calls:
        call()
        owner.index += 1
        with pytest.raises(fxp.FxpError, match="another device"):
            call()
        owner.index -= 1
    with pytest.raises(fxp.FxpError, match="dtype"):
        fxp.kv_load(cache, tab.runs, 2, dtype=torch.int8)
    torch.cuda.synchronize()
