"""The operators together, as a decoder block uses them: a prompt and then single tokens through 4-bit products, the writer that turns queries and keys, and attention; and
a block's training step with the rotation's gradient between the products'.  Each against 64 bits, fed with what the calls themselves stored."""
import numpy as np
import pytest

from tests import mx4_ref, rotary_ref
from tests.gpu_util import dev, host, say

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def fxp():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: there is no CPU path in libfxp")
    from paper_2207_08822_amd import fxp as binding
    binding.lib()
    return binding


def four(x, word=None):
    return mx4_ref.values(*mx4_ref.encode(x, word))


def product_bound(a, b, want, eps):
    """K sums, each cut by at most 2^-23 of the magnitudes' sum, and the type's rounding."""
    return np.abs(a) @ np.abs(b) * (a.shape[1] * 2.0 ** -23) + np.abs(want) * eps / 2 * 1.01 + 2.0 ** -126


@pytest.mark.parametrize("near", [False, True])
def test_serving(fxp, near):
    say("prompt and single tokens", near)
    WIDTH, QH, H, D = 200, 6, 2, 32
    rng = np.random.default_rng(3)
    W, V = rng.standard_normal((WIDTH, (QH + 2 * H) * D)) * WIDTH ** -0.5, rng.standard_normal((QH * D, WIDTH)) * (QH * D) ** -0.5
    into, out = (fxp.mx4_map(torch.tensor(m, dtype=torch.float32, device="cuda"), rounding=fxp.NEAREST, want_q=False, want_qT=True)[1] for m in (W, V))
    into64, out64 = host(fxp.mx4_unmap(into).double()).T, host(fxp.mx4_unmap(out).double()).T
    assert np.array_equal(into64, four(W.astype(np.float32).astype(np.float64).T).T)
    rope = fxp.Rotary(D, interleaved=near)
    cache = fxp.KvCache(12, H, D)
    kept = {b: [] for b in range(3)}           # places of each request's tokens
    tabs = {}

    def tables(tokens):
        """Tables of a step of `tokens` rows that go on with the first one's requests."""
        if tokens not in tabs:
            tabs[tokens] = tab = fxp.KvTables(3, 4, tokens, 12)
            if len(tabs) > 1:
                for name in ("block_table", "lens", "free", "n_free"):
                    getattr(tab, name).copy_(getattr(last[0], name))
        last[:] = [tabs[tokens]]
        return tabs[tokens]

    last = []
    for n_new in ([70, 0, 5], [1, 3, 0], [1, 1, 1], [1, 1, 1]):
        T = sum(n_new)
        tab = tables(T)
        x = torch.tensor(rng.standard_normal((T, WIDTH)), dtype=torch.float32, device="cuda")
        fxp.kv_tables(dev(np.array(n_new, np.int32)), tab)
        qkv = fxp.mx4_linear(x, into)
        x64 = four(host(x.double()))
        want = x64 @ into64
        assert np.all(np.abs(host(qkv.double()) - want) <= product_bound(x64, into64, want, 2.0 ** -23))
        parts = qkv.unflatten(1, (QH + 2 * H, D))
        q, k, v = parts[:, :QH], parts[:, QH:QH + H], parts[:, QH + H:]
        positions = host(tab.positions)
        q_want = rotary_ref.turn(host(q.double()), positions, rope)
        q_before = host(q.double())
        q = fxp.kv_append_rotary(k, v, cache, tab, rope, q=q, out=q)
        assert rotary_ref.within(host(q.double()), q_want, q_before, rope, 2.0 ** -23)
        t = 0
        for b, n in enumerate(n_new):
            kept[b] += host(tab.slots)[t:t + n].tolist()
            t += n
        # the new keys as they are stored: turned, then at most a step of their page from what they were
        runs = host(tab.runs)
        kl, vl = fxp.kv_load(cache, tab.runs, T)
        k_want = rotary_ref.turn(host(k.double()), positions, rope)
        e = host(cache.ek)
        step = np.zeros((T, H, 1))
        for first, count, page, _ in runs.tolist():
            step[first:first + count] = 2.0 ** (e[page] - 133.0)[:, None]
        assert np.all(np.abs(host(kl.double()) - k_want) <= step)
        o = fxp.kv_attention(q, cache, tab)
        o_want, t = np.zeros((T, QH, D)), 0
        ks = host(cache.kq).astype(np.float64) * 2.0 ** (host(cache.ek) - 133.0)[:, :, None, None]
        vs = host(cache.vq).transpose(0, 1, 2, 4, 3).reshape(12, H, 64, D) * 2.0 ** (host(cache.ev) - 133.0)[:, :, None, None]
        for b, n in enumerate(n_new):
            at = np.array(kept[b], int)
            for i in range(n):
                seen = at[:len(at) - n + i + 1]
                for h in range(QH):
                    kk, vv = ks[seen // 64, h // (QH // H), seen % 64], vs[seen // 64, h // (QH // H), seen % 64]
                    a = kk @ host(q.double())[t + i, h] * D ** -0.5
                    w = np.exp(a - a.max())
                    o_want[t + i, h] = w @ vv / w.sum()
            t += n
        # rows and weights in 23 bits, sums of fp32 over at most 73 tokens: far below 2^-14 of the values, which stay below 8
        assert np.abs(host(o.double()) - o_want).max() < 8 * 2.0 ** -14
        y = fxp.mx4_linear(o.flatten(1), out)
        o64 = four(host(o.flatten(1).double()))
        want = o64 @ out64
        assert np.all(np.abs(host(y.double()) - want) <= product_bound(o64, out64, want, 2.0 ** -23))


def test_training(fxp):
    """Queries and keys of a projection, turned, and back: Y = X W, Z = turned(Y), a loss with gradient dZ; dX and dW are the products' of turned-back dZ."""
    say("projection, rotation and their gradients")
    B, S, H, D, WIDTH = 2, 37, 3, 32, 96
    rng = np.random.default_rng(4)
    M, N = B * S, H * D
    X, W, dZ = (torch.tensor(rng.standard_normal(s), dtype=torch.float32, device="cuda") for s in ((M, WIDTH), (WIDTH, N), (B, S, H, D)))
    rope, positions = fxp.Rotary(D, interleaved=True), torch.arange(S, dtype=torch.int32, device="cuda")
    buf = fxp.Mx4LayerBuffers(M, WIDTH, N)
    Y = fxp.mx4_linear_fwd(X, W, buf, seed=6, step=2).view(B, S, H, D)
    Z = fxp.rotary(Y, positions, rope)
    places = np.broadcast_to(np.arange(S), (B, S))
    assert rotary_ref.within(host(Z.double()), rotary_ref.turn(host(Y.double()), places, rope), host(Y.double()), rope, 2.0 ** -23)
    dY = fxp.rotary_bwd(dZ, positions, rope)
    assert rotary_ref.within(host(dY.double()), rotary_ref.turn(host(dZ.double()), places, rope, True), host(dZ.double()), rope, 2.0 ** -23)
    dX, dW = fxp.mx4_linear_bwd(dY.view(M, N), buf, seed=6, step=2)
    words = [mx4_ref.words(*s, 6, (2 << 8) | tag) for tag, s in enumerate(((M, WIDTH), (WIDTH, N), (M, N)))]
    x, w, g = (host(t.double()) for t in (X, W, dY.view(M, N)))
    for got, a, b in ((Y.view(M, N), four(x, words[0]), four(w.T, words[1].T).T), (dX, four(g, words[2]), four(w, words[1]).T), (dW, four(x.T, words[0].T), four(g.T, words[2].T).T)):
        want = a @ b
        assert np.all(np.abs(host(got.double()) - want) <= product_bound(a, b, want, 2.0 ** -23))
