"""The serving entry points validate their arguments on the host, before anything touches a device."""
import ctypes as c

import pytest

from paper_2207_08822_amd import fxp
from tests.test_abi import load

BIG = 1 << 20          # an address that is never dereferenced: every call below fails validation or has nothing to do


@pytest.fixture(scope="module")
def L():
    load()
    return fxp.lib()


def cache(**over):
    a = dict(kq=BIG, vq=BIG, ek=BIG, ev=BIG, pages=10, heads=2, dim=64, bits=8) | over
    return c.byref(fxp._KvCache(*[a[n] for n, _ in fxp._KvCache._fields_]))


def step(**over):
    a = dict(requests=3, blocks=4, tokens=5, pages=6) | over
    return c.byref(fxp._KvStep(*[a.get(n, BIG) for n, _ in fxp._KvStep._fields_]))


def test_most_runs(L):
    assert [L.fxp_kv_max_runs(b, t) for b, t in ((1, 1), (1, 64), (1, 66), (256, 256), (2, 200), (-1, 4), (1, 1 << 31))] == [1, 2, 3, 256, 7, 0, 0]


def test_tables(L):
    f = L.fxp_kv_tables
    assert f(None, BIG, None, 0, None) == -1 and f(step(), None, None, 0, None) == -1
    for name in ("requests", "blocks", "tokens", "pages"):
        assert f(step(**{name: -1}), BIG, None, 0, None) == -2 and f(step(**{name: 1 << 31}), BIG, None, 0, None) == -2
    for name in ("lens", "free_pages", "n_free", "block_table", "lens_after", "n_free_after", "first", "slots", "positions", "runs", "refused"):
        assert f(step(**{name: None}), BIG, None, 0, None) == -1, name
        assert f(step(**{name: BIG + 2}), BIG, None, 0, None) == -3, name
    assert f(step(runs=BIG + 4), BIG, None, 0, None) == -3 and f(step(slots=BIG + 4), BIG, None, 0, None) == -3
    # lengths updated in place need the workspace
    assert f(step(), BIG, None, 0, None) == -4 and f(step(), BIG, BIG, 255, None) == -4 and f(step(n_free_after=2 * BIG), BIG, None, 0, None) == -4
    assert f(step(), BIG, BIG + 1, 256, None) == -3


def test_append_and_load(L):
    def append(ca=cache(), type=1, k=BIG, kt=128, kh=64, v=BIG, vt=128, vh=64, tokens=4, runs=BIG, n=4):
        return L.fxp_kv_append(ca, type, k, kt, kh, v, vt, vh, tokens, runs, n, None)

    def load_(ca=cache(), type=1, k=BIG, v=BIG, tokens=4, runs=BIG, n=4):
        return L.fxp_kv_load(ca, type, k, v, tokens, runs, n, None)

    for f in append, load_:
        for over, rc in ((dict(kq=None), -1), (dict(ev=None), -1), (dict(pages=0), -2), (dict(pages=1 << 31), -2), (dict(heads=0), -2),
                         (dict(heads=65536), -2), (dict(dim=24), -2), (dict(dim=272), -2), (dict(dim=0), -2), (dict(bits=1), -6), (dict(bits=9), -6),
                         (dict(kq=BIG + 8), -3), (dict(ek=BIG + 2), -3)):
            assert f(ca=cache(**over)) == rc, over
        assert f(ca=None) == -1 and f(type=3) == -9 and f(type=-1) == -9 and f(tokens=-1) == -2 and f(n=-1) == -2 and f(n=1 << 24) == -2
        assert f(k=None) == -1 and f(v=None) == -1 and f(runs=None) == -1 and f(runs=BIG + 4) == -3 and f(k=BIG + 1) == -3
        assert f(tokens=0) == 0 and f(n=0) == 0                                      # nothing to do
    assert append(kt=-1) == -2 and append(vh=-64) == -2 and append(v=BIG + 2, type=0) == -3


def test_attention(L):
    need = L.fxp_kv_attention_workspace_bytes
    assert need(3, 5, 4, 2, 64) > 0
    assert [need(*a) for a in ((0, 5, 4, 2, 64), (3, -1, 4, 2, 64), (3, 5, 3, 2, 64), (3, 5, 4, 2, 40), (3, 5, 4, 0, 64), (3, 1 << 30, 4, 2, 64))] == [0] * 6

    def f(ca=cache(), st=step(), type=1, q=BIG, qt=256, qh=64, heads=4, scale=0.125, window=0, out=BIG, ot=256, oh=64, lse=None, ws=BIG, n=1 << 30):
        return L.fxp_kv_attention(ca, st, type, q, qt, qh, heads, scale, window, out, ot, oh, lse, ws, n, None)

    assert f(ca=None) == -1 and f(st=None) == -1 and f(ca=cache(dim=20)) == -2 and f(type=7) == -9
    assert f(heads=3) == -2 and f(heads=0) == -2 and f(window=-1) == -2 and f(qt=-1) == -2 and f(oh=-1) == -2
    assert f(st=step(requests=0)) == -2 and f(st=step(blocks=0)) == -2 and f(st=step(blocks=1 << 25)) == -2 and f(st=step(tokens=1 << 30)) == -2
    for scale in (0.0, -1.0, float("nan"), float("inf"), 2.0 ** 64):
        assert f(scale=scale) == -10
    assert f(q=None) == -1 and f(out=None) == -1 and f(q=BIG + 1) == -3 and f(out=BIG + 1) == -3 and f(lse=BIG + 2) == -3
    for name in ("first", "lens_after", "block_table"):
        assert f(st=step(**{name: None})) == -1 and f(st=step(**{name: BIG + 2})) == -3
    assert f(ws=None) == -4 and f(n=need(3, 5, 4, 2, 64) - 1) == -4 and f(ws=BIG + 128) == -3
    assert f(st=step(tokens=0)) == 0


def test_w4(L):
    assert L.fxp_w4_packed_bytes(128, 16) == 1024 and L.fxp_w4_packed_bytes(129, 17) == 4096 and L.fxp_w4_packed_bytes(0, 4) == 0
    assert L.fxp_w4_packed_bytes((1 << 20) + 1, 4) == 0 and L.fxp_w4_packed_bytes(4, (1 << 24) + 1) == 0
    assert [L.fxp_w4_scale_bytes(129, 17, g) for g in (32, 64, 128, 16, 256)] == [256, 128, 64, 0, 0]
    need = L.fxp_w4_workspace_bytes
    assert need(0, 4, 300, 64) > 0 and need(3, 4, 300, 64) == 0 and need(1, 0, 300, 64) == 0 and need(1, 4, 300, 48) == 0

    def pack(type=0, W=BIG, ldw=20, K=10, N=20, group=64, packed=BIG, scales=BIG):
        return L.fxp_w4_pack(type, W, ldw, K, N, group, packed, scales, None)

    assert pack(type=4) == -9 and pack(group=16) == -10 and pack(ldw=19) == -2 and pack(K=0) == -2 and pack(N=0) == -2
    assert pack(W=None) == -1 and pack(packed=None) == -1 and pack(scales=None) == -1
    assert pack(W=BIG + 2) == -3 and pack(packed=BIG + 4) == -3 and pack(scales=BIG + 1) == -3

    def linear(type=1, X=BIG, ldx=300, M=4, K=300, N=20, packed=BIG, scales=BIG, group=64, Y=BIG, ldy=20, ws=BIG, n=1 << 30):
        return L.fxp_w4_linear(type, X, ldx, M, K, N, packed, scales, group, Y, ldy, ws, n, None)

    assert linear(type=4) == -9 and linear(group=0) == -10 and linear(ldx=299) == -2 and linear(ldy=19) == -2 and linear(M=-1) == -2
    assert linear(M=1 << 20) == -2 and linear(X=None) == -1 and linear(Y=None) == -1 and linear(packed=None) == -1
    assert linear(X=BIG + 1) == -3 and linear(packed=BIG + 8) == -3 and linear(ws=None) == -4 and linear(n=need(1, 4, 300, 64) - 1) == -4
    assert linear(ws=BIG + 16) == -3 and linear(M=0) == 0
    assert fxp.lib().fxp_strerror(-9) == b"unknown element type" and fxp.lib().fxp_strerror(-10) == b"a scalar argument outside its range"


def test_the_binding_refuses_tensors_on_the_cpu():
    import torch
    with pytest.raises(fxp.FxpError):
        fxp.KvCache(2, 1, 64, device="cpu")
    with pytest.raises(fxp.FxpError):
        fxp.pack4(torch.zeros(64, 16))


def test_whether_rows_share_elements():
    """Against sets of addresses: exact for strides that are alike, never a no where elements are shared."""
    import random

    import torch
    rng = random.Random(1)
    room = torch.zeros(4000)

    def elements(t):
        return set((t.storage_offset() + sum(i * s for i, s in zip(at, t.stride()))) for at in torch.cartesian_prod(
            *[torch.arange(n) for n in t.shape]).view(-1, t.dim()).tolist())

    seen = {True: 0, False: 0}
    for trial in range(600):
        lead = [rng.choice([1, 2, 3, 5]) for _ in range(rng.choice([1, 2]))]
        strides = [[rng.choice([0, 1, 4, 7, 8, 16, 33, 100]) for _ in lead] for _ in range(2)]
        if rng.random() < 0.8:
            strides[1] = [y if n == 1 else x for x, y, n in zip(*strides, lead)]
        lasts = rng.choice([1, 3, 4, 8]), rng.choice([1, 3, 4, 8])
        a, b = (room.as_strided(lead + [m], st + [1], rng.randrange(120)) for m, st in zip(lasts, strides))
        want, got = bool(elements(a) & elements(b)), fxp._share(a, b)
        alike = all(n == 1 or x == y for n, x, y in zip(lead, *strides))
        assert got == want if alike else got or not want, (a.shape, a.stride(), a.storage_offset(), b.shape, b.stride(), b.storage_offset())
        assert got == fxp._share(b, a)
        seen[got] += 1
        if lasts[0] == lasts[1]:
            assert fxp._same_rows(a, b) == (alike and a.data_ptr() == b.data_ptr())
    assert min(seen.values()) > 100
    assert not fxp._share(room[:0], room) and not fxp._share(room.view(20, 200)[:, :0], room.view(20, 200))


def rotation(**over):
    a = dict(turns=BIG, rot=32, interleaved=0, amplitude=1.0) | over
    return c.byref(fxp._Rotation(*[a[n] for n, _ in fxp._Rotation._fields_]))


def test_rotary(L):
    def f(rot=rotation(), back=0, type=1, batch=2, tokens=4, heads=2, dim=64, x=BIG, xb=512, xt=128, xh=64, p=BIG, pb=0, y=BIG, yb=512, yt=128, yh=64):
        return L.fxp_rotary(rot, back, type, batch, tokens, heads, dim, x, xb, xt, xh, p, pb, y, yb, yt, yh, None)

    assert f(rot=None) == -1 and f(rot=rotation(turns=None)) == -1 and f(rot=rotation(turns=BIG + 4)) == -3
    for rot in (0, 1, 3, 66, -2):
        assert f(rot=rotation(rot=rot)) == -2
    assert f(rot=rotation(rot=1026), dim=2000) == -2
    for amplitude in (0.0, -1.0, float("nan"), float("inf")):
        assert f(rot=rotation(amplitude=amplitude)) == -10
    assert f(type=3) == -9 and f(batch=-1) == -2 and f(tokens=-1) == -2 and f(tokens=1 << 31) == -2 and f(heads=65536) == -2 and f(dim=65537) == -2
    assert f(xt=-1) == -2 and f(yh=-1) == -2 and f(xb=-1) == -2 and f(pb=-1) == -2 and f(yb=1 << 40) == -2 and f(batch=1 << 30, tokens=1 << 12) == -2
    assert f(x=None) == -1 and f(y=None) == -1 and f(p=None) == -1 and f(x=BIG + 1) == -3 and f(y=BIG + 1) == -3 and f(p=BIG + 2) == -3
    assert f(batch=0) == 0 and f(tokens=0) == 0 and f(heads=0) == 0


def test_append_rotary(L):
    def f(ca=cache(), st=step(), rot=rotation(), type=1, k=BIG, kt=128, kh=64, v=BIG, q=BIG, qt=256, qh=64, heads=4, out=BIG, ot=256, oh=64):
        return L.fxp_kv_append_rotary(ca, st, rot, type, k, kt, kh, v, 128, 64, q, qt, qh, heads, out, ot, oh, None)

    assert f(ca=None) == -1 and f(ca=cache(dim=24)) == -2 and f(ca=cache(bits=9)) == -6 and f(st=None) == -1 and f(rot=None) == -1
    assert f(rot=rotation(rot=66)) == -2 and f(rot=rotation(rot=33)) == -2 and f(rot=rotation(amplitude=0.0)) == -10 and f(type=4) == -9
    assert f(st=step(requests=0)) == -2 and f(st=step(tokens=-1)) == -2 and f(st=step(requests=1 << 31)) == -2 and f(st=step(tokens=1 << 30)) == -2
    assert f(heads=3) == -2 and f(heads=0) == -2 and f(heads=16386) == -2 and f(kt=-1) == -2 and f(qt=-1) == -2 and f(oh=-1) == -2
    assert f(st=step(runs=None)) == -1 and f(st=step(positions=None)) == -1 and f(k=None) == -1 and f(v=None) == -1 and f(out=None) == -1
    assert f(st=step(runs=BIG + 4)) == -3 and f(st=step(positions=BIG + 2)) == -3 and f(k=BIG + 1) == -3 and f(q=BIG + 1) == -3 and f(out=BIG + 1) == -3
    assert f(st=step(tokens=0)) == 0 and f(st=step(tokens=0), q=None, heads=0) == 0


def mx4(**over):
    a = dict(data=BIG, scales=BIG << 4, rows=5, cols=70) | over
    return c.byref(fxp._Mx4(*[a[n] for n, _ in fxp._Mx4._fields_]))


def test_mx4_sizes(L):
    assert L.fxp_mx4_data_bytes(5, 70) == 5 * 128 and L.fxp_mx4_scale_bytes(5, 70) == 5 * 8 and L.fxp_mx4_data_bytes(3, 257) == 2 * 3 * 128
    assert L.fxp_mx4_data_bytes(0, 9) == 0 and L.fxp_mx4_data_bytes(-1, 9) == 0 and L.fxp_mx4_data_bytes(9, 1 << 24) == 0


def test_mx4_map_and_unmap(L):
    def f(type=0, x=BIG, ld=70, rows=5, cols=70, q=mx4(), t=mx4(data=BIG << 1, scales=BIG << 5, rows=70, cols=5), rounding=0):
        return L.fxp_mx4_map(type, x, ld, rows, cols, q, t, 0, 0, rounding, None)

    assert f(q=None, t=None) == -1 and f(type=5) == -9 and f(rounding=2) == -5 and f(x=None) == -1 and f(x=BIG + 2) == -3 and f(ld=69) == -2
    assert f(rows=-1) == -2 and f(cols=1 << 24, ld=1 << 24) == -2 and f(q=mx4(rows=6)) == -2 and f(t=mx4()) == -2
    for same in (dict(data=BIG + 512), dict(scales=BIG + 16), dict(scales=(BIG << 4) + 32)):          # in q's bytes
        assert f(t=mx4(**(dict(data=BIG << 1, scales=BIG << 5, rows=70, cols=5) | same))) == -10
    for bad, rc in ((dict(data=None), -1), (dict(scales=None), -1), (dict(data=BIG + 8), -3), (dict(scales=BIG + 4), -3), (dict(rows=-1), -2)):
        assert f(q=mx4(**bad)) == rc and f(t=mx4(**(dict(data=BIG << 1, scales=BIG << 5, rows=70, cols=5) | bad))) == rc
        assert L.fxp_mx4_unmap(mx4(**bad), 0, BIG, 70, None) == rc
    assert L.fxp_mx4_unmap(None, 0, BIG, 70, None) == -1 and L.fxp_mx4_unmap(mx4(), 3, BIG, 70, None) == -9 and L.fxp_mx4_unmap(mx4(), 0, BIG, 69, None) == -2
    assert L.fxp_mx4_unmap(mx4(), 0, None, 70, None) == -1 and L.fxp_mx4_unmap(mx4(), 0, BIG + 2, 70, None) == -3
    assert f(x=None, rows=0, q=mx4(rows=0), t=mx4(rows=70, cols=0)) == 0 and L.fxp_mx4_unmap(mx4(rows=0, data=None), 0, None, 70, None) == 0


def test_mx4_products(L):
    def f(A=mx4(rows=4), B=mx4(rows=9), type=0, C=BIG, ldc=9, ws=None, n=0):
        return L.fxp_mx4_gemm(A, B, type, C, ldc, ws, n, None)

    assert f(A=None) == -1 and f(B=None) == -1 and f(A=mx4(data=None)) == -1 and f(type=3) == -9 and f(ldc=8) == -2 and f(A=mx4(cols=71)) == -2
    assert f(C=None) == -1 and f(C=BIG + 2) == -3 and f(A=mx4(rows=0), C=None) == 0 and f(B=mx4(rows=0), C=None) == 0
    need = L.fxp_mx4_gemm_workspace_bytes(100, 100, 10000)
    big = dict(A=mx4(rows=100, cols=10000), B=mx4(rows=100, cols=10000), ldc=100)
    assert need > 0 and f(**big) == -4 and f(**big, ws=BIG, n=need - 1) == -4 and f(**big, ws=BIG + 8, n=need) == -3
    assert L.fxp_mx4_gemm_workspace_bytes(-1, 4, 4) == 0 and L.fxp_mx4_linear_workspace_bytes(4, 4, 1 << 24) == 0 and L.fxp_mx4_layer_workspace_bytes(1, -1, 1) == 0

    assert L.fxp_mx4_linear_workspace_bytes(4, 9, 70) == 0

    def g(type=0, X=BIG, ldx=70, M=5, W=mx4(rows=9), Y=BIG, ldy=9, ws=BIG, n=1 << 20):
        return L.fxp_mx4_linear(type, X, ldx, M, W, Y, ldy, ws, n, None)

    assert g(W=None) == -1 and g(type=3) == -9 and g(X=None) == -1 and g(Y=None) == -1 and g(ldx=69) == -2 and g(ldy=8) == -2 and g(M=-1) == -2
    assert g(X=BIG + 2) == -3 and g(Y=BIG + 1) == -3 and g(ws=None) == -4 and g(n=100) == -4 and g(ws=BIG + 128) == -3 and g(M=0, X=None, Y=None, ws=None) == 0


def test_mx4_layers(L):
    M, K, N = 4, 70, 9
    shapes = dict(X=(M, K), XT=(K, M), W=(K, N), WT=(N, K), dY=(M, N), dYT=(N, M))

    def layer(**over):
        make = lambda i, n, s: fxp._Mx4(*(over.get(n) or (BIG << i, BIG << (6 + i), *s)))  # noqa: E731
        return c.byref(fxp._Mx4Layer(*[make(i, n, s) for i, (n, s) in enumerate(shapes.items())]))

    def fwd(type=0, X=BIG, W=BIG, M=M, K=K, N=N, Y=BIG, l=layer(), rounding=0, ws=BIG, n=1 << 20):
        return L.fxp_mx4_linear_fwd(type, X, W, M, K, N, Y, l, 0, 0, rounding, ws, n, None)

    def bwd(type=0, dY=BIG, l=layer(), M=M, K=K, N=N, dX=BIG, dW=BIG, rounding=0, ws=BIG, n=1 << 20):
        return L.fxp_mx4_linear_bwd(type, dY, l, M, K, N, dX, dW, 0, 0, rounding, ws, n, None)

    for f, first in ((fwd, "X"), (bwd, "dY")):
        assert f(l=None) == -1 and f(type=3) == -9 and f(rounding=2) == -5 and f(ws=None) == -4 and f(n=255) == -4 and f(ws=BIG + 16) == -3 and f(M=-1) == -2 and f(N=1 << 24) == -2
        assert f(M=M + 1) == -2 and f(**{first: None}) == -1 and f(**{first: BIG + 2}) == -3
    assert fwd(W=None) == -1 and fwd(Y=None) == -1 and fwd(Y=BIG + 2) == -3 and bwd(dX=BIG + 2) == -3 and bwd(dW=BIG + 1) == -3 and bwd(dX=None, dW=None) == 0
    for name in ("X", "WT"):
        assert fwd(l=layer(**{name: (None, None, *shapes[name])})) == -1 and fwd(l=layer(**{name: ((BIG << 21) + 8, BIG << 22, *shapes[name])})) == -3
    assert fwd(l=layer(W=(BIG, BIG << 20, *shapes["W"]))) == -10 and bwd(l=layer(dYT=(BIG << 2, BIG << 20, *shapes["dYT"]))) == -10          # two in one place
    for name in ("dY", "W", "dYT", "XT"):
        assert bwd(l=layer(**{name: (None, None, *shapes[name])})) == -1 and bwd(l=layer(**{name: (BIG << 21, (BIG << 22) + 4, *shapes[name])})) == -3
