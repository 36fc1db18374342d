"""What is measured of the operators of a decoder block with rotary positions whose products run in microscaled 4-bit floating point: the
rotation and its gradient (fxp.rotary, fxp.rotary_bwd), the cache's writer with the rotation on the way (fxp.kv_append_rotary), the mapping to 4 bits and its
inverse (fxp.mx4_map, fxp.mx4_unmap), the product of floating rows with mapped weights (fxp.mx4_linear) and a layer's training step
(fxp.mx4_linear_fwd, fxp.mx4_linear_bwd).

Rotation: pair i of `rot / 2` at position p turns by p * f_i, f_i = base^(-2 i / rot), stretched for long contexts where a case says so.  Pairs are
neighbouring elements or elements rot / 2 apart; elements from `rot` on stay.

4-bit numbers: 32 elements along the contraction share a scale 2^(s - 127), the smallest under which the largest of them is at most 6; an element is
a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6.  Rounding is to nearest, ties to even, or stochastic: up where the top 22 bits of the element's
random word are less than the 22 bits that are cut off.  Element i has word i mod 4 of block i / 4 of a Philox4x32-10 stream.
A mapped matrix [rows, cols] lies in panels of 256 columns, [panels, rows, 128] bytes (even elements in the low halves) with scales [panels, rows, 8],
those of the blocks 0, 2, 4, 6, 1, 3, 5, 7 of the panel; columns up to the panel's end are zeros.
"""
import math
import random

import numpy
import torch

own = False

PAGE = 64
BLOCK, PANEL = 32, 256
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
ORDER = (0, 2, 4, 6, 1, 3, 5, 7)        # blocks of a panel in the order of their scales
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BASE = 10000.0


def listed():
    return [
        # one token of one request: the heads of ViT-B (synth.WORKLOADS), fp32 as the framework's layers give them
        dict(name="rotary_one", kind="rotary", B=1, T=1, heads=12, dim=64, rot=64, near=0, order="tokens", type="fp32", far=2000, scaling="none", back=0, mix=1),
        # queries of a serving step of many prompt tokens, part of one projection's rows, contexts stretched by parts
        dict(name="rotary_chunk", kind="rotary", B=1, T=16384, heads=32, dim=128, rot=128, near=0, order="tokens", type="bf16", far=130000, scaling="parts", back=0, mix=2),
        # gradient of the rotation in training: a batch of sequences with the heads outside, as the framework's batched products take them
        dict(name="rotary_back", kind="rotary", B=64, T=197, heads=12, dim=64, rot=64, near=1, order="heads", type="fp32", far=0, scaling="none", back=1, mix=3),
        # a decode step's keys and values into the cache, and its queries: 256 running requests
        dict(name="append_decode", kind="append", B=256, lo=1, hi=4000, n_lo=1, n_hi=1, q_heads=32, heads=8, dim=128, rot=128, near=0, scaling="none", type="bf16", bits=8, mix=4),
        # chunks of prompts of odd lengths, some behind earlier chunks; half of each head is rotated
        dict(name="append_prompt", kind="append", B=7, lo=0, hi=5000, n_lo=100, n_hi=4000, q_heads=16, heads=4, dim=128, rot=64, near=1, scaling="linear", type="fp16", bits=8, mix=5),
        # the upstream gradient of a layer of ViT-B, for both of its products, rounded stochastically
        dict(name="map_gradient", kind="map", rows=12608, cols=768, type="fp32", stochastic=1, both=1),
        # a large weight matrix, for the forward and the backward product, rounded to nearest
        dict(name="map_weights", kind="map", rows=8192, cols=8192, type="bf16", stochastic=0, both=1),
        # one token through a large square layer
        dict(name="linear_vector", kind="linear", M=1, K=8192, N=8192, type="bf16"),
        # a few tokens through a layer of odd sizes
        dict(name="linear_few", kind="linear", M=37, K=4100, N=9001, type="fp16"),
        # a batch of ViT-B's tokens through its qkv layer, in fp32 as the framework's layers have them: bound by what is written
        dict(name="linear_batch", kind="linear", M=12608, K=768, N=2304, type="fp32"),
        # the large square layer
        dict(name="linear_square", kind="linear", M=8192, K=8192, N=8192, type="bf16"),
        # a training step of ViT-B's projection layer: forward, both gradients
        dict(name="step_layer", kind="step", M=12608, K=768, N=768, type="fp32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    what = rng.choice(["rotary", "rotary", "append", "append", "map", "map", "linear", "linear", "linear", "step"])
    mix = rng.randint(0, 1 << 30)
    kind = rng.choice(["fp32", "bf16", "bf16", "fp16"])
    scaling = rng.choice(["none", "none", "linear", "base", "parts"])
    if what in ("rotary", "append"):
        heads = rng.choice([1, 2, 3, 4, 8, 12])
        dim = rng.choice([16, 48, 64, 64, 80, 96, 112, 128, 128, 128, 160, 192, 256])
        rot = rng.choice([dim, dim, dim, max(2, dim // 2 // 2 * 2), max(2, dim // 4 // 2 * 2)])
        near = rng.randint(0, 1)
    if what == "rotary":
        dim += rng.choice([0, 0, 0, 1, 2])
        tokens = _log_int(rng, 1, 16384 * 32 * 128 // (heads * dim * (2 if kind == "fp32" else 1)))
        B = rng.choice([1, 1, 2, 7, 64])
        return dict(kind="rotary", B=B, T=max(1, min(tokens // B, 40000)), heads=heads * rng.choice([1, 1, 4]) if tokens < 4000 else heads, dim=dim, rot=rot, near=near,
                    order=rng.choice(["tokens", "heads"]), type=kind, far=rng.choice([0, 2000, 130000, 1000000]), scaling=scaling, back=rng.randint(0, 1), mix=mix)
    if what == "append":
        q_heads = heads * rng.choice([0, 1, 1, 2, 4, 7, 8])
        tokens = 8000 * 1024 // ((heads * 2 + q_heads) * dim)
        bits = 8 if rng.random() < 0.8 else rng.randint(4, 7)
        if rng.random() < 0.5:
            return dict(kind="append", B=_log_int(rng, 1, max(2, min(300, tokens))), lo=0, hi=_log_int(rng, 10, 4000), n_lo=1, n_hi=1, q_heads=q_heads, heads=heads, dim=dim,
                        rot=rot, near=near, scaling=scaling, type=kind, bits=bits, mix=mix)
        B = _log_int(rng, 1, 24)
        return dict(kind="append", B=B, lo=0, hi=_log_int(rng, 10, 4000), n_lo=0, n_hi=_log_int(rng, 2, max(3, min(4000, tokens // B))), q_heads=q_heads, heads=heads,
                    dim=dim, rot=rot, near=near, scaling=scaling, type=kind, bits=bits, mix=mix)
    if what == "map":
        rows = _log_int(rng, 1, 12000)
        cols = _log_int(rng, 1, min(12000, 8192 * 8192 // rows))
        if rng.random() < 0.4:
            cols = -(-cols // 32) * 32
        stochastic = rng.randint(0, 1)
        if stochastic:
            rows = max(1, min(rows, 12608 * 768 // cols))
        return dict(kind="map", rows=rows, cols=cols, type=kind, stochastic=stochastic, both=rng.randint(0, 1))
    K, N = _log_int(rng, 16, 12000), _log_int(rng, 16, 12000)
    if what == "linear":
        M = rng.choice([1, 1, 2, 7, _log_int(rng, 3, 200), _log_int(rng, 100, 12000), _log_int(rng, 100, 12000)])
        while K * N > 8192 * 8192 or M * K * N > 8192 ** 3 or M * N > 8192 * 8192:
            M, K, N = max(1, (M * 7) // 8), (K * 7) // 8, (N * 7) // 8
        return dict(kind="linear", M=M, K=K, N=N, type=kind)
    M = _log_int(rng, 16, 12000)
    while M * (K + N) + K * N > 12608 * 768 * 2:
        M, K, N = (M * 7) // 8, (K * 7) // 8, (N * 7) // 8
    return dict(kind="step", M=M, K=K, N=N, type="fp32")


def _lengths(case):
    """(tokens held before, new tokens) of each request; the first of several requests is empty or the shortest, the last the longest."""
    rng = random.Random(case["mix"])
    B, lo, hi = case["B"], case["lo"], case["hi"]
    held = [_log_int(rng, lo + 1, hi + 1) - 1 for _ in range(B)]
    new = [_log_int(rng, case["n_lo"] + 1, case["n_hi"] + 1) - 1 for _ in range(B)]
    if B > 1:
        held[0], held[-1] = lo, hi
    if sum(new) == 0:
        new[0] = max(1, case["n_lo"])
    return held, new


def _pages(n):
    return (n + PAGE - 1) // PAGE


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _runs(held, new):
    """[(first token, tokens, block of the request, offset in it, request)] of the new tokens."""
    runs, t = [], 0
    for b, (h, n) in enumerate(zip(held, new)):
        at = h
        while at < h + n:
            k = min(h + n, (at // PAGE + 1) * PAGE) - at
            runs.append((t, k, at // PAGE, at % PAGE, b))
            t, at = t + k, at + k
    return runs


def _max_runs(B, T):
    return min(T, (T + 126 * B) // PAGE)


def _pow2(n):
    """2^n in 64 bits, exactly, for whole numbers n."""
    return ((n.long() + 1023) << 52).view(torch.float64)


def _mantissas(shape, bits, g):
    """Mantissas with a bell-shaped distribution whose largest values fill the width."""
    top = 2 ** (bits - 1) - 1
    a = torch.randint(-top, top + 1, shape, dtype=torch.int8, device="cuda", generator=g)
    b = torch.randint(-top, top + 1, shape, dtype=torch.int8, device="cuda", generator=g)
    return (a >> 1) + (b >> 1)


# how contexts are stretched: arguments of fxp.Rotary
SCALINGS = {"none": {}, "linear": dict(scaling="linear", factor=4.0), "base": dict(scaling="base", factor=4.0),
            "parts": dict(scaling="parts", factor=16.0, original=8192, low=1.0, high=32.0, amplitude=1.2772588722239782)}


def _frequencies(case):
    """(angle of each pair a position, amplitude), in 64 bits."""
    how, n = SCALINGS[case["scaling"]], case["rot"]
    i = torch.arange(0, n, 2, dtype=torch.float64)
    factor = how.get("factor", 1.0)
    base = BASE * factor ** (n / (n - 2)) if case["scaling"] == "base" and n > 2 else BASE
    f = base ** (-i / n)
    if case["scaling"] == "linear":
        f = f / factor
    if case["scaling"] == "parts":
        share = ((how["original"] * f / (2 * math.pi) - how["low"]) / (how["high"] - how["low"])).clamp(0, 1)
        f = f * (share + (1 - share) / factor)
    return f.cuda(), how.get("amplitude", 1.0)


def _rope(fxp, case):
    return fxp.Rotary(case["rot"], base=BASE, interleaved=bool(case["near"]), **SCALINGS[case["scaling"]])


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    return {"rotary": _prepare_rotary, "append": _prepare_append, "map": _prepare_map, "linear": _prepare_linear, "step": _prepare_step}[case["kind"]](case, g)


def _normal(shape, g, dtype=torch.float32):
    return torch.randn(shape, device="cuda", generator=g).to(dtype)


def _prepare_rotary(case, g):
    B, T, H, D = case["B"], case["T"], case["heads"], case["dim"]
    s = dict(kind="rotary", case=case)
    if case["order"] == "heads":
        s["x"] = _normal((B, H, T, D), g, TYPES[case["type"]]).transpose(1, 2)
    else:       # part of the rows of one projection: keys and values of half as many elements beside them
        s["x"] = _normal((B, T, H * D + H // 2 * D), g, TYPES[case["type"]])[..., :H * D].unflatten(-1, (H, D))
    if case["far"]:     # tokens of several requests
        s["positions"] = torch.randint(0, case["far"], (B, T), dtype=torch.int32, device="cuda", generator=g)
    else:               # training: the same positions in every sequence
        s["positions"] = torch.arange(T, dtype=torch.int32, device="cuda")
    s["f"], s["amplitude"] = _frequencies(case)
    if own:
        from paper_2207_08822_amd import fxp
        s["fxp"], s["rope"] = fxp, _rope(fxp, case)
    return s


def _prepare_append(case, g):
    held, new = _lengths(case)
    B, T = case["B"], sum(new)
    H, Q, D, bits, dtype = case["heads"], case["q_heads"], case["dim"], case["bits"], TYPES[case["type"]]
    after = [h + n for h, n in zip(held, new)]
    pages = sum(_pages(a) for a in after) + 5
    order = torch.randperm(pages, device="cuda", generator=g).tolist()
    start = [0]
    for a in after:
        start.append(start[-1] + _pages(a))
    runs = [(t, n, order[start[b] + j], off) for t, n, j, off, b in _runs(held, new)]
    s = dict(kind="append", case=case, T=T, kq=_mantissas((pages, H, PAGE, D), bits, g), vq=_mantissas((pages, H, PAGE // 16, D, 16), bits, g),
             ek=torch.randint(127, 130, (pages, H), dtype=torch.int32, device="cuda", generator=g),
             ev=torch.randint(124, 129, (pages, H), dtype=torch.int32, device="cuda", generator=g))
    s["runs"] = _ints([list(r) for r in runs] + [[0, 0, -1, 0]] * (_max_runs(B, T) - len(runs)))
    s["positions"] = _ints([h + i for h, n in zip(held, new) for i in range(n)])
    read, t = [], 0
    for _, n, page, off in runs:            # what is read back: the tokens of every page written to
        read.append([t, off + n, page, 0])
        t += off + n
    s["read"], s["T_read"] = _ints(read), t
    # queries, keys and values are slices of one projection's output; some tokens are larger than what their page holds
    qkv = _normal((T, (Q + 2 * H) * D), g) * torch.exp2(torch.randint(-2, 3, (T, 1), device="cuda", generator=g).float())
    s["q"], s["k"], s["v"] = qkv.to(dtype).unflatten(1, (-1, D)).split((Q, H, H), 1)
    s["f"], s["amplitude"] = _frequencies(case)
    if own:
        from paper_2207_08822_amd import fxp
        s["fxp"], s["rope"], s["cache"] = fxp, _rope(fxp, case), fxp.KvCache.of(s["kq"], s["vq"], s["ek"], s["ev"], bits)
        s["tab"] = tab = fxp.KvTables(B, max(1, max(_pages(a) for a in after)), T, 1)
        tab.runs.copy_(s["runs"])
        tab.positions.copy_(s["positions"])
    return s


def _prepare_map(case, g):
    # rows and columns of very different sizes, as those of gradients and weights are
    x = _normal((case["rows"], case["cols"]), g)
    x *= torch.exp2(_normal((case["rows"], 1), g))
    x *= torch.exp2(_normal((1, case["cols"]), g))
    s = dict(kind="map", case=case, x=x.to(TYPES[case["type"]]), seed=int(torch.randint(0, 1 << 30, (1,), device="cuda", generator=g)), stream=(5 << 8) | 2)
    if own:
        from paper_2207_08822_amd import fxp
        s["fxp"] = fxp
    return s


def _prepare_linear(case, g):
    M, K, N = case["M"], case["K"], case["N"]
    panels = -(-K // PANEL)
    data = torch.randint(0, 256, (panels, N, PANEL // 2), dtype=torch.uint8, device="cuda", generator=g)
    k = torch.arange(panels * PANEL, device="cuda").view(panels, 1, PANEL // 2, 2) < K
    data &= 15 * k[..., 0].to(torch.uint8) + 240 * k[..., 1].to(torch.uint8)
    scales = torch.randint(117, 121, (panels, N, PANEL // BLOCK), dtype=torch.uint8, device="cuda", generator=g)
    # activations: a few channels far larger than the rest
    x = _normal((M, K), g) * torch.exp2(_normal((1, K), g))
    s = dict(kind="linear", case=case, x=x.to(TYPES[case["type"]]), data=data, scales=scales)
    if own:
        from paper_2207_08822_amd import fxp
        s["fxp"], s["w"] = fxp, fxp.Mx4.of(data, scales, N, K)
    return s


def _prepare_step(case, g):
    M, K, N = case["M"], case["K"], case["N"]
    dY = _normal((M, N), g) * 1e-3 * torch.exp2(_normal((M, 1), g))
    s = dict(kind="step", case=case, X=_normal((M, K), g), W=_normal((K, N), g) * 0.02, dY=dY, seed=int(torch.randint(0, 1 << 30, (1,), device="cuda", generator=g)), step=7)
    if own:
        from paper_2207_08822_amd import fxp
        s["fxp"], s["buf"] = fxp, fxp.Mx4LayerBuffers(M, K, N)
    return s


def run(s):
    if own:
        return _own(s)
    return {"rotary": _rotary, "append": _append, "map": _map, "linear": _linear, "step": _step}[s["kind"]](s)


def _own(s):
    fxp, case = s["fxp"], s["case"]
    if s["kind"] == "rotary":
        return dict(y=(fxp.rotary_bwd if case["back"] else fxp.rotary)(s["x"], s["positions"], s["rope"]))
    if s["kind"] == "append":
        q = fxp.kv_append_rotary(s["k"], s["v"], s["cache"], s["tab"], s["rope"], q=s["q"] if case["q_heads"] else None)
        k, v = fxp.kv_load(s["cache"], s["read"], s["T_read"])
        out = dict(k=k, v=v, ek=s["ek"], ev=s["ev"])
        return dict(out, q=q) if case["q_heads"] else out
    if s["kind"] == "map":
        rounding = fxp.STOCHASTIC if case["stochastic"] else fxp.NEAREST
        q, qT = fxp.mx4_map(s["x"], seed=s["seed"], stream_id=s["stream"], rounding=rounding, want_qT=bool(case["both"]))
        out = dict(q=fxp.mx4_unmap(q, s["x"].dtype))
        return dict(out, qT=fxp.mx4_unmap(qT, s["x"].dtype)) if case["both"] else out
    if s["kind"] == "linear":
        return dict(y=fxp.mx4_linear(s["x"], s["w"]))
    Y = fxp.mx4_linear_fwd(s["X"], s["W"], s["buf"], seed=s["seed"], step=s["step"])
    dX, dW = fxp.mx4_linear_bwd(s["dY"], s["buf"], seed=s["seed"], step=s["step"])
    return dict(Y=Y, dX=dX, dW=dW)


# ---- plain forms ----

def _turn(x, positions, f, amplitude, near, back=False):
    """x [..., heads, dim] with the first 2 * len(f) elements of its heads turned by positions [...] * f, in 64 bits."""
    n = f.numel()
    a = positions.double()[..., None, None] * f
    c, s = torch.cos(a) * amplitude, torch.sin(a) * (-amplitude if back else amplitude)
    x = x.double()
    u, w = (x[..., 0:2 * n:2], x[..., 1:2 * n:2]) if near else (x[..., :n], x[..., n:2 * n])
    u, w = u * c - w * s, u * s + w * c
    turned = torch.stack((u, w), -1).flatten(-2) if near else torch.cat((u, w), -1)
    return torch.cat((turned, x[..., 2 * n:]), -1)


def _rotary(s):
    case = s["case"]
    y = _turn(s["x"], s["positions"], s["f"], s["amplitude"], case["near"], case["back"])
    return dict(y=y.to(s["x"].dtype))


def _write(x, q, e, runs, bits):
    """New values x[T, H, D] (64 bits) into pages q[pages, H, 64, D] (int8) under the scales e[pages, H]: the pages written, and what is written."""
    first, count, page, off = runs.long().unbind(1)
    keep = torch.nonzero(count > 0)[:, 0]
    first, count, page, off = first[keep], count[keep], page[keep], off[keep]
    at = torch.arange(PAGE, device=x.device)
    new = ((at >= off[:, None]) & (at < (off + count)[:, None]))[:, :, None, None]
    y = x[(first[:, None] + at - off[:, None]).clamp(0, x.shape[0] - 1)]
    y = torch.where(new, y, torch.zeros_like(y))                                   # [R, 64, H, D]
    top = y.abs().amax((1, 3))
    e_new = (((top.view(torch.int64) >> 52) & 2047) - 896).clamp(1, 255)           # [R, H]
    e_old = torch.where(off[:, None] > 0, e[page], torch.ones_like(e[page]))
    e_all = torch.maximum(e_new, e_old)
    unit = _pow2(125 + bits - e_all)[:, None, :, None]
    mapped = torch.floor(y.abs() * unit + 0.5).clamp(max=2 ** (bits - 1) - 1) * y.sign()
    old = q[page].permute(0, 2, 1, 3).int()
    d = (e_all - e_old).clamp(max=16)[:, None, :, None]
    moved = torch.where(d > 0, ((old.abs() + (1 << (d - 1).clamp(min=0))) >> d) * old.sign(), old)
    return page, torch.where(new, mapped.to(torch.int8), moved.to(torch.int8)).permute(0, 2, 1, 3), e_all.int()


def _rows(vq):
    """Value pages [..., 4, dim, 16] as rows [..., 64, dim]."""
    return vq.transpose(-1, -2).flatten(-3, -2)


def _values(q, e, bits):
    return q.float() * _pow2(e - 125 - bits).float()[:, :, None, None]


def _read(values, runs):
    """The tokens of `runs` out of pages values[R, H, 64, D]: [tokens, H, D]."""
    at = torch.arange(PAGE, device=runs.device)
    r, p = torch.nonzero(at < runs[:, 1:2], as_tuple=True)
    return values[r, :, p].contiguous()


def _append(s):
    case = s["case"]
    bits, turned = case["bits"], (s["positions"], s["f"], s["amplitude"], case["near"])
    page, q, e = _write(_turn(s["k"], *turned), s["kq"], s["ek"], s["runs"], bits)
    s["kq"][page], s["ek"][page] = q, e
    page, q, e = _write(s["v"].double(), _rows(s["vq"]), s["ev"], s["runs"], bits)
    s["vq"][page], s["ev"][page] = q.unflatten(2, (PAGE // 16, 16)).transpose(3, 4), e
    at = s["read"][:, 2].long()
    k = _read(_values(s["kq"][at], s["ek"][at], bits), s["read"])
    v = _read(_values(_rows(s["vq"][at]), s["ev"][at], bits), s["read"])
    out = dict(k=k, v=v, ek=s["ek"], ev=s["ev"])
    return dict(out, q=_turn(s["q"], *turned).to(s["q"].dtype)) if case["q_heads"] else out


def _philox(rows, cols, seed, stream, device):
    """The random word of each element of a matrix, as whole numbers [rows, cols]."""
    n = rows * cols
    low = 0xFFFFFFFF
    c = [torch.arange((n + 3) // 4, device=device), torch.zeros((), dtype=torch.long, device=device)]
    c += [torch.full((), v, dtype=torch.long, device=device) for v in (stream & low, stream >> 32)]
    keys = [(seed & low, seed >> 32)]
    keys += [((keys[0][0] + r * 0x9E3779B9) & low, (keys[0][1] + r * 0xBB67AE85) & low) for r in range(1, 10)]

    def product(m, x):      # (high, low) halves of the product of two 32-bit numbers
        p, q = (x >> 16) * m, (x & 0xFFFF) * m
        return (p + (q >> 16)) >> 16, ((p << 16) + q) & low

    for k0, k1 in keys:
        h0, l0 = product(0xD2511F53, c[0])
        h1, l1 = product(0xCD9E8D57, c[2])
        c = [h1 ^ c[1] ^ k0, l1, h0 ^ c[3] ^ k1, l0]
    return torch.stack(torch.broadcast_tensors(*c), -1).flatten()[:n].view(rows, cols)


def _mapped(x, word=None):
    """The values that a matrix has in 4 bits, blocks along its rows; word: the elements' random words, for stochastic rounding."""
    rows, cols = x.shape
    x = torch.nn.functional.pad(x.float(), (0, -cols % BLOCK)).view(rows, -1, BLOCK)
    top = x.abs().amax(-1, keepdim=True).contiguous().view(torch.int32)
    s = ((top >> 23) - 2 + ((top & 0x7FFFFF) > 0x400000).int()).clamp(min=0)
    m = x.abs().double() * _pow2(127 - s)
    step = torch.where(m < 2, 0.5, torch.where(m < 4, 1.0, 2.0))
    if word is None:
        y = torch.round(m / step) * step
    else:
        # what is cut off, in 22 bits, against the word's top 22
        unit = torch.floor(m / step * (1 << 22)).long()
        word = torch.nn.functional.pad(word, (0, -cols % BLOCK)).view(rows, -1, BLOCK)
        y = ((unit >> 22) + ((word >> 10) < (unit & 0x3FFFFF))) * step
    return (y * _pow2(s - 127) * x.sign()).float().view(rows, -1)[:, :cols]


def _map(s):
    case, x = s["case"], s["x"]
    word = _philox(case["rows"], case["cols"], s["seed"], s["stream"], x.device) if case["stochastic"] else None
    out = dict(q=_mapped(x, word).to(x.dtype))
    return dict(out, qT=_mapped(x.T, word.T if word is not None else None).to(x.dtype)) if case["both"] else out


def _unpack(data, scales, cols, dtype):
    """The values [rows, cols] of a matrix mapped to 4 bits."""
    panels, rows, _ = data.shape
    code = torch.stack((data & 15, data >> 4), -1).view(panels, rows, PANEL // BLOCK, BLOCK)
    value = torch.tensor(GRID + tuple(-v for v in GRID), dtype=dtype, device=data.device)[code.int()]
    place = torch.empty(PANEL // BLOCK, dtype=torch.long, device=data.device)
    place[list(ORDER)] = torch.arange(PANEL // BLOCK, device=data.device)
    value = value * _pow2(scales.int() - 127).to(dtype)[..., place, None]
    return value.view(panels, rows, PANEL).transpose(0, 1).reshape(rows, -1)[:, :cols]


def _linear(s):
    w = _unpack(s["data"], s["scales"], s["case"]["K"], torch.float32)
    return dict(y=(_mapped(s["x"]) @ w.T).to(s["x"].dtype))


def _step(s):
    X, W, dY = s["X"], s["W"], s["dY"]
    words = [_philox(*x.shape, s["seed"], (s["step"] << 8) | tag, x.device) for tag, x in enumerate((X, W, dY))]
    Y = _mapped(X, words[0]) @ _mapped(W.T, words[1].T).T
    dX = _mapped(dY, words[2]) @ _mapped(W, words[1]).T
    dW = _mapped(X.T, words[0].T) @ _mapped(dY.T, words[2].T).T
    return dict(Y=Y, dX=dX, dW=dW)


def work(case):
    size = TYPES[case["type"]].itemsize
    kind = case["kind"]
    if kind == "rotary":
        n = case["B"] * case["T"] * case["heads"] * case["dim"]
        return {"bytes": 2 * n * size + 4 * case["T"] * (case["B"] if case["far"] else 1), "flops": 3 * n * case["rot"] // case["dim"]}
    if kind == "append":
        held, new = _lengths(case)
        T, read = sum(new), sum(n + off for _, n, _, off, _ in _runs(held, new))
        return {"bytes": 2 * case["heads"] * case["dim"] * (T * (size + 1) + read * (1 + 4)) + 2 * T * case["q_heads"] * case["dim"] * size, "flops": 0}
    if kind == "map":
        # the copies are written, read again and written as values
        n, copies = case["rows"] * case["cols"], 1 + case["both"]
        return {"bytes": n * (size + copies * (size + 17 / 16)), "flops": 0}
    M, K, N = case["M"], case["K"], case["N"]
    if kind == "linear":
        return {"bytes": N * K * 17 / 32 + M * (K + N) * size, "flops": 2 * M * K * N}
    return {"bytes": size * 2 * (M * K + K * N + M * N), "flops": 6 * M * K * N}


# ---- from the definitions, in 64 bits ----

def _rotated(x, position, case):
    """x [heads, tokens, dim] in 64 bits on the host, by complex products."""
    how, n = SCALINGS[case["scaling"]], case["rot"]
    out = numpy.array(x, dtype=numpy.float64)
    position = numpy.asarray(position, dtype=numpy.float64)
    for i in range(n // 2):
        f = BASE ** (-2 * i / n)
        if case["scaling"] == "linear":
            f /= how["factor"]
        elif case["scaling"] == "base" and n > 2:
            f = (BASE * how["factor"] ** (n / (n - 2))) ** (-2 * i / n)
        elif case["scaling"] == "parts":
            share = min(1.0, max(0.0, (how["original"] / (2 * math.pi / f) - how["low"]) / (how["high"] - how["low"])))
            f = share * f + (1 - share) * f / how["factor"]
        a, b = (2 * i, 2 * i + 1) if case["near"] else (i, i + n // 2)
        z = (x[..., a] + 1j * x[..., b]) * how.get("amplitude", 1.0) * numpy.exp((-1j if case.get("back") else 1j) * position * f)
        out[..., a], out[..., b] = z.real, z.imag
    return out


def _host(t):
    return t.double().cpu().numpy()


def _words(rows, cols, seed, stream):
    """Philox4x32-10 with numpy's unsigned numbers."""
    n = rows * cols
    u = numpy.uint64
    mask, shift = u(0xFFFFFFFF), u(32)
    blocks = numpy.arange((n + 3) // 4, dtype=u)
    a, b = blocks & mask, blocks >> shift
    c, d = numpy.full_like(a, stream & 0xFFFFFFFF), numpy.full_like(a, stream >> 32)
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(10):
        p, q = a * u(0xD2511F53), c * u(0xCD9E8D57)
        a, b, c, d = (q >> shift) ^ b ^ u(k0), q & mask, (p >> shift) ^ d ^ u(k1), p & mask
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return torch.from_numpy(numpy.stack([a, b, c, d], 1).reshape(-1)[:n].astype(numpy.int64)).view(rows, cols).cuda()


def _in_four(x, word=None):
    """x [rows, cols] in 4 bits, in 64: the two neighbours of each magnitude on the grid, and which of them it goes to."""
    rows, cols = x.shape
    blocks = torch.zeros((rows, -(-cols // BLOCK) * BLOCK), dtype=torch.float64, device=x.device)
    blocks[:, :cols] = x
    blocks = blocks.view(rows, -1, BLOCK)
    largest = blocks.abs().amax(-1, keepdim=True)
    scale = torch.exp2(torch.ceil(torch.log2(largest / 6).clamp(min=-127)))
    scale = torch.where(largest > 6 * scale, scale * 2, scale)                       # where the logarithm was rounded
    scale = torch.where((largest <= 3 * scale) & (scale > 2.0 ** -127), scale / 2, scale)
    m = blocks.abs() / scale
    grid = torch.tensor(GRID, dtype=torch.float64, device=x.device)
    up = torch.bucketize(m, grid).clamp(max=7)                                       # grid[up - 1] < m <= grid[up]
    low, high = grid[(up - 1).clamp(min=0)], grid[up]
    if word is None:
        nearer, tie = m - low > high - m, m - low == high - m
        take = nearer | (tie & (up % 2 == 0))
    else:
        r = torch.zeros((rows, blocks.shape[1] * BLOCK), dtype=torch.int64, device=x.device)
        r[:, :cols] = word
        share = torch.where(high > low, (m - low) / (high - low), torch.zeros_like(m))
        take = (r.view(blocks.shape) // 1024).double() < torch.floor(share * 2.0 ** 22)
        take = take | (m == high)
    return (torch.where(take, high, low) * scale * blocks.sign()).reshape(rows, -1)[:, :cols]


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "rotary":
        if case["B"] * case["T"] * case["heads"] * case["dim"] > 1 << 27:
            return None
        x = _host(s["x"])                                                            # [B, T, H, D]
        position = numpy.broadcast_to(s["positions"].cpu().numpy(), x.shape[:2])[:, :, None]
        return dict(y=torch.from_numpy(_rotated(x, position, case)))
    if kind == "append":
        bits, H, D = case["bits"], case["heads"], case["dim"]
        position = s["positions"].cpu().numpy()[:, None]
        out = {}
        keys = torch.from_numpy(_rotated(_host(s["k"]), position, case))
        for name, x, q, e in (("k", keys, s["kq"], s["ek"]), ("v", s["v"].double().cpu(), s["vq"].permute(0, 1, 2, 4, 3).reshape(-1, H, PAGE, D), s["ev"])):
            q, e, rows = q.cpu(), e.cpu(), []
            for t, n, page, off in s["runs"].tolist():
                if n == 0:
                    continue
                for h in range(H):
                    new = x[t:t + n, h]
                    scale = max(1, int(torch.frexp(new.abs().max())[1]) + 126, int(e[page, h]) if off else 1)
                    step = 2.0 ** (scale - 125 - bits)
                    new = torch.sign(new) * torch.clamp(torch.floor(new.abs() / step + 0.5), max=2 ** (bits - 1) - 1)
                    old = q[page, h, :off].double() * 2.0 ** (int(e[page, h]) - 125 - bits)
                    old = torch.sign(old) * torch.floor(old.abs() / step + 0.5) if off and scale > int(e[page, h]) else old / step
                    rows.append(torch.cat([old, new]) * step)
            rows = [torch.stack(rows[i:i + H], 1) for i in range(0, len(rows), H)]
            out[name] = torch.cat(rows)
        out = dict(k=out["k"], v=out["v"], ek=None, ev=None)
        return dict(out, q=torch.from_numpy(_rotated(_host(s["q"]), position, case))) if case["q_heads"] else out
    if kind == "map":
        word = _words(case["rows"], case["cols"], s["seed"], s["stream"]) if case["stochastic"] else None
        x = s["x"].double()
        out = dict(q=_in_four(x, word))
        return dict(out, qT=_in_four(x.T, word.T if word is not None else None)) if case["both"] else out
    if kind == "linear":
        K, N = case["K"], case["N"]
        w = torch.zeros((N, s["data"].shape[0] * PANEL), dtype=torch.float64, device="cuda")
        for k in range(PANEL):
            code = (s["data"][:, :, k // 2].int() >> (4 * (k % 2))) & 15             # [panels, N]
            size = torch.tensor(GRID, dtype=torch.float64, device="cuda")[code % 8]
            scale = s["scales"][:, :, ORDER.index(k // BLOCK)].double()
            w[:, k::PANEL] = (torch.where(code >= 8, -size, size) * 2.0 ** (scale - 127)).T
        return dict(y=_in_four(s["x"].double()) @ w[:, :K].T.contiguous())
    X, W, dY = (s[n].double() for n in ("X", "W", "dY"))
    r = [_words(*x.shape, s["seed"], (s["step"] << 8) + tag) for tag, x in enumerate((X, W, dY))]
    return dict(Y=_in_four(X, r[0]) @ _in_four(W.T, r[1].T).T.contiguous(), dX=_in_four(dY, r[2]) @ _in_four(W, r[1]).T.contiguous(),
                dW=_in_four(X.T, r[0].T) @ _in_four(dY.T, r[2].T).T.contiguous())
