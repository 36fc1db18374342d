"""Plain 64-bit definitions of the serving operators (not collected by pytest): loops over requests, runs and rows."""
import math

import numpy as np

PAGE = 64


def tables(lens, n_new, table, free, n_free, tokens, rows):
    """Every output of kv_tables, from the definition."""
    table, B, blocks = table.copy(), len(lens), table.shape[1]
    first, after, refused, taken, sum_need = [0], [], [], 0, 0
    slots, positions = np.full(tokens, -1, np.int64), np.full(tokens, -1, np.int64)
    runs = []
    for b in range(B):
        asked, at = int(n_new[b]), int(lens[b])
        n = min(asked, tokens)
        need = -(-(at + n) // PAGE) - -(-at // PAGE)
        fits = at + n <= blocks * PAGE and asked == n
        if fits:
            sum_need += need
        served = fits and (need == 0 or sum_need <= n_free) and (n == 0 or first[-1] + n <= tokens)
        if served:
            for j in range(need):
                table[b, -(-at // PAGE) + j] = free[n_free - 1 - taken - j]
            taken += need
        t, end = first[-1], at + n
        while at < end:
            k = min(end, (at // PAGE + 1) * PAGE) - at
            page = int(table[b, at // PAGE]) if served else -1
            runs.append((t, k, page, at % PAGE))
            for i in range(max(min(k, tokens - t), 0)):
                positions[t + i] = at + i
                slots[t + i] = page * PAGE + at % PAGE + i if page >= 0 else -1
            t, at = t + k, at + k
        first.append(t)
        after.append(int(lens[b]) + n if served else int(lens[b]))
        refused.append(not served)
    runs = runs[:rows]
    runs += [(0, 0, -1, 0)] * (rows - len(runs))
    return dict(block_table=table, first=np.array(first), lens_after=np.array(after), n_free_after=np.array([n_free - taken]), slots=slots,
                positions=positions, runs=np.array(runs).reshape(rows, 4), refused=np.array(refused, dtype=np.int64))


def exponent(x):
    """The biased exponent field of the largest magnitude, at least 1."""
    m = float(np.max(np.abs(x))) if x.size else 0.0
    return max(1, math.frexp(m)[1] + 126) if m else 1


def to_units(x, e, bits):
    q = np.floor(np.abs(x) * 2.0 ** (125 + bits - e) + 0.5)
    return np.sign(x) * np.minimum(q, 2 ** (bits - 1) - 1)


class Cache:
    """q[pages, heads, 64, dim] and e[pages, heads] of keys or values, as float64 and int."""

    def __init__(self, q, e, bits):
        self.q, self.e, self.bits = q.astype(np.float64), e.astype(np.int64), bits

    def append(self, x, runs):
        for first, count, page, off in runs.tolist():
            if count <= 0 or page < 0 or page >= len(self.q):
                continue
            for h in range(self.q.shape[1]):
                new = x[first:first + count, h].astype(np.float64)
                e = exponent(new)
                if off:
                    old = int(self.e[page, h])
                    e = max(e, old)
                    if e > old:
                        q = self.q[page, h, :off]
                        self.q[page, h, :off] = np.sign(q) * np.floor(np.abs(q) / 2.0 ** (e - old) + 0.5)
                self.e[page, h] = e
                self.q[page, h, off:off + count] = to_units(new, e, self.bits)

    def values(self):
        return self.q * 2.0 ** (self.e - 125 - self.bits)[:, :, None, None]


def rows_of(vq):
    """Value pages [pages, heads, 4, dim, 16] as [pages, heads, 64, dim]."""
    p, h, _, d, _ = vq.shape
    return vq.transpose(0, 1, 2, 4, 3).reshape(p, h, PAGE, d)


def attention(q, k, v, first, lens, table, scale, window, unit_bits, half_step):
    """(out, lse, how far out may be off) of q[tokens, q_heads, dim] over pages k, v[pages, heads, 64, dim] in 64 bits.

    The bound follows the arithmetic that the interface states.  An element of q is rounded to a unit u = 2^(e - 126 - unit_bits), e the exponent
    of its row's largest element (one more where that is within 2^-7 of the next binade), so a score is off by at most scale * u/2 * sum|k|, and by
    a few fp32 roundings of a value of its size; a weight w_j = exp(s_j) then by a factor within exp(+-d).  The weights of a page are rounded to
    half a unit of 1/32639 (1/8355711) of the page's largest weight.  fp32 sums of a page's products and of the pages add roundings of 2^-24 each,
    counted once per page and then some.  A weight below 2^-126 of the largest is no normal fp32 number: 2^-126 |v| each may be lost (a token
    that weighs 1e-44 gives 0, not 1e-44 v).  The output is rounded once, by half a step."""
    T, QH, D = q.shape
    H = k.shape[1]
    G, most = QH // H, 32639 if unit_bits == 15 else 8355711
    out, lse, off = np.zeros((T, QH, D)), np.full((T, QH), -np.inf), np.zeros((T, QH, D))
    for b in range(len(lens)):
        n, L = int(first[b + 1] - first[b]), int(lens[b])
        pages = table[b, :-(-L // PAGE)]
        ok = (pages >= 0) & (pages < len(k))
        if n == 0 or L == 0:
            continue
        rows, j = slice(int(first[b]), int(first[b]) + n), np.arange(L)
        place = (L - n + np.arange(n))[:, None]
        m = np.repeat(ok, PAGE)[:L] & (j <= place) & ((j > place - window) if window else True)
        some = m.any(1)
        for h in range(QH):
            kk, vv = (np.concatenate([x[p if o else 0, h // G] for p, o in zip(pages, ok)])[:L] for x in (k, v))
            x = q[rows, h]
            s = scale * (x @ kk.T)
            top_s = np.where(some, np.where(m, s, -np.inf).max(1), 0.0)[:, None]
            w = np.where(m, np.exp(np.minimum(s - top_s, 0.0)), 0.0)
            l = np.where(some, w.sum(1), 1.0)[:, None]
            o = w @ vv / l
            out[rows, h] = np.where(some[:, None], o, 0.0)
            lse[rows, h] = np.where(some, top_s[:, 0] + np.log(l[:, 0]), -np.inf)
            u = np.array([2.0 ** (exponent(r * (1 + 2.0 ** -6)) - 126 - unit_bits) for r in x])[:, None]
            d = np.where(m, scale * u / 2 * np.abs(kk).sum(1) + 8 * 2.0 ** -24 * (np.abs(s) + scale * np.abs(x) @ np.abs(kk).T + 1), 0.0).max(1)[:, None]
            mass = w @ np.abs(vv) / l
            rounded = np.zeros_like(o)
            for p in range(0, L, PAGE):
                part = w[:, p:p + PAGE]
                rounded += part.max(1, keepdims=True) * ((part > 0) @ np.abs(vv[p:p + PAGE])) * 0.5 / most / l
            inner = (np.expm1(2 * d) + 2.0 ** -24 * (2 * len(pages) + 80)) * mass + rounded * np.exp(2 * d) + 2.0 ** -126 * np.abs(vv).sum(0)
            off[rows, h] = np.where(some[:, None], half_step * (np.abs(o) + inner) + inner, 0.0)
    return out, lse, off


def unpack4(packed, scales, K, N, group):
    """(mantissas, scales as numbers) [K, N] of the packed layout, byte by byte."""
    S, kt = min(group, 64), -(-K // 128)
    packed, scales = packed.reshape(-1, kt, 64, 16), scales.reshape(-1, kt * 128 // group, 16)
    q, e = np.zeros((K, N)), np.zeros((K, N))
    for k in range(K):
        kk = k % 128
        byte = packed[:, k // 128, 16 * (kk % S // (S // 4)):, kk // S * (S // 8) + kk % (S // 8)][:, :16].reshape(-1)[:N].astype(np.int64)
        nib = (byte & 15) if kk % (S // 4) < S // 8 else byte >> 4
        q[k] = np.where(nib > 7, nib - 16, nib)
        e[k] = scales[:, k // group].reshape(-1)[:N]
    return q, 2.0 ** (e - 129)
