"""Whether the turned queries share elements with the step's keys and values: exact for the layouts of a fused projection, by the elements themselves."""
import random

import torch

from paper_2207_08822_amd import fxp

ROOM = torch.zeros(6000)


def elements(t):
    at = torch.arange(t.shape[0])[:, None, None] * t.stride(0) + torch.arange(t.shape[1])[:, None] * t.stride(1) + torch.arange(t.shape[2])
    return set((at + t.storage_offset()).flatten().tolist())


def test_layouts_of_a_fused_projection():
    """Queries, keys and values of a token beside each other, and of a head beside each other; of one token and of several."""
    T, H, D = 5, 3, 16
    for tokens in (1, T):
        q, k, v = ROOM[:tokens * 3 * H * D].view(tokens, 3, H, D).unbind(1)
        assert not fxp._meet(q, k) and not fxp._meet(q, v) and fxp._meet(q, q)
        q, k, v = ROOM[:tokens * H * 3 * D].view(tokens, H, 3, D).unbind(2)
        assert not fxp._meet(q, k) and not fxp._meet(q, v) and fxp._meet(q, q) and fxp._meet(v, ROOM[2 * D - 1:][:tokens * H * 3 * D].as_strided(v.shape, v.stride(), 2 * D - 1))
        # heads outside of tokens
        q, k, v = ROOM[:tokens * H * 3 * D].view(3, H, tokens, D).transpose(1, 2).unbind(0)
        assert not fxp._meet(q, k) and not fxp._meet(k, v)
        q, k = ROOM[:tokens * H * 2 * D].view(H, tokens, 2, D).transpose(0, 1).unbind(2)
        assert not fxp._meet(q, k) and fxp._meet(k, k)
    # more query heads than keys'
    both = ROOM[:T * 8 * D].view(T, 8, D)
    assert not fxp._meet(both[:, :6], both[:, 6:7]) and fxp._meet(both[:, :6], both[:, 5:6])


def test_against_the_elements():
    rng = random.Random(3)
    seen = {True: 0, False: 0}
    for trial in range(3000):
        T, D = rng.choice([1, 2, 3, 5]), rng.choice([2, 4, 8])
        heads = [rng.choice([1, 2, 3, 4])] * 2
        strides = [[rng.choice([8, 16, 24, 64, 96]), rng.choice([2, 4, 8, 24, 40])] for _ in range(2)]
        alike = rng.random() < 0.8
        if alike:
            strides[1] = strides[0]
        elif rng.random() < 0.5:
            heads[1] = rng.choice([1, 2, 3, 4])
        a, b = (ROOM.as_strided((T, h, D), (*s, 1), rng.randrange(150)) for h, s in zip(heads, strides))
        want, got = bool(elements(a) & elements(b)), fxp._meet(a, b)
        assert got == want if alike else got or not want, (a.shape, a.stride(), a.storage_offset(), b.shape, b.stride(), b.storage_offset())
        seen[got] += 1
    assert min(seen.values()) > 300
