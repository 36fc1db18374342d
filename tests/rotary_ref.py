"""Plain 64-bit definition of rotary positions (not collected by pytest)."""
import math

import numpy as np


def angles(rope, positions):
    """Angles [..., pairs] of positions, reduced to one turn in whole numbers of 2^-64 turns as the operators define them."""
    turns = [int(t) & (2 ** 64 - 1) for t in rope.turns.tolist()]
    return np.array([[(t * int(p) % 2 ** 64) * (2 * math.pi / 2 ** 64) for t in turns] for p in np.ravel(positions)]).reshape(*np.shape(positions), len(turns))


def turn(x, positions, rope, backward=False):
    """x [..., heads, dim] turned by positions [...]; 64 bits."""
    x = np.array(x, dtype=np.float64)
    a = angles(rope, positions)[..., None, :] * (-1 if backward else 1)
    n = rope.dim
    first, second = (slice(0, n, 2), slice(1, n, 2)) if rope.interleaved else (slice(0, n // 2), slice(n // 2, n))
    u, w = x[..., first].copy(), x[..., second].copy()
    x[..., first] = rope.amplitude * (u * np.cos(a) - w * np.sin(a))
    x[..., second] = rope.amplitude * (u * np.sin(a) + w * np.cos(a))
    return x


def within(got, want, x, rope, eps):
    """|got - want| within: the rounding to the type, eps / 2 of the result; and of the arithmetic in 32 bits (2^-24 a rounding): the cosine and the sine
    are off by the angle's 2^-33 turns (2^-30.3), the series' 2^-24 each for its sum, the conversion, factor and product of the reduced angle (three of 2^-24 of at most
    0.8) and the amplitude's product with its own rounding to 32 bits (two): 2^-24 * (1 + 2.4 + 2 + 0.02) of u and of w; two products and a sum: three
    more of 2^-24.  Together below 2^-20.9 * amplitude * (|u| + |w|)."""
    n = rope.dim
    size = np.abs(np.array(x, dtype=np.float64))
    first, second = (slice(0, n, 2), slice(1, n, 2)) if rope.interleaved else (slice(0, n // 2), slice(n // 2, n))
    both = size[..., first] + size[..., second]
    bound = np.zeros_like(size)
    bound[..., first] = bound[..., second] = both * rope.amplitude * 2.0 ** -20.9
    bound += np.abs(want) * (eps / 2) * (1 + 2.0 ** -20) + 2.0 ** -25        # 2^-25: half of the smallest fp16
    return np.all(np.abs(got - want) <= bound)
