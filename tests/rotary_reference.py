"""Turned positions in 64 bits from the definition, with a bound for a kernel's error.

The bound.  The angle is a whole number modulo one turn, cut to 32 bits (2^-32 of a turn: 1.5e-9).  What is left of it behind the nearest
quarter turn, at most 0.7854, is rounded when it becomes fp32, when it is multiplied, and in the factor: 3 * 0.7854 * 2^-24 = 1.4e-7.
The series leaves out 2.5e-8 and rounds its result, at most 1, and the term before it: 1.0e-7.  gain times a sine is rounded (2^-24),
so is each product and their sum (2 * 2^-24 of what is added).  Together 4.5e-7 < 2^-21 of gain (|a| + |b|), then the result's rounding."""
import math

import torch

ROUND = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
LEAST = {torch.float32: 2.0 ** -126, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -126}


def angles(positions, turns):
    """[tokens, pairs] in 64 bits: the product is taken modulo 2^64, so whole turns fall away by themselves."""
    return (positions.long()[:, None] * turns[None, :]).double() * (2 * math.pi / 2.0 ** 64)


def rotate_reference(x, positions, turns, halves=False, gain=1.0, back=False):
    """(y, bound) of x [tokens, heads, width] at positions int64 [tokens] (host tensors)."""
    r, y, size = 2 * turns.numel(), x.double().clone(), torch.zeros(x.shape, dtype=torch.float64)
    t = angles(positions, turns)[:, None] * (-1 if back else 1)
    a, b = (slice(0, r // 2), slice(r // 2, r)) if halves else (slice(0, r, 2), slice(1, r, 2))
    p, q = x.double()[..., a], x.double()[..., b]
    y[..., a], y[..., b] = gain * (p * t.cos() - q * t.sin()), gain * (p * t.sin() + q * t.cos())
    size[..., a] = size[..., b] = abs(gain) * (p.abs() + q.abs())
    bound = 2.0 ** -21 * size
    bound[..., :r] += ROUND[x.dtype] * y[..., :r].abs() + LEAST[x.dtype]
    return y, bound


def within(got, want, bound):
    over = (got.double().cpu() - want).abs() - bound
    assert torch.isfinite(over).all() and float(over.max()) <= 0, float(over.max())


def places(offsets, tokens):
    """Places in their texts of the tokens, -1 where no text has them."""
    at = torch.full((tokens,), -1, dtype=torch.int64)
    for a, b in zip(offsets[:-1], offsets[1:]):
        at[a:b] = torch.arange(b - a)
    return at
