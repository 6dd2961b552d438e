"""How far the dense operators' results are from 64 bits in the root mean square: as far as the roundings that they document, and no further.

A bound on each element has to allow for the worst order of a sum, which a second rounding of an operand or a result stays below.  In the root mean square
it does not: r, the distance of the 64-bit result from itself rounded once, is what a result may be off, and another rounding of like size makes 1.41 r
of it.  On top of r: 5 % for operands whose fp32 value falls on the other side of a rounding's border (2^-20 of a value against steps of 2^-10: one
in 512, each off by a step instead of 0.29 of one, 1.2 % in the root mean square) and for the draw, and the fp32 sum itself: at most K / 8 + 16 additions
in a row, each off by 2^-23 of the terms' absolute sum."""
import torch


def rms(t):
    return float(t.double().square().mean().sqrt())


def check_rms(got, want, terms, absum, what):
    """got: the result; want: the formula in 64 bits of the operands as they enter the product; terms, absum: of the fp32 sum."""
    r = rms(want.to(got.dtype).double() - want)
    bound = 1.05 * r + (terms / 8 + 16) * 2.0 ** -23 * rms(absum)
    off = rms(got.double() - want)
    assert bound <= 1.35 * r, (what, "a second rounding would not show", bound / r)
    assert off <= bound, (what, off / r, bound / r)


def rounded(t, dtype):
    return t.to(dtype).double()
