"""The 2-norm that fp32 results of the calls for many adapters are held to: three bf16 parts to a number, sums emptied every 256 terms.

An output goes through two sums of products, one after the other (u, then Y or dB; du, then dX or dA).  In each
  parts    three parts leave 2^-24 of a number at worst and 2^-28 in root mean square; two would leave 2^-18.6 in root mean square,
           (0.4 2^-8)^2 with 0.4 2^-8 for the rounding of evenly spread mantissas, and products of parts that are left out (0 x 2) as much;
  sums     a tensor core's step of 16 terms loses up to 2^-26 of the sum so far, towards zero: 2^-22 in the 16 steps between two emptyings;
           fp32 additions of pooling (64 neighbours at most here), of the emptied sums and of the warps' are off by 0.4 2^-24 of the sum so far
           each, with either sign: below 2^-23 for a hundred of them.
Together 2 (2^-22 + 2^-23 + 2^-27) < 2^-20 of the result's 2-norm.
"""
LIMIT = 2.0 ** -20


def off(got, want):
    """2-norm of the error over that of the result."""
    got = got.double()
    return float((got - want).norm() / want.norm())


def split(x, parts):
    """What `parts` bf16 numbers hold of x (fp32)."""
    held, rest = x.double() * 0, x.float()
    for _ in range(parts):
        h = rest.bfloat16()
        held += h.double()
        rest = rest - h.float()
    return held
