"""What the tests of the attention of prompts and of drafted trees share: how far results may be off.

Tolerances count roundings, as decode_parity.py does: with u = 2^-24 a logit is off by e = (2 d + 8) u terms + 2^-21, a softmax weight of n keys by
r = 2 e + (n / 16 + 64) u of itself.  Weights enter the products with V in the type of the queries: half a step h of themselves more (2^-8 bf16, 2^-11 fp16; fp16
ones that are less than 2^-26 of the largest, 2^-37 of that).  So with S = sum p |v| an output is off by (r + h) S, for fp16 by 2^-36 max |v| n more,
and the rounding to its own type, half a step of the result: of |o| and of what it is off by."""

import numpy as np

from decode_parity import HALF_STEP, close, f64


def check_outputs(dtype, d, keys, out, lse, o, l, terms, spread, vmax=0.0):
    """Results against the oracle's; keys: of the longest sequence."""
    u, h = 2.0 ** -24, HALF_STEP[dtype]
    e = (2 * d + 8) * u * terms + 2.0 ** -21
    r = 2 * e + (keys / 16 + 64) * u
    off = (r[..., None] + (0.0 if dtype == "f32" else h)) * spread + (2.0 ** -36 * vmax * keys if dtype == "f16" else 0.0)
    close(f64(out), o, off + h * (np.abs(o) + off), "out")
    close(f64(lse), l, r + 2.0 ** -22 * np.abs(np.where(np.isfinite(l), l, 0)), "lse")
