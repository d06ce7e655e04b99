"""Values that name the block they belong to: with v = the unit vector (block % D), component d of
an output is the mass of the weights in the blocks d, d + D, .. of the request.  A step of 32 keys
that is lost, read twice or joined with a wrong factor then moves two components by a good part of
themselves, where the bound is a few roundings of them."""
import numpy as np

UNIT = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}


def weights(q, k, scale, p, window=0, softcap=0.0):
    """fp64 scores' softmax of one row and head over the keys k [L, D]; -infinity where hidden.
    Returns the weights, and what fp32 may move an exponent by (see kv_cases)."""
    s = scale * (k @ q)
    ds = (k.shape[1] + 4) * 2.0 ** -24 * abs(scale) * (np.abs(k) @ np.abs(q)).max()
    if softcap:
        s = softcap * np.tanh(s / softcap)
        ds += 2.0 ** -21 * softcap
    ds += 4 * 2.0 ** -23 * (np.abs(s).max() + 1)
    j = np.arange(len(k))
    s = np.where((j <= p) & ((p - j < window) if window else True), s, -np.inf)
    e = np.exp(s - s.max())
    return e / e.sum(), ds


def masses(w, block, D):
    """Component d: the mass of the blocks d, d + D, .."""
    per = np.add.reduceat(w, np.arange(0, len(w), block))
    return np.bincount(np.arange(len(per)) % D, per, D)


def bound(mass, keys, ds, dtype):
    """How far an output component may be off.  Its values are 1 and its weights positive, so errors
    are relative: weights and output rounded to 16 bits 2 u; scores ds each; at most keys / 4
    weights a lane and as many products a sum, one after the other, in fp32.  f16: weights below
    its normal numbers are off by 2^-32 of the largest, outputs by 2^-25; an output of bf16 has no
    such end here."""
    u = UNIT[dtype]
    small = keys * 2.0 ** -32 + 2.0 ** -25 if dtype == "f16" else 2.0 ** -100
    return (2 * u + np.expm1(2 * ds) + 2 * (keys / 4 + 8) * 2.0 ** -24) * mass + small
