"""The sums of parts as which values go into the products of the layer for a few tokens, in 64 bits from their definition."""
import numpy as np

from tests import fp4_reference as f4

GROUP = 32
# parts of a value: {bits of the weights: {bytes of a value: parts}}
PARTS = {8: {2: 5, 4: 5}, 4: {2: 7, 4: 9}}
LARGEST = {8: 448.0, 4: 6.0}


def below(bits, p):
    """How far part p's power of two is below the first's: what a part leaves fits there."""
    return 0 if p == 0 else 4 + 5 * (p - 1) if bits == 8 else 2 + 3 * (p - 1)


def round_part(y, bits):
    """To the nearest e4m3 or e2m1 value, ties to even; |y| at most the largest."""
    if bits == 4:
        codes = f4.to_codes(y)
        return np.where(codes & 8, -1.0, 1.0) * f4.VALUES[codes & 7]
    e = np.maximum(np.floor(np.log2(np.maximum(np.abs(y), 2.0**-40))), -6)
    step = 2.0 ** (e - 3)
    return np.clip(np.round(y / step) * step, -448.0, 448.0)


def split(v, bits, parts):
    """v [..., cols] float64, cols a multiple of 32: the sum of the parts."""
    g = v.reshape(*v.shape[:-1], -1, GROUP)
    amax = np.abs(g).max(-1, keepdims=True)
    s = np.ceil(np.log2(np.maximum(amax, 1e-300) / LARGEST[bits]))
    s += amax > LARGEST[bits] * 2.0**s
    s -= amax <= LARGEST[bits] * 2.0 ** (s - 1)
    s = np.where(amax == 0, 0.0, np.maximum(s, -126))
    rest, out = g.copy(), np.zeros_like(g)
    for p in range(parts):
        unit = 2.0 ** np.maximum(s - below(bits, p), -126)
        part = round_part(rest / unit, bits) * unit
        out += part
        rest -= part
    return out.reshape(v.shape)


def bound(v, bits, parts):
    """What the parts leave out at most: 8 bits half a step of four bits and a sign each (2^-4 of a value's power of two, then 2^-5 each), down
    to half a step of the last part, which is 2^-10 of its power; 4 bits half of the last part's power.  The largest of 32 is more than
    half of what the first power is chosen for."""
    g = v.reshape(*v.shape[:-1], -1, GROUP)
    amax = np.abs(g).max(-1, keepdims=True)
    last = 2.0 ** -below(bits, parts - 1)
    if bits == 8:
        b = np.maximum(2.0 ** (1 - 5 * parts) * np.abs(g), last * 2.0**-10 * amax / 224)
    else:
        b = np.broadcast_to(last / 2 * amax / 3, g.shape)
    return b.reshape(v.shape)
