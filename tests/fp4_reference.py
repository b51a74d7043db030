"""Operands in e2m1 with a power of two for each 32 values, and the MoE layer for a few tokens, in 64 bits from their definitions."""
import numpy as np
import torch

from tests import moe_reference as ref

GROUP = 32
VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def exponent(amax):
    """The least s >= -126 with amax <= 6 * 2^s; 0 for amax 0; None for a group that is not finite."""
    if not np.isfinite(amax):
        return None
    if amax == 0:
        return 0
    s = max(-126, int(np.floor(np.log2(amax))) - 4)
    while amax > 6.0 * 2.0**s:
        s += 1
    return s


def to_codes(y):
    """Codes of the nearest e2m1 values (ties to the even code) of every y in [-6, 6]."""
    a = np.abs(y)
    hi = np.clip(np.searchsorted(VALUES, a), 0, 7)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - VALUES[lo], VALUES[hi] - a
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return code | np.where(np.signbit(y), 8, 0)


def quantize(y):
    """y [rows, cols] float64 -> codes [rows, cols], scale bytes [rows, groups]"""
    rows, cols = y.shape
    n = -(-cols // GROUP)
    codes, s = np.zeros((rows, cols), np.int64), np.zeros((rows, n), np.int64)
    for g in range(n):
        part = y[:, g * GROUP : (g + 1) * GROUP]
        for r in range(rows):
            e = exponent(np.abs(part[r]).max() if not np.isnan(part[r]).any() else np.nan)
            s[r, g] = 255 if e is None else e + 127
            if e is not None:
                codes[r, g * GROUP : (g + 1) * GROUP] = to_codes(part[r] / 2.0**e)
    return codes, s


def unpack(q, cols):
    """bytes [..., ceil(cols / 2)] -> codes [..., cols]"""
    q = q.cpu().numpy().astype(np.int64)
    return np.stack([q & 15, q >> 4], -1).reshape(*q.shape[:-1], -1)[..., :cols]


def pack(codes):
    codes = np.concatenate([codes, np.zeros((*codes.shape[:-1], codes.shape[-1] % 2), np.int64)], -1)
    return (codes[..., 0::2] | codes[..., 1::2] << 4).astype(np.uint8)


def scale_bytes(atoms, rows, cols):
    """atoms [lines, atoms, 512] -> bytes [rows, groups], one look-up for each"""
    a = atoms.cpu().numpy()
    r, g = np.arange(rows)[:, None], np.arange(-(-cols // GROUP))[None]
    return a[r // 128, g // 4, 16 * (r % 32) + 4 * (r % 128 // 32) + g % 4].astype(np.int64)


def to_atoms(s, fill=127):
    rows, groups = s.shape
    a = np.full((-(-rows // 128), -(-groups // 4), 512), fill, np.uint8)
    for r in range(rows):
        for g in range(groups):
            a[r // 128, g // 4, 16 * (r % 32) + 4 * (r % 128 // 32) + g % 4] = s[r, g]
    for r in range(rows):  # behind the last group of a row
        for g in range(groups, a.shape[1] * 4):
            a[r // 128, g // 4, 16 * (r % 32) + 4 * (r % 128 // 32) + g % 4] = 127
    return a


def values(codes, s):
    """float64 [rows, cols]; NaN where the byte is 255"""
    v = np.where(codes & 8, -1.0, 1.0) * VALUES[codes & 7]
    f = np.where(s == 255, np.nan, 2.0 ** (s - 127.0))
    return v * np.repeat(f, GROUP, axis=-1)[..., : codes.shape[-1]]


def random_operand(rows, cols, seed, spread=8):
    """Codes and scale bytes as a quantisation of ordinary numbers makes them, with scales over 2^spread."""
    g = np.random.default_rng(seed)
    y = g.standard_normal((rows, cols)) * 2.0 ** g.integers(-spread, 1, (rows, -(-cols // GROUP))).repeat(GROUP, 1)[:, :cols]
    return quantize(y)


def operand_tensors(codes, s, device):
    """Padded to rows of 16 bytes: (view of the codes, atoms)."""
    p = pack(codes)
    buf = torch.zeros(*p.shape[:-1], -(-p.shape[-1] // 16) * 16, dtype=torch.uint8, device=device)
    buf[..., : p.shape[-1]] = torch.from_numpy(p).to(device)
    return buf[..., : p.shape[-1]], torch.from_numpy(to_atoms(s)).to(device)


def layer(x, logits, bias, w1, w2, config, score):
    """x [T, d], w1 [E, 2 f, d], w2 [E, d, f] in float64: out, choice, weights, and the sum of the magnitudes of what out is made
    of, with what h is made of in the place of h."""
    ids, weights = ref.route(logits, bias, config["top_k"], score, config.get("n_groups", 1), config.get("top_groups", 1),
                             config.get("group_best", 2), config.get("renormalise", False), config.get("scale", 1.0))
    T, d = x.shape
    out, size = torch.zeros(T, d, dtype=torch.float64, device=x.device), torch.zeros(T, d, dtype=torch.float64, device=x.device)
    for e in range(w1.shape[0]):
        t, j = np.nonzero(ids == e)
        if not len(t):
            continue
        t = torch.from_numpy(t).to(x.device)
        c = torch.from_numpy(weights[ids == e]).to(x.device)[:, None]
        h, hs = x[t] @ w1[e].T, x[t].abs() @ w1[e].abs().T
        f = h.shape[1] // 2
        g, u, gs, us = h[:, :f], h[:, f:], hs[:, :f], hs[:, f:]
        a = g / (1 + torch.exp(-g)) * u
        # |silu'| is at most 1.1, |silu(g)| at most |g|
        spread = 1.1 * gs * u.abs() + g.abs() * us
        out.index_add_(0, t, c * (a @ w2[e].T))
        size.index_add_(0, t, c.abs() * (spread @ w2[e].abs().T))
    return out, ids, weights, size
