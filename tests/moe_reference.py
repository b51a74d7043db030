"""The operators behind the gather of a MoE layer, in 64 bits, written from their definitions with loops and numpy."""
import numpy as np
import torch

BLOCK = 128


def open_logits(logits):
    x = logits.double().cpu().numpy().copy()
    x[np.isnan(x)] = -np.inf
    return np.minimum(x, np.finfo(np.float32).max)


def scores(logits, score):
    """[T, E] float64; 0 for a closed logit."""
    x = open_logits(logits)
    shut = np.isneginf(x)
    if score == "sigmoid":
        with np.errstate(over="ignore"):
            s = 1.0 / (1.0 + np.exp(-x))
    else:
        m = np.where(np.all(shut, 1, keepdims=True), 0.0, x.max(1, keepdims=True))
        e = np.where(shut, 0.0, np.exp(np.where(shut, 0.0, x - m)))
        t = e.sum(1, keepdims=True)
        s = e / np.where(t > 0, t, 1.0)
    return np.where(shut, 0.0, s), shut


def route(logits, bias, top_k, score, n_groups=1, top_groups=1, group_best=2, renormalise=False, scale=1.0):
    s, shut = scores(logits, score)
    T, E = s.shape
    ids = np.full((T, top_k), -1, np.int64)
    w = np.zeros((T, top_k))
    per = E // n_groups
    for t in range(T):
        c = s[t] + (0.0 if bias is None else bias.double().cpu().numpy())
        c = [-np.inf if shut[t, e] or np.isnan(c[e]) else c[e] for e in range(E)]
        if top_groups < n_groups:
            value = []
            for g in range(n_groups):
                best = sorted([v for v in c[g * per : (g + 1) * per] if v > -np.inf], reverse=True)[:group_best]
                value.append(sum(best[1:], best[0]) if best else -np.inf)
            keep = sorted((g for g in range(n_groups) if value[g] > -np.inf), key=lambda g: (-value[g], g))[:top_groups]
            c = [c[e] if e // per in keep else -np.inf for e in range(E)]
        order = sorted((e for e in range(E) if c[e] > -np.inf), key=lambda e: (-c[e], e))[:top_k]
        ids[t, : len(order)] = order
        w[t, : len(order)] = s[t, order]
        if renormalise:
            total = w[t].sum()
            w[t] = w[t] / total if total > 0 else 0.0
    return ids, w * scale


def route_backward(logits, experts, dweights, score, renormalise=False, scale=1.0):
    s, shut = scores(logits, score)
    T, E = s.shape
    ids = experts.cpu().numpy()
    dw = dweights.double().cpu().numpy()
    out = np.zeros((T, E))
    for t in range(T):
        some = [j for j in range(ids.shape[1]) if 0 <= ids[t, j] < E]
        sk = np.array([s[t, ids[t, j]] for j in some])
        d = np.array([dw[t, j] for j in some]) * scale
        if renormalise:
            total = sk.sum()
            d = (d - (d * sk).sum() / total) / total if total > 0 else d * 0
        ds = np.zeros(E)
        for j, v in zip(some, d):
            ds[ids[t, j]] += v
        out[t] = ds * s[t] * (1 - s[t]) if score == "sigmoid" else s[t] * (ds - (ds * s[t]).sum())
    out[shut] = 0.0
    return out


def layout(experts, n_experts):
    """starts, counts, row_of_slot, {row: slot or -1}"""
    flat = experts.reshape(-1).cpu().tolist()
    by = [[i for i, e in enumerate(flat) if e == x] for x in range(n_experts)]
    starts, slot_of_row, row_of_slot = [0], {}, [-1] * len(flat)
    for slots in by:
        n = -(-len(slots) // BLOCK) * BLOCK
        for r in range(n):
            slot_of_row[starts[-1] + r] = slots[r] if r < len(slots) else -1
            if r < len(slots):
                row_of_slot[slots[r]] = starts[-1] + r
        starts.append(starts[-1] + n)
    return starts, [len(s) for s in by], row_of_slot, slot_of_row


def exponent(amax):
    """The least s >= -126 with amax <= 448 * 2^s; 0 for amax 0; None for a block that is not finite."""
    if not np.isfinite(amax):
        return None
    if amax == 0:
        return 0
    s = -126
    while amax > 448.0 * 2.0**s:
        s += 1
    return s


_E4M3 = None


def e4m3_values():
    """byte -> value, from the format's definition (4 exponent bits, bias 7, 3 mantissa bits; 0x7f and 0xff are NaN)."""
    global _E4M3
    if _E4M3 is None:
        v = np.zeros(256)
        for b in range(256):
            e, m = (b >> 3) & 15, b & 7
            x = m * 2.0**-9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
            v[b] = np.nan if b & 127 == 127 else (-x if b & 128 else x)
        _E4M3 = v
    return _E4M3


def to_e4m3(y):
    """Nearest e4m3 value (ties to the even byte) of every y in [-448, 448], as values."""
    pos = e4m3_values()[:127]
    a = np.abs(y)
    hi = np.clip(np.searchsorted(pos, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - pos[lo], pos[hi] - a
    pick = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return np.sign(y) * pos[pick]


def quantize_rows(y):
    """y [rows, cols] float64 -> values before scaling [rows, cols], scale bytes [blocks, rows]"""
    rows, cols = y.shape
    nb = -(-cols // BLOCK)
    q, s = np.zeros_like(y), np.zeros((nb, rows), np.int64)
    for b in range(nb):
        part = y[:, b * BLOCK : (b + 1) * BLOCK]
        for r in range(rows):
            e = exponent(np.abs(part[r]).max() if not np.isnan(part[r]).any() else np.nan)
            s[b, r] = 255 if e is None else e + 127
            q[r, b * BLOCK : (b + 1) * BLOCK] = np.nan if e is None else to_e4m3(part[r] / 2.0**e)
    return q, s


def quantize_blocks(w):
    rows, cols = w.shape
    rb, cb = -(-rows // BLOCK), -(-cols // BLOCK)
    q, s = np.zeros_like(w), np.zeros((rb, cb), np.int64)
    for i in range(rb):
        for j in range(cb):
            at = np.s_[i * BLOCK : (i + 1) * BLOCK, j * BLOCK : (j + 1) * BLOCK]
            e = exponent(np.abs(w[at]).max() if not np.isnan(w[at]).any() else np.nan)
            s[i, j] = 255 if e is None else e + 127
            q[at] = np.nan if e is None else to_e4m3(w[at] / 2.0**e)
    return q, s


def swiglu(x):
    f = x.shape[1] // 2
    g, u = x[:, :f], x[:, f:]
    return g / (1 + np.exp(-g)) * u


def swiglu_backward(x, grad):
    f = x.shape[1] // 2
    g, u = x[:, :f], x[:, f:]
    s = 1 / (1 + np.exp(-g))
    return np.concatenate([grad * u * s * (1 + g * (1 - s)), grad * g * s], 1)


def operand_values(q, scales):
    """e4m3 tensor [rows, cols] and scale bytes [blocks, >= rows] -> float64 values on the tensor's device"""
    s = torch.exp2(scales[:, : q.shape[0]].double() - 127).t()
    return q.double() * s.repeat_interleave(BLOCK, 1)[:, : q.shape[1]]


def matrix_values(q, scales):
    """e4m3 [matrices, rows, cols] and scale bytes [matrices, row blocks, column blocks] -> float64 values"""
    s = torch.exp2(scales.double() - 127)
    return q.double() * s.repeat_interleave(BLOCK, 1).repeat_interleave(BLOCK, 2)[:, : q.shape[1], : q.shape[2]]
