"""The operators that a MoE layer answers with: weights and rows in 4 bits, their products, and the whole layer for a few tokens.

``own = False``: every operator in elementary torch operations, in 32 bits or more.  ``own = True``: the calls that a
program makes of ``paper_2609_04609_b200.ciera``.  Both work on what ``prepare`` makes.

4 bits are e2m1 (0, 1/2, 1, 3/2, 2, 3, 4, 6 and their negatives), two values to a byte, the even column in the low half, and
one power of two for each 32 values of a row.  Its scale bytes (exponent + 127) lie in atoms of 512 bytes, one for 128 rows
and 128 columns: row r's four bytes at 16 * (r % 32) + 4 * (r % 128 // 32).

The operators, by ``case["op"]``:

* ``quantize``         rows, gathered in the experts' order or silu(g) * u, rounded to 4 bits; and the values they then stand for
* ``quantize_weights`` matrices rounded to 4 bits along their rows, as a product with them needs them; and their values
* ``product``          product of such operands: one matrix, or a matrix for each expert's rows
* ``tokens``           a whole MoE layer for at most 64 tokens, from logits to output: routing, gate and up product, silu(g) * u,
                       down product, weighted sum, with the experts' matrices in 8 or 4 bits
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
SEGMENT = 128  # rows that an expert's segment is a multiple of; rows and columns of an atom of scales
GROUP = 32     # values that share a scale in 4 bits
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
NBYTES = {"bf16": 2, "fp16": 2, "fp32": 4}
E4M3 = torch.float8_e4m3fn
NEG = float("-inf")


def _cdiv(a, b):
    return -(-a // b)


def _up(a, b):
    return _cdiv(a, b) * b


def _quantize(name, source, tokens, top_k, experts, cols, dtype):
    """``source``: plain (``tokens`` rows), gather or swiglu (rows of a layout of ``tokens`` x ``top_k`` slots)."""
    c = {"op": "quantize", "source": source, "tokens": tokens, "top_k": top_k, "experts": experts, "cols": cols, "dtype": dtype,
         "skew": 0.5}
    return {"name": name, **c} if name else c


def _weights(name, matrices, rows, cols, dtype):
    c = {"op": "quantize_weights", "matrices": matrices, "rows": rows, "cols": cols, "dtype": dtype}
    return {"name": name, **c} if name else c


def _product(name, mode, tokens, n, k, out, top_k=1, experts=1, skew=0.5):
    """``dense``: [tokens, k] x [n, k].  ``rows``: the rows of ``tokens`` x ``top_k`` slots, each expert's with its own [n, k]."""
    c = {"op": "product", "mode": mode, "tokens": tokens, "n": n, "k": k, "out": out, "top_k": top_k, "experts": experts,
         "skew": skew}
    return {"name": name, **c} if name else c


def _tokens(name, tokens, experts, top_k, d_model, d_ff, bits, dtype, score="softmax", groups=1, top_groups=1, bias=False,
            renorm=False, scale=1.0, masked=0.0):
    c = {"op": "tokens", "tokens": tokens, "experts": experts, "top_k": top_k, "d_model": d_model, "d_ff": d_ff, "bits": bits,
         "dtype": dtype, "score": score, "groups": groups, "top_groups": top_groups, "bias": bias, "renorm": renorm,
         "scale": scale, "masked": masked}
    return {"name": name, **c} if name else c


def listed():
    return [
        # generation with the gathered weights: one new token through the OLMoE-shaped layer, 8-bit experts; only latency counts
        _tokens("tokens_one", 1, 64, 8, 2048, 1024, 8, "bf16"),
        # the same on experts in 4 bits, half the bytes
        _tokens("tokens_one_4bit", 1, 64, 8, 2048, 1024, 4, "bf16"),
        # five sequences that are continued together on 256 fine-grained experts, chosen within groups and balanced by a bias
        _tokens("tokens_fine_4bit", 5, 256, 8, 2048, 512, 4, "fp16", "sigmoid", 8, 4, True, True, 2.5),
        # the most tokens of such a call: 64 sequences, which between them reach every expert
        _tokens("tokens_batch", 64, 64, 8, 2048, 1024, 8, "bf16"),
        # one token's rows on the way to the product, where only the launch counts
        _quantize("quantize_one_token", "gather", 1, 8, 64, 2048, "bf16"),
        # a prompt of 4096 tokens: rows in the experts' order
        _quantize("quantize_dispatch", "gather", 4096, 8, 64, 2048, "bf16"),
        # a prompt of odd length between the layer's two products, a width that is no multiple of anything
        _quantize("quantize_swiglu_odd", "swiglu", 1001, 8, 64, 1001, "fp16"),
        # one of a layer's three stacks of matrices as it comes out of the gather, turned as the product needs it
        _weights("quantize_weights", 64, 2048, 1024, "bf16"),
        # gate and up product of one token over the 8 experts it reaches; each weight is read once
        _product("product_one_token", "rows", 1, 2048, 2048, "bf16", 8, 64),
        # the same of a prompt of 4096 tokens
        _product("product_prompt", "rows", 4096, 2048, 2048, "bf16", 8, 64),
        # one large matrix
        _product("product_square", "dense", 8192, 8192, 8192, "bf16"),
        # a small one with odd sizes on every side
        _product("product_odd", "dense", 1001, 1111, 777, "fp32"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["quantize", "quantize_weights", "product", "product", "tokens", "tokens", "tokens"])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    if op == "quantize":
        source = rng.choice(["plain", "gather", "swiglu"])
        cols = rng.randint(32, 2048) if rng.random() < 0.5 else 128 * rng.randint(1, 16)
        top_k = 1 if source == "plain" else rng.randint(1, 8)
        return _quantize(None, source, _log(rng, 1, 4096), top_k, rng.randint(max(2, top_k), 64), cols, dtype)
    if op == "quantize_weights":
        rows, cols = rng.randint(16, 2048), rng.randint(16, 2048)
        return _weights(None, _log(rng, 1, min(64, (64 * 2048 * 1024) // (rows * cols))), rows, cols, dtype)
    if op == "product":
        n, k = rng.randint(16, 2048), rng.randint(16, 2048)
        if rng.random() < 0.4:
            n, k = _up(n, 128), _up(k, 128)
        if rng.random() < 0.5:
            return _product(None, "dense", _log(rng, 1, 16384), n, k, dtype)
        top_k = rng.randint(1, 8)
        return _product(None, "rows", _log(rng, 1, 4096), n, k, dtype, top_k, rng.randint(max(2, top_k), 64),
                        rng.choice([0.0, 0.5, 1.0]))
    d_model, d_ff = 128 * rng.randint(1, 16), 128 * rng.randint(1, 16)
    most = min(256, (64 * 2048 * 1024) // (d_model * d_ff))  # experts of this size that the largest case's memory holds
    groups = rng.choice([1, 1, 2, 4])
    experts = groups * rng.randint(2, max(2, most // groups))
    top_groups = rng.randint(1, groups)
    top_k = rng.randint(1, min(10, top_groups * (experts // groups)))
    return _tokens(None, _log(rng, 1, 64), experts, top_k, d_model, d_ff, rng.choice([8, 4]), dtype,
                   rng.choice(["softmax", "sigmoid"]), groups, top_groups, rng.random() < 0.5, rng.random() < 0.5,
                   rng.choice([1.0, 2.5]), rng.choice([0.0, 0.0, 0.3]))


# ------------------------------------------------------------------------------------------------ inputs


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _choices(g, case):
    """int32 [tokens, top_k]: a router's choices, some experts more popular than others."""
    liked = _randn(g, case["experts"]) * case["skew"]
    return (_randn(g, case["tokens"], case["experts"]) + liked).topk(case["top_k"], dim=1).indices.to(torch.int32).contiguous()


def _rows_capacity(n_slots, experts):
    """Rows that segments of a multiple of 128 can take at most."""
    return SEGMENT * (n_slots // SEGMENT + min(experts, n_slots))


def _layout(ids, experts):
    """starts [E + 1] and slot_of_row [capacity] (-1: no slot): the slots in the order of the experts."""
    flat = ids.reshape(-1).long()
    n = flat.numel()
    counts = torch.bincount(flat, minlength=experts)
    starts = torch.zeros(experts + 1, dtype=torch.int64, device=ids.device)
    starts[1:] = ((counts + SEGMENT - 1) // SEGMENT * SEGMENT).cumsum(0)
    order = torch.sort(flat, stable=True).indices
    rank = torch.empty_like(order)
    rank[order] = torch.arange(n, device=ids.device)
    row = starts[flat] + rank - (counts.cumsum(0) - counts)[flat]
    slot_of_row = torch.full((_rows_capacity(n, experts),), -1, dtype=torch.int64, device=ids.device)
    slot_of_row[row] = torch.arange(n, device=ids.device)
    return starts.int(), slot_of_row.int()


def _pow2(s):
    return ((s + 127) << 23).view(torch.float32)


def _exponents4(amax):
    """The least s >= -126 with amax <= 6 * 2^s; 0 for an empty group."""
    m, e = torch.frexp(amax)
    s = e - 3 + (m > 0.75).int()
    return torch.where(amax == 0, torch.zeros_like(s), s.clamp(min=-126))


def _round4(y):
    """y in [-6, 6] to the nearest e2m1 value, ties to the even one."""
    a = y.abs()
    step = torch.where(a < 2, torch.full_like(a, 0.5), torch.where(a < 4, torch.ones_like(a), torch.full_like(a, 2.0)))
    return torch.copysign(torch.round(a / step) * step, y)


def _group4(x):
    """x [..., cols] in 32 or 64 bits: e2m1 values [..., cols] in fp32 and exponents [..., groups of 32]."""
    cols = x.shape[-1]
    g = _cdiv(cols, GROUP)
    y = torch.nn.functional.pad(x, (0, g * GROUP - cols)).reshape(*x.shape[:-1], g, GROUP)
    s = _exponents4(y.abs().amax(-1))
    v = _round4((y * _pow2(-s)[..., None]).float())
    return v.reshape(*x.shape[:-1], g * GROUP)[..., :cols], s


def _values4(v, s):
    """What e2m1 values with these exponents stand for, in fp32."""
    return v * _pow2(s).repeat_interleave(GROUP, dim=-1)[..., : v.shape[-1]]


def _pack4(v):
    """e2m1 values [..., cols] -> bytes [..., cols / 2], rows at multiples of 16 bytes, a last odd column beside a zero."""
    edges = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=v.device)
    code = torch.bucketize(v.abs(), edges).to(torch.uint8) | (torch.signbit(v).to(torch.uint8) << 3)
    code = torch.nn.functional.pad(code, (0, v.shape[-1] % 2))
    buf = _pitched4(*v.shape)
    buf.copy_(code[..., 0::2] | code[..., 1::2] << 4)
    return buf


def _unpack4(q, cols, dtype=torch.float32):
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=dtype, device=q.device)
    table = torch.cat([table, -table])
    return torch.stack([table[(q & 15).int()], table[(q >> 4).int()]], -1).reshape(*q.shape[:-1], -1)[..., :cols]


def _pitched4(*shape):
    """Zero bytes for [..., cols] values of 4 bits whose rows start at multiples of 16 bytes."""
    line = _cdiv(max(shape[-1], 1), 2)
    return torch.zeros(*shape[:-1], _up(line, 16), dtype=torch.uint8, device=DEV)[..., :line]


def _no_atoms(*shape):
    """Scale bytes of [..., rows, cols] before anything is written: all 127."""
    rows, cols = shape[-2:]
    return torch.full((*shape[:-2], _cdiv(rows, SEGMENT), _cdiv(cols, SEGMENT), 512), 127, dtype=torch.uint8, device=DEV)


def _atoms(s):
    """Exponents [..., rows, groups] -> scale bytes [..., ceil(rows / 128), ceil(groups / 4), 512]; 127 in the rest of an atom."""
    rows, groups = s.shape[-2:]
    rb, kb = _cdiv(rows, SEGMENT), _cdiv(groups, 4)
    b = torch.nn.functional.pad(s + 127, (0, kb * 4 - groups, 0, rb * SEGMENT - rows), value=127).to(torch.uint8)
    b = b.reshape(-1, rb, 4, 32, kb, 4).permute(0, 1, 4, 3, 2, 5)
    return b.reshape(*s.shape[:-2], rb, kb, 512).contiguous()


def _from_atoms(a, rows, cols):
    """Exponents [..., rows, groups of 32] out of scale bytes."""
    rb, kb = a.shape[-3:-1]
    s = a.reshape(-1, rb, kb, 32, 4, 4).permute(0, 1, 4, 3, 2, 5).reshape(*a.shape[:-3], rb * SEGMENT, kb * 4)
    return s[..., :rows, : _cdiv(cols, GROUP)].int() - 127


def _group_blocks8(w):
    """w [matrices, rows, cols] -> e4m3 and scale bytes [matrices, row blocks, column blocks], one for each 128 x 128."""
    m, r, c = w.shape
    y = w.reshape(m, r // 128, 128, c // 128, 128)
    f, e = torch.frexp(y.abs().amax((2, 4)))
    s = (e - 9 + (f > 0.875).int()).clamp(min=-126)
    return (y * _pow2(-s)[:, :, None, :, None]).reshape(m, r, c).to(E4M3), (s + 127).to(torch.uint8)


def _values8(q, s, dtype=torch.float32):
    """The same back: [rows, cols] of one matrix or [matrices, rows, cols]."""
    f = torch.exp2(s.double() - 127).to(dtype)
    return q.to(dtype) * f.repeat_interleave(128, -2).repeat_interleave(128, -1)


def _expert_weights(g, experts, rows, cols, bits):
    """The operand and the scales of a stack of random matrices, in 8 or 4 bits, a few experts at a time."""
    parts = []
    for lo in range(0, experts, 16):
        w = _randn(g, min(16, experts - lo), rows, cols) * 0.02
        if bits == 8:
            parts.append(_group_blocks8(w))
        else:
            v, s = _group4(w)
            parts.append((_pack4(v), _atoms(s)))
    return torch.cat([q.view(torch.uint8) for q, _ in parts]).view(E4M3 if bits == 8 else torch.uint8), torch.cat([s for _, s in parts])


def _route_config(case):
    from paper_2609_04609_b200 import ciera

    return ciera.RouteConfig(n_experts=case["experts"], top_k=case["top_k"], n_groups=case["groups"],
                             top_groups=case["top_groups"], group_best=2,
                             score={"softmax": ciera.SCORE_SOFTMAX, "sigmoid": ciera.SCORE_SIGMOID}[case["score"]],
                             renormalise=int(case["renorm"]), scale=case["scale"])


def prepare(case, seed):
    g = _gen(seed)
    op = case["op"]
    st = {"case": case}
    if op == "quantize":
        cols, dt, t = case["cols"], DTYPES[case["dtype"]], case["tokens"]
        rows = t
        if case["source"] != "plain":
            ids = _choices(g, case)
            st["starts"], st["slot_of_row"] = _layout(ids, case["experts"])
            rows = st["slot_of_row"].numel()
        if case["source"] == "swiglu":
            st["x"] = (_randn(g, rows, 2 * cols) * (st["slot_of_row"] >= 0)[:, None]).to(dt)
        else:
            st["x"] = _randn(g, t, cols).to(dt)
        st["q"], st["s"], st["values"] = _pitched4(rows, cols), _no_atoms(rows, cols), torch.zeros(rows, cols, dtype=dt, device=DEV)
        return st
    if op == "quantize_weights":
        m, r, c, dt = case["matrices"], case["rows"], case["cols"], DTYPES[case["dtype"]]
        st["w"] = (_randn(g, m, r, c) * 0.02).to(dt)
        st["qt"], st["s_t"], st["values"] = _pitched4(m, c, r), _no_atoms(m, c, r), torch.zeros(m, c, r, dtype=dt, device=DEV)
        return st
    if op == "product":
        t, n, k, e = case["tokens"], case["n"], case["k"], case["experts"]
        if case["mode"] == "dense":
            a, shape = _randn(g, t, k), (n, k)
        else:
            st["starts"], slots = _layout(_choices(g, case), e)
            a, shape = _randn(g, slots.numel(), k) * (slots >= 0)[:, None], (e, n, k)
            st["longest"] = int((st["starts"][1:] - st["starts"][:-1]).max())  # what the plain form pads every segment to
        for name, x in (("a", a), ("b", _randn(g, *shape) * 0.02)):
            v, s = _group4(x)
            st[name], st[name + "_s"] = _pack4(v), _atoms(s)
        st["out"] = torch.zeros(a.shape[0], n, dtype=DTYPES[case["out"]], device=DEV)
        return st
    t, e, k, d, f, dt = (case["tokens"], case["experts"], case["top_k"], case["d_model"], case["d_ff"], DTYPES[case["dtype"]])
    logits = (_randn(g, t, e) * 1.5).to(dt)
    if case["masked"]:  # experts that are out of reach for a token
        logits = logits.masked_fill(torch.rand(t, e, generator=g, device=DEV) < case["masked"], NEG)
    st["logits"], st["x"] = logits, _randn(g, t, d).to(dt)
    st["bias"] = (torch.rand(e, generator=g, device=DEV) - 0.5) * 0.1 if case["bias"] else None
    st["w1"], st["w1_s"] = _expert_weights(g, e, 2 * f, d, case["bits"])
    st["w2"], st["w2_s"] = _expert_weights(g, e, d, f, case["bits"])
    st["out"] = torch.zeros(t, d, dtype=dt, device=DEV)
    st["experts"] = torch.zeros(t, k, dtype=torch.int32, device=DEV)
    st["weights"] = torch.zeros(t, k, dtype=torch.float32, device=DEV)
    if own:
        from paper_2609_04609_b200 import ciera

        st["config"] = _route_config(case)
        st["workspace"] = torch.zeros(ciera.expert_tokens_workspace_bytes(st["config"], t, d, f), dtype=torch.uint8, device=DEV)
    return st


# ------------------------------------------------------------------------------------------------ plain forms


def _plain_quantize(st):
    case, x = st["case"], st["x"]
    if case["source"] == "plain":
        y = x.float()
    elif case["source"] == "gather":
        slot = st["slot_of_row"].long()
        y = torch.where((slot >= 0)[:, None], x.float()[(slot // case["top_k"]).clamp(min=0)], torch.zeros(1, device=DEV))
    else:  # in 64 bits: a group's largest value may be next to the border of its scale
        gate, up = x[:, : case["cols"]].double(), x[:, case["cols"] :].double()
        y = gate * torch.sigmoid(gate) * up
    v, s = _group4(y)
    return _values4(v, s).to(x.dtype), _atoms(s)


def _plain_weights(st):
    v, s = _group4(st["w"].float().transpose(1, 2))
    return _values4(v, s).to(st["w"].dtype), _atoms(s)


def _operand4(q, s, cols):
    return _values4(_unpack4(q, cols), _from_atoms(s, q.shape[-2], cols))


def _plain_product(st):
    case, dt = st["case"], st["out"].dtype
    a, b = _operand4(st["a"], st["a_s"], case["k"]), _operand4(st["b"], st["b_s"], case["k"])
    if case["mode"] == "dense":
        return (a @ b.t()).to(dt)
    starts = st["starts"].long()
    at = starts[:-1, None] + torch.arange(st["longest"], device=a.device)[None]  # every segment as long as the longest
    live = at < starts[1:, None]
    c = torch.bmm(a[torch.where(live, at, torch.zeros_like(at))] * live[:, :, None], b.transpose(1, 2))
    out = torch.zeros(a.shape[0] + 1, case["n"], device=a.device)
    out[torch.where(live, at, torch.full_like(at, a.shape[0])).reshape(-1)] = c.reshape(-1, case["n"])
    return out[:-1].to(dt)


def _plain_route(case, logits, bias):
    """Scores and choice in 64 bits: two experts' scores may be next to each other."""
    t, e = logits.shape
    g, k = case["groups"], case["top_k"]
    x = logits.double()
    open_ = x != NEG
    if case["score"] == "sigmoid":
        s = torch.sigmoid(x)
    else:
        s = torch.exp(x - x.amax(1, keepdim=True).clamp(min=-1e300)) * open_
        s = s / s.sum(1, keepdim=True).clamp(min=1e-300)
    c = (s if bias is None else s + bias.double()).masked_fill(~open_, NEG)
    if g > 1:
        by = c.reshape(t, g, e // g).sort(dim=2, descending=True).values[:, :, :2]
        value = torch.where(by == NEG, torch.zeros_like(by), by).sum(2).masked_fill(by[:, :, 0] == NEG, NEG)
        best = value.sort(dim=1, descending=True, stable=True).indices[:, : case["top_groups"]]
        keep = torch.zeros(t, g, dtype=torch.bool, device=c.device).scatter_(1, best, True)
        c = c.masked_fill(~keep.repeat_interleave(e // g, dim=1), NEG)
    v, i = c.sort(dim=1, descending=True, stable=True)
    v, i = v[:, :k], i[:, :k]
    w = s.gather(1, i).masked_fill(v == NEG, 0.0)
    if case["renorm"]:
        w = w / w.sum(1, keepdim=True).clamp(min=1e-300)
    return i.masked_fill(v == NEG, -1).int(), (w * case["scale"]).float()


def _matrix(st, name, e, cols):
    """Matrices e (a number or a tensor of them) of a stack of experts' weights, in fp32."""
    q, s = st[name], st[name + "_s"]
    return _values8(q.view(torch.uint8)[e].view(E4M3), s[e]) if st["case"]["bits"] == 8 else _operand4(q[e], s[e], cols)


def _plain_tokens(st):
    case = st["case"]
    t, k, d, f = case["tokens"], case["top_k"], case["d_model"], case["d_ff"]
    ids, weights = _plain_route(case, st["logits"], st["bias"])
    x = st["x"].float()

    def middle(h):
        return h[..., :f] * torch.sigmoid(h[..., :f]) * h[..., f:]

    if t * k <= 64:  # the chosen matrices, slot by slot
        e = ids.reshape(-1).long().clamp(min=0)
        h = torch.bmm(_matrix(st, "w1", e, d), x.repeat_interleave(k, 0)[:, :, None])[:, :, 0]
        y = torch.bmm(_matrix(st, "w2", e, f), middle(h)[:, :, None])[:, :, 0].reshape(t, k, d)
        out = (y * (weights * (ids >= 0))[:, :, None]).sum(1)
    else:  # all tokens on all experts, of which the chosen ones count
        share = torch.zeros(t, case["experts"], device=DEV).scatter_add_(1, ids.long().clamp(min=0), weights * (ids >= 0))
        out = torch.zeros(t, d, device=DEV)
        for e in range(case["experts"]):
            out += share[:, e, None] * (middle(x @ _matrix(st, "w1", e, d).t()) @ _matrix(st, "w2", e, f).t())
    return out.to(st["x"].dtype), ids, weights


def _run_plain(st):
    return {"quantize": _plain_quantize, "quantize_weights": _plain_weights, "product": _plain_product,
            "tokens": _plain_tokens}[st["case"]["op"]](st)


# ------------------------------------------------------------------------------------------------ the framework's calls


def _run_own(st):
    from paper_2609_04609_b200 import ciera

    case = st["case"]
    op = case["op"]
    if op == "quantize":
        ciera.fp4_quantize_rows(st["x"], st["q"], st["s"],
                                kind=ciera.SOURCE_SWIGLU if case["source"] == "swiglu" else ciera.SOURCE_ROWS,
                                slot_of_row=st.get("slot_of_row"), top_k=case["top_k"], starts=st.get("starts"))
        ciera.fp4_values(st["q"], st["s"], st["values"])
        return st["values"], st["s"]
    if op == "quantize_weights":
        ciera.fp4_quantize_matrices(st["w"], qt=st["qt"], scales_t=st["s_t"])
        ciera.fp4_values(st["qt"], st["s_t"], st["values"])
        return st["values"], st["s_t"]
    if op == "product":
        ciera.fp4_matmul(st["a"], st["a_s"], st["b"], st["b_s"], st["out"], starts=st.get("starts"))
        return st["out"]
    ciera.expert_tokens(st["config"], st["x"], st["logits"], st["bias"], st["w1"], st["w1_s"], st["w2"], st["w2_s"], st["out"],
                        st["experts"], st["weights"], st["workspace"])
    return st["out"], st["experts"], st["weights"]


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------------------------------------ what a pass cannot do without


def _bytes4(rows, cols):
    """Of rows in 4 bits, with their scales."""
    return rows * (_cdiv(cols, 2) + _cdiv(cols, GROUP))


def work(case):
    op = case["op"]
    t = case.get("tokens", 0)
    if op == "quantize":
        v, cols = NBYTES[case["dtype"]], case["cols"]
        rows = t * case["top_k"]
        read = (2 * rows if case["source"] == "swiglu" else t) * cols * v + (0 if case["source"] == "plain" else 4 * rows)
        # written once as 4 bits, and once as the values they stand for
        return {"bytes": read + _bytes4(rows, cols) + rows * cols * v, "flops": 2 * rows * cols}
    if op == "quantize_weights":
        m, r, c, v = case["matrices"], case["rows"], case["cols"], NBYTES[case["dtype"]]
        return {"bytes": 2 * m * r * c * v + _bytes4(m * c, r), "flops": 2 * m * r * c}
    if op == "product":
        n, k, v, rows = case["n"], case["k"], NBYTES[case["out"]], t * case["top_k"]
        matrices = min(case["experts"], rows) if case["mode"] == "rows" else 1
        return {"bytes": _bytes4(rows, k) + matrices * _bytes4(n, k) + rows * n * v, "flops": 2 * rows * n * k}
    e, k, d, f, v = case["experts"], case["top_k"], case["d_model"], case["d_ff"], NBYTES[case["dtype"]]
    reached = round(e * (1 - (1 - k / e) ** t))  # experts that t tokens with k each reach between them
    one = 3 * d * f if case["bits"] == 8 else _bytes4(2 * f, d) + _bytes4(d, f)
    return {"bytes": reached * one + t * (2 * d * v + e * v + 8 * k), "flops": 6 * t * k * d * f}


# ------------------------------------------------------------------------------------------------ 64 bits


def _exact_exponent4(amax):
    """The least s >= -126 with amax <= 6 * 2^s."""
    s = torch.ceil(torch.log2(amax.clamp(min=1e-300) / 6.0))
    s = torch.where(amax > 6.0 * torch.exp2(s), s + 1, s)
    s = torch.where(amax <= 6.0 * torch.exp2(s - 1), s - 1, s).clamp(min=-126)
    return torch.where(amax == 0, torch.zeros_like(s), s)


def _exact_rows4(y):
    """The values that rows in 64 bits are rounded to, from the format's definition: one bit of mantissa, least exponent 0."""
    out = torch.zeros_like(y)
    for lo in range(0, y.shape[-1], GROUP):
        part = y[..., lo : lo + GROUP]
        unit = torch.exp2(_exact_exponent4(part.abs().amax(-1, keepdim=True)))
        _, e = torch.frexp(part / unit)
        step = unit * torch.exp2((e - 1).clamp(min=0).double() - 1)
        out[..., lo : lo + GROUP] = torch.round(part / step) * step
    return out


def _exact_operand4(q, s, cols):
    """From codes: sign, two bits of exponent (bias 1), one of mantissa; times the row's power of two for 32 columns."""
    code = torch.stack([q & 15, q >> 4], -1).reshape(*q.shape[:-1], -1)[..., :cols].double()
    sign = torch.where(code >= 8, -1.0, 1.0).double()
    code = code % 8
    e, m = torch.floor(code / 2), code % 2
    value = torch.where(e == 0, m / 2, torch.exp2(e - 1) * (1 + m / 2))
    row, col = torch.arange(q.shape[-2], device=q.device)[:, None], torch.arange(cols, device=q.device)[None]
    byte = s[..., row // 128, col // 128, 16 * (row % 32) + 4 * (row % 128 // 32) + col % 128 // 32]
    return sign * value * torch.exp2(byte.double() - 127)


def _exact_route(case, logits, bias):
    """One choice after the other."""
    x = logits.double()
    t, e = x.shape
    g = case["groups"]
    can = x > NEG
    z = torch.where(can, x, torch.zeros_like(x))
    if case["score"] == "sigmoid":
        s = torch.where(can, 1 / (1 + torch.exp(-z)), torch.zeros_like(z))
    else:
        p = torch.where(can, torch.exp(z), torch.zeros_like(z))
        s = p / p.sum(1, keepdim=True).clamp(min=1e-300)
    key = s + (0 if bias is None else bias.double()[None])
    if g > 1:
        inner = torch.where(can, key, torch.full_like(key, NEG)).reshape(t, g, -1)
        first = inner.amax(2)
        rest = inner.scatter(2, inner.argmax(2, keepdim=True), NEG).amax(2) if inner.shape[2] > 1 else torch.full_like(first, NEG)
        total = first + torch.where(rest == NEG, torch.zeros_like(rest), rest)
        left = torch.ones(t, g, dtype=torch.bool, device=x.device)
        for _ in range(case["top_groups"]):
            left.scatter_(1, torch.where(left, total, torch.full_like(total, NEG)).argmax(1, keepdim=True), False)
        can = can & ~left.repeat_interleave(e // g, 1)
    ids, ws = [], []
    for _ in range(case["top_k"]):
        top = torch.where(can, key, torch.full_like(key, NEG)).argmax(1, keepdim=True)
        some = can.any(1, keepdim=True)
        ids.append(torch.where(some, top, torch.full_like(top, -1)))
        ws.append(torch.where(some, s.gather(1, top), torch.zeros_like(s[:, :1])))
        can = can.scatter(1, top, False)
    w = torch.cat(ws, 1)
    if case["renorm"]:
        total = w.sum(1, keepdim=True)
        w = torch.where(total > 0, w / torch.where(total > 0, total, torch.ones_like(total)), w)
    return torch.cat(ids, 1).int(), w * case["scale"]


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op == "quantize":
        x, cols = st["x"].double(), case["cols"]
        if case["source"] == "plain":
            return _exact_rows4(x), None
        y = torch.zeros(st["slot_of_row"].numel(), cols, dtype=torch.float64, device=DEV)
        row = (st["slot_of_row"] >= 0).nonzero()[:, 0]
        if case["source"] == "gather":
            y[row] = x[st["slot_of_row"][row].long() // case["top_k"]]
        else:
            y[row] = x[row, :cols] * x[row, cols:] / (1 + torch.exp(-x[row, :cols]))
        return _exact_rows4(y), None
    if op == "quantize_weights":
        return _exact_rows4(st["w"].double().transpose(1, 2).contiguous()), None
    if op == "product":
        k = case["k"]
        a = _exact_operand4(st["a"], st["a_s"], k)
        if case["mode"] == "dense":
            return a @ _exact_operand4(st["b"], st["b_s"], k).t()
        starts = st["starts"].tolist()
        out = torch.zeros(st["out"].shape, dtype=torch.float64, device=DEV)
        for e in range(case["experts"]):
            if starts[e] < starts[e + 1]:
                out[starts[e] : starts[e + 1]] = a[starts[e] : starts[e + 1]] @ _exact_operand4(st["b"][e], st["b_s"][e], k).t()
        return out
    d, f = case["d_model"], case["d_ff"]
    ids, weights = _exact_route(case, st["logits"], st["bias"])
    x = st["x"].double()
    out = torch.zeros(x.shape, dtype=torch.float64, device=DEV)

    def matrix(name, e, cols):
        q, s = st[name][e], st[name + "_s"][e]
        return _values8(q, s, torch.float64) if case["bits"] == 8 else _exact_operand4(q, s, cols)

    for e in ids.unique().tolist():
        if e < 0:
            continue
        t, j = (ids == e).nonzero(as_tuple=True)
        h = x[t] @ matrix("w1", e, d).t()
        a = h[:, :f] * h[:, f:] / (1 + torch.exp(-h[:, :f]))
        out.index_add_(0, t, weights[t, j].double()[:, None] * (a @ matrix("w2", e, f).t()))
    return out, ids, weights
