"""The operators of a MoE layer that follow the gather of its experts' weights, as a list of cases with sizes.

``own = False``: every operator in elementary torch operations, in 32 bits or more.  ``own = True``: the calls that a
program makes of ``paper_2609_04609_b200.ciera``.  Both work on what ``prepare`` makes.

The operators, by ``case["op"]``:

* ``route``, ``route_backward``      scores of the experts, top k within the best groups, weights; gradient of the logits
* ``layout``                         the slots (token, choice) in the order of the experts, segments of 128 rows
* ``quantize``                       rows of a product's operand, formed and rounded to e4m3 with one power of two for each
                                     128 values of a row; also transposed, with one for each 128 rows
* ``quantize_blocks``                matrices in e4m3 with one power of two for each block of 128 x 128
* ``product``                        product of such operands: one matrix, a matrix for each expert's rows, or one result
                                     for each expert (gradient of the weights)
* ``combine``, ``combine_backward``  weighted sum of a token's rows; gradients of weights and rows
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
B = 128  # values that share a scale; rows that a segment is a multiple of
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
NBYTES = {"bf16": 2, "fp16": 2, "fp32": 4}
E4M3 = torch.float8_e4m3fn
NEG = float("-inf")


def _cdiv(a, b):
    return -(-a // b)


def _up(a, b):
    return _cdiv(a, b) * b


def _route(name, op, tokens, experts, top_k, dtype, score="softmax", groups=1, top_groups=1, bias=False, renorm=False,
           scale=1.0, masked=0.0):
    c = {"op": op, "tokens": tokens, "experts": experts, "top_k": top_k, "dtype": dtype, "score": score, "groups": groups,
         "top_groups": top_groups, "bias": bias, "renorm": renorm, "scale": scale, "masked": masked}
    return {"name": name, **c} if name else c


def _layout(name, tokens, top_k, experts, skew=0.5, dropped=0.0):
    c = {"op": "layout", "tokens": tokens, "top_k": top_k, "experts": experts, "skew": skew, "dropped": dropped}
    return {"name": name, **c} if name else c


def _quantize(name, source, tokens, top_k, experts, cols, dtype, transposed, skew=0.5):
    """``source``: plain (``tokens`` rows), gather, weighted, swiglu, swiglu_backward (rows of a layout)."""
    c = {"op": "quantize", "source": source, "tokens": tokens, "top_k": top_k, "experts": experts, "cols": cols,
         "dtype": dtype, "transposed": transposed, "skew": skew}
    return {"name": name, **c} if name else c


def _blocks(name, matrices, rows, cols, dtype, transposed):
    c = {"op": "quantize_blocks", "matrices": matrices, "rows": rows, "cols": cols, "dtype": dtype, "transposed": transposed}
    return {"name": name, **c} if name else c


def _product(name, mode, tokens, n, k, out, top_k=1, experts=1, skew=0.5, b_rows=False):
    """``dense``: [tokens, k] x [n, k].  ``rows``: the rows of ``tokens`` x ``top_k`` slots, each expert's with its own
    [n, k].  ``contract``: for each expert [n, its rows] x [k, its rows]."""
    c = {"op": "product", "mode": mode, "tokens": tokens, "n": n, "k": k, "out": out, "top_k": top_k, "experts": experts,
         "skew": skew, "b_rows": b_rows}
    return {"name": name, **c} if name else c


def _combine(name, op, tokens, top_k, experts, cols, dtype, weighted=True, dropped=0.0):
    c = {"op": op, "tokens": tokens, "top_k": top_k, "experts": experts, "cols": cols, "dtype": dtype, "weighted": weighted,
         "dropped": dropped, "skew": 0.5}
    return {"name": name, **c} if name else c


def listed():
    return [
        # serving: the router on one new token of the OLMoE-shaped layer; only latency counts
        _route("route_one_token", "route", 1, 64, 8, "bf16"),
        # fine-grained experts (256), balanced by a bias, chosen within groups: a training batch
        _route("route_groups", "route", 16384, 256, 8, "bf16", "sigmoid", 8, 4, True, True, 2.5),
        # the same training step backwards, on the 64 experts of the OLMoE-shaped layer
        _route("route_backward", "route_backward", 32768, 64, 8, "fp32"),
        # a small batch of tokens being served: 33 tokens, ragged
        _layout("layout_serving", 33, 8, 64),
        # a long training batch over fine-grained experts
        _layout("layout_training", 32771, 8, 256, 0.8),
        # dispatch: tokens gathered into the experts' order for the first product and for the weights' gradient
        _quantize("quantize_dispatch", "gather", 4096, 8, 64, 2048, "bf16", True),
        # one of a layer's three stacks of matrices as it comes out of the gather, both orientations
        _blocks("quantize_weights", 64, 2048, 1024, "bf16", True),
        # serving: gate and up product of one token over the 8 experts it reaches; each weight is read once
        _product("product_one_token", "rows", 1, 2048, 2048, "bf16", 8, 64),
        # training: gate and up product of a batch of 4096 tokens, each on 8 experts
        _product("product_forward", "rows", 4096, 2048, 2048, "bf16", 8, 64),
        # training: gradient of the same weights
        _product("product_weight_gradient", "contract", 4096, 2048, 2048, "fp32", 8, 64, b_rows=True),
        # the experts' rows back to their tokens, a width that is no multiple of anything
        _combine("combine_odd", "combine", 1023, 8, 64, 2050, "bf16"),
        # training: the gradients of the same sum
        _combine("combine_backward", "combine_backward", 4096, 8, 64, 2048, "bf16"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["route", "route", "layout", "quantize", "quantize", "quantize_blocks", "product", "product", "product",
                     "combine"])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    if op == "route":
        groups = rng.choice([1, 1, 2, 4, 8])
        experts = groups * rng.randint(max(1, 8 // groups), 256 // groups)
        top_groups = rng.randint(1, groups)
        top_k = rng.randint(1, min(12, top_groups * (experts // groups)))
        tokens = _log(rng, 1, min(32768, (16384 * 256) // experts))
        score = rng.choice(["softmax", "sigmoid"])
        return _route(None, rng.choice(["route", "route", "route_backward"]), tokens, experts, top_k, dtype, score, groups,
                      top_groups, rng.random() < 0.5, rng.random() < 0.5, rng.choice([1.0, 2.5]), rng.choice([0.0, 0.0, 0.3]))
    if op == "layout":
        top_k = rng.randint(1, 10)
        return _layout(None, _log(rng, 1, 262144 // top_k), top_k, rng.randint(max(2, top_k), 320), rng.choice([0.0, 0.5, 1.5]),
                       rng.choice([0.0, 0.1]))
    if op == "quantize":
        source = rng.choice(["plain", "gather", "weighted", "swiglu", "swiglu_backward"])
        cols = rng.randint(64, 2048) if rng.random() < 0.5 else 128 * rng.randint(1, 16)
        cols += cols % 2 if source == "swiglu_backward" else 0
        top_k = 1 if source == "plain" else rng.randint(1, 8)
        return _quantize(None, source, _log(rng, 1, 4096), top_k, rng.randint(max(2, top_k), 64), cols, dtype,
                         rng.random() < 0.5)
    if op == "quantize_blocks":
        rows, cols = rng.randint(16, 2048), rng.randint(16, 2048)
        return _blocks(None, _log(rng, 1, min(64, (64 * 2048 * 1024) // (rows * cols))), rows, cols, dtype, rng.random() < 0.5)
    if op == "product":
        mode = rng.choice(["dense", "rows", "contract"])
        n, k = rng.randint(16, 2048), rng.randint(16, 2048)
        if rng.random() < 0.4:
            n, k = _up(n, 128), _up(k, 128)
        if mode == "dense":
            return _product(None, mode, _log(rng, 1, 16384), n, k, dtype, b_rows=rng.random() < 0.5)
        top_k = rng.randint(1, 8)
        return _product(None, mode, _log(rng, 1, 4096), n, k, dtype, top_k, rng.randint(max(2, top_k), 64),
                        rng.choice([0.0, 0.5, 1.0]), mode == "contract")
    top_k = rng.randint(1, 8)
    return _combine(None, rng.choice(["combine", "combine_backward"]), _log(rng, 1, 4096), top_k, rng.randint(max(2, top_k), 64),
                    rng.randint(64, 2048), dtype, rng.random() < 0.7, rng.choice([0.0, 0.1]))


# ------------------------------------------------------------------------------------------------ inputs


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _choices(g, case):
    """int32 [tokens, top_k]: a router's choices, some experts more popular than others; some dropped (-1)."""
    t, e = case["tokens"], case["experts"]
    liked = _randn(g, e) * case["skew"]
    ids = (_randn(g, t, e) + liked).topk(case["top_k"], dim=1).indices.to(torch.int32)
    if case.get("dropped"):
        ids = torch.where(torch.rand(ids.shape, generator=g, device=DEV) < case["dropped"], torch.full_like(ids, -1), ids)
    return ids.contiguous()


def _rows_capacity(n_slots, experts):
    """Rows that segments of a multiple of 128 can take at most."""
    return B * (n_slots // B + min(experts, n_slots))


def _plain_layout(ids, experts):
    """starts [E + 1], counts [E], row_of_slot [slots], slot_of_row [capacity] (-1: no slot)."""
    flat = ids.reshape(-1).long()
    n = flat.numel()
    ok = (flat >= 0) & (flat < experts)
    key = torch.where(ok, flat, torch.full_like(flat, experts))
    counts = torch.bincount(key, minlength=experts + 1)[:experts]
    starts = torch.zeros(experts + 1, dtype=torch.int64, device=ids.device)
    starts[1:] = ((counts + B - 1) // B * B).cumsum(0)
    first = torch.zeros(experts + 1, dtype=torch.int64, device=ids.device)
    first[1:] = counts.cumsum(0)
    order = torch.sort(key, stable=True).indices
    place = torch.empty_like(order)
    place[order] = torch.arange(n, device=ids.device)
    row = torch.where(ok, starts[key.clamp(max=experts)] + place - first[key.clamp(max=experts)], torch.full_like(flat, -1))
    slot_of_row = torch.full((_rows_capacity(n, experts) + 1,), -1, dtype=torch.int64, device=ids.device)
    slot_of_row[torch.where(ok, row, torch.full_like(row, -1))] = torch.arange(n, device=ids.device)
    return (starts.int(), counts.int(), row.int().reshape(ids.shape), slot_of_row[:-1].int())


def _exponents(amax):
    """amax: the exponent s of the scale 2^s, the least with amax <= 448 * 2^s, at least -126; 0 for an empty group."""
    m, e = torch.frexp(amax)
    s = e - 9 + (m > 0.875).int()
    return torch.where(amax == 0, torch.zeros_like(s), s.clamp(min=-126))


def _pow2(s):
    return ((s + 127) << 23).view(torch.float32)


def _group(x):
    """x [rows, cols] in 32 or 64 bits -> e4m3 [rows, cols] and scale bytes [blocks of 128 columns, rows]."""
    rows, cols = x.shape
    kb = _cdiv(cols, B)
    y = torch.nn.functional.pad(x, (0, kb * B - cols)).reshape(rows, kb, B)
    s = _exponents(y.abs().amax(2))
    q = (y * _pow2(-s)[:, :, None]).reshape(rows, kb * B)[:, :cols].float().to(E4M3)
    return q, (s + 127).to(torch.uint8).t()


def _group_blocks(w):
    """w [matrices, rows, cols] -> e4m3 and scale bytes [matrices, row blocks, column blocks]."""
    m, r, c = w.shape
    rb, cb = _cdiv(r, B), _cdiv(c, B)
    y = torch.nn.functional.pad(w.float(), (0, cb * B - c, 0, rb * B - r)).reshape(m, rb, B, cb, B)
    s = _exponents(y.abs().amax((2, 4)))
    q = (y * _pow2(-s)[:, :, None, :, None]).reshape(m, rb * B, cb * B)[:, :r, :c].to(E4M3)
    return q, (s + 127).to(torch.uint8)


def _pitched(*shape, dtype=E4M3):
    """Zeros whose rows start at multiples of 16 bytes."""
    return torch.zeros(*shape[:-1], _up(max(shape[-1], 1), 16), dtype=torch.uint8, device=DEV).view(dtype)[..., : shape[-1]]


def _scales(blocks, rows):
    return torch.zeros(blocks, _up(max(rows, 1), 16), dtype=torch.uint8, device=DEV)


def _put(buf, q):
    buf.view(torch.uint8).copy_(q.view(torch.uint8))
    return buf


def _put_rows(s, rows):
    buf = _scales(s.shape[0], rows)
    buf[:, :rows] = s
    return buf


def _score_names():
    from paper_2609_04609_b200 import ciera

    return {"softmax": ciera.SCORE_SOFTMAX, "sigmoid": ciera.SCORE_SIGMOID}


def _route_config(case):
    from paper_2609_04609_b200 import ciera

    return ciera.RouteConfig(n_experts=case["experts"], top_k=case["top_k"], n_groups=case["groups"],
                             top_groups=case["top_groups"], group_best=2, score=_score_names()[case["score"]],
                             renormalise=int(case["renorm"]), scale=case["scale"])


def prepare(case, seed):
    g = _gen(seed)
    op = case["op"]
    st = {"case": case}
    if op in ("route", "route_backward"):
        t, e, k = case["tokens"], case["experts"], case["top_k"]
        logits = (_randn(g, t, e) * 1.5).to(DTYPES[case["dtype"]])
        if case["masked"]:
            gone = torch.rand(t, e, generator=g, device=DEV) < case["masked"]
            gone[::97] = True
            logits = logits.masked_fill(gone, NEG)
        st["logits"] = logits
        st["bias"] = (torch.rand(e, generator=g, device=DEV) - 0.5) * 0.1 if case["bias"] else None
        st["experts"] = torch.zeros(t, k, dtype=torch.int32, device=DEV)
        st["weights"] = torch.zeros(t, k, dtype=torch.float32, device=DEV)
        if op == "route_backward":
            st["experts"] = _plain_route(case, logits, st["bias"])[0]
            st["dweights"] = _randn(g, t, k) * 1e-2
            st["dlogits"] = torch.zeros_like(logits)
        if own:
            st["config"] = _route_config(case)
        return st
    if op == "quantize_blocks":
        m, r, c = case["matrices"], case["rows"], case["cols"]
        st["w"] = (_randn(g, m, r, c) * 0.02).to(DTYPES[case["dtype"]])
        st["q"], st["s"] = _pitched(m, r, c), torch.zeros(m, _cdiv(r, B), _cdiv(c, B), dtype=torch.uint8, device=DEV)
        st["qt"], st["s_t"] = _pitched(m, c, r), torch.zeros(m, _cdiv(c, B), _cdiv(r, B), dtype=torch.uint8, device=DEV)
        return st
    if op == "product" and case["mode"] == "dense":
        t, n, k = case["tokens"], case["n"], case["k"]
        qa, sa = _group(_randn(g, t, k))
        st["a"], st["a_s"] = _put(_pitched(t, k), qa), _put_rows(sa, t)
        w = _randn(g, n, k) * 0.02
        if case["b_rows"]:
            qb, sb = _group(w)
            st["b"], st["b_s"] = _put(_pitched(n, k), qb), _put_rows(sb, n)
        else:
            qb, sb = _group_blocks(w[None])
            st["b"], st["b_s"] = _put(_pitched(1, n, k), qb), sb
        st["out"] = torch.zeros(t, n, dtype=DTYPES[case["out"]], device=DEV)
        return st
    if op == "quantize" and case["source"] == "plain":
        rows, dt = case["tokens"], DTYPES[case["dtype"]]
        st["x"] = (_randn(g, rows, case["cols"])).to(dt)
        return _quantize_outputs(st, rows, case["cols"])
    ids = _choices(g, case)
    e, n_slots = case["experts"], ids.numel()
    cap = _rows_capacity(n_slots, e)
    st["ids"] = ids
    if op == "layout":
        st["starts"] = torch.zeros(e + 1, dtype=torch.int32, device=DEV)
        st["counts"] = torch.zeros(e, dtype=torch.int32, device=DEV)
        st["row_of_slot"] = torch.zeros_like(ids)
        st["slot_of_row"] = torch.full((cap,), -1, dtype=torch.int32, device=DEV)
        if own:
            from paper_2609_04609_b200 import ciera

            st["workspace"] = torch.zeros(ciera.expert_layout_workspace_bytes(n_slots, e), dtype=torch.uint8, device=DEV)
        return st
    starts, counts, row_of_slot, slot_of_row = _plain_layout(ids, e)
    st.update(starts=starts, counts=counts, row_of_slot=row_of_slot, slot_of_row=slot_of_row)
    live = (slot_of_row >= 0)[:, None]
    if op == "quantize":
        cols, dt = case["cols"], DTYPES[case["dtype"]]
        if case["source"] in ("gather", "weighted"):
            st["x"] = _randn(g, case["tokens"], cols).to(dt)
            if case["source"] == "weighted":
                st["row_weights"] = torch.rand(case["tokens"], case["top_k"], generator=g, device=DEV)
        else:
            f = cols if case["source"] == "swiglu" else cols // 2
            st["x"] = (_randn(g, cap, 2 * f) * live).to(dt)
            if case["source"] == "swiglu_backward":
                st["grad"] = (_randn(g, cap, f) * 1e-3 * live).to(dt)
        return _quantize_outputs(st, cap, cols)
    if op == "product":
        n, k = case["n"], case["k"]
        if case["mode"] == "rows":
            qa, sa = _group(_randn(g, cap, k) * live)
            qb, sb = _group_blocks(_randn(g, e, n, k) * 0.02)
            st["a"], st["a_s"] = _put(_pitched(cap, k), qa), _put_rows(sa, cap)
            st["b"], st["b_s"] = _put(_pitched(e, n, k), qb), sb
            st["out"] = torch.zeros(cap, n, dtype=DTYPES[case["out"]], device=DEV)
        else:
            for name, width, size in (("a", n, 1e-3), ("b", k, 1.0)):
                q, s = _group((_randn(g, cap, width) * live * size).t())
                st[name], st[name + "_s"] = _put(_pitched(width, cap), q), _put_rows(s, width)
            st["out"] = torch.zeros(e, n, k, dtype=DTYPES[case["out"]], device=DEV)
        # the longest segment: what the plain form pads every segment to
        st["longest"] = int((starts[1:] - starts[:-1]).max())
        return st
    cols, dt = case["cols"], DTYPES[case["dtype"]]
    st["rows"] = (_randn(g, cap, cols) * live).to(dt)
    st["weights"] = torch.rand(case["tokens"], case["top_k"], generator=g, device=DEV) if case["weighted"] else None
    st["out"] = torch.zeros(case["tokens"], cols, dtype=dt, device=DEV)
    if op == "combine_backward":
        st["dout"] = (_randn(g, case["tokens"], cols) * 1e-2).to(dt)
        st["dweights"] = torch.zeros(case["tokens"], case["top_k"], device=DEV)
        st["drows"] = torch.zeros(cap, cols, dtype=dt, device=DEV)
    return st


def _quantize_outputs(st, rows, cols):
    st["q"], st["s"] = _pitched(rows, cols), _scales(_cdiv(cols, B), rows)
    st["qt"], st["s_t"] = _pitched(cols, rows), _scales(_cdiv(rows, B), cols)
    return st


# ------------------------------------------------------------------------------------------------ plain forms


def _scores(case, logits):
    """Scores in 64 bits (two experts' scores plus bias may be next to each other) and which experts may be chosen."""
    x = logits.double()
    open_ = ~torch.isnan(x) & (x != NEG)
    x = torch.where(open_, x, torch.full_like(x, NEG)).clamp(max=torch.finfo(torch.float32).max)
    if case["score"] == "sigmoid":
        return torch.sigmoid(x), open_
    s = torch.exp(x - x.amax(1, keepdim=True).clamp(min=torch.finfo(torch.float32).min))
    return s / s.sum(1, keepdim=True).clamp(min=1e-300), open_


def _plain_route(case, logits, bias):
    t, e = logits.shape
    g, k = case["groups"], case["top_k"]
    s, open_ = _scores(case, logits)
    c = s if bias is None else s + bias.double()
    c = c.masked_fill(~open_, NEG)
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


def _plain_route_backward(case, logits, experts, dweights):
    s, open_ = _scores(case, logits)
    chosen = experts >= 0
    i = experts.long().clamp(min=0)
    sk = s.gather(1, i) * chosen
    d = dweights.double() * chosen * case["scale"]
    if case["renorm"]:
        total = sk.sum(1, keepdim=True).clamp(min=1e-300)
        d = (d - (d * sk).sum(1, keepdim=True) / total) / total * chosen
    ds = torch.zeros_like(s).scatter_add_(1, i, d)
    if case["score"] == "sigmoid":
        dl = ds * s * (1 - s)
    else:
        dl = s * (ds - (ds * s).sum(1, keepdim=True))
    return dl.masked_fill(~open_, 0.0).to(logits.dtype)


def _source(st):
    """The rows that are rounded, in 32 bits (in 64 behind an exponential: a group's largest value may be next to the
    border of its scale), and how many of them are written."""
    case, x = st["case"], st["x"]
    src = case["source"]
    if src == "plain":
        return x.float()
    if src in ("gather", "weighted"):
        slot = st["slot_of_row"].long()
        y = x.float()[(slot // case["top_k"]).clamp(min=0)]
        if src == "weighted":
            y = y * st["row_weights"].reshape(-1)[slot.clamp(min=0)][:, None]
        return torch.where((slot >= 0)[:, None], y, torch.zeros_like(y))
    live = (st["slot_of_row"] >= 0)[:, None]
    f = x.shape[1] // 2
    gate, up = x[:, :f].double(), x[:, f:].double()
    sig = torch.sigmoid(gate)
    if src == "swiglu":
        return torch.where(live, gate * sig * up, torch.zeros_like(gate))
    d = torch.where(live, st["grad"].double(), torch.zeros_like(gate))
    return torch.cat([d * up * sig * (1 + gate * (1 - sig)), d * gate * sig], 1)


def _plain_quantize(st):
    case, y = st["case"], _source(st)
    rows = y.shape[0]
    used = torch.arange(rows, device=y.device) < (rows if case["source"] == "plain" else st["starts"][-1])
    q, s = _group(y)
    q = torch.where(used[:, None], q.view(torch.uint8), torch.zeros_like(q.view(torch.uint8))).view(E4M3)
    outs = [q, torch.nn.functional.pad(torch.where(used[None], s, torch.zeros_like(s)), (0, _up(rows, 16) - rows))]
    if case["transposed"]:
        qt, s_t = _group(y.t())
        qt = torch.where(used[None], qt.view(torch.uint8), torch.zeros_like(qt.view(torch.uint8))).view(E4M3)
        s_t = torch.where(used[::B][:, None], s_t, torch.zeros_like(s_t))
        outs += [qt, torch.nn.functional.pad(s_t, (0, _up(y.shape[1], 16) - y.shape[1]))]
    return outs


def _values(q, s, dtype=torch.float32):
    """e4m3 [rows, cols] and scale bytes [blocks, rows or more] -> the values they stand for."""
    f = torch.exp2(s[:, : q.shape[0]].to(torch.float64) - 127).to(dtype).t()
    return q.to(dtype) * f.repeat_interleave(B, dim=1)[:, : q.shape[1]]


def _values_blocks(q, s, dtype=torch.float32):
    f = torch.exp2(s.to(torch.float64) - 127).to(dtype)
    return q.to(dtype) * f.repeat_interleave(B, 1).repeat_interleave(B, 2)[:, : q.shape[1], : q.shape[2]]


def _plain_product(st):
    case = st["case"]
    a = _values(st["a"], st["a_s"])
    b = _values(st["b"], st["b_s"]) if st["b"].dim() == 2 else _values_blocks(st["b"], st["b_s"])
    dt = st["out"].dtype
    if case["mode"] == "dense":
        return (a @ b.reshape(case["n"], case["k"]).t()).to(dt)
    starts = st["starts"].long()
    at = starts[:-1, None] + torch.arange(st["longest"], device=a.device)[None]  # every segment as long as the longest
    live = at < starts[1:, None]
    at = torch.where(live, at, torch.zeros_like(at))
    if case["mode"] == "contract":
        pa = a.t()[at] * live[:, :, None]
        pb = b.t()[at] * live[:, :, None]
        return torch.bmm(pa.transpose(1, 2), pb).to(dt)
    c = torch.bmm(a[at] * live[:, :, None], b.transpose(1, 2))
    out = torch.zeros(a.shape[0] + 1, case["n"], device=a.device)
    out[torch.where(live, at, torch.full_like(at, a.shape[0])).reshape(-1)] = c.reshape(-1, case["n"])
    return out[:-1].to(dt)


def _plain_combine(rows, row_of_slot, weights):
    t, k = row_of_slot.shape
    y = rows[row_of_slot.long().clamp(min=0).reshape(-1)].float().reshape(t, k, -1)
    w = torch.ones(t, k, device=rows.device) if weights is None else weights
    return ((w * (row_of_slot >= 0))[:, :, None] * y).sum(1).to(rows.dtype)


def _plain_combine_backward(st):
    rows, at, dout, weights = st["rows"], st["row_of_slot"], st["dout"].float(), st["weights"]
    t, k = at.shape
    chosen = at >= 0
    y = rows[at.long().clamp(min=0).reshape(-1)].float().reshape(t, k, -1)
    dw = (y * dout[:, None, :]).sum(2) * chosen
    w = torch.ones(t, k, device=rows.device) if weights is None else weights
    drows = torch.zeros(rows.shape[0] + 1, rows.shape[1], device=rows.device)
    drows[torch.where(chosen, at.long(), torch.full_like(at.long(), rows.shape[0])).reshape(-1)] = \
        (w[:, :, None] * dout[:, None, :]).reshape(t * k, -1)
    return dw, drows[:-1].to(rows.dtype)


def _run_plain(st):
    case = st["case"]
    op = case["op"]
    if op == "route":
        return _plain_route(case, st["logits"], st["bias"])
    if op == "route_backward":
        return _plain_route_backward(case, st["logits"], st["experts"], st["dweights"])
    if op == "layout":
        return _plain_layout(st["ids"], case["experts"])
    if op == "quantize":
        return _plain_quantize(st)
    if op == "quantize_blocks":
        q, s = _group_blocks(st["w"])
        return [q, s, q.transpose(1, 2).contiguous(), s.transpose(1, 2).contiguous()] if case["transposed"] else [q, s]
    if op == "product":
        return _plain_product(st)
    if op == "combine":
        return _plain_combine(st["rows"], st["row_of_slot"], st["weights"])
    return _plain_combine_backward(st)


# ------------------------------------------------------------------------------------------------ the framework's calls


def _run_own(st):
    from paper_2609_04609_b200 import ciera

    case = st["case"]
    op = case["op"]
    if op == "route":
        ciera.route(st["config"], st["logits"], st["bias"], st["experts"], st["weights"])
        return st["experts"], st["weights"]
    if op == "route_backward":
        ciera.route_backward(st["config"], st["logits"], st["experts"], st["dweights"], st["dlogits"])
        return st["dlogits"]
    if op == "layout":
        ciera.expert_layout(st["ids"], case["experts"], st["starts"], st["counts"], st["row_of_slot"], st["slot_of_row"],
                            st["workspace"])
        return st["starts"], st["counts"], st["row_of_slot"], st["slot_of_row"]
    if op == "quantize":
        kind = {"plain": ciera.SOURCE_ROWS, "gather": ciera.SOURCE_ROWS, "weighted": ciera.SOURCE_ROWS,
                "swiglu": ciera.SOURCE_SWIGLU, "swiglu_backward": ciera.SOURCE_SWIGLU_BACKWARD}[case["source"]]
        both = case["transposed"]
        ciera.fp8_quantize_rows(st["x"], st["q"], st["s"], st["qt"] if both else None, st["s_t"] if both else None, kind=kind,
                                grad=st.get("grad"), slot_of_row=st.get("slot_of_row"), top_k=case["top_k"],
                                row_weights=st.get("row_weights"), starts=st.get("starts"))
        return [st["q"], st["s"], st["qt"], st["s_t"]] if both else [st["q"], st["s"]]
    if op == "quantize_blocks":
        both = case["transposed"]
        ciera.fp8_quantize_blocks(st["w"], st["q"], st["s"], st["qt"] if both else None, st["s_t"] if both else None)
        return [st["q"], st["s"], st["qt"], st["s_t"]] if both else [st["q"], st["s"]]
    if op == "product":
        ciera.fp8_matmul(st["a"], st["a_s"], st["b"], st["b_s"], st["out"], starts=st.get("starts"),
                         contract=case["mode"] == "contract")
        return st["out"]
    if op == "combine":
        ciera.expert_combine(st["rows"], st["row_of_slot"], st["weights"], st["out"])
        return st["out"]
    ciera.expert_combine_backward(st["dout"], st["rows"], st["row_of_slot"], st["weights"], st["dweights"], st["drows"])
    return st["dweights"], st["drows"]


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------------------------------------ what a pass cannot do without


def work(case):
    op = case["op"]
    t = case.get("tokens", 0)
    if op in ("route", "route_backward"):
        e, k, v = case["experts"], case["top_k"], NBYTES[case["dtype"]]
        if op == "route":
            return {"bytes": t * (e * v + 8 * k) + (4 * e if case["bias"] else 0), "flops": 4 * t * e}
        return {"bytes": t * (2 * e * v + 8 * k), "flops": 6 * t * e}
    if op == "quantize_blocks":
        n = case["matrices"] * case["rows"] * case["cols"]
        return {"bytes": n * (NBYTES[case["dtype"]] + (2 if case["transposed"] else 1)), "flops": 2 * n}
    if op == "quantize":
        v, cols = NBYTES[case["dtype"]], case["cols"]
        rows = t * case["top_k"]
        read = {"plain": t * cols, "gather": t * cols, "weighted": t * cols, "swiglu": 2 * rows * cols,
                "swiglu_backward": rows * (cols + cols // 2)}[case["source"]] * v
        index = 0 if case["source"] == "plain" else 4 * rows
        return {"bytes": read + index + rows * cols * (2 if case["transposed"] else 1), "flops": 2 * rows * cols}
    if op == "layout":
        n = t * case["top_k"]
        return {"bytes": 4 * n * 3 + 8 * case["experts"], "flops": n}
    if op == "product":
        n, k, v = case["n"], case["k"], NBYTES[case["out"]]
        if case["mode"] == "dense":
            return {"bytes": t * k + n * k + t * n * v, "flops": 2 * t * n * k}
        rows, e = t * case["top_k"], case["experts"]
        if case["mode"] == "contract":
            return {"bytes": rows * (n + k) + e * n * k * v, "flops": 2 * rows * n * k}
        return {"bytes": rows * k + min(e, rows) * n * k + rows * n * v, "flops": 2 * rows * n * k}
    v, cols, k = NBYTES[case["dtype"]], case["cols"], case["top_k"]
    if op == "combine":
        return {"bytes": t * k * cols * v + t * cols * v + 8 * t * k, "flops": 2 * t * k * cols}
    return {"bytes": 2 * t * k * cols * v + t * cols * v + 12 * t * k, "flops": 3 * t * k * cols}


# ------------------------------------------------------------------------------------------------ 64 bits


def _exact_route(case, logits, bias):
    """One choice after the other."""
    x = logits.double()
    t, e = x.shape
    g = case["groups"]
    can = ~torch.isnan(x) & (x > NEG)
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
            top = torch.where(left, total, torch.full_like(total, NEG)).argmax(1, keepdim=True)
            left.scatter_(1, top, False)
        can = can & ~left.repeat_interleave(e // g, 1)
    ids, ws = [], []
    for _ in range(case["top_k"]):
        now = torch.where(can, key, torch.full_like(key, NEG))
        top = now.argmax(1, keepdim=True)
        some = can.any(1, keepdim=True)
        ids.append(torch.where(some, top, torch.full_like(top, -1)))
        ws.append(torch.where(some, s.gather(1, top), torch.zeros_like(s[:, :1])))
        can = can.scatter(1, top, False)
    w = torch.cat(ws, 1)
    if case["renorm"]:
        total = w.sum(1, keepdim=True)
        w = torch.where(total > 0, w / torch.where(total > 0, total, torch.ones_like(total)), w)
    return torch.cat(ids, 1).int(), w * case["scale"]


def _exact_route_backward(case, logits, experts, dweights):
    """The Jacobian of the chosen weights by the scores, times that of the scores by the logits, token by token in one product."""
    x = logits.double()
    can = ~torch.isnan(x) & (x > NEG)
    z = torch.where(can, x, torch.zeros_like(x))
    if case["score"] == "sigmoid":
        s = torch.where(can, 1 / (1 + torch.exp(-z)), torch.zeros_like(z))
    else:
        p = torch.where(can, torch.exp(z), torch.zeros_like(z))
        s = p / p.sum(1, keepdim=True).clamp(min=1e-300)
    hit = (torch.arange(x.shape[1], device=x.device)[None, None] == experts[:, :, None]).double()  # [T, k, E]
    d = dweights.double() * case["scale"]
    if case["renorm"]:
        sk = torch.einsum("tke,te->tk", hit, s)
        total = sk.sum(1, keepdim=True)
        total = torch.where(total > 0, total, torch.ones_like(total))
        ok = hit.sum(2)
        d = d / total - ok * (d * sk).sum(1, keepdim=True) / total ** 2
    ds = torch.einsum("tk,tke->te", d, hit)
    if case["score"] == "sigmoid":
        return ds * s * (1 - s)
    return ds * s - s * torch.einsum("te,te->t", ds, s)[:, None]


def _exact_source(st):
    case = st["case"]
    x = st["x"].double()
    src = case["source"]
    if src == "plain":
        return x
    out = torch.zeros(st["slot_of_row"].numel(), case["cols"], dtype=torch.float64, device=DEV)
    row = (st["slot_of_row"] >= 0).nonzero()[:, 0]
    slot = st["slot_of_row"][row].long()
    if src == "gather":
        out[row] = x[slot // case["top_k"]]
    elif src == "weighted":
        out[row] = x[slot // case["top_k"]] * st["row_weights"].double().reshape(-1, 1)[slot]
    else:
        f = x.shape[1] // 2
        g, u = x[row, :f], x[row, f:]
        z = torch.exp(-g)
        if src == "swiglu":
            out[row] = g * u / (1 + z)
        else:
            d = st["grad"].double()[row]
            out[row, :f] = d * u * (1 + z + g * z) / (1 + z) ** 2
            out[row, f:] = d * g / (1 + z)
    return out


def _exact_e4m3(x, dim_blocks):
    """e4m3 of x / 2^s, ties to even, from the format's definition: 3 bits of mantissa, least exponent -6, most 448."""
    y = x / torch.exp2(dim_blocks)
    _, e = torch.frexp(y)
    step = torch.exp2((e - 1).clamp(min=-6).double() - 3)
    return (torch.round(y / step) * step).clamp(-448.0, 448.0)


def _exact_exponent(amax):
    """The least s with amax <= 448 * 2^s."""
    s = torch.ceil(torch.log2(amax.clamp(min=1e-300) / 448.0))
    s = torch.where(amax > 448.0 * torch.exp2(s), s + 1, s)
    s = torch.where(amax <= 448.0 * torch.exp2(s - 1), s - 1, s).clamp(min=-126)
    return torch.where(amax == 0, torch.zeros_like(s), s)


def _exact_rows(y, rows_used):
    rows, cols = y.shape
    s = torch.zeros(_cdiv(cols, B), rows, dtype=torch.float64, device=DEV)
    q = torch.zeros_like(y)
    for b in range(_cdiv(cols, B)):
        part = y[:, b * B : (b + 1) * B]
        s[b] = _exact_exponent(part.abs().amax(1))
        q[:, b * B : (b + 1) * B] = _exact_e4m3(part, s[b][:, None])
    return q


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op == "route":
        return _exact_route(case, st["logits"], st["bias"])
    if op == "route_backward":
        return _exact_route_backward(case, st["logits"], st["experts"], st["dweights"])
    if op == "layout":
        return None
    if op == "quantize":
        y = _exact_source(st)
        q = _exact_rows(y, None)
        return [q, None, _exact_rows(y.t().contiguous(), None), None] if case["transposed"] else [q, None]
    if op == "quantize_blocks":
        w = st["w"].double()
        q = torch.zeros_like(w)
        for i in range(0, w.shape[1], B):
            for j in range(0, w.shape[2], B):
                part = w[:, i : i + B, j : j + B]
                q[:, i : i + B, j : j + B] = _exact_e4m3(part, _exact_exponent(part.abs().amax((1, 2)))[:, None, None])
        return [q, None, q.transpose(1, 2).contiguous(), None] if case["transposed"] else [q, None]
    if op == "product":
        a = _values(st["a"], st["a_s"], torch.float64)
        b = _values(st["b"], st["b_s"], torch.float64) if st["b"].dim() == 2 else _values_blocks(st["b"], st["b_s"], torch.float64)
        if case["mode"] == "dense":
            return a @ b.reshape(case["n"], case["k"]).t()
        starts = st["starts"].tolist()
        out = torch.zeros(st["out"].shape, dtype=torch.float64, device=DEV)
        for e in range(case["experts"]):
            lo, hi = starts[e], starts[e + 1]
            if case["mode"] == "contract":
                out[e] = a[:, lo:hi] @ b[:, lo:hi].t()
            else:
                out[lo:hi] = a[lo:hi] @ b[e].t()
        return out
    at = st["row_of_slot"].long()
    w = torch.ones(at.shape, device=DEV) if st["weights"] is None else st["weights"]
    y = st["rows"].double()
    if op == "combine":
        out = torch.zeros(at.shape[0], case["cols"], dtype=torch.float64, device=DEV)
        for j in range(case["top_k"]):
            t = (at[:, j] >= 0).nonzero()[:, 0]
            out[t] += w[t, j].double()[:, None] * y[at[t, j]]
        return out
    dout = st["dout"].double()
    dw = torch.zeros(at.shape, dtype=torch.float64, device=DEV)
    drows = torch.zeros_like(y)
    for j in range(case["top_k"]):
        t = (at[:, j] >= 0).nonzero()[:, 0]
        dw[t, j] = torch.einsum("th,th->t", dout[t], y[at[t, j]])
        drows[at[t, j]] = w[t, j].double()[:, None] * dout[t]
    return dw, drows
