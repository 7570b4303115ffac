"""The operators on a key-value cache held in 8 bits, as measurable cases.

The cache keeps K and V as 8-bit codes (E4M3 or signed integers) with a power of two as the scale of
each block of tokens of a head, so that value = code * scale.  Three kinds of call:

  write    new rows of K and V are quantised into the cache, and rows around them are read back in the
           type of the keys and values
  sparse   attention of each query head over the rows of its own index list (the decode step's
           last part), over the 8-bit cache
  dense    attention of the last n_q tokens of each sequence over the whole cache before them (the
           layers that keep full attention), one token or several, with a length for each sequence

With `own` false they are computed in plain tensor operations in 32 bits, with `own` true by the
package's own calls.  Head layouts and lengths are those of `workload.CONFIGS` and of `perf/cases.py`;
keys and queries come from two nearly orthogonal cones, as in `workload.py`, and rows differ in size,
so that blocks have scales of their own.
"""
import math

import torch

own = False

D = 128
DEVICE = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
CODES = {"e4m3": torch.float8_e4m3fn, "i8": torch.int8}
SCALE = 1.0 / math.sqrt(D)


def _write(name, batch, hkv, first, rows, block, code="e4m3", kv="bf16", ragged=False):
    return {"name": name, "kind": "write", "batch": batch, "hkv": hkv, "first": first, "rows": rows, "block": block,
            "code": code, "kv": kv, "ragged": ragged}


def _sparse(name, batch, hq, hkv, tokens, topk, block, code="e4m3", kv="bf16"):
    return {"name": name, "kind": "sparse", "batch": batch, "hq": hq, "hkv": hkv, "tokens": tokens, "topk": topk,
            "block": block, "code": code, "kv": kv}


def _dense(name, batch, hq, hkv, tokens, queries, block, code="e4m3", kv="bf16", ragged=False):
    return {"name": name, "kind": "dense", "batch": batch, "hq": hq, "hkv": hkv, "tokens": tokens, "queries": queries,
            "block": block, "code": code, "kv": kv, "ragged": ragged}


def listed():
    return [
        # the new token of a decode step, 8 key-value heads: the smallest write, nothing but latency
        _write("write-1row-8head", 1, 8, 8191, 1, 64),
        # the new tokens of a serving batch whose sequences have lengths of their own
        _write("write-1row-b16-ragged", 16, 8, 8192, 1, 32, code="i8", ragged=True),
        # a prompt of 128K tokens has just been prefilled, 32 key-value heads
        _write("write-prefill-32head-128k", 1, 32, 0, 131072, 64),
        # binary32 keys and values, an odd number of rows behind an odd number of tokens
        _write("write-4head-10k-f32", 1, 4, 33, 10007, 16, code="i8", kv="f32"),
        # a single head, 4096 tokens, binary32 queries: the smallest attention, launches and latency
        _sparse("sparse-1head-4k-f32", 1, 1, 1, 4096, 128, 64, kv="f32"),
        # a 7B layer without grouped heads at 512K tokens, 2 % kept: the length the method is quoted at
        _sparse("sparse-32head-512k", 1, 32, 32, 524288, 10486, 64),
        # grouped heads, a serving batch at 128K tokens
        _sparse("sparse-gqa4-b16-128k", 16, 32, 8, 131072, 2048, 32, code="i8"),
        # full attention of one token over a short cache, one head, binary32 queries
        _dense("dense-1head-4k-f32", 1, 1, 1, 4096, 1, 16, kv="f32"),
        # a layer with full attention and grouped heads, one token at 128K
        _dense("dense-gqa4-128k", 1, 32, 8, 131072, 1, 64),
        # groups of seven, a serving batch with lengths of its own up to an odd number of tokens
        _dense("dense-gqa7-b16-ragged", 16, 28, 4, 32769, 1, 32, code="i8", ragged=True),
        # a few tokens at once behind a running cache: speculative decoding, small prompt chunks
        _dense("dense-17q-b8", 8, 8, 8, 8209, 17, 64, code="i8"),
        # a chunk of a prompt behind 32K tokens
        _dense("dense-128q-gqa4-32k", 1, 32, 8, 32768, 128, 64),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    block, code = rng.choice([16, 32, 64, 128]), rng.choice(["e4m3", "i8"])
    kv = rng.choice(["bf16", "bf16", "f32"])
    kind = rng.choice(["write", "sparse", "dense", "dense"])
    hkv = rng.choice([1, 2, 3, 4, 8, 16, 20, 32])
    batch = _spread(rng, 1, 16)
    if kind == "write":
        rows = rng.choice([1, 1, _spread(rng, 2, 64), _spread(rng, 64, 100000)])
        while batch * hkv * rows > 32 * 131072 // (2 if kv == "f32" else 1):
            rows = max(1, rows // 2)
        ragged = rows <= 64 and rng.random() < 0.5
        c = _write("", batch, hkv, _spread(rng, 1, 20000) + (256 if ragged else -1), rows, block, code, kv, ragged)
    else:
        group = rng.choice([1, 2, 3, 4, 5, 7, 8])
        tokens = _spread(rng, 100, 300000)
        while batch * hkv * tokens > 32 * 131072:
            tokens = max(100, tokens // 2)
        if kind == "sparse":
            topk = max(1, min(tokens, int(tokens * rng.uniform(0.005, 0.06))))
            while batch * hkv * group * topk > 32 * 10486:
                topk = max(1, topk // 2)
            c = _sparse("", batch, hkv * group, hkv, tokens, topk, block, code, kv)
        else:
            queries = rng.choice([1, 1, 1, rng.randint(2, 9), _spread(rng, 10, 128)])
            while batch * hkv * group * queries * tokens > 32 * 128 * 32768:
                queries, tokens = max(1, queries // 2), tokens if queries > 1 else max(100, tokens // 2)
            c = _dense("", batch, hkv * group, hkv, tokens, queries, block, code, kv, rng.random() < 0.5)
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------- inputs

def _quantise(x, code, block):
    """Rows [heads, n, D] (n a multiple of block) as codes and the scales of their blocks."""
    y = x.float().view(x.shape[0], -1, block, D)
    m, e = torch.frexp(y.abs().amax((2, 3)))
    e = (e - torch.where(m <= 0.875, 9, 8) if code == "e4m3" else e - torch.where(m <= 0.9921875, 7, 6)).clamp(min=-126)
    s = torch.ldexp(torch.ones_like(m), e)
    y = y / s[:, :, None, None]
    y = y.to(torch.float8_e4m3fn) if code == "e4m3" else y.round().to(torch.int8)
    return y.view(x.shape), s


def _rows(g, heads, n, centre, kv):
    """Rows of a cone around `centre` [heads, 1, D], with sizes that differ from token to token."""
    x = torch.randn(heads, n, D, generator=g, device=DEVICE)
    x += centre
    x *= torch.exp(0.5 * torch.randn(heads, n, 1, generator=g, device=DEVICE))
    return x.to(TYPES[kv])


def _cones(g, heads):
    mu = torch.randn(2, heads, 1, D, generator=g, device=DEVICE)
    k = mu[0] / mu[0].norm(dim=-1, keepdim=True)
    q = mu[1] - (mu[1] * k).sum(-1, keepdim=True) * k
    return 0.8 * k, 0.8 * q / q.norm(dim=-1, keepdim=True)


def _capacity(case):
    """Tokens the cache has room for: a little more than the case uses, not a multiple of a block; as many as there are queries, which
    a call asks for (a short cache drawn with more of them was refused)."""
    return (case["first"] + case["rows"] + 5 if case["kind"] == "write" else max(case["tokens"], case.get("queries", 1)) + 3)


def _window(case):
    """(rows before the first new one that are read back, rows read back) of a write case."""
    back = min(15, case["first"])
    return back, back + case["rows"]


def _lengths(case):
    b, n = case["batch"], case["tokens"]
    return [1 + (n - 1) * (i + 1) // b for i in range(b)] if case["ragged"] else [n] * b


def _positions(case):
    """The token at which the new rows of each sequence begin."""
    b, n = case["batch"], case["first"]
    return [15 + (n - 15) * (i + 1) // b for i in range(b)] if case["ragged"] else [n] * b


def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    b, hkv, block, code, kv = case["batch"], case["hkv"], case["block"], case["code"], case["kv"]
    n = _capacity(case)
    blocks = -(-n // block)
    ck, cq = _cones(g, b * hkv)
    cv = torch.zeros_like(ck)
    st = {"case": case}
    # the cache as earlier writes left it
    for name, centre in (("k", ck), ("v", cv)):
        st[name] = torch.zeros(b, hkv, n, D, dtype=torch.uint8, device=DEVICE).view(CODES[code])
        st[name + "_scale"] = torch.ones(b, hkv, blocks, device=DEVICE)
        filled = n if case["kind"] != "write" else case["first"]
        for h in range(b * hkv if filled else 0):
            room = -(-filled // block) * block
            c, s = _quantise(_rows(g, 1, room, centre[h], kv), code, block)
            st[name].view(torch.uint8).view(-1, n, D)[h, :filled] = c.view(torch.uint8)[0, :filled]
            st[name + "_scale"].view(-1, blocks)[h, :s.shape[1]] = s[0]
    if case["kind"] == "write":
        st["K"] = _rows(g, b * hkv, case["rows"], ck, kv).view(b, hkv, -1, D)
        st["V"] = _rows(g, b * hkv, case["rows"], cv, kv).view(b, hkv, -1, D)
        back, _ = _window(case)
        pos = torch.tensor(_positions(case), device=DEVICE, dtype=torch.int32)
        st["pos"] = pos[torch.randperm(b, generator=g, device=DEVICE)] if case["ragged"] else pos
        st["from"] = st["pos"] - back
        heads_q = hkv
    else:
        heads_q, group = case["hq"], case["hq"] // hkv
        nq = case.get("queries", 1)
        q = _rows(g, b * hkv, group * nq, cq, "f32")
        st["q"] = (2.0 * q).to(TYPES[kv]).view(b, heads_q, nq, D)
        if case["kind"] == "sparse":
            st["q"] = st["q"].view(b, heads_q, D)
            r = torch.rand(b * heads_q, case["tokens"], generator=g, device=DEVICE) if b * heads_q * case["tokens"] <= 1 << 28 else None
            if r is not None:
                idx = r.topk(case["topk"], dim=-1).indices
            else:   # distinct tokens of a long cache: one out of each of topk strata
                w = case["tokens"] // case["topk"]
                idx = torch.arange(case["topk"], device=DEVICE) * w + torch.randint(0, w, (b * heads_q, case["topk"]), generator=g, device=DEVICE)
            st["idx"] = idx.sort(-1).values.to(torch.int32).view(b, heads_q, -1).contiguous()
        else:
            lens = torch.tensor(_lengths(case), device=DEVICE, dtype=torch.int32)
            st["lens"] = lens[torch.randperm(b, generator=g, device=DEVICE)]
    if own:     # the context and the handle that a program keeps for a layer
        import paper_2508_19740_amd as sp
        st["ctx"] = sp.Spotlight(b, heads_q, hkv, 128, 256, n, case.get("topk", 1), kv_dtype=TYPES[kv], device=DEVICE)
        st["cache"] = sp.Cache(st["k"], st["v"], st["k_scale"], st["v_scale"], block)
    return st


# ------------------------------------------------------------------------------------- plain forms

def _power(amax, code):
    """The smallest power of two that brings amax into the code's range."""
    m, e = torch.frexp(amax)
    e = e - torch.where(m <= 0.875, 9, 8) if code == "e4m3" else e - torch.where(m <= 0.9921875, 7, 6)
    return torch.ldexp(torch.ones_like(amax), e.clamp(min=-126))


def _plain_write(st, name, x):
    case = st["case"]
    b, hkv, block, code, rows = case["batch"], case["hkv"], case["block"], case["code"], case["rows"]
    codes, scales = st[name], st[name + "_scale"]
    n, blocks = codes.shape[2], scales.shape[2]
    span = (rows + block - 2) // block + 1                            # blocks that rows rows can touch
    first = (st["pos"].long() // block)[:, None, None]                # [B, 1, 1]
    bi = torch.arange(b, device=x.device)[:, None, None]
    hi = torch.arange(hkv, device=x.device)[None, :, None]
    at_block = first + torch.arange(span, device=x.device)            # [B, 1, span]
    at = first * block + torch.arange(span * block, device=x.device)  # [B, 1, span * block]
    old_s = scales[bi, hi, at_block.clamp(max=blocks - 1)]            # [B, Hkv, span]
    new = at - st["pos"].long()[:, None, None]                        # index among the new rows
    is_new, is_old = (new >= 0) & (new < rows), new < 0
    y = x[bi, hi, new.clamp(0, rows - 1)].float() * is_new[..., None]
    amax = y.abs().amax(-1).view(b, hkv, span, block).amax(-1)
    keeps = is_old.view(b, 1, span, block).any(-1)
    s = _power(amax, code)
    s = torch.where(keeps, torch.maximum(s, old_s), s)
    row_s = s.repeat_interleave(block, 2)[..., None]
    # only the first block has rows from before
    lead = codes.view(torch.uint8)[bi, hi, at[..., :block].clamp(max=n - 1)].view(codes.dtype).float() * old_s[:, :, :1, None]
    y[:, :, :block] = torch.where(is_old[..., :block, None], lead, y[:, :, :block])
    y = y / row_s
    y = y.to(torch.float8_e4m3fn) if code == "e4m3" else y.round().to(torch.int8)
    use = (is_new | is_old).expand(b, hkv, -1)
    where = ((bi * hkv + hi) * n + at)[use]
    codes.view(torch.uint8).view(-1, D)[where] = y.view(torch.uint8)[use]
    touched = (is_new | is_old).view(b, 1, span, block).any(-1).expand(b, hkv, -1)
    scales.view(-1)[((bi * hkv + hi) * blocks + at_block)[touched]] = s[touched]


def _plain_read(st, name):
    case = st["case"]
    codes, scales = st[name], st[name + "_scale"]
    _, rows = _window(case)
    bi = torch.arange(case["batch"], device=codes.device)[:, None, None]
    hi = torch.arange(case["hkv"], device=codes.device)[None, :, None]
    at = st["from"].long()[:, None, None] + torch.arange(rows, device=codes.device)
    x = codes.view(torch.uint8)[bi, hi, at].view(codes.dtype).float()
    return (x * scales[bi, hi, at // case["block"]][..., None]).to(TYPES[case["kv"]])


def _plain_sparse(st):
    case = st["case"]
    b, hq, hkv, block = case["batch"], case["hq"], case["hkv"], case["block"]
    n, blocks = st["k"].shape[2], st["k_scale"].shape[2]
    head = (torch.arange(b * hq, device=DEVICE) // (hq // hkv))[:, None]
    idx = st["idx"].long().view(b * hq, -1)
    at, at_block = head * n + idx, head * blocks + idx // block
    k = st["k"].view(torch.uint8).view(-1, D)[at].view(CODES[case["code"]]).float() * st["k_scale"].view(-1)[at_block][..., None]
    v = st["v"].view(torch.uint8).view(-1, D)[at].view(CODES[case["code"]]).float() * st["v_scale"].view(-1)[at_block][..., None]
    s = (k * st["q"].float().view(b * hq, 1, D)).sum(-1) * SCALE
    p = torch.exp(s - s.amax(-1, keepdim=True))
    o = (p[..., None] * v).sum(1) / p.sum(-1, keepdim=True)
    return o.view(b, hq, D)


def _plain_dense(st):
    case = st["case"]
    b, hq, hkv, n, nq, block = case["batch"], case["hq"], case["hkv"], case["tokens"], case["queries"], case["block"]
    k = st["k"][:, :, :n].float() * st["k_scale"].repeat_interleave(block, 2)[:, :, :n, None]
    v = st["v"][:, :, :n].float() * st["v_scale"].repeat_interleave(block, 2)[:, :, :n, None]
    q = st["q"].float().view(b, hkv, -1, D)                           # rows: query heads of the group, then queries
    s = torch.matmul(q, k.transpose(2, 3)) * SCALE
    last = (st["lens"].long()[:, None] - nq + torch.arange(nq, device=DEVICE)).repeat(1, hq // hkv)   # [B, rows]
    seen = torch.arange(n, device=DEVICE) <= last[:, None, :, None]
    s = s.masked_fill(~seen, -math.inf)
    m = s.amax(-1, keepdim=True).clamp(min=-3e38)
    p = torch.exp(s - m)
    l = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v)
    return torch.where(l > 0, o / l, 0.0).view(b, hq, nq, D)


def run(state):
    case = state["case"]
    if own:
        ctx, cache = state["ctx"], state["cache"]
        if case["kind"] == "write":
            ctx.cache_write(cache, state["K"], state["V"], first=state["pos"])
            return ctx.cache_read(cache, _window(case)[1], first=state["from"])
        if case["kind"] == "sparse":
            return ctx.sparse_decode_cache(state["q"], cache, state["idx"])
        return ctx.dense_decode_cache(state["q"], cache, case["tokens"], lens=state["lens"])
    if case["kind"] == "write":
        _plain_write(state, "k", state["K"])
        _plain_write(state, "v", state["V"])
        return _plain_read(state, "k"), _plain_read(state, "v")
    return _plain_sparse(state) if case["kind"] == "sparse" else _plain_dense(state)


def work(case):
    e = 4 if case["kv"] == "f32" else 2
    b, block = case["batch"], case["block"]
    if case["kind"] == "write":
        heads, rows, back = b * case["hkv"], case["rows"], _window(case)[1]
        per = 2 * heads * (rows * D * (e + 1) + back * D * (e + 1) + 4 * (-(-rows // block) + -(-back // block)))
        return {"bytes": per + 8 * b, "flops": 4 * heads * (rows + back) * D}
    rows = b * case["hq"] * case.get("queries", 1)
    if case["kind"] == "sparse":
        # the lists of a group overlap little: each selected row is read for its own query head
        scales = min(case["hq"] // case["hkv"] * case["topk"], case["tokens"] // block + 1) * b * case["hkv"]
        return {"bytes": rows * (D * (e + 4) + case["topk"] * (2 * D + 4)) + 8 * scales, "flops": 4 * D * rows * case["topk"]}
    pairs = 0
    for n in _lengths(case):
        seen = [max(0, n - case["queries"] + 1 + i) for i in range(case["queries"])]
        pairs += sum(seen) * case["hq"]
    tokens = sum(_lengths(case))
    return {"bytes": rows * D * (e + 4) + case["hkv"] * tokens * (2 * D + 8 / block) + 4 * b, "flops": 4 * D * pairs}


# ------------------------------------------------------------------------------- the definition, 64 bits

def _nearest(y, code):
    """y rounded to the code's values, ties to even, in 64 bits."""
    if code == "i8":
        return torch.round(y)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3.0)
    return torch.round(y / step) * step


def _least_power(a, most):
    e = torch.ceil(torch.log2(a.clamp(min=2.0 ** -200) / most))
    e = torch.where(a > most * torch.exp2(e), e + 1, e)
    e = torch.where(a <= most * torch.exp2(e - 1), e - 1, e)
    return torch.exp2(e.clamp(min=-126.0))


def _exact_write(st, name, x):
    case = st["case"]
    block, code, rows = case["block"], case["code"], case["rows"]
    back, count = _window(case)
    most = 448.0 if code == "e4m3" else 127.0
    out = []
    for i, start in enumerate(st["pos"].tolist()):
        # the value of every row from the block of the first row read back on, and what the write makes of it
        lo = (start - back) // block * block
        tail = -(-(start + rows) // block) * block - (start + rows)
        s_old = st[name + "_scale"][i, :, lo // block: start // block + 1].double()
        old = st[name][i, :, lo:start].double() * s_old.repeat_interleave(block, 1)[:, :start - lo, None]
        for h in range(case["hkv"]):
            y = torch.cat([old[h], x[i, h].double(), torch.zeros(tail, D, dtype=torch.float64, device=x.device)]).view(-1, block, D)
            t = torch.arange(lo, lo + y.shape[0] * block, device=x.device).view(-1, block, 1)
            s = _least_power(torch.where(t >= start, y, 0.0).abs().amax((1, 2)), most)
            had = t[:, 0, 0] < start
            s_had = s_old[h, :int(had.sum())]
            s[:s_had.shape[0]] = torch.where(t[had][:, -1, 0] >= start, torch.maximum(s[:s_had.shape[0]], s_had), s_had)
            y = (_nearest(y / s[:, None, None], code) * s[:, None, None]).view(-1, D)
            out.append(y[start - back - lo: start - back - lo + count].to(torch.float32))
    return torch.stack(out).double().view(case["batch"], case["hkv"], count, D)


def _exact_head(q, k, v, seen):
    """softmax(q k^T) v in 64 bits of rows q over the rows that `seen` [rows, n] keeps."""
    s = (q @ k.T) * SCALE
    s = torch.where(seen, s, -math.inf)
    z = torch.logsumexp(s, -1, keepdim=True)
    return torch.where(torch.isinf(z), 0.0, torch.exp(s - z) @ v)


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "write":
        return _exact_write(st, "k", st["K"]), _exact_write(st, "v", st["V"])
    b, hq, hkv, block = case["batch"], case["hq"], case["hkv"], case["block"]
    group, nq = hq // hkv, case.get("queries", 1)
    out = torch.empty(b, hq, nq, D, dtype=torch.float64, device=DEVICE)
    for i in range(b):
        for h in range(hkv):
            ks, vs = (st[x][i, h].double().repeat_interleave(block)[:, None] for x in ("k_scale", "v_scale"))
            if case["kind"] == "sparse":
                for j in range(h * group, (h + 1) * group):
                    t = st["idx"][i, j].long()
                    k = st["k"][i, h].view(torch.uint8)[t].view(CODES[case["code"]]).double() * ks[t]
                    v = st["v"][i, h].view(torch.uint8)[t].view(CODES[case["code"]]).double() * vs[t]
                    out[i, j] = _exact_head(st["q"][i, j].double()[None], k, v, torch.ones(1, t.numel(), dtype=torch.bool, device=DEVICE))
                continue
            n = int(st["lens"][i])
            k, v = st["k"][i, h, :n].double() * ks[:n], st["v"][i, h, :n].double() * vs[:n]
            t = torch.arange(n, device=DEVICE)
            last = n - nq + torch.arange(nq, device=DEVICE)
            for j in range(h * group, (h + 1) * group):
                out[i, j] = _exact_head(st["q"][i, j].double(), k, v, t[None] <= last[:, None])
    return out.view(b, hq, D) if case["kind"] == "sparse" else out
