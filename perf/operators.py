"""Operators between the compressed rows and a language model's attention, as a serving program calls them.

Three of them: the norm and rotation of queries and keys by their (t, y, x) positions
(``ttf_qk_norm_rope``), the same with keys and values put into a paged cache (``ttf_cache_append``)
and the attention of a chunk of new rows, or of single tokens, over that cache
(``ttf_paged_attention``).  ``own`` false computes them in plain torch operations, in 32 bits with
angles in 64; ``own`` true makes the library's calls.

Rows are packed sequence after sequence, as ``ttf_compress`` packs clips.  Queries, keys and values
are slices of one projection's output, as they come out of it.
"""
import math

import torch

own = False

EPS = 1e-6
MOST_BYTES = 1 << 31                 # most cache bytes of a drawn case
MOST_PRODUCTS = 1 << 36              # most products q.k of a drawn case, rows x heads x keys x D (fp32: an eighth)


def _case(name, op, dtype, B, chunk, context, heads, kv_heads, D, **more):
    """B sequences that bring up to `chunk` new rows to up to `context` cached ones."""
    c = {"name": name, "op": op, "dtype": dtype, "B": B, "chunk": chunk, "context": context, "ragged": B > 1, "heads": heads,
         "kv_heads": kv_heads, "D": D, "slack": 0}
    if op != "attention":
        c |= {"rot": D, "layout": "half", "axes": 1, "norm": True, "base": 1e6, "factor": 1.0}
    if op != "rope":
        c |= {"page": 16, "heads_first": False}
    if op == "append":
        c |= {"queries": True}
    if op == "attention":
        c |= {"causal": True, "window": 0}
    return c | more


def listed():
    return [
        # one token of one request: launches and latency
        _case("rope_token", "rope", "bf16", 1, 1, 2900, 32, 8, 128),
        # a batch of 16 compressed clips (a third of 32 frames of 16x16 tokens is kept), three position axes, buffers with
        # room behind the last clip
        _case("rope_clips", "rope", "bf16", 16, 3600, 0, 32, 8, 128, axes=3, slack=1000),
        # fp32, neighbouring pairs, half of a head of 96, far positions of a stretched context, no norm, odd row count
        _case("rope_far_f32", "rope", "f32", 3, 2999, 900000, 20, 4, 96, rot=48, layout="interleaved", norm=False, factor=8.0),
        # one token each of a batch of requests
        _case("append_tokens", "append", "bf16", 64, 1, 1000, 32, 8, 128),
        # the compressed clips of a batch go into the cache, the queries rotated in the same call
        _case("append_clips", "append", "bf16", 16, 3600, 40, 32, 8, 128, axes=3, page=64, slack=1000),
        # fp32, a head of 80 with 32 rotated, pages of 24 slots with heads first, no queries, no norm
        _case("append_odd_f32", "append", "f32", 5, 333, 100, 6, 2, 80, rot=32, norm=False, page=24, heads_first=True, queries=False),
        # the next token after one compressed clip and its question
        _case("attn_token", "attention", "bf16", 1, 1, 2900, 32, 8, 128),
        # one token each of a batch whose contexts differ widely
        _case("attn_tokens", "attention", "bf16", 64, 1, 32000, 32, 8, 128, page=64),
        # tokens of long streams that look back over a window; older pages are gone
        _case("attn_window", "attention", "bf16", 12, 3, 130000, 16, 8, 64, page=32, heads_first=True, window=8192),
        # a chunk of text after long cached contexts
        _case("attn_chunk", "attention", "bf16", 4, 512, 8192, 32, 8, 128),
        # prefill of a batch of compressed clips
        _case("attn_clips", "attention", "bf16", 8, 3600, 0, 32, 8, 128, page=64, slack=500),
        # fp32, odd sizes all over, every row sees every key
        _case("attn_odd_f32", "attention", "f32", 3, 77, 1000, 6, 2, 80, page=24, causal=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "append", "attention", "attention"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    kv_heads, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 3, 4, 7, 8])
    D = rng.choice([128, 128, 64, rng.randint(4, 32) * 8])
    B = _log(rng, 1, 64)
    chunk = rng.choice([1, 1, _log(rng, 2, 64), _log(rng, 64, 4000)])
    context = _log(rng, 16, 130000) if op == "attention" else _log(rng, 16, 4000)
    row = kv_heads * D * (2 if dtype == "bf16" else 4)
    if op == "attention":
        context = max(16, min(context, MOST_BYTES // (2 * row * B) - chunk))
        most = MOST_PRODUCTS // (1 if dtype == "bf16" else 8)
        chunk = max(1, min(chunk, most // (B * kv_heads * group * (context + chunk) * D)))
    else:
        chunk = max(1, min(chunk, MOST_BYTES // 4 // (row * (group + 2) * B)))
    c = _case("", op, dtype, B, chunk, context, kv_heads * group, kv_heads, D, slack=rng.choice([0, 0, 37]))
    del c["name"]
    if op != "attention":
        c |= {"rot": rng.choice([D, D, D // 16 * 8]), "layout": rng.choice(["half", "interleaved"]), "axes": rng.choice([1, 3]),
              "norm": rng.random() < 0.6, "base": rng.choice([1e4, 1e6]), "factor": rng.choice([1.0, 4.0])}
    if op != "rope":
        c |= {"page": rng.choice([16, 64, rng.randint(1, 16) * 8]), "heads_first": rng.random() < 0.3}
    if op == "append":
        c |= {"queries": rng.random() < 0.7}
    if op == "attention":
        c |= {"causal": rng.random() < 0.8, "window": rng.choice([0, 0, 0, _log(rng, 16, 8192)])}
    return c


def _lengths(case):
    """New and cached rows of every sequence: spread between a quarter and all of the most; some bring nothing this time."""
    rows, cached = [], []
    for b in range(case["B"]):
        u, v = (0.25 + 0.75 * ((b + 1) * g % 1.0) if case["ragged"] else 1.0 for g in (0.6180339887, 0.4142135624))
        rows.append(0 if case["ragged"] and b % 8 == 5 else max(1, int(case["chunk"] * v)))
        cached.append(int(case["context"] * u))
    return rows, cached


def _first_seen(case, rows, cached):
    """The lowest key index that a row of the sequence sees."""
    return max(0, cached - case["window"] + 1) if case.get("window") and rows else 0


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _rope_inputs(s, case, rnd):
    """Positions of the rows, frequencies of the pairs and the axis each pair goes by."""
    rows, axes, half = s["rows"], case["axes"], case["rot"] // 2
    total, dev = s["total"], "cuda"
    j = torch.arange(half, device=dev)
    s["inv_freq"] = case["base"] ** (-2.0 * j.double() / case["rot"]) / case["factor"]
    s["attention_factor"] = 1.0 if case["factor"] == 1.0 else 0.1 * math.log(case["factor"]) + 1.0
    if axes == 1:                                          # the index in the sequence
        s["axis"] = None
        pos = (s["cached"].long()[s["seq"]] + s["within"])[None]
    else:                                                  # kept tokens of a clip of 16x16 grids, in ascending order
        turn = half * 5 // 16                              # pairs of y and of x; they take turns with those of t
        s["axis"] = torch.where((j % 3 > 0) & (j < 3 * turn), j % 3, 0).int()
        flat = (s["within"] * 3 + torch.randint(0, 3, (total,), **rnd))
        pos = torch.stack([flat // 256, flat // 16 % 16, flat % 16])
    s["pos"] = torch.zeros((axes, rows), dtype=torch.int32, device=dev)
    s["pos"][:, :total] = pos.int()
    D = case["D"]
    dt = _dtype(case)
    s["q_weight"], s["k_weight"] = [(1 + 0.2 * torch.randn(D, **rnd)).to(dt) if case["norm"] else None for _ in range(2)]


def _projected(case, rows, rnd):
    """q, k and v of all rows, slices of one projection's output."""
    hq, hk = case["heads"], case["kv_heads"]
    x = torch.randn((rows, hq + 2 * hk, case["D"]), **rnd)
    x *= torch.exp(0.3 * torch.randn((rows, hq + 2 * hk, 1), **rnd))
    x = x.to(_dtype(case))
    return x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = dict(device="cuda", generator=g)
    B, hq, hk, D, op, dt = case["B"], case["heads"], case["kv_heads"], case["D"], case["op"], _dtype(case)
    rows, cached = _lengths(case)
    total = sum(rows)
    s = {"case": case, "total": total, "rows": total + case["slack"], "longest": max(r + c for r, c in zip(rows, cached)),
         "most_rows": max(rows)}
    s["cached"] = torch.tensor(cached, dtype=torch.int32, device="cuda")
    ends = torch.tensor([0] + rows, device="cuda").cumsum(0)
    s["row_offsets"] = ends.int()
    s["seq"] = torch.repeat_interleave(torch.arange(B, device="cuda"), torch.tensor(rows, device="cuda"))
    s["within"] = torch.arange(total, device="cuda") - ends[s["seq"]]
    if op != "rope":
        S = case["page"]
        width = max(1, -(-s["longest"] // S))
        used = [-(-(r + c) // S) for r, c in zip(rows, cached)]
        behind = [_first_seen(case, r, c) // S for r, c in zip(rows, cached)]     # pages that no row looks at any more
        pages = sum(used) - sum(behind) + 3
        order = torch.randperm(pages, **rnd).int()
        p = torch.arange(width, device="cuda")[None]
        has = (p >= torch.tensor(behind, device="cuda")[:, None]) & (p < torch.tensor(used, device="cuda")[:, None])
        s["page_table"] = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
        s["page_table"][has] = order[:sum(used) - sum(behind)]
        shape = (pages, hk, S, D) if case["heads_first"] else (pages, S, hk, D)
        k, v = torch.randn(shape, **rnd).to(dt), (0.3 + torch.randn(shape, **rnd)).to(dt)
        s["k_cache"], s["v_cache"] = (x.transpose(1, 2) if case["heads_first"] else x for x in (k, v))
    if op == "attention":
        # some heads look at everything alike, some pick out a few keys
        peak = torch.linspace(0.5, 3.0, hq, device="cuda")[None, :, None]
        s["q"] = (peak * torch.randn((s["rows"], hq, D), **rnd)).to(dt)
        s["out"] = torch.zeros((s["rows"], hq, D), dtype=dt, device="cuda")
        s["lse"] = torch.zeros((s["rows"], hq), dtype=torch.float32, device="cuda")
        return s
    s["q"], s["k"], s["v"] = _projected(case, s["rows"], rnd)
    _rope_inputs(s, case, rnd)
    s["q_out"] = torch.zeros((s["rows"], hq, D), dtype=dt, device="cuda")
    s["k_out"] = torch.zeros((s["rows"], hk, D), dtype=dt, device="cuda")
    return s


# ------------------------------------------------------------------------------ plain forms
def _angles(s):
    """Cosines and sines of every row's pairs, [rows, 1, pairs]."""
    total = s["total"]
    pos = s["pos"][:, :total]
    pos = pos[s["axis"].long()].t() if s["axis"] is not None else pos[0][:, None]
    theta = pos.double() * s["inv_freq"]
    f = s["attention_factor"]
    return (theta.cos() * f).float()[:, None], (theta.sin() * f).float()[:, None]


def _norm_rotate(s, x, weight, angles):
    case = s["case"]
    x = x[:s["total"]].float()
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()
    c, si = angles
    rot = case["rot"]
    if case["layout"] == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        parts = [a * c - b * si, b * c + a * si]
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        parts = [torch.stack([a * c - b * si, b * c + a * si], -1).flatten(-2)]
    return torch.cat(parts + [x[..., rot:]], -1).to(_dtype(case))


def _plain_rope(s):
    angles, n = _angles(s), s["total"]
    s["q_out"][:n] = _norm_rotate(s, s["q"], s["q_weight"], angles)
    s["k_out"][:n] = _norm_rotate(s, s["k"], s["k_weight"], angles)
    return {"q": s["q_out"], "k": s["k_out"]}


def _plain_append(s):
    angles, n, S = _angles(s), s["total"], s["case"]["page"]
    at = s["cached"].long()[s["seq"]] + s["within"]
    page = s["page_table"][s["seq"], at // S].long()
    s["k_cache"][page, at % S] = _norm_rotate(s, s["k"], s["k_weight"], angles)
    s["v_cache"][page, at % S] = s["v"][:n]
    if not s["case"]["queries"]:
        return {"k": s["k_cache"], "v": s["v_cache"]}
    s["q_out"][:n] = _norm_rotate(s, s["q"], s["q_weight"], angles)
    return {"q": s["q_out"], "k": s["k_cache"], "v": s["v_cache"]}


def _plain_attention(s):
    case = s["case"]
    B, hq, hk, D, S = case["B"], case["heads"], case["kv_heads"], case["D"], case["page"]
    most, total = s["most_rows"], s["total"]
    behind = int(case["window"] > 0) * max(0, min(c for c in _lengths(case)[1]) - case["window"] + 1) // S
    table = s["page_table"][:, behind:].long()
    key = torch.arange(table.shape[1] * S, device="cuda") + behind * S          # index in the sequence
    there = (table >= 0).repeat_interleave(S, 1)                                # [B, L]
    k = s["k_cache"][table.clamp(min=0)].float().flatten(1, 2).permute(0, 2, 3, 1)   # [B, hk, D, L]
    q = torch.zeros((B, most, hq, D), device="cuda")
    q[s["seq"], s["within"]] = s["q"][:total].float()
    q = q.view(B, most, hk, hq // hk, D).permute(0, 2, 3, 1, 4).reshape(B, hk, -1, D)
    score = torch.matmul(q, k.contiguous()).mul_(D ** -0.5)
    del k, q
    at = s["cached"][:, None] + torch.arange(most, device="cuda")               # [B, most] index of the rows
    n = s["row_offsets"][1:] - s["row_offsets"][:-1]
    sees = (there & (key < (s["cached"] + n)[:, None]))[:, None].expand(B, most, key.numel())
    if case["causal"]:
        sees = sees & (key <= at[..., None])
    if case["window"]:
        sees = sees & (key > at[..., None] - case["window"])
    score = score.view(B, hk, hq // hk, most, -1).masked_fill_(~sees[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top > -math.inf, top, 0.0)
    p = score.sub_(top).exp_()
    z = p.sum(-1, keepdim=True)
    v = torch.where(there[..., None, None], s["v_cache"][table.clamp(min=0)].flatten(1, 2).float(), 0.0)
    v = v.permute(0, 2, 1, 3).contiguous()
    o = torch.matmul(p.view(B, hk, -1, key.numel()), v).view(B, hq, most, D) / z.view(B, hq, most, 1).clamp(min=1e-30)
    lse = (top + z.log()).view(B, hq, most)
    s["out"][:total] = o.transpose(1, 2)[s["seq"], s["within"]].to(_dtype(case))
    s["lse"][:total] = lse.transpose(1, 2)[s["seq"], s["within"]]
    return {"out": s["out"], "lse": s["lse"]}


# ------------------------------------------------------------------------------ the library's calls
def _own_rope(s):
    import paper_2605_07355_amd as ttf
    return ttf.TTFRope(s["inv_freq"], s["axis"], layout=s["case"]["layout"], attention_factor=s["attention_factor"])


def _own_run(s):
    import paper_2605_07355_amd as ttf
    case, op = s["case"], s["case"]["op"]
    if op == "rope":
        q, k = ttf.ttf_qk_norm_rope(s["q"], s["k"], s["pos"], _own_rope(s), q_weight=s["q_weight"], k_weight=s["k_weight"],
                                    eps=EPS, row_offsets=s["row_offsets"], q_out=s["q_out"], k_out=s["k_out"])
        return {"q": q, "k": k}
    cache = ttf.TTFKVCache(s["k_cache"], s["v_cache"], s["page_table"])
    if op == "attention":
        out = ttf.ttf_paged_attention(s["q"], cache, s["row_offsets"], s["cached"], max_rows=s["most_rows"], causal=case["causal"],
                                      window=case["window"], out=s["out"], lse=s["lse"])
        return {"out": out, "lse": s["lse"]}
    q = {"q": s["q"], "q_weight": s["q_weight"], "q_out": s["q_out"]} if case["queries"] else {}
    ttf.ttf_cache_append(cache, s["k"], s["v"], s["row_offsets"], s["cached"], pos=s["pos"], rope=_own_rope(s),
                         k_weight=s["k_weight"], eps=EPS, **q)
    return {"k": s["k_cache"], "v": s["v_cache"]} | ({"q": s["q_out"]} if case["queries"] else {})


def run(s):
    if own:
        return _own_run(s)
    return {"rope": _plain_rope, "append": _plain_append, "attention": _plain_attention}[s["case"]["op"]](s)


# ------------------------------------------------------------------------------ work and exact values
def work(case):
    rows, cached = _lengths(case)
    e, total, hq, hk, D = 2 if case["dtype"] == "bf16" else 4, sum(rows), case["heads"], case["kv_heads"], case["D"]
    if case["op"] != "attention":
        moved = hk * (2 if case["op"] == "append" else 1) + (hq if case.get("queries", True) else 0)
        rotated = hk + (hq if case.get("queries", True) else 0)
        return {"bytes": 2 * total * moved * D * e + 4 * total * case["axes"], "flops": 6.0 * total * rotated * D}
    w = case["window"]
    keys = sum(r + c - _first_seen(case, r, c) for r, c in zip(rows, cached) if r)
    pairs = 0
    for r, c in zip(rows, cached):
        if not case["causal"]:                             # row i sees from its window's start to the end
            pairs += sum(r + c - max(0, c + i - w + 1) for i in range(r)) if w else r * (r + c)
        elif not w:
            pairs += r * c + r * (r + 1) // 2
        else:
            pairs += sum(min(w, c + i + 1) for i in range(r))
    return {"bytes": 2 * keys * hk * D * e + 2 * total * hq * D * e + 4 * total * hq, "flops": 4.0 * D * hq * pairs}


def _exact_rotated(s, x, weight):
    """Row by row as complex numbers: every pair times s e^(i p f)."""
    case, n, rot = s["case"], s["total"], s["case"]["rot"]
    x = x[:n].double()
    if weight is not None:
        x = x / (x.square().sum(-1, keepdim=True) / case["D"] + EPS).sqrt() * weight.double()
    f = s["inv_freq"]
    which = s["axis"].long() if s["axis"] is not None else torch.zeros(rot // 2, dtype=torch.long, device=x.device)
    angle = torch.gather(s["pos"][:, :n].double().t(), 1, which.expand(n, -1)) * f
    turn = torch.polar(torch.full_like(angle, s["attention_factor"]), angle)[:, None]
    y = x.clone()
    if case["layout"] == "half":
        z = torch.complex(x[..., :rot // 2].contiguous(), x[..., rot // 2:rot].contiguous()) * turn
        y[..., :rot // 2], y[..., rot // 2:rot] = z.real, z.imag
    else:
        z = torch.view_as_complex(x[..., :rot].unflatten(-1, (-1, 2)).contiguous()) * turn
        y[..., :rot] = torch.view_as_real(z).flatten(-2)
    return y


def exact(case, seed):
    s = prepare(case, seed)
    n, S = s["total"], case.get("page")
    rows, cached = _lengths(case)
    if case["op"] == "rope":
        q, k = s["q_out"].double(), s["k_out"].double()
        q[:n], k[:n] = _exact_rotated(s, s["q"], s["q_weight"]), _exact_rotated(s, s["k"], s["k_weight"])
        return {"q": q, "k": k}
    if case["op"] == "append":
        k, v = s["k_cache"].double(), s["v_cache"].double()
        new, first = _exact_rotated(s, s["k"], s["k_weight"]), 0
        for b in range(case["B"]):                         # sequence by sequence
            if rows[b]:
                t = torch.arange(cached[b], cached[b] + rows[b], device="cuda")
                page = s["page_table"][b].long()[torch.div(t, S, rounding_mode="floor")]
                k[page, t % S] = new[first:first + rows[b]]
                v[page, t % S] = s["v"][first:first + rows[b]].double()
            first += rows[b]
        if not case["queries"]:
            return {"k": k, "v": v}
        q = s["q_out"].double()
        q[:n] = _exact_rotated(s, s["q"], s["q_weight"])
        return {"q": q, "k": k, "v": v}
    hq, hk, D = case["heads"], case["kv_heads"], case["D"]
    out, lse, first = s["out"].double(), s["lse"].double(), 0
    for b in range(case["B"]):                             # one sequence and one key head at a time
        r, c = rows[b], cached[b]
        if r:
            u = torch.arange(_first_seen(case, r, c), c + r, device="cuda")
            page = s["page_table"][b].long()[torch.div(u, S, rounding_mode="floor")]
            t = torch.arange(c, c + r, device="cuda")[:, None]
            hidden = torch.zeros((r, u.numel()), dtype=torch.bool, device="cuda")
            if case["causal"]:
                hidden |= u[None] > t
            if case["window"]:
                hidden |= u[None] <= t - case["window"]
            for h in range(hk):
                k, v = (x[page, u % S, h].double() for x in (s["k_cache"], s["v_cache"]))
                for i in range(h * (hq // hk), (h + 1) * (hq // hk)):
                    a = (s["q"][first:first + r, i].double() @ k.t() / math.sqrt(D)).masked_fill(hidden, -math.inf)
                    l = torch.logsumexp(a, 1)
                    out[first:first + r, i] = torch.exp(a - l[:, None]).nan_to_num(0.0) @ v
                    lse[first:first + r, i] = l
        first += r
    return {"out": out, "lse": lse}
