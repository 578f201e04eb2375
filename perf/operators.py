"""What stands between the compressed products of a decode step, as a list of cases that can be timed.

Sizes are those of the LLaMA-3.2 shapes that inputs/synth.py and bench.py name (1B: hidden 2048, 32 heads of 64, key/value
512 = 8 heads of 64, feed-forward 8192; 3B: 24 heads of 128, key/value 1024 = 8 heads of 128), with batches up to the 16 rows
of a product and contexts up to that family's 131072 tokens.

Kinds of case:
  norm     residual + product -> new residual, and the RMS-normalised row as the next product's bf16 x (or int8 with a scale)
  append   rotary positions on q and k, and the new keys and values into a paged cache (bf16, or int8 with scales)
  attend   one new token per row over its sequence's pages; with "track", the attention weights are added up per slot
  evict    a cache cut down to "keep" tokens per head, by accumulated attention weight

`own` False: elementary torch operations in 32 bits.  `own` True: the library's calls.
"""
import math

import torch

own = False

DEV = "cuda"
GRANDEST = {"norm": 4096 * 8192, "append": 8192 * 40 * 128, "attend": 16 * 32768 * 8 * 128, "evict": 16 * 32768 * 8 * 128}
EPS = 1e-5


def listed():
    return [
        # one token's row between two products of the 1B model: launch and latency
        {"name": "norm_1x2048", "kind": "norm", "rows": 1, "cols": 2048, "residual": "fp32", "out": "bf16"},
        # a few sequences of a model whose width is no multiple of anything, residual held in bf16
        {"name": "norm_13x2999_bf16", "kind": "norm", "rows": 13, "cols": 2999, "residual": "bf16", "out": "bf16"},
        # a long prompt's rows at the feed-forward width, 8-bit rows with scales
        {"name": "norm_4096x8192_int8", "kind": "norm", "rows": 4096, "cols": 8192, "residual": "fp32", "out": "int8"},
        # the new tokens of 16 sequences, 1B heads: one decode step
        {"name": "append_b16_1b", "kind": "append", "rows": 16, "seqs": 16, "heads": 32, "kv_heads": 8, "dim": 64, "page": 16, "context": 1000,
         "cache": "bf16"},
        # a prompt of 8192 tokens of one sequence, 3B heads, 8-bit cache
        {"name": "append_prompt_8192_3b_int8", "kind": "append", "rows": 8192, "seqs": 1, "heads": 24, "kv_heads": 8, "dim": 128, "page": 64,
         "context": 0, "cache": "int8"},
        # one sequence, a short context, 1B heads: the smallest attention there is in a chat's first answer
        {"name": "attend_1x200_1b", "kind": "attend", "rows": 1, "heads": 32, "kv_heads": 8, "dim": 64, "page": 16, "context": 200, "ragged": False,
         "cache": "bf16", "track": False},
        # 16 sequences of very different lengths up to 6000 tokens, one of them empty, 3B heads
        {"name": "attend_b16_ragged_3b", "kind": "attend", "rows": 16, "heads": 24, "kv_heads": 8, "dim": 128, "page": 16, "context": 6000,
         "ragged": True, "cache": "bf16", "track": False},
        # eight sequences whose weights are added up for a later eviction, 1B heads, a length that ends inside a page
        {"name": "attend_b8_track_1b", "kind": "attend", "rows": 8, "heads": 32, "kv_heads": 8, "dim": 64, "page": 32, "context": 8179,
         "ragged": False, "cache": "bf16", "track": True},
        # one sequence at the longest context of the family, 3B heads
        {"name": "attend_1x131071_3b", "kind": "attend", "rows": 1, "heads": 24, "kv_heads": 8, "dim": 128, "page": 64, "context": 131071,
         "ragged": False, "cache": "bf16", "track": False},
        # 16 long sequences on an 8-bit cache, 3B heads: the most a decode step reads here
        {"name": "attend_b16x32768_3b_int8", "kind": "attend", "rows": 16, "heads": 24, "kv_heads": 8, "dim": 128, "page": 64, "context": 32768,
         "ragged": False, "cache": "int8", "track": False},
        # one sequence, a budget of 1024 tokens and 128 tokens over it, 1B heads
        {"name": "evict_1x1152_1b", "kind": "evict", "seqs": 1, "kv_heads": 8, "dim": 64, "page": 16, "context": 1152, "keep": 1024, "recent": 256},
        # 16 sequences cut from 16384 tokens to half of them, 3B heads
        {"name": "evict_b16x16384_3b", "kind": "evict", "seqs": 16, "kv_heads": 8, "dim": 128, "page": 64, "context": 16384, "keep": 8192,
         "recent": 512},
    ]


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["norm", "append", "attend", "attend", "attend", "evict"])
    heads, kv_heads, dim = rng.choice([(32, 8, 64), (24, 8, 128), (32, 8, 128), (16, 16, 64), (12, 2, 128), (20, 4, 96), (8, 1, 256)])
    page = rng.choice([16, 16, 32, 64, 256])
    if kind == "norm":
        cols = _log_uniform(rng, 64, 8192)
        cols = max(64, cols // 64 * 64) if rng.random() < 0.6 else cols
        rows = _log_uniform(rng, 1, min(4096, GRANDEST["norm"] // cols))
        return {"kind": kind, "rows": rows, "cols": cols, "residual": rng.choice(["fp32", "fp32", "bf16"]), "out": rng.choice(["bf16", "bf16", "int8"])}
    heads_case = {"kv_heads": kv_heads, "dim": dim, "page": page}
    if kind == "append":
        case = dict(heads_case, kind=kind, heads=heads, cache=rng.choice(["bf16", "bf16", "int8"]))
        if rng.random() < 0.5:      # one new token for each of some sequences
            rows = _log_uniform(rng, 1, 64)
            return dict(case, rows=rows, seqs=rows, context=_log_uniform(rng, 1, 4000))
        rows = _log_uniform(rng, 16, min(8192, GRANDEST["append"] // ((heads + 2 * kv_heads) * dim)))
        return dict(case, rows=rows, seqs=1, context=rng.choice([0, _log_uniform(rng, 1, 4000)]))
    n = rng.choice([1, 1, 2, 3, 4, 8, 12, 16])
    most = min(131072, GRANDEST[kind] // (n * kv_heads * dim))
    if kind == "attend":
        cache, track = rng.choice(["bf16", "bf16", "int8"]), rng.random() < 0.25
        return dict(heads_case, kind=kind, heads=heads, rows=n, context=_log_uniform(rng, 1, most // 2 if cache == "bf16" else most),
                    ragged=rng.random() < 0.4, cache=cache, track=track)
    context = _log_uniform(rng, 64, min(65536, most // 2))
    keep = max(1, int(context * rng.choice([0.25, 0.5, 0.9, 0.99])))
    return dict(heads_case, kind=kind, seqs=n, context=context, keep=keep, recent=int(keep * rng.choice([0.0, 0.1, 0.25])))


# ---- inputs ----------------------------------------------------------------------------------------------------------

def _lengths(case):
    """Tokens of each row's sequence: the context, or spread below it with the last row empty."""
    n, c = case["rows"], case["context"]
    if not case["ragged"]:
        return [c] * n
    got = [1 + int((c - 1) * ((0.618034 * r + 0.9) % 1.0)) for r in range(n)]
    if n >= 4:
        got[-1] = 0
    return got


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32)


def _pages(g, n_seqs, seq_pages):
    """Page tables: every sequence's pages lie anywhere in the pool."""
    return torch.randperm(n_seqs * seq_pages, generator=g, device=DEV).to(torch.int32).view(n_seqs, seq_pages)


def _pool(g, kind, n_pages, kv_heads, page, dim):
    """One pool [page][head][slot][dim] of N(0, 1) values -> (values, scales or None)."""
    x = _normal(g, n_pages, kv_heads, page, dim)
    if kind == "bf16":
        return x.to(torch.bfloat16), None
    scale = x.abs().amax(dim=-1) / 127.0
    return torch.round(x / scale[..., None]).to(torch.int8), scale


def _scores(g, *shape):
    """Accumulated weights: many small ones, a few large ones, some never attended to (equal, zero)."""
    s = torch.exp(2.0 * _normal(g, *shape) - 4.0)
    return torch.where(torch.rand(shape, generator=g, device=DEV) < 0.05, torch.zeros_like(s), s)


def _rotation(n, dim):
    """cos and sin [positions][dim / 2] of the usual frequencies, base 500000, from 64 bits."""
    freq = 500000.0 ** (-torch.arange(0, dim, 2, device=DEV, dtype=torch.float64) / dim)
    angle = torch.arange(n, device=DEV, dtype=torch.float64)[:, None] * freq[None, :]
    return torch.cos(angle).float(), torch.sin(angle).float()


def _inputs(case, seed):
    """The tensors of a case, a function of the seed alone."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    kind = case["kind"]
    if kind == "norm":
        rows, cols = case["rows"], case["cols"]
        res = torch.bfloat16 if case["residual"] == "bf16" else torch.float32
        s = {"residual": (2.0 * _normal(g, rows, cols)).to(res), "delta": 0.5 * _normal(g, rows, cols),
             "weight": (1.0 + 0.2 * _normal(g, cols)).to(torch.bfloat16)}
        s["residual_out"] = torch.empty_like(s["residual"])
        s["out"] = torch.empty((rows, cols), dtype=torch.bfloat16 if case["out"] == "bf16" else torch.int8, device=DEV)
        if case["out"] == "int8":
            s["out_scale"] = torch.empty((rows, 1), device=DEV)
            s["out_values"] = torch.empty((rows, cols), dtype=torch.bfloat16, device=DEV)
        return s
    hk, d, page = case["kv_heads"], case["dim"], case["page"]
    if kind == "append":
        rows, n = case["rows"], case["seqs"]
        new = rows // n
        seq_pages = -(-(case["context"] + new) // page)
        s = {"q": _normal(g, rows, case["heads"], d), "k_new": _normal(g, rows, hk, d), "v_new": _normal(g, rows, hk, d),
             "tables": _pages(g, n, seq_pages)}
        s["k"], s["k_scale"] = _pool(g, case["cache"], n * seq_pages, hk, page, d)
        s["v"], s["v_scale"] = _pool(g, case["cache"], n * seq_pages, hk, page, d)
        s["seqs"] = torch.arange(rows, device=DEV, dtype=torch.int32) // new
        s["slots"] = case["context"] + torch.arange(rows, device=DEV, dtype=torch.int32) % new
        s["cos"], s["sin"] = _rotation(case["context"] + new, d)
        s["q_out"] = torch.empty_like(s["q"])
        if case["cache"] == "int8":
            s["k_values"], s["v_values"] = (torch.empty(s["k"].shape, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        return s
    if kind == "attend":
        rows = case["rows"]
        seq_pages = -(-case["context"] // page)
        s = {"q": 1.5 * _normal(g, rows, case["heads"], d), "tables": _pages(g, rows, seq_pages),
             "lengths": torch.tensor(_lengths(case), dtype=torch.int32, device=DEV)}
        s["k"], s["k_scale"] = _pool(g, case["cache"], rows * seq_pages, hk, page, d)
        s["v"], s["v_scale"] = _pool(g, case["cache"], rows * seq_pages, hk, page, d)
        s["out"] = torch.empty((rows, case["heads"], d), dtype=torch.bfloat16, device=DEV)
        if case["track"]:
            s["scores"] = _scores(g, rows, hk, seq_pages * page) / case["context"]      # as a few earlier tokens left them
        return s
    n = case["seqs"]
    seq_pages = -(-case["context"] // page)
    cap = seq_pages * page
    s = {"tables": _pages(g, n, seq_pages), "lengths": torch.full((n,), case["context"], dtype=torch.int32, device=DEV)}
    s["k"], s["v"] = (_pool(g, "bf16", n * seq_pages, hk, page, d)[0] for _ in range(2))
    s["scores"] = _scores(g, n, hk, cap)
    # positions as earlier evictions left them: each head has its own gaps, and an order in part
    step = torch.randint(1, 3, (n, hk, cap), generator=g, device=DEV)
    pos = torch.cumsum(step, dim=-1)
    first = min(case["keep"], cap)
    swap = torch.randperm(first, generator=g, device=DEV)
    s["positions"] = torch.cat([pos[..., :first][..., swap], pos[..., first:]], dim=-1).to(torch.int32).contiguous()
    newest = s["positions"][:, :, : case["context"]].amax(dim=(1, 2))
    s["since"] = newest + 1 - case["recent"] if case["recent"] else newest + 1
    s["since"] = s["since"].to(torch.int32)
    s["scores_out"], s["positions_out"], s["lengths_out"] = torch.zeros_like(s["scores"]), torch.zeros_like(s["positions"]), torch.zeros_like(s["lengths"])
    return s


def _ptr(t):
    return 0 if t is None else t.data_ptr()


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        s["call"] = _call(case, s)
    return s


def _call(case, s):
    """The prepared call a program keeps for its buffers."""
    import paper_2509_22951_amd as tq
    kind = case["kind"]
    if kind == "norm":
        return tq.AddNorm(residual=_ptr(s["residual"]), delta=_ptr(s["delta"]), weight=_ptr(s["weight"]), residual_out=_ptr(s["residual_out"]),
                          out=_ptr(s["out"]), out_scale=_ptr(s.get("out_scale")), rows=case["rows"], cols=case["cols"], eps=EPS,
                          residual_type=tq.TQ_BF16 if case["residual"] == "bf16" else tq.TQ_FP32, weight_type=tq.TQ_BF16,
                          out_type=tq.TQ_BF16 if case["out"] == "bf16" else tq.TQ_INT8)
    n_seqs, seq_pages = s["tables"].shape
    cache = tq.Cache(k=_ptr(s["k"]), v=_ptr(s["v"]), k_scale=_ptr(s.get("k_scale")), v_scale=_ptr(s.get("v_scale")), tables=_ptr(s["tables"]),
                     scores=_ptr(s.get("scores")), positions=_ptr(s.get("positions")),
                     type=tq.TQ_INT8 if case.get("cache") == "int8" else tq.TQ_BF16, n_pages=s["k"].shape[0], page_size=case["page"],
                     kv_heads=case["kv_heads"], head_dim=case["dim"], n_seqs=n_seqs, seq_pages=seq_pages)
    if kind == "append":
        return tq.CacheAppend(cache, q=_ptr(s["q"]), k=_ptr(s["k_new"]), v=_ptr(s["v_new"]), q_out=_ptr(s["q_out"]), seqs=_ptr(s["seqs"]),
                              slots=_ptr(s["slots"]), cos=_ptr(s["cos"]), sin=_ptr(s["sin"]), rows=case["rows"], heads=case["heads"],
                              rotary_dim=case["dim"], n_positions=s["cos"].shape[0], q_out_type=tq.TQ_FP32)
    if kind == "attend":
        fields = dict(q=_ptr(s["q"]), out=_ptr(s["out"]), lengths=_ptr(s["lengths"]), rows=case["rows"], heads=case["heads"],
                      scale=1.0 / math.sqrt(case["dim"]), q_type=tq.TQ_FP32, accumulate=int(case["track"]))
        s["workspace"] = torch.zeros(tq.Attend.workspace_bytes(cache, **fields), dtype=torch.uint8, device=DEV)
        return tq.Attend(cache, workspace=_ptr(s["workspace"]), workspace_bytes=s["workspace"].numel(), **fields)
    fields = dict(lengths=_ptr(s["lengths"]), lengths_out=_ptr(s["lengths_out"]), since=_ptr(s["since"]), scores_out=_ptr(s["scores_out"]),
                  positions_out=_ptr(s["positions_out"]), keep=case["keep"])
    s["workspace"] = torch.zeros(tq.CacheEvict.workspace_bytes(cache, **fields), dtype=torch.uint8, device=DEV)
    return tq.CacheEvict(cache, workspace=_ptr(s["workspace"]), workspace_bytes=s["workspace"].numel(), **fields)


# ---- one pass --------------------------------------------------------------------------------------------------------

def run(state):
    kind = state["case"]["kind"]
    if own:
        state["call"].launch(torch.cuda.current_stream().cuda_stream)
    else:
        {"norm": _plain_norm, "append": _plain_append, "attend": _plain_attend, "evict": _plain_evict}[kind](state)
    return _outputs(state)


def _outputs(s):
    """What a pass leaves; rows held in 8 bits as the values they stand for."""
    kind = s["case"]["kind"]
    if kind == "norm":
        if "out_values" in s:
            return {"residual": s["residual_out"], "out": torch.mul(s["out"], s["out_scale"], out=s["out_values"])}
        return {"residual": s["residual_out"], "out": s["out"]}
    if kind == "append":
        if "k_values" in s:
            return {"q": s["q_out"], "k": torch.mul(s["k"], s["k_scale"][..., None], out=s["k_values"]),
                    "v": torch.mul(s["v"], s["v_scale"][..., None], out=s["v_values"])}
        return {"q": s["q_out"], "k": s["k"], "v": s["v"]}
    if kind == "attend":
        return {"out": s["out"], "scores": s["scores"]} if "scores" in s else {"out": s["out"]}
    return {"k": s["k"], "v": s["v"], "scores": s["scores_out"], "positions": s["positions_out"], "lengths": s["lengths_out"]}


def _quantized(x, scale_out):
    """Rows along the last axis as int8 levels: scale = absmax / 127, round half to even."""
    scale = x.abs().amax(dim=-1)
    scale = scale / torch.full_like(scale, 127.0)
    safe = torch.where(scale > 0, scale, torch.ones_like(scale))
    scale_out.copy_(scale.view(scale_out.shape))
    return torch.clamp(torch.round(x / safe[..., None]), -127, 127).to(torch.int8)


def _plain_norm(s):
    h = s["residual"].float() + s["delta"]
    s["residual_out"].copy_(h)
    y = h * torch.rsqrt((h * h).mean(dim=-1, keepdim=True) + EPS) * s["weight"].float()
    s["out"].copy_(_quantized(y, s["out_scale"]) if "out_scale" in s else y)


def _rotated(x, cos, sin):
    a, b = x.chunk(2, dim=-1)
    return torch.cat([a * cos - b * sin, a * sin + b * cos], dim=-1)


def _plain_append(s):
    page = s["case"]["page"]
    slots, seqs = s["slots"].long(), s["seqs"].long()
    cos, sin = s["cos"][slots][:, None, :], s["sin"][slots][:, None, :]
    s["q_out"].copy_(_rotated(s["q"], cos, sin))
    at = (s["tables"][seqs, slots // page].long(), slice(None), slots % page)
    for new, name in ((_rotated(s["k_new"], cos, sin), "k"), (s["v_new"], "v")):
        if s[name + "_scale"] is not None:
            scale = torch.empty(new.shape[:2], device=new.device)
            new = _quantized(new, scale)
            s[name + "_scale"][at] = scale
        s[name][at] = new.to(s[name].dtype)


def _gathered(s, name):
    """A pool's values in sequence order, fp32 [seq][head][slot][dim]; slots past a length are zero."""
    x = s[name][s["tables"].long()].float()                               # [seq][page][head][slot][dim]
    if s[name + "_scale"] is not None:
        x = x * s[name + "_scale"][s["tables"].long()][..., None]
    x = x.transpose(1, 2).flatten(2, 3)
    there = torch.arange(x.shape[2], device=x.device)[None, :] < s["lengths"][:, None]
    return torch.where(there[:, None, :, None], x, torch.zeros_like(x)), there


def _plain_attend(s):
    case = s["case"]
    rows, hk, d = case["rows"], case["kv_heads"], case["dim"]
    k, there = _gathered(s, "k")
    q = s["q"].view(rows, hk, case["heads"] // hk, d) * (1.0 / math.sqrt(d))
    logits = torch.matmul(q, k.transpose(-1, -2).contiguous())
    del k
    there = there[:, None, None, :]
    logits = torch.where(there, logits, torch.full_like(logits, -math.inf))
    top = logits.amax(dim=-1, keepdim=True)
    p = torch.where(there, torch.exp(logits - torch.where(top == -math.inf, torch.zeros_like(top), top)), torch.zeros_like(logits))
    total = p.sum(dim=-1, keepdim=True)
    p = p / torch.where(total > 0, total, torch.ones_like(total))
    if "scores" in s:
        s["scores"].add_(p.sum(dim=2))
    v, _ = _gathered(s, "v")
    s["out"].copy_(torch.matmul(p, v).view(rows, case["heads"], d))


def _plain_evict(s):
    page, keep = s["case"]["page"], s["case"]["keep"]
    n, hk, cap = s["scores"].shape
    slot = torch.arange(cap, device=s["scores"].device)
    there = (slot[None, :] < s["lengths"][:, None])[:, None, :].expand(n, hk, cap)
    inf = torch.full_like(s["scores"], math.inf)
    key = torch.where(s["positions"] >= s["since"][:, None, None], inf, s["scores"])
    key = torch.where(there, key, -inf)
    order = torch.sort(key, dim=-1, descending=True, stable=True).indices     # equal ones: lowest slot first
    kept = torch.zeros_like(there.contiguous())
    kept.scatter_(-1, order[..., :keep], torch.ones_like(order[..., :keep], dtype=torch.bool))
    kept &= there
    to, of = (there & ~kept & (slot < keep)).nonzero(), (kept & (slot >= keep)).nonzero()
    s["lengths_out"].copy_(torch.clamp(s["lengths"], max=keep))
    stays = kept & (slot < keep)
    for name in ("scores", "positions"):
        out = s[name + "_out"]
        out.copy_(torch.where(stays, s[name], out))
        out[to[:, 0], to[:, 1], to[:, 2]] = s[name][of[:, 0], of[:, 1], of[:, 2]]
    for name in ("k", "v"):
        of_page, to_page = (s["tables"][x[:, 0], x[:, 2] // page].long() for x in (of, to))
        s[name][to_page, to[:, 1], to[:, 2] % page] = s[name][of_page, of[:, 1], of[:, 2] % page]


# ---- what a pass cannot do without, and what it gives in 64 bits -----------------------------------------------------

def work(case):
    kind = case["kind"]
    if kind == "norm":
        n, r = case["rows"] * case["cols"], 2 if case["residual"] == "bf16" else 4
        return {"bytes": n * (2 * r + 4 + (2 if case["out"] == "bf16" else 1)) + 2 * case["cols"], "flops": 6 * n}
    hk, d = case["kv_heads"], case["dim"]
    size = 1 if case.get("cache") == "int8" else 2
    if kind == "append":
        rows, h = case["rows"], case["heads"]
        positions = rows if case["seqs"] == 1 else 1
        return {"bytes": rows * (8 * h * d + hk * 2 * (4 * d + size * d + (4 if size == 1 else 0))) + 4 * d * positions, "flops": 3 * rows * (h + hk) * d}
    if kind == "attend":
        tokens = sum(_lengths(case))
        per = 2 * (size * d + (4 if size == 1 else 0)) + (8 if case["track"] else 0)
        return {"bytes": tokens * hk * per + 6 * case["rows"] * case["heads"] * d, "flops": 4 * tokens * case["heads"] * d}
    n, keep, context = case["seqs"], case["keep"], case["context"]
    # a kept token outside of the budget's slots is read and written; about keep * (context - keep) / context of them
    moved = keep * (context - keep) // context
    return {"bytes": n * hk * (8 * context + 8 * keep + moved * 2 * 2 * 2 * d), "flops": 0}


def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind == "norm":
        h = s["residual"].double() + s["delta"].double()
        y = h / torch.sqrt(h.square().mean(dim=1, keepdim=True) + EPS) * s["weight"].double()
        return {"residual": h, "out": _levels(y) if case["out"] == "int8" else y}
    if kind == "append":
        return _exact_append(case, s)
    if kind == "attend":
        return _exact_attend(case, s)
    return _exact_evict(case, s)


def _levels(y):
    """What 8 bits hold of rows along the last axis."""
    scale = y.abs().amax(dim=-1, keepdim=True) / 127.0
    return torch.round(y / torch.where(scale > 0, scale, torch.ones_like(scale))) * scale


def _exact_append(case, s):
    d, page = case["dim"], case["page"]

    def rotated(x):
        z = torch.complex(x[..., : d // 2].double(), x[..., d // 2:].double())
        at = s["slots"].long()
        z = z * torch.complex(s["cos"].double()[at], s["sin"].double()[at])[:, None, :]
        return torch.cat([z.real, z.imag], dim=-1)

    out = {"q": rotated(s["q"])}
    where = s["tables"].long()[s["seqs"].long(), s["slots"].long() // page] * page + s["slots"].long() % page
    for name, new in (("k", rotated(s["k_new"])), ("v", s["v_new"].double())):
        pool = s[name].double()
        if case["cache"] == "int8":
            pool, new = pool * s[name + "_scale"].double()[..., None], _levels(new)
        flat = pool.transpose(1, 2).reshape(-1, case["kv_heads"], d)
        flat[where] = new
        out[name] = flat.view(pool.shape[0], page, case["kv_heads"], d).transpose(1, 2).contiguous()
    return out


def _exact_attend(case, s):
    hk, d, group = case["kv_heads"], case["dim"], case["heads"] // case["kv_heads"]
    out = torch.zeros((case["rows"], case["heads"], d), dtype=torch.float64, device=DEV)
    scores = s["scores"].double() if case["track"] else None
    for r, length in enumerate(_lengths(case)):
        for h in range(hk if length else 0):
            at = s["tables"][r].long()
            k, v = (s[n][at, h].reshape(-1, d)[:length].double() for n in ("k", "v"))
            if case["cache"] == "int8":
                k, v = (x * s[n][at, h].reshape(-1, 1)[:length].double() for x, n in ((k, "k_scale"), (v, "v_scale")))
            logits = k @ s["q"][r, h * group:(h + 1) * group].double().T.contiguous() / math.sqrt(d)
            p = torch.softmax(logits, dim=0)
            out[r, h * group:(h + 1) * group] = p.T.contiguous() @ v
            if case["track"]:
                scores[r, h, :length] += p.sum(dim=1)
    return {"out": out, "scores": scores} if case["track"] else {"out": out}


def _exact_evict(case, s):
    page, keep, context = case["page"], case["keep"], case["context"]
    out = {"k": s["k"].double(), "v": s["v"].double(), "scores": s["scores_out"].double(), "positions": s["positions_out"].clone(),
           "lengths": torch.clamp(s["lengths"], max=keep)}
    scores, positions = s["scores"][..., :context].cpu(), s["positions"][..., :context].cpu()
    for n in range(case["seqs"]):
        for h in range(case["kv_heads"]):
            rank = torch.where(positions[n, h] >= int(s["since"][n]), torch.full_like(scores[n, h], math.inf), scores[n, h]).numpy()
            kept = sorted((-rank).argsort(kind="stable")[:keep].tolist())
            free = sorted(set(range(min(keep, context))) - set(kept))
            take = list(range(min(keep, context)))
            for to, of in zip(free, kept[len(kept) - len(free):]):
                take[to] = of
            to = torch.arange(len(take), device=DEV)
            of = torch.tensor(take, device=DEV)
            for name in ("scores", "positions"):
                out[name][n, h, : len(take)] = s[name][n, h, of].to(out[name].dtype)
            of_page, to_page = (s["tables"][n].long()[x // page] for x in (of, to))
            for name in ("k", "v"):
                out[name][to_page, h, to % page] = s[name][of_page, h, of % page].double()
    return out
