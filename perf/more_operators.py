"""What a decoder needs beyond one greedy token a step, as a list of cases that can be timed: queries and keys normed per head on
their way into the cache, attention of a tree of drafted tokens, tokens drawn from logits, and the accepted branch of a tree.

Sizes are those of the LLaMA-3.2 shapes that inputs/synth.py and bench.py name (1B: 32 heads of 64, key/value 512 = 8 heads of 64,
vocabulary 128256, 16 layers; 3B: 24 heads of 128, key/value 1024 = 8 heads of 128, 28 layers), contexts up to that family's 131072
tokens, and up to 64 nodes of a tree; 16 rows is what one product takes.

Kinds of case:
  normed   per-head root-mean-square norm of q and k, rotary positions, keys and values into a paged cache
  tree     every node of a drafted tree attends to its sequence's tokens and to its ancestors in the tree
  sample   one token per row of logits: temperature, top-k, top-p, min-p, from a given uniform number
  accept   the longest branch of a tree that the drawn tokens agree with; its keys and values moved together, in every layer

`own` False: elementary torch operations in 32 bits (drawing in 64).  `own` True: the library's calls.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
EPS = 1e-6
MOST_APPENDED, MOST_CACHED, MOST_PRODUCTS, MOST_LOGITS = 8192 * 40 * 128, 16 * 32768 * 8 * 128, 16 * 32768 * 24 * 128 * 16, 64 * 128256


def listed():
    return [
        # one decode step of 16 sequences, 1B heads: launch and latency
        {"name": "normed_b16_1b", "kind": "normed", "rows": 16, "seqs": 16, "heads": 32, "kv_heads": 8, "dim": 64, "page": 16, "context": 1000,
         "cache": "bf16", "weight": "bf16", "per_head": False},
        # four trees of 16 drafted tokens behind an odd context, 3B heads, 8-bit cache, weights of their own for every head
        {"name": "normed_tree_4x16_3b_int8", "kind": "normed", "rows": 64, "seqs": 4, "heads": 24, "kv_heads": 8, "dim": 128, "page": 16, "context": 333,
         "cache": "int8", "weight": "fp32", "per_head": True},
        # a prompt of 8192 tokens of one sequence, 3B heads: the most that goes into a cache at a time here
        {"name": "normed_prompt_8192_3b", "kind": "normed", "rows": 8192, "seqs": 1, "heads": 24, "kv_heads": 8, "dim": 128, "page": 64, "context": 0,
         "cache": "bf16", "weight": "bf16", "per_head": False},
        # a small tree in a chat's first answer, 1B heads: the smallest there is
        {"name": "tree_1x8_200_1b", "kind": "tree", "trees": 1, "nodes": 8, "heads": 32, "kv_heads": 8, "dim": 64, "page": 16, "context": 200,
         "ragged": False, "cache": "bf16"},
        # eight sequences of very different lengths up to 6001 tokens, one of them empty, trees of up to 15 nodes, 3B heads
        {"name": "tree_b8x15_ragged_3b", "kind": "tree", "trees": 8, "nodes": 15, "heads": 24, "kv_heads": 8, "dim": 128, "page": 16, "context": 6001,
         "ragged": True, "cache": "bf16"},
        # one sequence near the longest context of the family, a tree as large as trees get, 3B heads
        {"name": "tree_1x64_131000_3b", "kind": "tree", "trees": 1, "nodes": 64, "heads": 24, "kv_heads": 8, "dim": 128, "page": 64, "context": 131000,
         "ragged": False, "cache": "bf16"},
        # 16 long sequences on an 8-bit cache, 3B heads: the most a step of drafted tokens reads here
        {"name": "tree_b16x16_32700_3b_int8", "kind": "tree", "trees": 16, "nodes": 16, "heads": 24, "kv_heads": 8, "dim": 128, "page": 64,
         "context": 32700, "ragged": False, "cache": "int8"},
        # one row at the smaller vocabulary of the example decoder, as a chat program sets the filters
        {"name": "sample_1x32000", "kind": "sample", "rows": 1, "vocab": 32000, "filters": "chat"},
        # a product's 16 rows at the family's vocabulary, every row with filters of its own, one of them greedy, one without any
        {"name": "sample_16x128256_mixed", "kind": "sample", "rows": 16, "vocab": 128256, "filters": "mixed"},
        # all nodes of four trees of 16, no filter but the temperature: every token stays
        {"name": "sample_64x128256_open", "kind": "sample", "rows": 64, "vocab": 128256, "filters": "open"},
        # one small tree, 16 layers of 1B heads: launch and latency
        {"name": "accept_1x8_16l_1b", "kind": "accept", "trees": 1, "nodes": 8, "kv_heads": 8, "dim": 64, "page": 16, "context": 100, "layers": 16},
        # 16 trees of 64 nodes, 28 layers of 3B heads
        {"name": "accept_b16x64_28l_3b", "kind": "accept", "trees": 16, "nodes": 64, "kv_heads": 8, "dim": 128, "page": 16, "context": 75, "layers": 28},
    ]


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["normed", "tree", "tree", "tree", "sample", "sample", "accept"])
    if kind == "sample":
        vocab = _log_uniform(rng, 500, 128256)
        return {"kind": kind, "rows": _log_uniform(rng, 1, min(256, MOST_LOGITS // vocab)), "vocab": vocab, "filters": rng.choice(["chat", "mixed", "mixed", "open"])}
    heads, kv_heads, dim = rng.choice([(32, 8, 64), (24, 8, 128), (32, 8, 128), (16, 16, 64), (12, 2, 128), (20, 4, 96), (8, 1, 256)])
    page = rng.choice([16, 16, 32, 64, 256])
    case = {"kind": kind, "kv_heads": kv_heads, "dim": dim, "page": page}
    nodes = rng.choice([1, 2, 4, 5, 8, 11, 16, 16, 16, 31, 48, 64])
    if kind == "accept":
        layers = rng.choice([2, 4, 16, 28, 40])
        trees = _log_uniform(rng, 1, 16)
        context = _log_uniform(rng, 1, max(1, min(400, 28 * 16 * 139 * 1024 // (layers * trees * kv_heads * dim) - nodes)))
        return dict(case, trees=trees, nodes=nodes, context=context, layers=layers)
    if kind == "normed":
        case.update(heads=heads, cache=rng.choice(["bf16", "bf16", "int8"]), weight=rng.choice(["bf16", "fp32"]), per_head=rng.random() < 0.3)
        if rng.random() < 0.6:      # a tree, or one new token, for each of some sequences
            seqs = _log_uniform(rng, 1, 16)
            return dict(case, rows=seqs * nodes, seqs=seqs, context=_log_uniform(rng, 1, 4000))
        rows = _log_uniform(rng, 16, min(8192, MOST_APPENDED // ((heads + 2 * kv_heads) * dim)))
        return dict(case, rows=rows, seqs=1, context=rng.choice([0, _log_uniform(rng, 1, 4000)]))
    trees, cache = rng.choice([1, 1, 2, 3, 4, 8, 12, 16]), rng.choice(["bf16", "bf16", "int8"])
    most = min(131000, MOST_CACHED // (trees * kv_heads * dim) // (2 if cache == "bf16" else 1), MOST_PRODUCTS // (trees * heads * nodes * dim))
    return dict(case, trees=trees, nodes=nodes, heads=heads, context=_log_uniform(rng, 1, most - nodes), ragged=rng.random() < 0.4, cache=cache)


# ---- inputs ----------------------------------------------------------------------------------------------------------

def _lengths(case):
    """Tokens of each sequence ahead of its tree: the context, or spread below it with the last sequence empty."""
    n, c = case["trees"], case["context"]
    if not case.get("ragged"):
        return [c] * n
    got = [1 + int((c - 1) * ((0.618034 * r + 0.9) % 1.0)) for r in range(n)]
    if n >= 4:
        got[-1] = 0
    return got


def _sizes(case):
    """Nodes of each tree: all, or, with ragged sequences, some fewer."""
    return [max(1, case["nodes"] - (3 * t) % 5) if case.get("ragged") else case["nodes"] for t in range(case["trees"])]


def _parents(case, seed):
    """A tree for each sequence, node 0 its root, every other node the child of one shortly before it."""
    rng = random.Random(seed)
    return [[-1] + [rng.randint(max(0, i // 2 - 1), i - 1) for i in range(1, case["nodes"])] for _ in range(case["trees"])]


def _masks(parents):
    """For each node the nodes it attends to, itself and its ancestors, as bits."""
    rows = []
    for tree in parents:
        bits = []
        for i, p in enumerate(tree):
            bits.append((bits[p] if p >= 0 else 0) | 1 << i)
        rows.append([b - (1 << 64) if b >> 63 else b for b in bits])
    return torch.tensor(rows, dtype=torch.int64, device=DEV)


def _words(case, parents, seed):
    """Drafted and drawn tokens [trees][nodes]: at four of five nodes the drawn token is one of the children's."""
    rng = random.Random(seed + 1)
    drafted = [[rng.randrange(128256) for _ in tree] for tree in parents]
    drawn = []
    for tree, words in zip(parents, drafted):
        children = [[] for _ in tree]
        for i, p in enumerate(tree):
            if p >= 0:
                children[p].append(i)
        drawn.append([words[rng.choice(c)] if c and rng.random() < 0.8 else rng.randrange(128256) for c in children])
    return drafted, drawn


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


def _rotation(n, dim):
    """cos and sin [positions][dim / 2] of the usual frequencies, base 500000, from 64 bits."""
    freq = 500000.0 ** (-torch.arange(0, dim, 2, device=DEV, dtype=torch.float64) / dim)
    angle = torch.arange(n, device=DEV, dtype=torch.float64)[:, None] * freq[None, :]
    return torch.cos(angle).float(), torch.sin(angle).float()


def _filters(case, g):
    """temperature, top_k, top_p, min_p of each row."""
    n = case["rows"]
    if case["filters"] == "open":
        t, k, p, m = [1.0] * n, [0] * n, [1.0] * n, [0.0] * n
    elif case["filters"] == "chat":
        t, k, p, m = [0.8] * n, [50] * n, [0.95] * n, [0.0] * n
    else:
        kinds = [(0.7, 40, 0.9, 0.0), (1.0, 0, 0.95, 0.0), (1.2, 0, 1.0, 0.05), (0.0, 0, 1.0, 0.0), (1.0, 0, 1.0, 0.0), (0.6, 1000, 0.8, 0.02), (1.5, 200, 1.0, 0.1)]
        t, k, p, m = (list(x) for x in zip(*(kinds[r % len(kinds)] for r in range(n))))
    f = dict(dtype=torch.float32, device=DEV)
    return torch.tensor(t, **f), torch.tensor(k, dtype=torch.int32, device=DEV), torch.tensor(p, **f), torch.tensor(m, **f)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _inputs(case, seed):
    """The tensors of a case, a function of the seed alone."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    kind = case["kind"]
    if kind == "sample":
        n, vocab = case["rows"], case["vocab"]
        # logits as a model gives them: a broad bulk and, on top, a few tokens that stand out
        s = {"logits": 2.0 * _normal(g, n, vocab), "uniform": torch.rand((n,), generator=g, device=DEV)}
        at = torch.randint(0, vocab, (n, 12), generator=g, device=DEV)
        s["logits"].scatter_(1, at, 9.0 + 2.5 * _normal(g, n, 12))
        s["temperature"], s["top_k"], s["top_p"], s["min_p"] = _filters(case, g)
        s["tokens"], s["probs"] = torch.empty((n,), dtype=torch.int32, device=DEV), torch.empty((n,), device=DEV)
        return s
    hk, d, page = case["kv_heads"], case["dim"], case["page"]
    if kind == "normed":
        rows, n, h = case["rows"], case["seqs"], case["heads"]
        new = rows // n
        seq_pages = -(-(case["context"] + new) // page)
        s = {"q": 3.0 * _normal(g, rows, h, d), "k_new": 2.0 * _normal(g, rows, hk, d), "v_new": _normal(g, rows, hk, d), "tables": _pages(g, n, seq_pages)}
        s["k"], s["k_scale"] = _pool(g, case["cache"], n * seq_pages, hk, page, d)
        s["v"], s["v_scale"] = _pool(g, case["cache"], n * seq_pages, hk, page, d)
        kind_of = torch.bfloat16 if case["weight"] == "bf16" else torch.float32
        s["q_weight"], s["k_weight"] = ((1.0 + 0.3 * _normal(g, x if case["per_head"] else 1, d)).to(kind_of) for x in (h, hk))
        s["seqs"] = torch.arange(rows, device=DEV, dtype=torch.int32) // new
        s["slots"] = case["context"] + torch.arange(rows, device=DEV, dtype=torch.int32) % new
        if n == 1:       # a prompt: positions are slots
            s["positions"] = s["slots"].clone()
        else:            # a tree's tokens: as far behind the context as they lie deep in the tree
            depth = torch.sort(torch.randint(0, 1 + new // 2, (rows,), generator=g, device=DEV).view(n, new), dim=1).values
            s["positions"] = (case["context"] + depth).view(-1).to(torch.int32)
        s["cos"], s["sin"] = _rotation(case["context"] + new, d)
        s["q_out"] = torch.empty_like(s["q"])
        if case["cache"] == "int8":
            s["k_values"], s["v_values"] = (torch.empty(s["k"].shape, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        return s
    n, nodes = case["trees"], case["nodes"]
    seq_pages = -(-(case["context"] + nodes) // page)
    parents = _parents(case, seed)
    s = {"masks": _masks(parents), "sizes": _ints(_sizes(case)), "lengths": _ints(_lengths(case))}
    if kind == "tree":
        s["q"], s["tables"] = 1.5 * _normal(g, n * nodes, case["heads"], d), _pages(g, n, seq_pages)
        s["k"], s["k_scale"] = _pool(g, case["cache"], n * seq_pages, hk, page, d)
        s["v"], s["v_scale"] = _pool(g, case["cache"], n * seq_pages, hk, page, d)
        s["out"] = torch.empty((n * nodes, case["heads"], d), dtype=torch.bfloat16, device=DEV)
        return s
    drafted, drawn = _words(case, parents, seed)
    s["drafted"], s["sampled"] = _ints(drafted), _ints(drawn)
    s["tables"] = [_pages(g, n, seq_pages) for _ in range(case["layers"])]
    for name in ("k", "v"):
        s[name] = [_pool(g, "bf16", n * seq_pages, hk, page, d)[0] for _ in range(case["layers"])]
    s["path"], s["accepted"], s["next"], s["lengths_out"] = _ints([[0] * nodes] * n), _ints([0] * n), _ints([0] * n), _ints([0] * n)
    return s


def _ptr(t):
    return 0 if t is None else t.data_ptr()


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        s["call"] = _call(case, s)
    return s


def _cache(tq, case, k, v, tables, k_scale=None, v_scale=None):
    n_seqs, seq_pages = tables.shape
    return tq.Cache(k=_ptr(k), v=_ptr(v), k_scale=_ptr(k_scale), v_scale=_ptr(v_scale), tables=_ptr(tables),
                    type=tq.TQ_INT8 if case.get("cache") == "int8" else tq.TQ_BF16, n_pages=k.shape[0], page_size=case["page"],
                    kv_heads=case["kv_heads"], head_dim=case["dim"], n_seqs=n_seqs, seq_pages=seq_pages)


def _call(case, s):
    """The prepared call a program keeps for its buffers."""
    import paper_2509_22951_amd as tq
    kind = case["kind"]
    if kind == "sample":
        fields = dict(logits=_ptr(s["logits"]), temperature=_ptr(s["temperature"]), top_k=_ptr(s["top_k"]), top_p=_ptr(s["top_p"]), min_p=_ptr(s["min_p"]),
                      uniform=_ptr(s["uniform"]), tokens=_ptr(s["tokens"]), probs=_ptr(s["probs"]), rows=case["rows"], vocab=case["vocab"])
        s["workspace"] = torch.zeros(tq.Sample.workspace_bytes(**fields), dtype=torch.uint8, device=DEV)
        return tq.Sample(workspace=_ptr(s["workspace"]), workspace_bytes=s["workspace"].numel(), **fields)
    if kind == "normed":
        norm = tq.HeadNorm(q_weight=_ptr(s["q_weight"]), k_weight=_ptr(s["k_weight"]), q_weight_stride=case["dim"] if case["per_head"] else 0,
                           k_weight_stride=case["dim"] if case["per_head"] else 0, eps=EPS, weight_type=tq.TQ_BF16 if case["weight"] == "bf16" else tq.TQ_FP32)
        return tq.CacheAppendNormed(_cache(tq, case, s["k"], s["v"], s["tables"], s["k_scale"], s["v_scale"]), norm, q=_ptr(s["q"]), k=_ptr(s["k_new"]),
                                    v=_ptr(s["v_new"]), q_out=_ptr(s["q_out"]), seqs=_ptr(s["seqs"]), slots=_ptr(s["slots"]), positions=_ptr(s["positions"]),
                                    cos=_ptr(s["cos"]), sin=_ptr(s["sin"]), rows=case["rows"], heads=case["heads"], rotary_dim=case["dim"],
                                    n_positions=s["cos"].shape[0], q_out_type=tq.TQ_FP32)
    if kind == "tree":
        cache = _cache(tq, case, s["k"], s["v"], s["tables"], s["k_scale"], s["v_scale"])
        fields = dict(q=_ptr(s["q"]), out=_ptr(s["out"]), lengths=_ptr(s["lengths"]), sizes=_ptr(s["sizes"]), masks=_ptr(s["masks"]), trees=case["trees"],
                      nodes=case["nodes"], heads=case["heads"], scale=1.0 / math.sqrt(case["dim"]), q_type=tq.TQ_FP32)
        s["workspace"] = torch.zeros(tq.AttendTree.workspace_bytes(cache, **fields), dtype=torch.uint8, device=DEV)
        return tq.AttendTree(cache, workspace=_ptr(s["workspace"]), workspace_bytes=s["workspace"].numel(), **fields)
    caches = [_cache(tq, case, k, v, t) for k, v, t in zip(s["k"], s["v"], s["tables"])]
    return tq.TreeAccept(caches, masks=_ptr(s["masks"]), sizes=_ptr(s["sizes"]), lengths=_ptr(s["lengths"]), drafted=_ptr(s["drafted"]),
                         sampled=_ptr(s["sampled"]), path=_ptr(s["path"]), accepted=_ptr(s["accepted"]), next=_ptr(s["next"]),
                         lengths_out=_ptr(s["lengths_out"]), trees=case["trees"], nodes=case["nodes"])


# ---- one pass --------------------------------------------------------------------------------------------------------

def run(state):
    kind = state["case"]["kind"]
    if own:
        state["call"].launch(torch.cuda.current_stream().cuda_stream)
    else:
        {"normed": _plain_normed, "tree": _plain_tree, "sample": _plain_sample, "accept": _plain_accept}[kind](state)
    return _outputs(state)


def _outputs(s):
    """What a pass leaves; rows held in 8 bits as the values they stand for."""
    kind = s["case"]["kind"]
    if kind == "normed":
        if "k_values" in s:
            return {"q": s["q_out"], "k": torch.mul(s["k"], s["k_scale"][..., None], out=s["k_values"]),
                    "v": torch.mul(s["v"], s["v_scale"][..., None], out=s["v_values"])}
        return {"q": s["q_out"], "k": s["k"], "v": s["v"]}
    if kind == "tree":
        return {"out": s["out"]}
    if kind == "sample":
        return {"tokens": s["tokens"], "probs": s["probs"]}
    return {name: s[name] for name in ("path", "accepted", "next", "lengths_out", "k", "v")}


def _quantized(x):
    """Rows along the last axis as int8 levels and scales: scale = absmax / 127, round half to even."""
    scale = x.abs().amax(dim=-1)
    scale = scale / torch.full_like(scale, 127.0)
    safe = torch.where(scale > 0, scale, torch.ones_like(scale))
    return torch.clamp(torch.round(x / safe[..., None]), -127, 127).to(torch.int8), scale


def _plain_normed(s):
    page = s["case"]["page"]
    slots, seqs, positions = s["slots"].long(), s["seqs"].long(), s["positions"].long()
    cos, sin = s["cos"][positions][:, None, :], s["sin"][positions][:, None, :]

    def turned(x, weight):
        x = x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS) * weight.float()
        a, b = x.chunk(2, dim=-1)
        return torch.cat([a * cos - b * sin, a * sin + b * cos], dim=-1)

    s["q_out"].copy_(turned(s["q"], s["q_weight"]))
    at = (s["tables"][seqs, slots // page].long(), slice(None), slots % page)
    for new, name in ((turned(s["k_new"], s["k_weight"]), "k"), (s["v_new"], "v")):
        if s[name + "_scale"] is not None:
            new, s[name + "_scale"][at] = _quantized(new)
        s[name][at] = new.to(s[name].dtype)


def _plain_tree(s):
    case = s["case"]
    n, nodes, hk, d = case["trees"], case["nodes"], case["kv_heads"], case["dim"]
    group = case["heads"] // hk
    tables = s["tables"].long()

    def gathered(name):
        x = s[name][tables].float()                                       # [seq][page][head][slot][dim]
        if s[name + "_scale"] is not None:
            x = x * s[name + "_scale"][tables][..., None]
        return x.transpose(1, 2).flatten(2, 3)

    slot = torch.arange(tables.shape[1] * case["page"], device=DEV)
    node = slot[None, :] - s["lengths"][:, None]                          # of a slot, negative in the context
    bit = (s["masks"][:, :, None] >> node.clamp(0, nodes - 1)[:, None, :]) & 1
    sees = (node < 0)[:, None, :] | ((node >= 0) & (node < s["sizes"][:, None]))[:, None, :] & (bit == 1)
    sees = sees & (torch.arange(nodes, device=DEV)[None, :] < s["sizes"][:, None])[:, :, None]      # [tree][node][slot]
    used = (node < s["sizes"][:, None])[:, None, :, None]
    q = s["q"].view(n, nodes, hk, group, d).permute(0, 2, 1, 3, 4).reshape(n, hk, nodes * group, d) * (1.0 / math.sqrt(d))
    k = gathered("k")
    logits = torch.matmul(q, torch.where(used, k, torch.zeros_like(k)).transpose(-1, -2).contiguous()).view(n, hk, nodes, group, -1)
    del k
    sees = sees[:, None, :, None, :]
    logits = torch.where(sees, logits, torch.full_like(logits, -math.inf))
    top = logits.amax(dim=-1, keepdim=True)
    p = torch.exp(logits - torch.where(top == -math.inf, torch.zeros_like(top), top))
    del logits
    total = p.sum(dim=-1, keepdim=True)
    p = (p / torch.where(total > 0, total, torch.ones_like(total))).view(n, hk, nodes * group, -1)
    v = gathered("v")
    out = torch.matmul(p, torch.where(used, v, torch.zeros_like(v)))
    s["out"].copy_(out.view(n, hk, nodes, group, d).permute(0, 2, 1, 3, 4).reshape(s["out"].shape))


def _plain_sample(s):
    logits = s["logits"]
    t, top_p, min_p, u = (s[x].double()[:, None] for x in ("temperature", "top_p", "min_p", "uniform"))
    vocab = logits.shape[1]
    ranked, order = torch.sort(logits, dim=-1, descending=True, stable=True)      # equal ones: lowest token first
    warm = t > 0
    w = torch.exp((ranked.double() - ranked[:, :1].double()) / torch.where(warm, t, torch.ones_like(t)))
    upto = torch.cumsum(w, dim=-1)
    before = torch.cat([torch.zeros_like(upto[:, :1]), upto[:, :-1]], dim=-1)
    rank = torch.arange(vocab, device=DEV)[None, :]
    k = torch.where(s["top_k"] > 0, s["top_k"], torch.full_like(s["top_k"], vocab))[:, None]
    kept = (rank < k) & ((top_p >= 1) | (before < top_p * upto[:, -1:])) & (w >= min_p) & (warm | (rank == 0)) | (rank == 0)
    weight = torch.zeros_like(w).scatter_(1, order, torch.where(kept, w, torch.zeros_like(w)))
    upto = torch.cumsum(weight, dim=-1)                                           # by token
    token = (upto > u * upto[:, -1:]).to(torch.uint8).argmax(dim=-1)              # the first one beyond the uniform number's place
    s["tokens"].copy_(token)
    s["probs"].copy_(weight.gather(1, token[:, None])[:, 0] / upto[:, -1])


def _plain_accept(s):
    case = s["case"]
    n, nodes, page = case["trees"], case["nodes"], case["page"]
    masks, sizes, drafted, sampled = s["masks"], s["sizes"], s["drafted"], s["sampled"]
    index, one = torch.arange(nodes, device=DEV), torch.ones((), dtype=torch.int64, device=DEV)
    own_bit = one << index
    tree = torch.arange(n, device=DEV)
    at = torch.zeros(n, dtype=torch.int64, device=DEV)
    going = sizes > 0
    path = torch.full((n, nodes), -1, dtype=torch.int64, device=DEV)
    for step in range(nodes):
        path[:, step] = torch.where(going, at, path[:, step])
        s["next"].copy_(torch.where(going, sampled[tree, at], torch.full_like(s["next"], -1) if step == 0 else s["next"]))
        child = (masks == (masks[tree, at][:, None] | own_bit)) & (index[None, :] > at[:, None]) & (index[None, :] < sizes[:, None])
        child = child & (drafted == sampled[tree, at][:, None]) & going[:, None]
        going = child.any(dim=1)
        at = torch.where(going, child.to(torch.uint8).argmax(dim=1), at)
    s["path"].copy_(path)
    s["accepted"].copy_((path >= 0).sum(dim=1))
    torch.add(s["lengths"], s["accepted"], out=s["lengths_out"])
    t, i = (path > index[None, :]).nonzero().unbind(1)
    of, to = s["lengths"][t].long() + path[t, i], s["lengths"][t].long() + i
    for k, v, tables in zip(s["k"], s["v"], s["tables"]):
        of_page, to_page = (tables[t, x // page].long() for x in (of, to))
        for pool in (k, v):
            pool[to_page, :, to % page] = pool[of_page, :, of % page]


# ---- what a pass cannot do without, and what it gives in 64 bits -----------------------------------------------------

def work(case):
    kind = case["kind"]
    if kind == "sample":
        n = case["rows"] * case["vocab"]
        return {"bytes": 4 * n + 28 * case["rows"], "flops": 8 * n}
    hk, d = case["kv_heads"], case["dim"]
    size = 1 if case.get("cache") == "int8" else 2
    if kind == "normed":
        rows, h = case["rows"], case["heads"]
        positions = rows if case["seqs"] == 1 else 1
        weights = (h + hk if case["per_head"] else 2) * d * (2 if case["weight"] == "bf16" else 4)
        return {"bytes": rows * (8 * h * d + hk * 2 * (4 * d + size * d + (4 if size == 1 else 0))) + 4 * d * positions + weights,
                "flops": 7 * rows * (h + hk) * d}
    if kind == "tree":
        per = 2 * (size * d + (4 if size == 1 else 0))
        lengths, sizes = _lengths(case), _sizes(case)
        tokens = sum(lengths) + sum(sizes)
        pairs = sum(n * (c + (n + 1) // 2) for c, n in zip(lengths, sizes))
        return {"bytes": tokens * hk * per + 6 * case["trees"] * case["nodes"] * case["heads"] * d, "flops": 4 * pairs * case["heads"] * d}
    parents = _parents(case, 0)
    moved = sum(i != node for path, _ in _branches(case, 0, parents) for i, node in enumerate(path))
    return {"bytes": 16 * case["trees"] * case["nodes"] + moved * case["layers"] * hk * d * 2 * 2 * 2, "flops": 0}


def _branches(case, seed, parents):
    """The accepted nodes of each tree and the token behind them, from the parents."""
    drafted, drawn = _words(case, parents, seed)
    got = []
    for tree, words, draws, size in zip(parents, drafted, drawn, _sizes(case)):
        path, at = [], 0
        while at is not None:
            path.append(at)
            at = next((c for c in range(path[-1] + 1, size) if tree[c] == path[-1] and words[c] == draws[path[-1]]), None)
        got.append((path, draws[path[-1]]))
    return got


def exact(case, seed):
    s = _inputs(case, seed)
    return {"normed": _exact_normed, "tree": _exact_tree, "sample": _exact_sample, "accept": _exact_accept}[case["kind"]](case, s, seed)


def _levels(y):
    """What 8 bits hold of rows along the last axis."""
    scale = y.abs().amax(dim=-1, keepdim=True) / 127.0
    return torch.round(y / torch.where(scale > 0, scale, torch.ones_like(scale))) * scale


def _exact_normed(case, s, seed):
    d, page = case["dim"], case["page"]

    def turned(x, weight):
        x = x.double()
        x = x / torch.sqrt(x.square().sum(dim=-1, keepdim=True) / d + EPS) * weight.double()
        z = torch.complex(x[..., : d // 2].contiguous(), x[..., d // 2:].contiguous())
        at = s["positions"].long()
        z = z * torch.complex(s["cos"].double()[at], s["sin"].double()[at])[:, None, :]
        return torch.cat([z.real, z.imag], dim=-1)

    out = {"q": turned(s["q"], s["q_weight"])}
    where = s["tables"].long()[s["seqs"].long(), s["slots"].long() // page] * page + s["slots"].long() % page
    for name, new in (("k", turned(s["k_new"], s["k_weight"])), ("v", s["v_new"].double())):
        pool = s[name].double()
        if case["cache"] == "int8":
            pool, new = pool * s[name + "_scale"].double()[..., None], _levels(new)
        flat = pool.transpose(1, 2).reshape(-1, case["kv_heads"], d)
        flat[where] = new
        out[name] = flat.view(pool.shape[0], page, case["kv_heads"], d).transpose(1, 2).contiguous()
    return out


def _exact_tree(case, s, seed):
    hk, d, nodes, group = case["kv_heads"], case["dim"], case["nodes"], case["heads"] // case["kv_heads"]
    out = torch.zeros((case["trees"], nodes, case["heads"], d), dtype=torch.float64, device=DEV)
    q = s["q"].view(case["trees"], nodes, case["heads"], d)
    for t, (length, size, tree) in enumerate(zip(_lengths(case), _sizes(case), _parents(case, seed))):
        sees = torch.zeros((size, length + size), dtype=torch.bool)
        sees[:, :length] = True
        for i in range(size):
            a = i
            while a >= 0:
                sees[i, length + a] = True
                a = tree[a]
        sees = sees.to(DEV)[:, None, :].expand(size, group, -1).reshape(size * group, -1)
        at = s["tables"][t].long()
        for h in range(hk):
            k, v = (s[n][at, h].reshape(-1, d)[: length + size].double() for n in ("k", "v"))
            if case["cache"] == "int8":
                k, v = (x * s[n][at, h].reshape(-1, 1)[: length + size].double() for x, n in ((k, "k_scale"), (v, "v_scale")))
            of = q[t, :size, h * group:(h + 1) * group].reshape(size * group, d).double()
            logits = (of @ k.T.contiguous() / math.sqrt(d)).masked_fill(~sees, -math.inf)
            out[t, :size, h * group:(h + 1) * group] = (torch.softmax(logits, dim=-1) @ v).view(size, group, d)
    return {"out": out.view(s["out"].shape)}


def _exact_sample(case, s, seed):
    n, vocab = case["rows"], case["vocab"]
    tokens, probs = np.zeros(n, dtype=np.int32), np.zeros(n)
    logits, t, k, p, m, u = (s[x].cpu().numpy() for x in ("logits", "temperature", "top_k", "top_p", "min_p", "uniform"))
    for r in range(n):
        x = logits[r].astype(np.float64)
        by_rank = np.argsort(-x, kind="stable")
        if t[r] <= 0:
            tokens[r], probs[r] = by_rank[0], 1.0
            continue
        w = np.exp((x[by_rank] - x[by_rank[0]]) / float(t[r]))
        stay = vocab if k[r] <= 0 else min(vocab, int(k[r]))
        if p[r] < 1:
            stay = min(stay, 1 + int(np.searchsorted(np.cumsum(w), float(p[r]) * w.sum(), side="left")))
        stay = max(1, min(stay, int(np.searchsorted(-w, -float(m[r]), side="right"))))
        kept = np.sort(by_rank[:stay])
        w = np.exp((x[kept] - x[by_rank[0]]) / float(t[r]))
        upto = np.cumsum(w)
        at = min(int(np.searchsorted(upto, float(u[r]) * upto[-1], side="right")), stay - 1)
        tokens[r], probs[r] = kept[at], w[at] / upto[-1]
    return {"tokens": torch.from_numpy(tokens).to(DEV), "probs": torch.from_numpy(probs).to(DEV)}


def _exact_accept(case, s, seed):
    nodes, page = case["nodes"], case["page"]
    out = {"path": _ints([[-1] * nodes] * case["trees"]), "accepted": torch.zeros_like(s["accepted"]), "next": torch.zeros_like(s["next"])}
    out["k"], out["v"] = ([pool.double() for pool in s[name]] for name in ("k", "v"))
    for t, (path, token) in enumerate(_branches(case, seed, _parents(case, seed))):
        out["path"][t, : len(path)] = _ints(path)
        out["accepted"][t], out["next"][t] = len(path), token
        begin = _lengths(case)[t]
        for layer, tables in enumerate(s["tables"]):
            table = tables[t].tolist()
            for i, node in enumerate(path):
                of, to = begin + node, begin + i
                for name in ("k", "v"):
                    out[name][layer][table[to // page], :, to % page] = s[name][layer][table[of // page], :, of % page].double()
    out["lengths_out"] = s["lengths"] + out["accepted"]
    return {name: out[name] for name in ("path", "accepted", "next", "lengths_out", "k", "v")}
