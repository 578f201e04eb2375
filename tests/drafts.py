"""Trees of drafted tokens and drawing, for the tests: what the calls give, in 64 bits on the CPU."""
import math
import random

import numpy as np
import torch

import paper_2509_22951_amd as tq
from paged import ptr


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def signed(bits):
    return bits - (1 << 64) if bits >> 63 else bits


def random_parents(trees, nodes, seed=0):
    rng = random.Random(seed)
    return [[-1] + [rng.randint(max(0, i // 2 - 1), i - 1) for i in range(1, nodes)] for _ in range(trees)]


def bits_of(parents):
    got = []
    for tree in parents:
        bits = []
        for i, p in enumerate(tree):
            bits.append((bits[p] if p >= 0 else 0) | 1 << i)
        got.append(bits)
    return got


def masks_of(bits):
    return torch.tensor([[signed(b) for b in tree] for tree in bits], dtype=torch.int64, device="cuda")


def tree_call(cache, q, lengths, masks, sizes=None, seqs=None, scale=None, out=None, workspace=None, **more):
    """q: [trees][nodes][heads][dim]."""
    trees, nodes, heads, dim = q.shape
    out = torch.full((trees, nodes, heads, dim), float("nan"), dtype=torch.bfloat16, device="cuda") if out is None else out
    fields = dict(q=ptr(q), out=ptr(out), lengths=ptr(lengths), sizes=ptr(sizes), seqs=ptr(seqs), masks=ptr(masks), trees=trees, nodes=nodes, heads=heads,
                  scale=1 / math.sqrt(dim) if scale is None else scale, q_type=tq.TQ_FP32 if q.dtype == torch.float32 else tq.TQ_BF16, **more)
    n = tq.AttendTree.workspace_bytes(cache, **fields)
    ws = torch.full((n,), 0xEE, dtype=torch.uint8, device="cuda") if workspace is None else workspace
    call = tq.AttendTree(cache, workspace=ptr(ws), workspace_bytes=ws.numel(), **fields)
    call.keep = (ws, out, q, lengths, masks, sizes, seqs)
    return call, out


def tree_reference(p, q, lengths, bits, sizes=None, seqs=None, scale=None):
    trees, nodes, heads, dim = q.shape
    q, group = q.cpu().double(), heads // p.kv_heads
    scale = 1 / math.sqrt(dim) if scale is None else scale
    out = torch.zeros((trees, nodes, heads, dim), dtype=torch.float64)
    keys, vals = p.values("k"), p.values("v")
    for t in range(trees):
        s = t if seqs is None else int(seqs[t])
        if not 0 <= s < p.n_seqs:
            continue
        length = max(int(lengths[t]), 0)
        size = nodes if sizes is None else min(max(int(sizes[t]), 0), nodes)
        end = min(length + size, p.capacity)
        sees = torch.zeros((nodes, end), dtype=torch.bool)
        for i in range(size):
            sees[i, : min(length, end)] = True
            for j in range(size):
                if length + j < end and bits[t][i] >> j & 1:
                    sees[i, length + j] = True
        for h in range(p.kv_heads if end else 0):
            k, there = p.of_sequence(keys, s, h, end)
            v, _ = p.of_sequence(vals, s, h, end)
            for i in range(size):
                at = sees[i] & there
                if at.any():
                    w = torch.softmax(q[t, i, h * group:(h + 1) * group] @ k[at].T * scale, dim=-1)
                    out[t, i, h * group:(h + 1) * group] = w @ v[at]
    return out


def accept_reference(bits, sizes, drafted, sampled, nodes):
    """-> per tree (accepted nodes, the token behind them)."""
    got = []
    for tree, size, words, drawn in zip(bits, sizes, drafted, sampled):
        path = [0] if size > 0 else []
        while path:
            p = path[-1]
            child = next((c for c in range(p + 1, min(size, nodes)) if tree[c] == tree[p] | 1 << c and words[c] == drawn[p]), None)
            if child is None:
                break
            path.append(child)
        got.append((path, drawn[path[-1]] if path else -1))
    return got


def sample_reference(logits, temperature, top_k, top_p, min_p, uniform):
    """One row, fp32 values and Python numbers -> (token, probability, kept tokens)."""
    x = np.asarray(logits, dtype=np.float32).astype(np.float64)
    x[np.isnan(x)] = -np.inf
    order = np.argsort(-x, kind="stable")
    top = x[order[0]]
    if top == -np.inf:
        return -1, 0.0, []
    if not temperature > 0:
        return int(order[0]), 1.0, [int(order[0])]
    with np.errstate(over="ignore", invalid="ignore"):
        w = np.where(x == np.inf, 1.0, 0.0) if top == np.inf else np.where(x == -np.inf, 0.0, np.exp((x - top) / np.float64(np.float32(temperature))))
    ranked = w[order]
    stay = len(x) if top_k <= 0 else min(top_k, len(x))
    if top_p < 1:
        before = np.concatenate([[0.0], np.cumsum(ranked)[:-1]])
        stay = min(stay, int((before < np.float64(np.float32(top_p)) * ranked.sum()).sum()))
    if min_p > 0:
        stay = min(stay, int((ranked >= np.float64(np.float32(min_p))).sum()))
    kept = np.sort(order[: max(stay, 1)])
    kept = kept[w[kept] > 0]
    upto = np.cumsum(w[kept])
    beyond = np.nonzero(upto > np.float64(np.float32(uniform)) * upto[-1])[0]
    at = int(beyond[0]) if len(beyond) else len(kept) - 1
    return int(kept[at]), float(w[kept[at]] / upto[-1]), kept.tolist()
