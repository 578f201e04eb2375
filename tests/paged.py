"""Paged caches for the tests, and what the calls on them give, in 64 bits on the CPU."""
import math

import numpy as np
import torch

import paper_2509_22951_amd as tq


def ptr(t):
    return 0 if t is None else t.data_ptr()


def stream():
    return torch.cuda.current_stream().cuda_stream


class Paged:
    """A cache of random contents on the GPU.  order: how a pool lies in memory, "phtd" = [page][head][slot][dim]; every
    other order is a permuted view of such a buffer, with gaps."""

    def __init__(self, n_seqs, seq_pages, kv_heads=2, dim=64, page=16, kind="bf16", order="phtd", spare_pages=3, seed=0, marks=False, table_stride=0):
        g = torch.Generator().manual_seed(seed)
        self.n_pages, self.page, self.kv_heads, self.dim, self.kind = n_seqs * seq_pages + spare_pages, page, kv_heads, dim, kind
        self.n_seqs, self.seq_pages, self.capacity, self.marks = n_seqs, seq_pages, seq_pages * page, marks
        tables = torch.randperm(self.n_pages, generator=g)[: n_seqs * seq_pages].to(torch.int32).view(n_seqs, seq_pages)
        self.table_stride = table_stride or seq_pages
        wide = torch.full((n_seqs, self.table_stride), -1, dtype=torch.int32)
        wide[:, :seq_pages] = tables
        self.tables = wide.cuda()
        self.k, self.k_scale = self._pool(g, order)
        self.v, self.v_scale = self._pool(g, order)
        self.scores = self.positions = None
        if marks:
            self.scores = (torch.rand((n_seqs, kv_heads, self.capacity), generator=g) ** 4).cuda()
            self.positions = torch.arange(self.capacity, dtype=torch.int32).expand(n_seqs, kv_heads, -1).contiguous().cuda()
        self.strides = {} if order == "phtd" else {
            "page_stride": self.k.stride(0), "head_stride": self.k.stride(1), "slot_stride": self.k.stride(2)}

    def _pool(self, g, order):
        shape = {"p": self.n_pages, "h": self.kv_heads, "t": self.page, "d": self.dim}
        values = torch.randn([shape[a] for a in "phtd"], generator=g)
        scale = None
        if self.kind == "int8":
            scale = values.abs().amax(dim=-1) / 127
            values = torch.round(values / scale[..., None]).to(torch.int8)
            scale = scale.cuda()
        else:
            values = values.to(torch.bfloat16)
        if order == "phtd":
            return values.cuda(), scale
        sizes = [shape[a] for a in order]
        sizes[-1] += 16                              # gaps behind every head
        buf = torch.zeros(sizes, dtype=values.dtype).cuda()
        view = buf[..., : self.dim].permute([order.index(a) for a in "phtd"])
        view.copy_(values)
        return view, scale

    def describe(self, **more):
        fields = dict(k=ptr(self.k), v=ptr(self.v), k_scale=ptr(self.k_scale), v_scale=ptr(self.v_scale), tables=ptr(self.tables),
                      scores=ptr(self.scores), positions=ptr(self.positions), type=tq.TQ_INT8 if self.kind == "int8" else tq.TQ_BF16,
                      n_pages=self.n_pages, page_size=self.page, kv_heads=self.kv_heads, head_dim=self.dim, n_seqs=self.n_seqs,
                      seq_pages=self.seq_pages, table_stride=self.table_stride if self.table_stride != self.seq_pages else 0, **self.strides)
        fields.update(more)
        return tq.Cache(**fields)

    def values(self, name):
        """A pool's values in 64 bits, [page][head][slot][dim]."""
        x = getattr(self, name).cpu().double()
        scale = getattr(self, name + "_scale")
        return x if scale is None else x * scale.cpu().double()[..., None]

    def of_sequence(self, pool, s, h, length):
        """[length][dim] of values(...), and which of the tokens lie in a page that is there."""
        slots = torch.arange(length)
        pages = self.tables.cpu().long()[s, slots // self.page]
        there = (pages >= 0) & (pages < self.n_pages)
        return pool[pages.clamp(0, self.n_pages - 1), h, slots % self.page], there

    def set_slot(self, s, slot, value):
        """Puts a value (a NaN, an infinity) into a slot's keys and values; with 8 bits into its scales."""
        page, at = int(self.tables[s, slot // self.page]), slot % self.page
        for name in ("k", "v"):
            scale = getattr(self, name + "_scale")
            if scale is None:
                getattr(self, name)[page, :, at] = value
            else:
                scale[page, :, at] = value


def attend_call(cache, p, q, lengths, seqs=None, accumulate=False, scale=None, out=None, workspace=None, **more):
    rows, heads, dim = q.shape
    out = torch.full((rows, heads, dim), float("nan"), dtype=torch.bfloat16, device="cuda") if out is None else out
    fields = dict(q=ptr(q), out=ptr(out), seqs=ptr(seqs), lengths=ptr(lengths), rows=rows, heads=heads,
                  scale=1 / math.sqrt(dim) if scale is None else scale, q_type=tq.TQ_FP32 if q.dtype == torch.float32 else tq.TQ_BF16,
                  accumulate=int(accumulate), **more)
    n = tq.Attend.workspace_bytes(cache, **fields)
    ws = torch.zeros(n, dtype=torch.uint8, device="cuda") if workspace is None else workspace
    call = tq.Attend(cache, workspace=ptr(ws), workspace_bytes=ws.numel(), **fields)
    call.keep = (ws, out, q, lengths, seqs, p)
    return call, out


def attend_reference(p, q, lengths, seqs=None, scale=None):
    """-> (out, scores added) in 64 bits."""
    rows, heads, dim = q.shape
    q, group = q.cpu().double(), heads // p.kv_heads
    scale = 1 / math.sqrt(dim) if scale is None else scale
    out = torch.zeros((rows, heads, dim), dtype=torch.float64)
    added = torch.zeros((p.n_seqs, p.kv_heads, p.capacity), dtype=torch.float64)
    keys, vals = p.values("k"), p.values("v")
    for r in range(rows):
        s = r if seqs is None else int(seqs[r])
        length = min(max(int(lengths[r]), 0), p.capacity)
        if not 0 <= s < p.n_seqs or length == 0:
            continue
        for h in range(p.kv_heads):
            k, there = p.of_sequence(keys, s, h, length)
            v, _ = p.of_sequence(vals, s, h, length)
            if not there.any():
                continue
            slots = there.nonzero()[:, 0]
            w = torch.softmax(q[r, h * group:(h + 1) * group] @ k[there].T * scale, dim=-1)
            out[r, h * group:(h + 1) * group] = w @ v[there]
            added[s, h, slots] += w.sum(dim=0)
    return out, added


def evict_reference(p, lengths, keep, since=None):
    """-> per (sequence, head) {slot filled: slot it is filled from}, and the slots that stay where they are."""
    scores, positions, moves, stays = p.scores.cpu().numpy(), None if p.positions is None else p.positions.cpu().numpy(), {}, {}
    for s in range(p.n_seqs):
        n = min(max(int(lengths[s]), 0), p.capacity)
        for h in range(p.kv_heads):
            if n <= keep:
                moves[s, h], stays[s, h] = {}, list(range(n))
                continue
            rank = [(1, 0.0) if since is not None and positions[s, h, t] >= int(since[s]) else
                    (-1, 0.0) if np.isnan(scores[s, h, t]) else (0, float(scores[s, h, t])) for t in range(n)]
            kept = set(sorted(range(n), key=lambda t: (-rank[t][0], -rank[t][1], t))[:keep])
            free, late = [t for t in range(keep) if t not in kept], sorted(t for t in kept if t >= keep)
            moves[s, h], stays[s, h] = dict(zip(free, late)), sorted(t for t in kept if t < keep)
    return moves, stays
