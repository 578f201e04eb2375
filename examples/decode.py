"""A decoder whose matrices stay compressed, one token per sequence and step: norm -> q, k, v -> rotary positions and cache ->
attention -> output projection -> norm -> gated feed-forward, layer after layer, the whole step captured in one HIP graph.

Weights are random (0.02 * N(0, 1)); --budget keeps every sequence's cache at that many tokens per head, by accumulated attention
weight, the newest quarter of them (one token at least) protected.

  python examples/decode.py --layers 4 --hidden 2048 --heads 32 --kv-heads 8 --inter 8192 --batch 4 --tokens 64 --budget 48
"""
import argparse
import math
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2509_22951_amd as tq


def _ptr(t):
    return 0 if t is None else t.data_ptr()


class Decoder:
    """Fixed buffers and prepared calls of a decoder; step(tokens) -> logits.

    budget 0: the cache grows up to `context` tokens; else it is cut back to `budget` tokens after every step.  Either way there are
    angles for `context` positions: one more step is refused."""

    def __init__(self, layers, hidden, heads, kv_heads, inter, vocab, batch, context, budget=0, cache="bf16", page=16, seed=0, base=500000.0):
        self.batch, self.heads, self.kv_heads, self.dim, self.budget = batch, heads, kv_heads, hidden // heads, budget
        self.context, self.steps = context, 0
        rng, dev = np.random.default_rng(seed), "cuda"
        seq_pages = -(-((budget + 1) if budget else context) // page)
        n_pages, kv = batch * seq_pages, kv_heads * self.dim

        def matrix(rows, cols):
            self.blob = tq.tq_encode((rng.standard_normal((rows, cols)) * 0.02).astype(np.float32), dict_from=self.blob)
            return tq.Matrix(self.blob)

        def gated(rows, cols):
            g, u = ((rng.standard_normal((rows, cols)) * 0.02).astype(np.float32) for _ in range(2))
            self.blob = tq.tq_encode_gate_up(g, u, dict_from=self.blob)
            return tq.Matrix(self.blob)

        def norm_weight():
            return torch.from_numpy((1.0 + 0.1 * rng.standard_normal(hidden)).astype(np.float32)).to(dev).to(torch.bfloat16)

        def buffer(*shape, dtype=torch.float32):
            return torch.zeros(shape, dtype=dtype, device=dev)

        self.blob = None
        self.embedding = torch.from_numpy(rng.standard_normal((vocab, hidden)).astype(np.float32)).to(dev).to(torch.bfloat16)
        self.h, self.delta = buffer(batch, hidden), buffer(batch, hidden)
        self.x, self.attended = buffer(batch, hidden, dtype=torch.bfloat16), buffer(batch, hidden, dtype=torch.bfloat16)
        self.q, self.k, self.v = buffer(batch, hidden), buffer(batch, kv), buffer(batch, kv)
        self.gate, self.gate16 = buffer(batch, inter), buffer(batch, inter, dtype=torch.bfloat16)
        self.logits = buffer(batch, vocab)
        self.tokens = buffer(batch, dtype=torch.int64)
        # a token's slot, the tokens there are with it, its position, the positions from which on tokens are protected, what is left after eviction
        self.slots, self.lengths, self.positions, self.since, self.left = (buffer(batch, dtype=torch.int32) for _ in range(5))
        freq = base ** (-torch.arange(0, self.dim, 2, dtype=torch.float64) / self.dim)
        angle = torch.arange(context, dtype=torch.float64)[:, None] * freq[None, :]
        self.cos, self.sin = torch.cos(angle).float().to(dev), torch.sin(angle).float().to(dev)

        self.layers = []
        for n in range(layers):
            lay = {"q": matrix(hidden, hidden), "k": matrix(kv, hidden), "v": matrix(kv, hidden), "o": matrix(hidden, hidden),
                   "gate_up": gated(inter, hidden), "down": matrix(hidden, inter), "w1": norm_weight(), "w2": norm_weight()}
            pool = (n_pages, kv_heads, page, self.dim)
            lay["keys"], lay["values"] = (buffer(*pool, dtype=torch.int8 if cache == "int8" else torch.bfloat16) for _ in range(2))
            lay["scales"] = [buffer(*pool[:3]) for _ in range(2)] if cache == "int8" else [None, None]
            order = torch.from_numpy(rng.permutation(n_pages).astype(np.int32)).to(dev).view(batch, seq_pages)
            lay["tables"] = order
            marks = (batch, kv_heads, seq_pages * page)
            lay["scores"] = buffer(*marks) if budget else None
            lay["token"] = buffer(*marks, dtype=torch.int32) if budget else None
            lay["cache"] = tq.Cache(k=_ptr(lay["keys"]), v=_ptr(lay["values"]), k_scale=_ptr(lay["scales"][0]), v_scale=_ptr(lay["scales"][1]), tables=_ptr(order),
                                    scores=_ptr(lay["scores"]), positions=_ptr(lay["token"]), type=tq.TQ_INT8 if cache == "int8" else tq.TQ_BF16,
                                    n_pages=n_pages, page_size=page, kv_heads=kv_heads, head_dim=self.dim, n_seqs=batch, seq_pages=seq_pages)
            self._prepare(lay, first=n == 0)
            self.layers.append(lay)
        self.norm_out, self.w_out = None, norm_weight()
        self.norm_out = self._norm(self.w_out, delta=True)
        self.head = matrix(vocab, hidden)
        self.to_logits = tq.Step([self.head.handle], [_ptr(self.x)], [_ptr(self.logits)], batch)
        self.graph = None

    def _norm(self, weight, delta):
        return tq.AddNorm(residual=_ptr(self.h), delta=_ptr(self.delta) if delta else 0, weight=_ptr(weight), residual_out=_ptr(self.h) if delta else 0,
                          out=_ptr(self.x), rows=self.batch, cols=self.h.shape[1], eps=1e-5, residual_type=tq.TQ_FP32, weight_type=tq.TQ_BF16, out_type=tq.TQ_BF16)

    def _prepare(self, lay, first):
        x, batch = _ptr(self.x), self.batch
        lay["norm1"], lay["norm2"] = self._norm(lay["w1"], delta=not first), self._norm(lay["w2"], delta=True)
        lay["to_qkv"] = tq.Step([lay[n].handle for n in "qkv"], [x] * 3, [_ptr(self.q), _ptr(self.k), _ptr(self.v)], batch)
        lay["to_o"] = tq.Step([lay["o"].handle], [_ptr(self.attended)], [_ptr(self.delta)], batch)
        lay["to_gate"] = tq.Step([lay["gate_up"].handle], [x], [_ptr(self.gate)], batch, gate_up=True)
        lay["to_down"] = tq.Step([lay["down"].handle], [_ptr(self.gate16)], [_ptr(self.delta)], batch)
        lay["append"] = tq.CacheAppend(lay["cache"], q=_ptr(self.q), k=_ptr(self.k), v=_ptr(self.v), q_out=_ptr(self.q), slots=_ptr(self.slots),
                                       positions=_ptr(self.positions), cos=_ptr(self.cos), sin=_ptr(self.sin), rows=batch, heads=self.heads,
                                       rotary_dim=self.dim, n_positions=self.cos.shape[0], q_out_type=tq.TQ_FP32)
        fields = dict(q=_ptr(self.q), out=_ptr(self.attended), lengths=_ptr(self.lengths), rows=batch, heads=self.heads, scale=1.0 / math.sqrt(self.dim),
                      q_type=tq.TQ_FP32, accumulate=int(self.budget > 0))
        lay["attend_space"] = torch.zeros(tq.Attend.workspace_bytes(lay["cache"], **fields), dtype=torch.uint8, device="cuda")
        lay["attend"] = tq.Attend(lay["cache"], workspace=_ptr(lay["attend_space"]), workspace_bytes=lay["attend_space"].numel(), **fields)
        if self.budget:
            fields = dict(lengths=_ptr(self.lengths), lengths_out=_ptr(self.left), since=_ptr(self.since), keep=self.budget)
            lay["evict_space"] = torch.empty(tq.CacheEvict.workspace_bytes(lay["cache"], **fields), dtype=torch.uint8, device="cuda")
            lay["evict"] = tq.CacheEvict(lay["cache"], workspace=_ptr(lay["evict_space"]), workspace_bytes=lay["evict_space"].numel(), **fields)

    def _run(self):
        s = torch.cuda.current_stream().cuda_stream
        torch.add(self.slots, 1, out=self.lengths)
        self.h.copy_(self.embedding[self.tokens])
        for lay in self.layers:
            lay["norm1"].launch(s)
            lay["to_qkv"].launch(s)
            lay["append"].launch(s)
            lay["attend"].launch(s)
            lay["to_o"].launch(s)
            lay["norm2"].launch(s)
            lay["to_gate"].launch(s)
            self.gate16.copy_(self.gate)
            lay["to_down"].launch(s)
            if self.budget:
                lay["evict"].launch(s)
        self.norm_out.launch(s)
        self.to_logits.launch(s)
        # the next token's place
        self.slots.copy_(self.left if self.budget else self.lengths)
        self.positions.add_(1)
        # of the tokens that there are with the next one, the newest quarter is protected
        torch.sub(self.positions, max(1, self.budget // 4) - 1, out=self.since)

    def step(self, tokens, graph=False):
        """One token per sequence in, logits [batch][vocab] out (the decoder's own buffer)."""
        if self.steps == self.context:
            raise ValueError(f"this decoder has room for {self.context} tokens per sequence, and has had them")
        self.steps += 1
        self.tokens.copy_(tokens)
        if not graph:
            self._run()
            return self.logits
        if self.graph is None:
            graph = torch.cuda.CUDAGraph()
            torch.cuda.synchronize()
            with torch.cuda.graph(graph, stream=torch.cuda.Stream()):   # (recorded, not run)
                self._run()
            self.graph = graph
        self.graph.replay()
        return self.logits


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("layers", 4), ("hidden", 2048), ("heads", 32), ("kv-heads", 8), ("inter", 8192), ("vocab", 32000), ("batch", 4), ("tokens", 64), ("budget", 0)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--cache", choices=("bf16", "int8"), default="bf16")
    a = ap.parse_args()
    dec = Decoder(a.layers, a.hidden, a.heads, a.kv_heads, a.inter, a.vocab, a.batch, context=a.tokens + 8, budget=a.budget, cache=a.cache)
    token = torch.arange(a.batch, device="cuda")
    for _ in range(4):
        token = dec.step(token, graph=True).argmax(dim=1)
    torch.cuda.synchronize()
    began = time.perf_counter()
    for _ in range(a.tokens):
        token = dec.step(token, graph=True).argmax(dim=1)
    torch.cuda.synchronize()
    seconds = time.perf_counter() - began
    print(f"{a.layers} layers, batch {a.batch}: {a.tokens} steps, {1e3 * seconds / a.tokens:.3f} ms each, {a.batch * a.tokens / seconds:.0f} tokens/s; "
          f"cache holds {int(dec.slots.max())} tokens per sequence; last tokens {token.tolist()}")


if __name__ == "__main__":
    main()
