"""A decoder whose matrices stay compressed, one token per sequence and step: norm -> q, k, v -> rotary positions and cache ->
attention -> output projection -> norm -> gated feed-forward, layer after layer, the whole step captured in one HIP graph.

Weights are random (0.02 * N(0, 1)); --budget keeps every sequence's cache at that many tokens per head, by accumulated attention
weight, the newest quarter of them (one token at least) protected.  --temperature, --top-k, --top-p and --min-p say how tokens are drawn;
--head-norm norms queries and keys per head.  --draft runs a tree of that many tokens per sequence in every step, drafted from what the sequence
has held before, and keeps the branch that agrees with what is drawn (no more than 16 rows in all are one product).

  python examples/decode.py --layers 4 --hidden 2048 --heads 32 --kv-heads 8 --inter 8192 --batch 4 --tokens 64 --budget 48
  python examples/decode.py --layers 4 --hidden 2048 --heads 32 --kv-heads 8 --inter 8192 --batch 2 --tokens 64 --draft 8 --temperature 0.7 --top-p 0.9
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
    angles for `context` positions: one more step is refused.

    tree: the parents of a tree of drafted tokens (node 0 its root, parent -1, every other node behind its parent), or None.  With a tree a step is
    draft(tokens), tokens [batch][nodes].  filters: (temperature, top_k, top_p, min_p) of all rows; tokens are drawn into `sampled`."""

    def __init__(self, layers, hidden, heads, kv_heads, inter, vocab, batch, context, budget=0, cache="bf16", page=16, seed=0, base=500000.0, tree=None, head_norm=False,
                 filters=(0.0, 0, 1.0, 0.0)):
        if tree and budget:
            raise ValueError("a tree's tokens have no weights that a budget could go by")
        self.sequences, self.nodes = batch, len(tree) if tree else 1
        batch = batch * self.nodes      # rows of a step
        self.batch, self.heads, self.kv_heads, self.dim, self.budget = batch, heads, kv_heads, hidden // heads, budget
        self.context, self.steps = context, 0
        rng, dev = np.random.default_rng(seed), "cuda"
        seq_pages = -(-((budget + 1) if budget else context) // page)
        self.head_norm = head_norm
        n_pages, kv = self.sequences * seq_pages, kv_heads * self.dim

        def matrix(rows, cols):
            self.blob = tq.tq_encode((rng.standard_normal((rows, cols)) * 0.02).astype(np.float32), dict_from=self.blob)
            return tq.Matrix(self.blob)

        def gated(rows, cols):
            g, u = ((rng.standard_normal((rows, cols)) * 0.02).astype(np.float32) for _ in range(2))
            self.blob = tq.tq_encode_gate_up(g, u, dict_from=self.blob)
            return tq.Matrix(self.blob)

        def norm_weight(n=hidden):
            return torch.from_numpy((1.0 + 0.1 * rng.standard_normal(n)).astype(np.float32)).to(dev).to(torch.bfloat16)

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
        if tree:
            bits, depth = [], []
            for i, parent in enumerate(tree):
                bits.append((bits[parent] if i else 0) | 1 << i)
                depth.append(depth[parent] + 1 if i else 0)
            of_nodes = torch.tensor([b - (1 << 64) if b >> 63 else b for b in bits], dtype=torch.int64, device=dev)
            self.masks, self.depth = of_nodes.repeat(self.sequences, 1), torch.tensor(depth, dtype=torch.int32, device=dev)
            self.seqs = (torch.arange(batch, device=dev) // self.nodes).to(torch.int32)
            self.lengths, self.lengths_out, self.accepted, self.next = (buffer(self.sequences, dtype=torch.int32) for _ in range(4))
            self.drafted, self.path = (buffer(self.sequences, self.nodes, dtype=torch.int32) for _ in range(2))
        self.tree = tree
        freq = base ** (-torch.arange(0, self.dim, 2, dtype=torch.float64) / self.dim)
        angle = torch.arange(context, dtype=torch.float64)[:, None] * freq[None, :]
        self.cos, self.sin = torch.cos(angle).float().to(dev), torch.sin(angle).float().to(dev)

        self.layers = []
        for n in range(layers):
            lay = {"q": matrix(hidden, hidden), "k": matrix(kv, hidden), "v": matrix(kv, hidden), "o": matrix(hidden, hidden),
                   "gate_up": gated(inter, hidden), "down": matrix(hidden, inter), "w1": norm_weight(), "w2": norm_weight()}
            if head_norm:
                lay["q_norm"], lay["k_norm"] = norm_weight(self.dim), norm_weight(self.dim)
            pool = (n_pages, kv_heads, page, self.dim)
            lay["keys"], lay["values"] = (buffer(*pool, dtype=torch.int8 if cache == "int8" else torch.bfloat16) for _ in range(2))
            lay["scales"] = [buffer(*pool[:3]) for _ in range(2)] if cache == "int8" else [None, None]
            order = torch.from_numpy(rng.permutation(n_pages).astype(np.int32)).to(dev).view(self.sequences, seq_pages)
            lay["tables"] = order
            marks = (batch, kv_heads, seq_pages * page)
            lay["scores"] = buffer(*marks) if budget else None
            lay["token"] = buffer(*marks, dtype=torch.int32) if budget else None
            lay["cache"] = tq.Cache(k=_ptr(lay["keys"]), v=_ptr(lay["values"]), k_scale=_ptr(lay["scales"][0]), v_scale=_ptr(lay["scales"][1]), tables=_ptr(order),
                                    scores=_ptr(lay["scores"]), positions=_ptr(lay["token"]), type=tq.TQ_INT8 if cache == "int8" else tq.TQ_BF16,
                                    n_pages=n_pages, page_size=page, kv_heads=kv_heads, head_dim=self.dim, n_seqs=self.sequences, seq_pages=seq_pages)
            self._prepare(lay, first=n == 0)
            self.layers.append(lay)
        self.norm_out, self.w_out = None, norm_weight()
        self.norm_out = self._norm(self.w_out, delta=True)
        self.head = matrix(vocab, hidden)
        self.to_logits = tq.Step([self.head.handle], [_ptr(self.x)], [_ptr(self.logits)], batch)
        self.graph = None

        temperature, top_k, top_p, min_p = filters
        self.filters = [torch.full((batch,), x, dtype=d, device=dev) for x, d in ((temperature, torch.float32), (top_k, torch.int32), (top_p, torch.float32), (min_p, torch.float32))]
        self.uniform, self.sampled = buffer(batch), buffer(batch, dtype=torch.int32)
        fields = dict(logits=_ptr(self.logits), temperature=_ptr(self.filters[0]), top_k=_ptr(self.filters[1]), top_p=_ptr(self.filters[2]), min_p=_ptr(self.filters[3]),
                      uniform=_ptr(self.uniform), tokens=_ptr(self.sampled), rows=batch, vocab=vocab)
        self.sample_space = torch.empty(tq.Sample.workspace_bytes(**fields), dtype=torch.uint8, device=dev)
        self.sample = tq.Sample(workspace=_ptr(self.sample_space), workspace_bytes=self.sample_space.numel(), **fields)
        if tree:
            self.accept = tq.TreeAccept([lay["cache"] for lay in self.layers], masks=_ptr(self.masks), lengths=_ptr(self.lengths), drafted=_ptr(self.drafted),
                                        sampled=_ptr(self.sampled), path=_ptr(self.path), accepted=_ptr(self.accepted), next=_ptr(self.next),
                                        lengths_out=_ptr(self.lengths_out), trees=self.sequences, nodes=self.nodes)

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
        fields = dict(q=_ptr(self.q), k=_ptr(self.k), v=_ptr(self.v), q_out=_ptr(self.q), seqs=_ptr(self.seqs) if self.tree else 0, slots=_ptr(self.slots),
                      positions=_ptr(self.positions), cos=_ptr(self.cos), sin=_ptr(self.sin), rows=batch, heads=self.heads, rotary_dim=self.dim,
                      n_positions=self.cos.shape[0], q_out_type=tq.TQ_FP32)
        if self.head_norm:
            norm = tq.HeadNorm(q_weight=_ptr(lay["q_norm"]), k_weight=_ptr(lay["k_norm"]), eps=1e-6, weight_type=tq.TQ_BF16)
            lay["append"] = tq.CacheAppendNormed(lay["cache"], norm, **fields)
        else:
            lay["append"] = tq.CacheAppend(lay["cache"], **fields)
        if self.tree:
            fields = dict(q=_ptr(self.q), out=_ptr(self.attended), lengths=_ptr(self.lengths), masks=_ptr(self.masks), trees=self.sequences, nodes=self.nodes,
                          heads=self.heads, scale=1.0 / math.sqrt(self.dim), q_type=tq.TQ_FP32)
            lay["attend_space"] = torch.empty(tq.AttendTree.workspace_bytes(lay["cache"], **fields), dtype=torch.uint8, device="cuda")
            lay["attend"] = tq.AttendTree(lay["cache"], workspace=_ptr(lay["attend_space"]), workspace_bytes=lay["attend_space"].numel(), **fields)
            return
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
        if self.tree:
            node = torch.arange(self.nodes, dtype=torch.int32, device="cuda")
            torch.add(self.lengths[:, None], node[None, :], out=self.slots.view(self.sequences, self.nodes))
            torch.add(self.lengths[:, None], self.depth[None, :], out=self.positions.view(self.sequences, self.nodes))
        else:
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
        self.sample.launch(s)
        if self.tree:
            self.accept.launch(s)
            self.lengths.copy_(self.lengths_out)
            return
        # the next token's place
        self.slots.copy_(self.left if self.budget else self.lengths)
        self.positions.add_(1)
        # of the tokens that there are with the next one, the newest quarter is protected
        torch.sub(self.positions, max(1, self.budget // 4) - 1, out=self.since)

    def step(self, tokens, graph=False):
        """One token per sequence in, logits [batch][vocab] out (the decoder's own buffer)."""
        if self.steps == self.context:
            raise ValueError(f"this decoder has room for {self.context} tokens per sequence, and has had them")
        if self.tree:
            raise ValueError("a decoder with a tree takes draft(tokens)")
        self.steps += 1
        self.tokens.copy_(tokens)
        self._launch(graph)
        return self.logits

    def draft(self, tokens, graph=False):
        """A tree of drafted tokens per sequence in, node 0 the token drawn last: [batch][nodes] -> for every sequence the accepted tokens, and the one drawn behind them."""
        longest = int(self.lengths.max())
        if longest + self.nodes > self.context:
            raise ValueError(f"this decoder has room for {self.context} tokens per sequence, has {longest}, and a tree takes {self.nodes}")
        self.drafted.copy_(tokens)
        self.tokens.copy_(self.drafted.view(-1))
        self._launch(graph)
        return [([row[i] for i in path if i >= 0], after) for row, path, after in zip(self.drafted.tolist(), self.path.tolist(), self.next.tolist())]

    def _launch(self, graph):
        if not graph:
            return self._run()
        if self.graph is None:
            graph = torch.cuda.CUDAGraph()
            torch.cuda.synchronize()
            with torch.cuda.graph(graph, stream=torch.cuda.Stream()):   # (recorded, not run)
                self._run()
            self.graph = graph
        self.graph.replay()


def two_chains(nodes):
    """A tree of a root and two chains, the first the longer one."""
    first = nodes // 2
    return [-1] + [i - 1 for i in range(1, first + 1)] + [0 if i == first + 1 else i - 1 for i in range(first + 1, nodes)]


def guesses(history, tree):
    """Tokens for a tree behind the last one: what came behind earlier occurrences of it, the latest ones first; -1, which nothing drawn is, where there are none."""
    at = [i for i in range(len(history) - 2, -1, -1) if history[i] == history[-1]]
    chains = [i for i, parent in enumerate(tree) if parent == 0]
    tokens, begin = [history[-1]] + [-1] * (len(tree) - 1), {}
    for chain, place in zip(chains, at):
        begin[chain] = place + 1
    for i, parent in enumerate(tree):
        place = begin.get(i, begin[parent] + 1 if parent in begin else len(history))
        if i and place < len(history):
            begin[i], tokens[i] = place, history[place]
    return tokens


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("layers", 4), ("hidden", 2048), ("heads", 32), ("kv-heads", 8), ("inter", 8192), ("vocab", 32000), ("batch", 4), ("tokens", 64), ("budget", 0), ("draft", 0), ("top-k", 0)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--cache", choices=("bf16", "int8"), default="bf16")
    for name, value in (("temperature", 0.0), ("top-p", 1.0), ("min-p", 0.0)):
        ap.add_argument("--" + name, type=float, default=value)
    ap.add_argument("--head-norm", action="store_true")
    a = ap.parse_args()
    tree = two_chains(a.draft) if a.draft else None
    dec = Decoder(a.layers, a.hidden, a.heads, a.kv_heads, a.inter, a.vocab, a.batch, context=a.tokens + 8 + 2 * a.draft, budget=a.budget, cache=a.cache, tree=tree, head_norm=a.head_norm,
                  filters=(a.temperature, a.top_k, a.top_p, a.min_p))
    numbers = torch.Generator(device="cuda").manual_seed(0)
    if tree:
        texts, steps = [[i] for i in range(a.batch)], 0
        dec.draft(torch.zeros((a.batch, a.draft), dtype=torch.int32), graph=True)      # captured, and forgotten
        dec.lengths.zero_()
        torch.cuda.synchronize()
        began = time.perf_counter()
        while min(len(t) for t in texts) <= a.tokens and int(dec.lengths.max()) + a.draft <= dec.context:
            dec.uniform.uniform_(generator=numbers)
            tokens = torch.tensor([[max(t, 0) for t in guesses(text, tree)] for text in texts], dtype=torch.int32)
            for text, (kept, after) in zip(texts, dec.draft(tokens, graph=True)):
                text.extend(kept[1:] + [after])
            steps += 1
        seconds, made = time.perf_counter() - began, sum(len(t) - 1 for t in texts)
        print(f"{a.layers} layers, batch {a.batch}, trees of {a.draft}: {steps} steps, {1e3 * seconds / steps:.3f} ms each, {made / steps / a.batch:.2f} tokens a step and sequence, "
              f"{made / seconds:.0f} tokens/s; last tokens {[t[-1] for t in texts]}")
        return
    token = torch.arange(a.batch, device="cuda")
    for _ in range(4):
        dec.step(token, graph=True)
        token.copy_(dec.sampled)
    torch.cuda.synchronize()
    began = time.perf_counter()
    for _ in range(a.tokens):
        dec.uniform.uniform_(generator=numbers)
        dec.step(token, graph=True)
        token.copy_(dec.sampled)
    torch.cuda.synchronize()
    seconds = time.perf_counter() - began
    print(f"{a.layers} layers, batch {a.batch}: {a.tokens} steps, {1e3 * seconds / a.tokens:.3f} ms each, {a.batch * a.tokens / seconds:.0f} tokens/s; "
          f"cache holds {int(dec.slots.max())} tokens per sequence; last tokens {token.tolist()}")


if __name__ == "__main__":
    main()
