"""Drafted trees, head norms, drawing and accepted branches together, as the decode example uses them, against a plain decoder in 64 bits on the
expanded weights.

Tolerance of the logits as of the decoder without trees: a layer rounds to bf16 six times on the way, the last norm once: with two layers 13 * 2^-8 = 0.05 of
the logits, taken as a 2-norm.  (An 8-bit cache rounds about as bf16 does; head norms are fp32.)  What is drawn and accepted is checked exactly, from the logits that
the decoder itself has."""
import os
import sys
import time
import types

import numpy as np
import pytest

torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import decode
from decode import Decoder, guesses, two_chains
from drafts import sample_reference
from test_gpu_decode import Plain

pytestmark = pytest.mark.gpu

SHAPE = dict(layers=2, hidden=256, heads=8, kv_heads=2, inter=512, vocab=700, batch=2, context=96)
TREE = [-1, 0, 0, 1, 1, 2, 5, 3]


class Branching(Plain):
    """The plain decoder of one sequence, whose state can be left and come back to."""

    def __init__(self, dec, heads, kv_heads):
        super().__init__(dec, heads, kv_heads)
        self.norms = [(lay["q_norm"].double().cpu(), lay["k_norm"].double().cpu()) if dec.head_norm else None for lay in dec.layers]

    def state(self):
        return self.position, [(list(lay["keys"]), list(lay["values"])) for lay in self.layers]

    def back_to(self, state):
        self.position = state[0]
        for lay, (keys, values) in zip(self.layers, state[1]):
            lay["keys"], lay["values"] = list(keys), list(values)

    def step(self, tokens):
        turned = iter(x for pair in self.norms for x in (pair or (None, None)))      # q and k of layer after layer are rotated in this order
        plain = self.rotate

        def rotate(x):
            w = next(turned)
            return plain(x if w is None else x / torch.sqrt(x.square().mean(dim=-1, keepdim=True) + 1e-6) * w)

        self.rotate = rotate
        try:
            return super().step(tokens)
        finally:
            self.rotate = plain


@pytest.mark.parametrize("cache,head_norm,filters", [("bf16", False, (0.0, 0, 1.0, 0.0)), ("int8", True, (0.9, 40, 0.95, 0.0)), ("bf16", True, (1.3, 0, 0.9, 0.02))])
def test_trees_against_64_bits(cache, head_norm, filters):
    dec = Decoder(**SHAPE, cache=cache, tree=TREE, head_norm=head_norm, filters=filters)
    plains = [Branching(dec, SHAPE["heads"], SHAPE["kv_heads"]) for _ in range(SHAPE["batch"])]
    g = torch.Generator().manual_seed(3)
    last, lengths, longest = [1, 2], [0, 0], 0
    for step in range(9):
        drafted = torch.randint(0, SHAPE["vocab"], (SHAPE["batch"], len(TREE)), generator=g)
        uniform = torch.rand((SHAPE["batch"], len(TREE)), generator=g)
        dec.uniform.copy_(uniform.view(-1))
        states, want = [], torch.zeros((SHAPE["batch"], len(TREE), SHAPE["vocab"]), dtype=torch.float64)
        for s, plain in enumerate(plains):
            drafted[s, 0] = last[s]
            before, of_nodes = plain.state(), []
            for i, parent in enumerate(TREE):
                if parent >= 0 and i % 3 != 2:       # two of three drafts are what the plain decoder would draw itself
                    drafted[s, i] = sample_reference(want[s, parent].float().numpy(), *filters[:1], filters[1], filters[2], filters[3], float(uniform[s, parent]))[0]
                plain.back_to(of_nodes[parent] if parent >= 0 else before)
                want[s, i] = plain.step(drafted[s, i:i + 1])[0]
                of_nodes.append(plain.state())
            states.append(of_nodes)
        got = dec.draft(drafted, graph=step >= 2)
        logits = dec.logits.view(want.shape).cpu()
        for s in range(SHAPE["batch"]):
            for i in range(len(TREE)):
                assert (logits[s, i].double() - want[s, i]).norm() <= 0.05 * want[s, i].norm(), (step, s, i)
            drawn = [sample_reference(logits[s, i].numpy(), *filters[:1], filters[1], filters[2], filters[3], float(uniform[s, i]))[0] for i in range(len(TREE))]
            assert dec.sampled.view(SHAPE["batch"], -1)[s].tolist() == drawn
            path = [0]
            while True:
                child = next((c for c, p in enumerate(TREE) if p == path[-1] and int(drafted[s, c]) == drawn[path[-1]]), None)
                if child is None:
                    break
                path.append(child)
            assert got[s] == ([int(drafted[s, i]) for i in path], drawn[path[-1]])
            plains[s].back_to(states[s][path[-1]])
            lengths[s] += len(path)
            longest = max(longest, len(path))
            last[s] = drawn[path[-1]]
        assert dec.lengths.tolist() == lengths
    assert longest >= 3      # a branch of some length was accepted, so that keys and values have moved


def test_replays_equal_eager_steps():
    eager, replayed = (Decoder(**SHAPE, tree=TREE, head_norm=True, filters=(0.8, 20, 0.9, 0.0)) for _ in range(2))
    g = torch.Generator().manual_seed(5)
    last = [3, 4]
    for step in range(9):
        drafted = torch.randint(0, 5, (SHAPE["batch"], len(TREE)), generator=g)
        drafted[:, 0] = torch.tensor(last)
        for dec in (eager, replayed):
            dec.uniform.copy_(torch.full((16,), 0.1 * step))
        a, b = eager.draft(drafted), replayed.draft(drafted, graph=True)
        assert a == b and torch.equal(eager.logits, replayed.logits)
        last = [after for _, after in a]


def test_a_context_that_a_tree_does_not_fit_is_refused_and_budgets_are():
    dec = Decoder(**{**SHAPE, "layers": 1, "context": 10}, tree=TREE)
    for _ in range(2):
        dec.draft(torch.zeros((2, 8), dtype=torch.int64))
    while int(dec.lengths.max()) <= 2:
        dec.draft(torch.zeros((2, 8), dtype=torch.int64))
    with pytest.raises(ValueError, match="10 tokens"):
        dec.draft(torch.zeros((2, 8), dtype=torch.int64))
    with pytest.raises(ValueError, match="draft"):
        dec.step(torch.zeros(16, dtype=torch.int64))
    with pytest.raises(ValueError, match="budget"):
        Decoder(**SHAPE, budget=20, tree=TREE)


def test_guesses_are_what_came_behind_earlier_occurrences():
    tree = two_chains(8)
    assert tree == [-1, 0, 1, 2, 3, 0, 5, 6]
    assert guesses([7, 1, 2, 3, 7, 4, 5, 6, 9, 7], tree) == [7, 4, 5, 6, 9, 1, 2, 3]
    assert guesses([1, 2, 3], tree) == [3] + [-1] * 7
    assert guesses([5, 5], tree) == [5, 5, -1, -1, -1, -1, -1, -1]


def test_the_clock_starts_behind_the_capture(monkeypatch, capsys):
    """The program's steps are replays, as it says of the ones that it times; what it draws begins at the beginning."""
    happened, launch = [], Decoder._launch

    def recorded(self, graph):
        happened.append(("step", self.graph is not None, int(self.lengths.max())))
        return launch(self, graph)

    monkeypatch.setattr(Decoder, "_launch", recorded)
    monkeypatch.setattr(decode, "time", types.SimpleNamespace(perf_counter=lambda: happened.append(("clock",)) or time.perf_counter()))
    monkeypatch.setattr(sys, "argv", "decode.py --layers 1 --hidden 128 --heads 4 --kv-heads 2 --inter 256 --vocab 500 --batch 2 --tokens 12 --draft 6".split())
    decode.main()
    began, ended = (i for i, what in enumerate(happened) if what[0] == "clock")
    timed = happened[began + 1:ended]
    assert began == 1 and len(timed) >= 1 and all(what[1] for what in timed) and timed[0][2] == 0
    assert f"{len(timed)} steps" in capsys.readouterr().out
