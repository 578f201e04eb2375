"""The operators together, as the decode example uses them, against a plain decoder in 64 bits on the expanded weights.

Tolerance of the logits: a layer rounds to bf16 six times on the way (two norms' x, attention's result, the gated product, a key and
a value; 2^-8 at most each), the last norm once: with two layers 13 * 2^-8 = 0.05 of the logits, taken as a 2-norm."""
import os
import sys

import pytest

torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
from decode import Decoder

pytestmark = pytest.mark.gpu

SHAPE = dict(layers=2, hidden=256, heads=8, kv_heads=2, inter=512, vocab=700, batch=3, context=64)


def expanded(m, stream):
    out = torch.empty((m.info["rows"], m.info["cols"]), dtype=torch.int8, device="cuda")
    m.decompress(out.data_ptr(), stream)
    # the scales by a product with unit rows: y = scale * Q x
    x = torch.zeros((1, m.info["cols"]), dtype=torch.bfloat16, device="cuda")
    q, scale = out.double().cpu(), torch.zeros(m.info["rows"], dtype=torch.float64)
    y = torch.zeros((1, m.info["rows"]), device="cuda")
    top = q.abs().argmax(dim=1)
    for col in top.unique():
        x.zero_()
        x[0, col] = 1
        m.matvec(x.data_ptr(), y.data_ptr(), 1, stream)
        rows = top == col
        scale[rows] = (y[0].double().cpu() / q[:, col].where(q[:, col] != 0, torch.ones(())))[rows]
    return q * scale[:, None]


class Plain:
    def __init__(self, dec, heads, kv_heads):
        stream = torch.cuda.current_stream().cuda_stream
        self.heads, self.kv_heads, self.dim = heads, kv_heads, dec.dim
        self.embedding, self.w_out, self.head = dec.embedding.double().cpu(), dec.w_out.double().cpu(), expanded(dec.head, stream)
        self.layers = [{**{n: expanded(lay[n], stream) for n in ("q", "k", "v", "o", "gate_up", "down")}, "w1": lay["w1"].double().cpu(),
                        "w2": lay["w2"].double().cpu(), "keys": [], "values": []} for lay in dec.layers]
        self.cos, self.sin, self.position = dec.cos.double().cpu(), dec.sin.double().cpu(), 0

    def norm(self, h, w):
        return h / torch.sqrt(h.square().mean(dim=1, keepdim=True) + 1e-5) * w

    def rotate(self, x):
        a, b = x.chunk(2, dim=-1)
        c, s = self.cos[self.position], self.sin[self.position]
        return torch.cat([a * c - b * s, a * s + b * c], dim=-1)

    def step(self, tokens):
        h = self.embedding[tokens]
        rows = h.shape[0]
        for lay in self.layers:
            x = self.norm(h, lay["w1"])
            q = self.rotate((x @ lay["q"].T).view(rows, self.heads, self.dim))
            lay["keys"].append(self.rotate((x @ lay["k"].T).view(rows, self.kv_heads, self.dim)))
            lay["values"].append((x @ lay["v"].T).view(rows, self.kv_heads, self.dim))
            k, v = (torch.stack(lay[n], dim=2) for n in ("keys", "values"))        # [row][head][token][dim]
            q = q.view(rows, self.kv_heads, -1, self.dim)
            p = torch.softmax(q @ k.transpose(-1, -2) / self.dim ** 0.5, dim=-1)
            h = h + (p @ v).reshape(rows, -1) @ lay["o"].T
            x = self.norm(h, lay["w2"])
            y = x @ lay["gate_up"].T
            g, u = y[:, 0::2], y[:, 1::2]
            h = h + (g / (1 + torch.exp(-g)) * u) @ lay["down"].T
        self.position += 1
        return self.norm(h, self.w_out) @ self.head.T


@pytest.mark.parametrize("cache", ["bf16", "int8"])
@pytest.mark.parametrize("budget", [0, 40])
def test_decoder_against_64_bits(cache, budget):
    """budget 40 evicts nothing in 30 steps, but runs everything that eviction needs.  (An 8-bit cache rounds keys and values to 1 / 254 of
    their largest value, about as bf16 does.)"""
    dec = Decoder(**SHAPE, cache=cache, budget=budget)
    plain = Plain(dec, SHAPE["heads"], SHAPE["kv_heads"])
    g = torch.Generator().manual_seed(1)
    for i in range(30):
        tokens = torch.randint(0, SHAPE["vocab"], (SHAPE["batch"],), generator=g)
        got = dec.step(tokens.cuda(), graph=i >= 5).double().cpu()
        want = plain.step(tokens)
        assert (got - want).norm() <= 0.05 * want.norm(), i


def test_a_budget_holds_and_replays_equal_eager_steps():
    budget = 20
    eager, replayed = Decoder(**SHAPE, budget=budget), Decoder(**SHAPE, budget=budget)
    g = torch.Generator().manual_seed(2)
    for i in range(50):
        tokens = torch.randint(0, SHAPE["vocab"], (SHAPE["batch"],), generator=g).cuda()
        a, b = eager.step(tokens), replayed.step(tokens, graph=True)
        assert torch.isfinite(a).all() and torch.equal(a, b), i
        assert eager.slots.tolist() == [min(i + 1, budget)] * SHAPE["batch"]
    for lay in eager.layers:
        kept = lay["token"][:, :, :budget].sort(dim=-1).values
        assert (kept[..., 1:] > kept[..., :-1]).all()                       # every token once
        assert (kept[..., -budget // 4:] == torch.arange(50 - budget // 4, 50, device="cuda")).all()      # the newest quarter is there
        assert (kept[..., 0] < 50 - budget).any()                           # and something old


@pytest.mark.parametrize("budget", [1, 2, 7, 8])
def test_the_newest_quarter_and_nothing_else_is_protected(budget):
    """One token where a quarter is less; of a budget of one it is the token of the step itself."""
    dec = Decoder(**{**SHAPE, "layers": 1}, budget=budget)
    quarter = max(1, budget // 4)
    for i in range(3 * budget + 4):
        dec.step(torch.arange(3, device="cuda"), graph=i >= 2)
        kept = dec.layers[0]["token"][:, :, :min(i + 1, budget)].sort(dim=-1).values
        newest = torch.arange(max(0, i + 1 - quarter), i + 1, device="cuda", dtype=kept.dtype)
        assert (kept[..., -len(newest):] == newest).all()
        # the next eviction protects the quarter that the next token completes
        assert dec.since.tolist() == [i + 2 - quarter] * 3


@pytest.mark.parametrize("budget", [0, 5])
@pytest.mark.parametrize("graph", [False, True])
def test_a_context_that_is_full_is_refused(budget, graph):
    dec = Decoder(**{**SHAPE, "layers": 1, "context": 9}, budget=budget)
    for _ in range(9):
        was = dec.step(torch.arange(3, device="cuda"), graph=graph).clone()
    with pytest.raises(ValueError, match="9 tokens"):
        dec.step(torch.arange(3, device="cuda"), graph=graph)
    assert torch.equal(dec.logits, was) and dec.positions.tolist() == [9] * 3
