"""tq_tree_accept: branches and everything that is moved, bit for bit."""
import random

import pytest

torch = pytest.importorskip("torch")

import paper_2509_22951_amd as tq
from drafts import accept_reference, bits_of, ints, masks_of, random_parents
from paged import Paged, ptr, stream

pytestmark = pytest.mark.gpu


def words(parents, seed, likely=0.8, vocabulary=5):
    """Drafted and drawn tokens; few different ones, so that siblings share some."""
    rng = random.Random(seed)
    drafted = [[rng.randrange(vocabulary) for _ in tree] for tree in parents]
    drawn = []
    for tree, of in zip(parents, drafted):
        children = [[c for c, p in enumerate(tree) if p == i] for i in range(len(tree))]
        drawn.append([of[rng.choice(c)] if c and rng.random() < likely else rng.randrange(vocabulary) for c in children])
    return drafted, drawn


def accept(caches, bits, drafted, drawn, lengths, sizes=None, seqs=None):
    trees, nodes = len(bits), len(bits[0])
    masks, d, s = masks_of(bits), ints(drafted), ints(drawn)
    path, accepted, after, lengths_out = ints([[77] * nodes] * trees), ints([77] * trees), ints([77] * trees), ints([77] * trees)
    made = tq.TreeAccept(caches, masks=ptr(masks), sizes=ptr(sizes), seqs=ptr(seqs), lengths=ptr(lengths), drafted=ptr(d), sampled=ptr(s), path=ptr(path),
                         accepted=ptr(accepted), next=ptr(after), lengths_out=ptr(lengths_out), trees=trees, nodes=nodes)
    made.keep = (masks, d, s, sizes, seqs, lengths)
    return made, path, accepted, after, lengths_out


def everything(p):
    return {n: getattr(p, n).cpu().clone() for n in ("k", "v", "k_scale", "v_scale", "scores", "positions") if getattr(p, n) is not None}


def moved(p, before, branches, lengths, seqs):
    """What the cache holds afterwards."""
    want = {n: t.clone() for n, t in before.items()}
    table = p.tables.cpu().tolist()
    for t, (path, _) in enumerate(branches):
        s, begin = t if seqs is None else int(seqs[t]), max(int(lengths[t]), 0)
        if not 0 <= s < p.n_seqs:
            continue
        for i, node in enumerate(path):
            to, of = begin + i, begin + node
            if node == i or of >= p.capacity:
                continue
            to_page, of_page = table[s][to // p.page], table[s][of // p.page]
            if not (0 <= to_page < p.n_pages and 0 <= of_page < p.n_pages):
                continue
            for n in ("k", "v", "k_scale", "v_scale"):
                if n in want:
                    want[n][to_page, :, to % p.page] = before[n][of_page, :, of % p.page]
            for n in ("scores", "positions"):
                if n in want:
                    want[n][s, :, to] = before[n][s, :, of]
    return want


def check(ps, parents, lengths, seed=0, sizes=None, seqs=None, likely=0.8, strides=None):
    bits = bits_of(parents)
    trees, nodes = len(parents), len(parents[0])
    drafted, drawn = words(parents, seed, likely)
    lengths = ints(lengths)
    host_sizes = [nodes] * trees if sizes is None else sizes
    branches = accept_reference(bits, host_sizes, drafted, drawn, nodes)
    before = [everything(p) for p in ps]
    made, path, accepted, after, lengths_out = accept([p.describe() for p in ps], bits, drafted, drawn, lengths, None if sizes is None else ints(sizes),
                                                      None if seqs is None else ints(seqs))
    made.launch(stream())
    torch.cuda.synchronize()
    assert path.tolist() == [got + [-1] * (nodes - len(got)) for got, _ in branches]
    assert accepted.tolist() == [len(got) for got, _ in branches] and after.tolist() == [token for _, token in branches]
    assert lengths_out.tolist() == [max(int(n), 0) + len(got) for n, (got, _) in zip(lengths, branches)]
    for p, was in zip(ps, before):
        want, got = moved(p, was, branches, lengths, seqs), everything(p)
        for n in want:
            assert torch.equal(got[n], want[n]), n
    return branches


@pytest.mark.parametrize("nodes", [1, 2, 3, 8, 9, 16, 17, 33, 63, 64])
@pytest.mark.parametrize("kind", ["bf16", "int8"])
def test_trees(nodes, kind):
    p = Paged(5, 8, kind=kind, marks=True, seed=nodes)
    branches = check([p], random_parents(5, nodes, nodes), [0, 1, 40, 63, 64], seed=nodes, likely=0.95)
    assert nodes < 8 or max(len(path) for path, _ in branches) > 2


def test_a_chain_is_accepted_as_far_as_it_agrees():
    p = Paged(3, 8)
    chain = [list(range(-1, 63))] * 3
    check([p], chain, [3, 17, 60], likely=1.0)          # all of it: nothing moves
    check([p], chain, [3, 17, 60], likely=0.9)


def test_a_branch_of_late_nodes_moves_through_slots_that_it_reads():
    """Two chains, node by node in turn: the accepted one is every second node, so each token moves to where another one of the branch lay."""
    parents = [[-1, 0, 0] + [i - 2 for i in range(3, 64)]] * 2
    bits = bits_of(parents)
    p = Paged(2, 8, kind="int8", marks=True)
    drafted = [[100 + i for i in range(64)]] * 2
    drawn = [[drafted[0][2]] + [drafted[0][i + 2] if i + 2 < 64 else 5 for i in range(1, 64)]] * 2
    lengths, before = ints([5, 30]), everything(p)
    made, path, accepted, after, _ = accept([p.describe()], bits, drafted, drawn, lengths)
    made.launch(stream())
    torch.cuda.synchronize()
    branch = [0] + list(range(2, 64, 2))
    assert path[0].tolist() == branch + [-1] * (64 - len(branch)) and after.tolist() == [5, 5]
    want, got = moved(p, before, [(branch, 5)] * 2, lengths, None), everything(p)
    for n in want:
        assert torch.equal(got[n], want[n]), n


@pytest.mark.parametrize("dim,kv_heads,page,order", [(16, 1, 16, "phtd"), (80, 3, 32, "pthd"), (128, 8, 64, "hptd"), (256, 2, 16, "tphd"), (96, 17, 1024, "phtd")])
@pytest.mark.parametrize("kind", ["bf16", "int8"])
def test_caches_of_any_shape(dim, kv_heads, page, order, kind):
    p = Paged(3, max(2, -(-90 // page)), kv_heads=kv_heads, dim=dim, page=page, kind=kind, order=order, marks=True, seed=dim)
    check([p], random_parents(3, 20, dim), [10, 50, 27], seed=dim, likely=0.95)


def test_layers_of_different_shapes_more_than_a_launch_takes():
    ps = [Paged(2, 5 + n % 3, kv_heads=1 + n % 2, dim=(16, 48, 64)[n % 3], page=(16, 32)[n % 2], kind=("bf16", "int8")[n % 2], marks=n % 5 == 0, seed=n) for n in range(70)]
    check(ps, random_parents(2, 16, 1), [20, 40], likely=1.0)


@pytest.mark.parametrize("layers", [2, 7, 40])
@pytest.mark.parametrize("shared", [("positions",), ("scores",), ("scores", "positions")])
def test_layers_that_share_scores_or_positions(layers, shared):
    """Without eviction the positions of all layers are alike, and one array holds them: it moves once."""
    ps = [Paged(2, 8, kind=("bf16", "int8")[n % 2], marks=True, seed=n) for n in range(layers)]
    for p in ps[1:]:
        for name in shared:
            setattr(p, name, getattr(ps[0], name))
    nodes = [[-1, 0, 0] + [i - 2 for i in range(3, 64)]] * 2         # two chains in turn: a slot that is read is written, too
    drafted = [[100 + i for i in range(64)]] * 2
    drawn = [[drafted[0][2]] + [drafted[0][i + 2] if i + 2 < 64 else 5 for i in range(1, 64)]] * 2
    lengths, before = ints([5, 30]), [everything(p) for p in ps]
    made, *_ = accept([p.describe() for p in ps], bits_of(nodes), drafted, drawn, lengths)
    made.launch(stream())
    torch.cuda.synchronize()
    branch = [0] + list(range(2, 64, 2))
    for p, was in zip(ps, before):
        want, got = moved(p, was, [(branch, 5)] * 2, lengths, None), everything(p)
        for n in want:
            assert torch.equal(got[n], want[n]), n


def test_without_caches():
    check([], random_parents(200, 16, 2), [7] * 200, seed=3)


def test_sizes_sequences_and_what_is_not_there():
    p = Paged(6, 4, spare_pages=1, marks=True)           # 64 tokens of room
    p.tables[1, 1], p.tables[2, 2], p.tables[4] = -1, p.n_pages, 2 ** 30
    check([p], random_parents(8, 16, 5), [20, 10, 20, 60, 5, -4, 2 ** 31 - 200, 30], seqs=[0, 1, 2, 3, 4, 5, -1, 6], likely=1.0)
    check([p], random_parents(6, 16, 6), [20, 10, 20, 60, 5, 99999], sizes=[0, 3, 16, 99, -1, 7], likely=1.0)


def test_children_of_the_same_token_lowest_first_and_masks_of_other_kinds():
    p = Paged(2, 4)
    bits = [[1, 3, 5, 9, 1 | 4 | 16, 1 | 2 | 32], [0, 0, 0, 0, 0, 0]]
    made, path, accepted, after, lengths_out = accept([p.describe()], bits, [[9, 4, 4, 4, 7, 8]] * 2, [[4, 8, 7, 1, 2, 3]] * 2, ints([3, 3]))
    made.launch(stream())
    torch.cuda.synchronize()
    assert path.tolist() == [[0, 1, 5, -1, -1, -1], [0, -1, -1, -1, -1, -1]] and after.tolist() == [3, 4] and lengths_out.tolist() == [6, 4]


def test_a_pool_beyond_32_bits_of_offset():
    p = Paged(1, 2, kv_heads=2, dim=64)
    base = 2 ** 31 // (2 * 16 * 64) + 5
    far = p.n_pages + base
    small = {n: getattr(p, n).clone() for n in ("k", "v")}
    for name in ("k", "v"):
        pool = torch.empty((far, 2, 16, 64), dtype=torch.bfloat16, device="cuda")
        pool[base:] = small[name]
        setattr(p, name, pool)
    p.tables += base
    p.n_pages = far
    bits = bits_of([[-1, 0, 0, 2]])
    made, path, *_ = accept([p.describe()], bits, [[0, 1, 2, 3]], [[2, 0, 3, 0]], ints([15]))
    made.launch(stream())
    torch.cuda.synchronize()
    assert path.tolist() == [[0, 2, 3, -1]]
    pages = (p.tables[0] - base).tolist()
    for n in ("k", "v"):
        got, want = getattr(p, n)[base:], small[n].clone()
        want[pages[1], :, 0], want[pages[1], :, 1] = small[n][pages[1], :, 1], small[n][pages[1], :, 2]
        assert torch.equal(got, want)


def test_captured_and_replayed():
    p = Paged(2, 8, kind="int8", marks=True)
    parents = random_parents(2, 12, 8)
    bits = bits_of(parents)
    drafted, drawn = words(parents, 1)
    lengths = ints([10, 20])
    made, path, accepted, after, lengths_out = accept([p.describe()], bits, drafted, drawn, lengths)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        made.launch(stream())
    for step in range(4):
        drafted, drawn = words(parents, step)
        made.keep[1].copy_(ints(drafted)), made.keep[2].copy_(ints(drawn))
        before, was = everything(p), lengths.clone()
        graph.replay()
        torch.cuda.synchronize()
        branches = accept_reference(bits, [12, 12], drafted, drawn, 12)
        want, got = moved(p, before, branches, was, None), everything(p)
        assert all(torch.equal(got[n], want[n]) for n in want) and accepted.tolist() == [len(b) for b, _ in branches]
        lengths.copy_(lengths_out)
