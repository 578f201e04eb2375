"""tq_sample against the formula in 64 bits: the tokens are equal, probabilities one rounding to fp32 (2^-24) and the sums' 2^-30 apart."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2509_22951_amd as tq
from drafts import sample_reference
from paged import ptr, stream

pytestmark = pytest.mark.gpu

FILTERS = [(1.0, 0, 1.0, 0.0), (0.7, 40, 0.9, 0.0), (1.3, 0, 0.95, 0.0), (1.0, 0, 1.0, 0.05), (0.0, 5, 0.5, 0.0), (0.5, 3, 1.0, 0.9), (2.0, 1, 1.0, 0.0), (1.0, 1000, 0.999, 0.001),
           (0.05, 0, 0.3, 0.0), (1.0, 0, 0.0, 0.0), (-1.0, 0, 1.0, 0.0), (1.5, 7, 1.0, 0.0), (100.0, 0, 0.5, 0.0)]


def call(logits, t, k, p, m, u, stride=0, workspace=None, keep=None):
    rows, vocab = logits.shape
    cast = lambda x, d: None if x is None else torch.tensor(x, dtype=d).cuda()
    t, p, m, u, k = (*(cast(x, torch.float32) for x in (t, p, m, u)), cast(k, torch.int32))
    tokens, probs = torch.full((rows,), -7, dtype=torch.int32, device="cuda"), torch.full((rows,), -7.0, device="cuda")
    fields = dict(logits=ptr(logits), temperature=ptr(t), top_k=ptr(k), top_p=ptr(p), min_p=ptr(m), uniform=ptr(u), tokens=ptr(tokens), probs=ptr(probs), rows=rows,
                  vocab=vocab, logits_stride=stride)
    ws = torch.full((tq.Sample.workspace_bytes(**fields),), 0xEE, dtype=torch.uint8, device="cuda") if workspace is None else workspace
    made = tq.Sample(workspace=ptr(ws), workspace_bytes=ws.numel(), **fields)
    made.keep = (logits, t, p, m, u, k, ws)
    return made, tokens, probs


def check(logits, t, k, p, m, u, **more):
    made, tokens, probs = call(logits, t, k, p, m, u, **more)
    made.launch(stream())
    torch.cuda.synchronize()
    host = logits.cpu().numpy()
    rows = host.shape[0]
    pick = lambda x, r, default: default if x is None else x[r]
    for r in range(rows):
        token, prob, kept = sample_reference(host[r], pick(t, r, 1.0), pick(k, r, 0), pick(p, r, 1.0), pick(m, r, 0.0), u[r])
        assert int(tokens[r]) == token, (r, int(tokens[r]), token, len(kept))
        assert abs(float(probs[r]) - prob) <= prob * (2.0 ** -24 + 2.0 ** -30), (r, float(probs[r]), prob)
    return tokens, probs


def peaked(rows, vocab, seed, width=2.0):
    g = torch.Generator().manual_seed(seed)
    x = width * torch.randn((rows, vocab), generator=g)
    at = torch.randint(0, vocab, (rows, min(10, vocab)), generator=g)
    return x.scatter_(1, at, 8 + 2 * torch.randn(at.shape, generator=g)).cuda()


@pytest.mark.parametrize("vocab", [1, 2, 3, 63, 64, 65, 255, 1000, 1023, 4096, 4097, 32000, 50001, 128256, 200003])
def test_sizes(vocab):
    n = len(FILTERS)
    g = np.random.default_rng(vocab)
    t, k, p, m = zip(*FILTERS)
    check(peaked(n, vocab, vocab), t, k, p, m, g.random(n, dtype=np.float32).tolist())


@pytest.mark.parametrize("seed", range(6))
def test_filters_drawn_at_random(seed):
    g = np.random.default_rng(seed)
    rows, vocab = 40, int(g.integers(100, 20000))
    t = np.exp(g.uniform(-2, 2, rows)).astype(np.float32).tolist()
    k = np.where(g.random(rows) < 0.4, 0, g.integers(1, vocab + 10, rows)).tolist()
    p = np.where(g.random(rows) < 0.3, 1.0, g.random(rows)).astype(np.float32).tolist()
    m = np.where(g.random(rows) < 0.5, 0.0, g.random(rows) ** 4).astype(np.float32).tolist()
    check(peaked(rows, vocab, seed, width=float(g.uniform(0.1, 5))), t, k, p, m, g.random(rows, dtype=np.float32).tolist())


@pytest.mark.parametrize("scale", [1e-30, 1e-3, 30.0, 1e4, 1e30])
def test_logits_of_any_size(scale):
    g = np.random.default_rng(3)
    t, k, p, m = zip(*FILTERS)
    n = len(FILTERS)
    check(peaked(n, 5000, 9) * scale, [x * scale for x in t], k, p, m, g.random(n, dtype=np.float32).tolist())
    check(peaked(n, 5000, 10) * scale + 7 * scale, t, k, p, m, g.random(n, dtype=np.float32).tolist())


def test_equal_logits_are_cut_at_the_lowest_tokens():
    """All weights are 1: every sum is exact, and so is every border."""
    vocab = 10000
    x = torch.full((8, vocab), -3.25, device="cuda")
    tokens, _ = check(x, [1.0] * 8, [0, 0, 4, 0, 5000, 0, 1, 9999], [1.0, 0.5, 1.0, 0.25, 0.75, 1.0, 1.0, 1.0], [0, 0, 0, 0, 0, 1.0, 0, 0.5],
                      [0.5, 0.5, 0.5, 0.75, 0.5, 0.0, 0.99, 0.9999999])
    assert tokens.tolist() == [5000, 2500, 2, 1875, 2500, 0, 0, 9998]


def test_few_values_many_of_each():
    """Ties across the cut: 30000 tokens of five values, some of them zeros of both signs."""
    g = np.random.default_rng(5)
    x = torch.tensor(g.choice(np.array([1.5, 0.0, -0.0, -2.0, 2.5], dtype=np.float32), (10, 30000))).cuda()
    k = [1, 100, 5999, 6001, 12001, 20000, 29999, 30000, 0, 0]
    p = [1.0] * 7 + [0.9, 0.3, 0.999]
    check(x, [1.0] * 10, k, p, [0.0] * 10, g.random(10, dtype=np.float32).tolist())


def test_masked_tokens_rows_of_them_infinities_and_nan():
    inf, nan, low = float("inf"), float("nan"), torch.finfo(torch.float32).min
    x = peaked(12, 3000, 1)
    x[0] = -inf
    x[1] = nan
    x[2, 1:] = -inf
    x[3, :2999] = nan
    x[4, 100] = inf
    x[5, [7, 1000, 2999]] = inf
    x[6, ::2] = -inf
    x[7, ::3] = nan
    x[8] = low
    x[9, 5:] = low
    x[10, :-1], x[10, -1] = -inf, low
    x[11] = torch.where(torch.arange(3000, device="cuda") % 2 == 0, torch.tensor(low, device="cuda"), torch.tensor(-low, device="cuda"))
    for f in FILTERS[:5] + [(1.0, 2500, 1.0, 0.0), (1.0, 0, 0.9999, 0.0)]:
        check(x, [f[0]] * 12, [f[1]] * 12, [f[2]] * 12, [f[3]] * 12, [0.37] * 12)
    tokens, probs = check(x, None, None, None, None, [0.9] * 12)
    assert tokens[:2].tolist() == [-1, -1] and probs[:2].tolist() == [0, 0] and tokens[5] == 2999


def test_numbers_at_the_ends_and_parameters_that_are_not_numbers():
    x = peaked(6, 700, 4)
    x[:, 0], x[:, 699] = 3.0, 3.0
    tokens, _ = check(x, None, None, None, None, [0.0, float(np.nextafter(np.float32(1), np.float32(0))), 1.0, 5.0, -1.0, 0.0])
    assert tokens.tolist() == [0, 699, 699, 699, 0, 0]
    nan = float("nan")
    made, got, _ = call(x, [nan, 1, 1, float("inf"), 1, 1], [0] * 6, [1, nan, 1, 1, 2.5, 1], [0, 0, nan, 0, 0, -3], [0.4] * 6)
    made.launch(stream())
    same, want, _ = call(x, [0, 1, 1, 1, 1, 1], [0] * 6, [1] * 6, [0] * 6, [0.4] * 6)
    same.launch(stream())
    torch.cuda.synchronize()
    assert [int(v) for i, v in enumerate(got) if i != 3] == [int(v) for i, v in enumerate(want) if i != 3]
    assert int(got[3]) == 280      # at an infinite temperature all tokens are alike: the first beyond 0.4f * 700 of them
    tokens, _ = check(x, [1.0] * 6, [0] * 6, [1.0] * 6, [2.0] * 6, [0.9] * 6)
    assert torch.equal(tokens.long(), x.argmax(dim=1))      # beyond every weight: the first token stays


def test_rows_with_gaps_at_any_address_and_no_probabilities():
    buf = peaked(1, 9 * 1003 + 1, 6)[0]
    x = buf[1:].view(9, 1003)[:, :1000]
    t, k, p, m = zip(*FILTERS[:9])
    check(x, t, k, p, m, [0.1 * r for r in range(9)], stride=1003)
    made, tokens, probs = call(x, t, k, p, m, [0.1 * r for r in range(9)], stride=1003)
    made.args.probs = 0
    made.launch(stream())
    torch.cuda.synchronize()
    assert (probs == -7).all() and (tokens >= 0).all()


def test_results_repeat_on_another_stream_with_a_workspace_of_other_calls():
    wide = peaked(30, 40000, 7)
    t, k, p, m = ([FILTERS[r % len(FILTERS)][i] for r in range(30)] for i in range(4))
    u = np.random.default_rng(1).random(30, dtype=np.float32).tolist()
    made, tokens, probs = call(wide, t, k, p, m, u)
    made.launch(stream())
    torch.cuda.synchronize()
    first = tokens.clone(), probs.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for vocab in (3, 1000, 40000):
            check(wide[:, :vocab], t, k, p, m, u, stride=40000, workspace=made.keep[-1])
        for _ in range(3):
            tokens.zero_()
            made.launch(stream())
            torch.cuda.synchronize()
            assert torch.equal(tokens, first[0]) and torch.equal(probs, first[1])


@pytest.mark.parametrize("rows,vocab", [(48, 100000), (3, 70001), (300, 9000), (7, 15000)])
def test_rows_without_filters_beside_others(rows, vocab):
    """Their weights are summed relative to each part's own largest logit: parts of masked tokens, parts far below the others, parts with infinities."""
    inf = float("inf")
    x = peaked(rows, vocab, rows)
    x[0, : vocab // 2] = -inf
    x[1, 5000:] = float("nan")
    x[2, : vocab // 3] -= 60
    if rows > 3:
        x[3, [17, vocab - 1]] = inf
        x[4, 4096:8192] = inf
        x[5, : vocab - 1] = -inf
        x[6] = 0.25
    few = [FILTERS[0] if r % 3 else FILTERS[r % len(FILTERS)] for r in range(rows)]
    t, k, p, m = zip(*few)
    u = np.random.default_rng(rows).random(rows, dtype=np.float32).tolist()
    check(x, t, k, p, m, u)
    check(x, None, None, None, None, u)
    check(x, [0.01] * rows, [vocab] * rows, [1.0] * rows, None, u)      # (top_k of all tokens leaves none out)


def test_graphs_that_share_a_workspace():
    made = []
    shared = torch.full((1 << 26,), 0xEE, dtype=torch.uint8, device="cuda")
    for rows, vocab, seed in ((5, 30000, 11), (40, 60000, 12), (1, 777, 13)):
        t, k, p, m = ([FILTERS[(r + seed) % len(FILTERS)][i] for r in range(rows)] for i in range(4))
        made.append(call(peaked(rows, vocab, seed), t, k, p, m, np.random.default_rng(seed).random(rows, dtype=np.float32).tolist(), workspace=shared))
    wants, graphs = [], []
    for one, tokens, probs in made:
        one.launch(stream())
        torch.cuda.synchronize()
        wants.append((tokens.clone(), probs.clone()))
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=torch.cuda.Stream()):
            one.launch(stream())
    for _ in range(3):
        for graph, (_, tokens, probs) in zip(graphs, made):
            tokens.zero_(), probs.zero_()
            graph.replay()
        torch.cuda.synchronize()
        for (_, tokens, probs), want in zip(made, wants):
            assert torch.equal(tokens, want[0]) and torch.equal(probs, want[1])


@pytest.mark.parametrize("vocab", [1500, 2047, 2048, 2049, 4095, 4096, 4097, 8191, 12289])
def test_around_the_sizes_of_parts(vocab):
    """Rows of one workgroup and of several, more tokens of one bin than LDS has room for, and everything else that rows of a single workgroup have to themselves."""
    inf, n = float("inf"), len(FILTERS)
    g = np.random.default_rng(vocab)
    t, k, p, m = zip(*FILTERS)
    x = peaked(n, vocab, vocab)
    check(x, t, k, p, m, g.random(n, dtype=np.float32).tolist())
    x[:, : vocab - 40] = 1.25                                 # one bin, equal logits: the lowest tokens stay
    check(x, [1.0] * n, [vocab - 60 + r for r in range(n)], [0.9, 1.0] * (n // 2) + [0.5], None, g.random(n, dtype=np.float32).tolist())
    x = 1 + 1e-4 * torch.rand((n, vocab), generator=torch.Generator().manual_seed(vocab)).cuda()      # one bin, different ones
    x[1, ::3], x[2, 5:9], x[3, :-1] = -inf, inf, float("nan")
    check(x, [0.9] * n, [0, vocab // 2, 3] + [vocab // 3 + r for r in range(n - 3)], [0.7] * n, [0.0, 0.5] * (n // 2) + [0.0], g.random(n, dtype=np.float32).tolist())


@pytest.mark.parametrize("vocab", [700, 2500, 4096, 30000, 128256])
@pytest.mark.parametrize("mask", [float("-inf"), float("nan"), torch.finfo(torch.float32).min, -1e4])
def test_most_of_a_vocabulary_masked(vocab, mask):
    """Ten tokens that are not: fewer than, as many as and more than top_k asks for, with the other filters."""
    n, g = 12, np.random.default_rng(vocab)
    x = torch.full((n, vocab), mask, device="cuda")
    at = torch.stack([torch.randperm(vocab, generator=torch.Generator().manual_seed(r))[:10] for r in range(n)]).cuda()
    x.scatter_(1, at, peaked(n, 10, vocab))
    x[1, 5:], x[2] = mask, mask                       # (fewer still; none but, perhaps, a mask that is a number)
    k = [50, 50, 50, 9, 10, 11, 0, 50, vocab - 1, 50, 0, 3]
    p = [1.0, 1.0, 1.0, 1.0, 1.0, 1.0, 0.9, 0.9, 0.999, 1.0, 0.9999999, 0.5]
    m = [0.0] * 9 + [0.05, 0.0, 0.01]
    check(x, [0.8] * n, k, p, m, g.random(n, dtype=np.float32).tolist())
    check(x, [0.8] * n, k, None, m, [float(np.nextafter(np.float32(1), np.float32(0)))] * n)
    check(x, [0.8] * n, None, p, m, [0.0] * n)


@pytest.mark.parametrize("k,p", [(50, 1.0), (50, 0.9), (0, 0.95)])
def test_masked_tokens_are_not_listed(k, p):
    """Eight bytes a token that a cut could leave out or not: a cut beyond all tokens that have any weight lists none of the others, whose order nobody needs."""
    vocab = 128256
    x = torch.full((1, vocab), float("-inf"), device="cuda")
    x[0, 1000:1010] = peaked(1, 10, 1)[0]
    made, tokens, _ = call(x, [0.8], [k], [p], None, [0.4])
    made.launch(stream())
    torch.cuda.synchronize()
    assert 1000 <= int(tokens[0]) < 1010
    written = int((made.keep[-1] != 0xEE).sum())
    assert written < 2 * vocab, written                # (bins and what the parts leave each other: some 30000 bytes)


@pytest.mark.parametrize("vocab", [100, 2048, 2049, 4096, 4097, 30000, 70001])
@pytest.mark.parametrize("filters", ["all", "top_k", "top_p", "none"])
def test_nothing_is_written_behind_the_room_that_is_asked_for(vocab, filters):
    """Equal logits: as many keys are listed as there can be."""
    rows = 3
    k, p = ([vocab // 2] * rows if filters in ("all", "top_k") else None), ([0.5] * rows if filters in ("all", "top_p") else None)
    x = torch.zeros((rows, vocab), device="cuda")
    made, _, _ = call(x, [1.0] * rows, k, p, [0.5] * rows, [0.4] * rows)
    need = made.keep[-1].numel()
    room = torch.full((need + (1 << 22),), 0xEE, dtype=torch.uint8, device="cuda")
    made.args.workspace = ptr(room)
    made.launch(stream())
    torch.cuda.synchronize()
    assert (room[need:] == 0xEE).all()
    check(x, [1.0] * rows, k, p, [0.5] * rows, [0.4] * rows, workspace=room[:need])


@pytest.mark.parametrize("rows,vocab", [(1, 1 << 20), (2, (1 << 20) - 1), (5, 1 << 20), (13, 1000003), (2, 600000)])
def test_the_largest_vocabularies(rows, vocab):
    """Up to 512 parts a row, two to a thread of the workgroup that draws; numbers that fall into the first ones, the middle and the last."""
    f = [FILTERS[r % len(FILTERS)] for r in range(rows)]
    t, k, p, m = zip(*f)
    u = np.linspace(0.02, 0.999, rows, dtype=np.float32).tolist()
    x = peaked(rows, vocab, vocab)
    check(x, t, k, p, m, u)
    check(x, None, None, None, None, u[::-1])
    check(x, [1.2] * rows, [60000] * rows, [0.97] * rows, [1e-4] * rows, u)


def test_how_often_tokens_are_drawn():
    """4096 evenly spaced numbers: every token is drawn as often as its share says, give or take the two ends."""
    x = torch.tensor([2.0, 1.0, 0.0, -1.0, 1.5, -30.0], device="cuda")
    n = 4096
    made, tokens, _ = call(x.expand(n, 6).contiguous(), [0.8] * n, [4] * n, None, None, [(i + 0.5) / n for i in range(n)])
    made.launch(stream())
    w = torch.exp(x.double().cpu() / np.float32(0.8).item())
    w[[3, 5]] = 0
    counts = torch.bincount(tokens.cpu().long(), minlength=6)
    assert ((counts - n * w / w.sum()).abs() <= 1).all() and counts[3] == counts[5] == 0


def test_captured_and_replayed():
    x = peaked(5, 30000, 8)
    t, k, p, m = zip(*FILTERS[:5])
    made, tokens, probs = call(x, t, k, p, m, [0.5] * 5)
    u = made.keep[4]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        made.launch(stream())
    for step in range(4):
        u.copy_(torch.rand(5, generator=torch.Generator().manual_seed(step)))
        x.add_(torch.randn(x.shape, generator=torch.Generator().manual_seed(step)).cuda())
        tokens.fill_(-9)
        graph.replay()
        torch.cuda.synchronize()
        want = [sample_reference(x[r].cpu().numpy(), t[r], k[r], p[r], m[r], float(u[r]))[0] for r in range(5)]
        assert tokens.tolist() == want
