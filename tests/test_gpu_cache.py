"""tq_cache_append and tq_cache_evict: rotation and quantization against the formulas in 64 bits, everything that is moved bit for bit.

Tolerances of the rotation: two fp32 products and a sum, 3 * 2^-24 of |a| + |b| at most (taken as 2^-22); stored as bf16 2^-8 of the value
more; in 8 bits half a step of the scale, the scale 2^-22 off, in steps 127 * 2^-21."""
import pytest

torch = pytest.importorskip("torch")

import paper_2509_22951_amd as tq
from paged import Paged, attend_call, evict_reference, ptr, stream

pytestmark = pytest.mark.gpu


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def angles(n, rotary_dim):
    a = torch.arange(n, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, max(rotary_dim, 2), 2, dtype=torch.float64) / max(rotary_dim, 2))
    return torch.cos(a).float(), torch.sin(a).float()


def rotated(x, cos, sin, rotary_dim, adjacent):
    """fp32 [rows][heads][dim], angles [rows][rotary_dim / 2] -> (64 bits, what a value is off by in 2^-22)."""
    y, mag = x.double().clone(), x.double().abs().clone()
    half = rotary_dim // 2
    if half:
        a, b = (slice(0, rotary_dim, 2), slice(1, rotary_dim, 2)) if adjacent else (slice(0, half), slice(half, rotary_dim))
        c, s = cos.double()[:, None], sin.double()[:, None]
        xa, xb = x[..., a].double(), x[..., b].double()
        y[..., a], y[..., b] = xa * c - xb * s, xa * s + xb * c
        mag[..., a] = mag[..., b] = xa.abs() + xb.abs()
    return y, mag


def new_tokens(rows, heads, kv_heads, dim, seed=0):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn((rows, n, dim), generator=g) for n in (heads, kv_heads, kv_heads)]


def append(p, q, k, v, seqs, slots, positions, cos, sin, rotary_dim, adjacent=False, q_out=None, q16=False, gap=0, offset=0, in_place=False):
    rows, heads, dim = q.shape

    def placed(t):
        wide = t.shape[1] * dim + gap
        buf = torch.zeros(rows * wide + offset, device="cuda")
        view = buf[offset:].view(rows, wide)[:, : t.shape[1] * dim]
        view.copy_(t.reshape(rows, -1))
        return view

    qd, kd, vd, cd, sd = placed(q), placed(k), placed(v), cos.cuda(), sin.cuda()
    out = qd if in_place else torch.full((rows, heads * dim), 7, dtype=torch.bfloat16 if q16 else torch.float32, device="cuda")
    tq.CacheAppend(p.describe(), q=ptr(qd), k=ptr(kd), v=ptr(vd), q_out=ptr(out), seqs=ptr(seqs), slots=ptr(slots), positions=ptr(positions), cos=ptr(cd),
                   sin=ptr(sd), rows=rows, heads=heads, rotary_dim=rotary_dim, n_positions=cos.shape[0], q_stride=qd.stride(0), k_stride=kd.stride(0),
                   v_stride=vd.stride(0), q_out_stride=out.stride(0), q_out_type=tq.TQ_BF16 if q16 else tq.TQ_FP32, pairing=int(adjacent)).launch(stream())
    torch.cuda.synchronize()
    return out.cpu().reshape(rows, heads, dim)


def check_append(p, before, q_got, q, k, v, seqs, slots, positions, cos, sin, rotary_dim, adjacent=False):
    """before: (k, v, k_scale, v_scale) on the CPU, as the cache was."""
    rows = q.shape[0]
    seqs = list(range(rows)) if seqs is None else seqs.tolist()
    slots = slots.tolist()
    positions = slots if positions is None else positions.tolist()
    there = [0 <= s < p.n_seqs and 0 <= t < p.capacity and (rotary_dim == 0 or 0 <= x < cos.shape[0]) for s, t, x in zip(seqs, slots, positions)]
    at = torch.tensor([x if ok else 0 for x, ok in zip(positions, there)])
    want_q, mag_q = rotated(q, cos[at % cos.shape[0]], sin[at % cos.shape[0]], rotary_dim, adjacent)
    want_k, mag_k = rotated(k, cos[at % cos.shape[0]], sin[at % cos.shape[0]], rotary_dim, adjacent)
    ok = torch.tensor(there)
    assert (q_got[~ok] == 0).all()
    off = (q_got.double() - want_q).abs()
    more = 2.0 ** -8 * want_q.abs() if q_got.dtype == torch.bfloat16 else 0
    assert (off <= mag_q * 2.0 ** -22 + more)[ok].all()
    touched = torch.zeros(p.n_pages, p.page, dtype=torch.bool)
    pools = {n: getattr(p, n).cpu() for n in ("k", "v")}
    scales = {n: None if p.k_scale is None else getattr(p, n + "_scale").cpu() for n in ("k", "v")}
    table = p.tables.cpu()
    for r in range(rows):
        if not there[r]:
            continue
        page, t = int(table[seqs[r], slots[r] // p.page]), slots[r] % p.page
        if not 0 <= page < p.n_pages:
            continue
        touched[page, t] = True
        for n, want, mag in (("k", want_k[r], mag_k[r]), ("v", v[r].double(), torch.zeros_like(mag_k[r]))):
            got = pools[n][page, :, t]
            if scales[n] is None:
                assert ((got.double() - want).abs() <= want.abs() * 2.0 ** -8 + mag * 2.0 ** -22).all()
                if n == "v":
                    assert torch.equal(got, v[r].to(torch.bfloat16))
            else:
                s = want.abs().amax(dim=1) / 127
                got_s = scales[n][page, :, t].double()
                assert ((got_s - s).abs() <= mag.amax(dim=1) / 127 * 2.0 ** -21 + s * 2.0 ** -22).all()
                assert ((got.double() * got_s[:, None] - want).abs() <= s[:, None] * (0.5 + 127 * 2.0 ** -20)).all()
        if p.scores is not None:
            assert (p.scores[seqs[r], :, slots[r]] == 0).all() and (p.positions[seqs[r], :, slots[r]] == positions[r]).all()
    for n, was, was_scale in (("k", before[0], before[2]), ("v", before[1], before[3])):
        rest = ~touched[:, None, :].expand(-1, p.kv_heads, -1)
        assert torch.equal(pools[n][rest], was[rest])
        if was_scale is not None:
            assert torch.equal(scales[n][rest], was_scale[rest])


def snapshot(p):
    return [None if t is None else t.cpu().clone() for t in (p.k, p.v, p.k_scale, p.v_scale)]


@pytest.mark.parametrize("dim,rotary_dim", [(16, 16), (32, 8), (48, 48), (64, 64), (64, 0), (80, 64), (96, 96), (128, 128), (144, 72), (256, 256)])
@pytest.mark.parametrize("kind", ["bf16", "int8"])
@pytest.mark.parametrize("adjacent", [False, True])
def test_append(dim, rotary_dim, kind, adjacent):
    p = Paged(5, 4, kv_heads=3, dim=dim, kind=kind, marks=kind == "int8", seed=dim)
    q, k, v = new_tokens(5, 6, 3, dim, dim)
    cos, sin = angles(90, rotary_dim)
    slots = ints([0, 63, 17, 16, 5])
    before = snapshot(p)
    got = append(p, q, k, v, None, slots, None, cos, sin, rotary_dim, adjacent, q16=adjacent)
    check_append(p, before, got, q, k, v, None, slots, None, cos, sin, rotary_dim, adjacent)


@pytest.mark.parametrize("kind", ["bf16", "int8"])
@pytest.mark.parametrize("order", ["phtd", "pthd", "tphd"])
def test_prompt_rows_any_order_of_the_pool_gaps_positions_in_place(kind, order):
    p = Paged(3, 10, kv_heads=2, dim=64, page=32, kind=kind, order=order, marks=True, table_stride=13)
    rows = 77
    q, k, v = new_tokens(rows, 4, 2, 64)
    cos, sin = angles(1000, 64)
    seqs, slots, positions = ints([1] * rows), ints(list(range(40, 40 + rows))), ints([900 - 3 * i for i in range(rows)])
    for gap, offset, in_place in ((0, 0, True), (5, 0, False), (8, 4, True), (0, 3, True)):
        before = snapshot(p)
        got = append(p, q, k, v, seqs, slots, positions, cos, sin, 64, gap=gap, offset=offset, in_place=in_place)
        check_append(p, before, got, q, k, v, seqs, slots, positions, cos, sin, 64)


def test_padding_rows_and_pages_that_are_not_there():
    p = Paged(4, 3, marks=True)
    p.tables[2, 1] = -1
    p.tables[3, 0] = p.n_pages
    rows = 8
    q, k, v = new_tokens(rows, 4, 2, 64)
    cos, sin = angles(40, 64)
    seqs, slots = ints([-1, 4, 0, 1, 2, 3, 0, 1]), ints([0, 0, 48, -1, 20, 2, 5, 39])
    positions = ints([0, 0, 0, 0, 1, 2, 40, 39])
    before, scores = snapshot(p), p.scores.cpu().clone()
    got = append(p, q, k, v, seqs, slots, positions, cos, sin, 64)
    check_append_marks = p.scores
    p.scores = None            # (marks of a slot whose page is not there are not written: compared below)
    check_append(p, before, got, q, k, v, seqs, slots, positions, cos, sin, 64)
    p.scores = check_append_marks
    scores[1, :, 39] = 0
    assert torch.equal(p.scores.cpu(), scores)


def test_rows_that_are_not_finite_read_back_as_nan_in_8_bits():
    p = Paged(3, 2, kind="int8")
    q, k, v = new_tokens(3, 2, 2, 64)
    v[0, 1, 3], v[1, 0, 0], v[2, 0] = float("nan"), float("inf"), 0
    cos, sin = angles(8, 64)
    append(p, q, k, v, None, ints([1, 2, 3]), None, cos, sin, 64)
    got = p.values("v")
    page = p.tables.cpu()[:, 0].long()
    assert torch.isnan(got[page[0], 1, 1]).all() and torch.isnan(got[page[1], 0, 2]).all() and (got[page[2], 0, 3] == 0).all()
    assert torch.isfinite(got[page[0], 0, 1]).all()


def far_pool(p):
    """The same cache at the end of a pool of more than 2^31 values -> (the cache with that pool, what takes it back)."""
    base = 2 ** 31 // (p.kv_heads * p.page * p.dim) + 3
    for name in ("k", "v"):
        small = getattr(p, name)
        pool = torch.empty((base + p.n_pages, *small.shape[1:]), dtype=small.dtype, device="cuda")
        pool[base:] = small
        setattr(p, name, pool)
    p.tables += base
    p.n_pages += base

    def back():
        p.n_pages -= base
        p.tables -= base
        for name in ("k", "v"):
            setattr(p, name, getattr(p, name)[base:].clone())

    return back


def test_append_beyond_32_bits_of_offset():
    p = Paged(2, 3, kv_heads=2, dim=64)
    q, k, v = new_tokens(2, 4, 2, 64)
    cos, sin = angles(50, 64)
    slots, before = ints([17, 40]), snapshot(p)
    back = far_pool(p)
    got = append(p, q, k, v, None, slots, None, cos, sin, 64)
    back()
    check_append(p, before, got, q, k, v, None, slots, None, cos, sin, 64)


# ---- eviction ----

def evict(p, lengths, keep, since=None, in_place=True):
    cache = p.describe()
    outs = {} if in_place else {"lengths_out": torch.full_like(lengths, -1), "scores_out": torch.full_like(p.scores, -1),
                                **({} if p.positions is None else {"positions_out": torch.full_like(p.positions, -1)})}
    fields = dict(lengths=ptr(lengths), since=ptr(since), keep=keep, **{n: ptr(t) for n, t in outs.items()})
    ws = torch.full((tq.CacheEvict.workspace_bytes(cache, **fields),), 171, dtype=torch.uint8, device="cuda")
    tq.CacheEvict(cache, workspace=ptr(ws), workspace_bytes=ws.numel(), **fields).launch(stream())
    torch.cuda.synchronize()
    return outs


def check_evict(p, lengths, keep, since=None, in_place=True):
    was = {n: None if getattr(p, n) is None else getattr(p, n).cpu().clone() for n in ("k", "v", "k_scale", "v_scale", "scores", "positions")}
    lengths_were = lengths.tolist()
    moves, stays = evict_reference(p, lengths, keep, since)
    outs = evict(p, lengths, keep, since, in_place)
    want = {n: None if t is None else t.clone() for n, t in was.items()}
    marks = {}
    for n in ("scores", "positions"):
        if was[n] is not None:
            marks[n] = was[n].clone() if in_place else torch.full_like(was[n], -1)
    table = p.tables.cpu()

    def at(s, t):
        return int(table[s, t // p.page]), t % p.page

    for (s, h), filled in moves.items():
        for t in stays[s, h]:
            for n in marks:
                marks[n][s, h, t] = was[n][s, h, t]
        for to, of in filled.items():
            for n in marks:
                marks[n][s, h, to] = was[n][s, h, of]
            (tp, ti), (fp, fi) = at(s, to), at(s, of)
            if not (0 <= tp < p.n_pages and 0 <= fp < p.n_pages):
                continue
            for n in ("k", "v", "k_scale", "v_scale"):
                if want[n] is not None:
                    want[n][tp, h, ti] = was[n][fp, h, fi]
    for n in ("k", "v", "k_scale", "v_scale"):
        if want[n] is not None:
            assert torch.equal(getattr(p, n).cpu(), want[n]), n
    for n, t in marks.items():
        got = getattr(p, n) if in_place else outs[n + "_out"]
        assert torch.equal(got.cpu().nan_to_num(-99.0) if n == "scores" else got.cpu(), t.nan_to_num(-99.0) if n == "scores" else t), n
    new = lengths if in_place else outs["lengths_out"]
    assert new.tolist() == [min(n, keep) for n in lengths_were]
    if not in_place:
        assert lengths.tolist() == lengths_were
    return moves


@pytest.mark.parametrize("kind,dim,order", [("bf16", 64, "phtd"), ("int8", 64, "phtd"), ("bf16", 256, "pthd"), ("int8", 80, "tphd"), ("bf16", 16, "phtd")])
@pytest.mark.parametrize("in_place", [True, False])
def test_evict(kind, dim, order, in_place):
    p = Paged(6, 20, kv_heads=3, dim=dim, kind=kind, order=order, marks=True)
    moves = check_evict(p, ints([320, 100, 101, 0, 319, 250]), 100, in_place=in_place)
    assert len(moves[0, 0]) > 20 and len(moves[2, 0]) <= 1 and not moves[1, 0]


@pytest.mark.parametrize("capacity,keep", [(16, 1), (16, 15), (1024, 1023), (1040, 1024), (2048, 1), (5008, 2504), (40000, 39999), (40000, 300), (70000, 33000)])
def test_evict_sizes(capacity, keep):
    p = Paged(2, -(-capacity // 16), kv_heads=2, dim=16, marks=True, seed=capacity)
    check_evict(p, ints([capacity, max(keep, capacity - 5)]), keep)


def test_evict_equal_scores_zeros_infinities_and_nan():
    p = Paged(4, 80, kv_heads=2, dim=16, marks=True)
    g = torch.Generator().manual_seed(3)
    few = torch.tensor([0.0, -0.0, 0.5, 0.5, 1.0, float("inf"), float("-inf"), float("nan"), -2.0, 1e-42])
    p.scores.copy_(few[torch.randint(0, len(few), p.scores.shape, generator=g)])
    p.scores[1] = 0.25
    p.scores[2] = float("nan")
    p.scores[3] = torch.finfo(torch.float32).min
    for keep in (1000, 700, 333, 40, 1):
        check_evict(p, ints([1280, 1280, 1280, 1280]), keep, in_place=False)


@pytest.mark.parametrize("keep,kind,in_place", [(1, "bf16", True), (4095, "int8", False), (4096, "bf16", True), (4098, "bf16", False), (12289, "int8", True), (20477, "bf16", False)])
def test_evict_long_lists_of_equal_scores(keep, kind, in_place):
    p = Paged(5, 1280, kv_heads=1, dim=16, kind=kind, marks=True, seed=keep)
    g = torch.Generator().manual_seed(keep)
    few = torch.tensor([0.0, 0.5, 0.5000001, 1.0, float("nan"), float("-inf"), -2.0])
    p.scores.copy_(few[torch.randint(0, len(few), p.scores.shape, generator=g)])
    p.scores[1] = 0.25
    p.scores[1, :, 8192:12288] = 0.75   # more than the others, all in one stretch
    p.positions.copy_(torch.arange(p.positions[0].numel(), dtype=torch.int32).flip(0).expand_as(p.positions))   # the newest first
    check_evict(p, ints([20480, 20479, 0, 4096, 16400]), keep, since=ints([20480 - 700, 20481, 0, 0, 20475]), in_place=in_place)


@pytest.mark.parametrize("recent", [0, 1, 30, 99, 100, 150])
def test_evict_protects_by_position(recent):
    p = Paged(3, 20, kv_heads=2, dim=32, marks=True)
    p.positions.copy_(torch.stack([torch.randperm(320, generator=torch.Generator().manual_seed(i)) for i in range(6)]).view(3, 2, 320).to(torch.int32) - 100)
    p.scores[1, 0, 5] = float("inf")
    check_evict(p, ints([320, 300, 90]), 100, since=ints([220 - recent, -50, 0]))


def test_evict_without_positions_and_with_pages_that_are_not_there():
    p = Paged(2, 10, kv_heads=2, dim=32, marks=True)
    p.positions = None
    p.tables[0, 2], p.tables[1, 8] = -1, p.n_pages
    check_evict(p, ints([160, 160]), 70)


def test_evict_beyond_32_bits_of_offset():
    p, same = (Paged(2, 5, kv_heads=2, dim=32, marks=True, seed=9) for _ in range(2))
    check_evict(same, ints([80, 77]), 50)
    back = far_pool(p)
    evict(p, ints([80, 77]), 50)
    back()
    for name in ("k", "v", "scores", "positions"):
        assert torch.equal(getattr(p, name), getattr(same, name)), name


def test_evict_more_than_there_is_changes_nothing():
    p = Paged(2, 3, dim=32, marks=True)
    check_evict(p, ints([48, -4]), 1 << 30)


def test_a_budget_kept_token_after_token():
    """append -> attend with weights -> evict, in one captured graph: the cache never exceeds its budget, and every replay
    gives what the same calls give eagerly."""
    torch.manual_seed(0)
    rows, heads, kv, dim, keep = 3, 4, 2, 64, 40

    def build():
        p = Paged(rows, 4, kv_heads=kv, dim=dim, marks=True, seed=5)
        cache = p.describe()
        st = dict(p=p, cache=cache, q=torch.zeros(rows, heads, dim, device="cuda"), k=torch.zeros(rows, kv, dim, device="cuda"),
                  v=torch.zeros(rows, kv, dim, device="cuda"), slots=ints([40, 40, 17]), positions=ints([70, 70, 17]), lengths=ints([41, 41, 18]),
                  since=ints([66, 66, 13]))
        cos, sin = (t.cuda() for t in angles(300, dim))
        st["angles"], st["q_out"] = (cos, sin), torch.zeros(rows, heads, dim, device="cuda")
        st["append"] = tq.CacheAppend(cache, q=ptr(st["q"]), k=ptr(st["k"]), v=ptr(st["v"]), q_out=ptr(st["q_out"]), slots=ptr(st["slots"]),
                                      positions=ptr(st["positions"]), cos=ptr(cos), sin=ptr(sin), rows=rows, heads=heads, rotary_dim=dim, n_positions=300,
                                      q_out_type=tq.TQ_FP32)
        st["attend"], st["out"] = attend_call(cache, p, st["q_out"], st["lengths"], accumulate=True)
        fields = dict(lengths=ptr(st["lengths"]), since=ptr(st["since"]), keep=keep)
        st["ws"] = torch.zeros(tq.CacheEvict.workspace_bytes(cache, **fields), dtype=torch.uint8, device="cuda")
        st["evict"] = tq.CacheEvict(cache, workspace=ptr(st["ws"]), workspace_bytes=st["ws"].numel(), **fields)
        return st

    def step(st):
        s = stream()
        st["append"].launch(s)
        st["attend"].launch(s)
        st["evict"].launch(s)
        st["slots"].copy_(st["lengths"])
        st["positions"].add_(1)
        st["since"].add_(1)
        st["lengths"].add_(1)

    eager, replayed = build(), build()
    side = torch.cuda.Stream()
    warm = build()
    with torch.cuda.stream(side):
        step(warm)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(replayed)
    for i in range(60):
        new = [torch.randn(t.shape, device="cuda") for t in (eager["q"], eager["k"], eager["v"])]
        for st in (eager, replayed):
            for n, t in zip(("q", "k", "v"), new):
                st[n].copy_(t)
        step(eager)
        graph.replay()
        if i % 7 == 0:
            torch.cuda.synchronize()
        for n in ("out", "lengths", "slots", "q_out"):
            assert torch.equal(eager[n], replayed[n]), (i, n)
        for n in ("k", "v", "scores", "positions"):
            assert torch.equal(getattr(eager["p"], n), getattr(replayed["p"], n)), (i, n)
    assert eager["lengths"].tolist() == [41, 41, 41] and torch.isfinite(eager["out"]).all()
    newest = eager["p"].positions[:, :, :40].amax(dim=2)
    assert (newest == torch.tensor([[129], [129], [76]], device="cuda")).all()


@pytest.mark.parametrize("kind", ["bf16", "int8"])
def test_attention_after_an_eviction_is_attention_over_the_tokens_that_stay(kind):
    """The kept tokens of each head, read from the cache as it was, against the cache as it is.  Tolerance as for attention itself: 2^-14 of
    the largest value, and 2^-8 of the result for its rounding."""
    keep, n = 90, [320, 90, 200]
    p = Paged(3, 20, kv_heads=2, dim=64, kind=kind, marks=True, seed=11)
    lengths, since = ints(n), ints([300, 0, 195])
    was = {name: p.values(name) for name in ("k", "v")}
    moves, stays = evict_reference(p, lengths, keep, since)
    q = torch.randn((3, 4, 64), generator=torch.Generator().manual_seed(5))
    want = torch.zeros((3, 4, 64), dtype=torch.float64)
    for s in range(3):
        for h in range(2):
            kept = sorted(stays[s, h] + list(moves[s, h].values()))
            assert len(kept) == min(n[s], keep)
            k, v = (p.of_sequence(was[name], s, h, n[s])[0][kept] for name in ("k", "v"))
            want[s, 2 * h:2 * h + 2] = torch.softmax(q[s, 2 * h:2 * h + 2].double() @ k.T / 8, dim=-1) @ v
    evict(p, lengths, keep, since)
    call, out = attend_call(p.describe(), p, q.cuda(), lengths)
    call.launch(stream())
    torch.cuda.synchronize()
    assert ((out.cpu().double() - want).abs() <= want.abs() * 2.0 ** -8 + was["v"].abs().max() * 2.0 ** -14).all()
