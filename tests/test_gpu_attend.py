"""tq_attend against the formula in 64 bits.

Tolerances.  A logit in units of log 2 is a sum of fp32 products of exact operands: with dims of N(0, 1) keys and queries its terms
add up to some 2^5 in magnitude, so it is off by at most 2^5 * 2^-22, and a weight relatively as much; a weight enters the second
product with 16 bits (2^-17); the sums are fp32.  All in all 2^-15 of sum p |v| <= 2^-15 max |v|, taken twice; rounding the result
to bf16 adds 2^-8 of it.  Scores: the weights' 2^-15, taken twice, of what is added, and fp32's rounding of the sum."""
import pytest

torch = pytest.importorskip("torch")

import paper_2509_22951_amd as tq
from paged import Paged, attend_call, attend_reference, ptr, stream

pytestmark = pytest.mark.gpu


def queries(rows, heads, dim, seed=0, dtype=torch.float32):
    return torch.randn((rows, heads, dim), generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def close(out, want, p):
    vmax = p.values("v").nan_to_num(0, 0, 0).abs().max()
    off = (out.cpu().double() - want).abs()
    assert (off <= want.abs() * 2.0 ** -8 + vmax * 2.0 ** -14).all(), float((off - want.abs() * 2.0 ** -8).max() / vmax)


def run(p, q, lengths, **more):
    call, out = attend_call(p.describe(), p, q, lengths, **more)
    call.launch(stream())
    torch.cuda.synchronize()
    return out


@pytest.mark.parametrize("length", [1, 2, 15, 16, 17, 31, 33, 100, 127, 128, 129, 500, 1023, 1024, 1025, 2000, 4100])
@pytest.mark.parametrize("kind", ["bf16", "int8"])
def test_lengths(length, kind):
    p = Paged(2, -(-length // 16) + 1, kind=kind, seed=length)
    q = queries(2, 8, 64, length)
    lengths = ints([length, max(1, length - 7)])
    close(run(p, q, lengths), attend_reference(p, q, lengths)[0], p)


@pytest.mark.parametrize("dim", [16, 32, 48, 64, 80, 96, 112, 128, 144, 192, 240, 256])
@pytest.mark.parametrize("kind", ["bf16", "int8"])
def test_head_dims(dim, kind):
    p = Paged(3, 5, dim=dim, page=32, kind=kind, seed=dim)
    q = queries(3, 6, dim, dim)
    lengths = ints([150, 7, 64])
    close(run(p, q, lengths), attend_reference(p, q, lengths)[0], p)


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (2, 2), (3, 1), (8, 1), (9, 1), (16, 1), (24, 8), (20, 4), (34, 2), (71, 1)])
@pytest.mark.parametrize("kind", ["bf16", "int8"])
def test_groups_of_query_heads(heads, kv_heads, kind):
    p = Paged(2, 5, kv_heads=kv_heads, dim=64, kind=kind, seed=heads)
    q = queries(2, heads, 64, heads)
    lengths = ints([70, 33])
    close(run(p, q, lengths), attend_reference(p, q, lengths)[0], p)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 1024])
def test_pages(page):
    for kind in ("bf16", "int8"):
        p = Paged(3, -(-1500 // page), page=page, kind=kind, seed=page)
        q = queries(3, 4, 64, page)
        lengths = ints([1500, 1, 777])
        close(run(p, q, lengths), attend_reference(p, q, lengths)[0], p)


@pytest.mark.parametrize("order", ["pthd", "hptd", "tphd"])
@pytest.mark.parametrize("kind", ["bf16", "int8"])
def test_pools_in_another_order_with_gaps(order, kind):
    p = Paged(2, 6, kv_heads=3, dim=80, kind=kind, order=order, table_stride=11)
    q = queries(2, 6, 80)
    lengths = ints([90, 41])
    close(run(p, q, lengths), attend_reference(p, q, lengths)[0], p)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_query_types_strides_and_addresses(dtype):
    p = Paged(3, 4, dim=64)
    buf = queries(3, 9, 64, dtype=dtype).view(3, -1)
    q = buf.as_strided((3, 8, 64), (buf.stride(0), 64, 1), 3)
    out = torch.full((3, 700), 7, dtype=torch.bfloat16, device="cuda")
    lengths = ints([60, 3, 17])
    o = out.as_strided((3, 8, 64), (700, 64, 1), 1)
    run(p, q, lengths, out=o, q_stride=buf.stride(0), out_stride=700)
    close(o, attend_reference(p, q, lengths)[0], p)
    assert (out[:, 0] == 7).all() and (out[:, 513:] == 7).all()


def test_rows_without_tokens_and_sequences_that_are_not_there():
    p = Paged(4, 3)
    q = queries(6, 4, 64)
    lengths, seqs = ints([0, -5, 20, 20, 48, 99999]), ints([0, 1, -1, 4, 3, 2])
    out = run(p, q, lengths, seqs=seqs)
    assert (out[:4] == 0).all()
    close(out, attend_reference(p, q, lengths, seqs)[0], p)


@pytest.mark.parametrize("kind", ["bf16", "int8"])
def test_what_lies_beyond_a_length_is_not_used(kind):
    p = Paged(3, 4, kind=kind)
    q = queries(3, 4, 64)
    lengths = ints([0, 21, 33])
    want = attend_reference(p, q, lengths)[0]
    for s, n in enumerate([0, 21, 33]):
        for t in range(n, p.capacity):
            p.set_slot(s, t, [float("nan"), float("inf"), float("-inf"), torch.finfo(torch.bfloat16).min][t % 4])
    close(run(p, q, lengths), want, p)


@pytest.mark.parametrize("kind", ["bf16", "int8"])
def test_pages_that_are_not_there_are_masked(kind):
    p = Paged(3, 80, kind=kind)
    p.tables[0, ::2] = -1
    p.tables[1] = p.n_pages
    p.tables[2, 0], p.tables[2, 1], p.tables[2, 70:] = -1, 2 ** 31 - 1, -7
    q = queries(3, 4, 64)
    lengths = ints([1280, 1280, 1279])
    out = run(p, q, lengths)
    assert (out[1] == 0).all()
    close(out, attend_reference(p, q, lengths)[0], p)


def test_large_logits_and_equal_ones():
    p = Paged(2, 70)
    p.k[:] = p.k * 30
    q = queries(2, 4, 64) * 20
    q[1] = 0
    lengths = ints([1100, 1100])
    want, _ = attend_reference(p, q, lengths)
    out = run(p, q, lengths)
    # logits in the thousands: their fp32 error, 2^13 * 2^-22, is what their weights are off
    vmax = p.values("v").abs().max()
    assert ((out[0].cpu().double() - want[0]).abs() <= want[0].abs() * 2.0 ** -8 + vmax * 2.0 ** -8).all()
    close(out[1], want[1], p)


def test_a_nan_within_the_length_reaches_the_result():
    p = Paged(2, 70)
    p.set_slot(0, 1050, float("nan"))
    q = queries(2, 4, 64)
    lengths = ints([1060, 1060])
    out = run(p, q, lengths)
    assert torch.isnan(out[0]).all() and torch.isfinite(out[1]).all()


def test_rows_of_one_sequence_are_a_causal_prompt():
    p = Paged(2, 10, kv_heads=2)
    q = queries(40, 4, 64)
    lengths, seqs = ints(list(range(100, 140))), ints([1] * 40)
    close(run(p, q, lengths, seqs=seqs), attend_reference(p, q, lengths, seqs)[0], p)


@pytest.mark.parametrize("kind", ["bf16", "int8"])
@pytest.mark.parametrize("heads,kv_heads,dim", [(8, 2, 64), (24, 8, 128), (18, 2, 96), (4, 4, 256)])
def test_weights_are_added_to_the_scores(kind, heads, kv_heads, dim):
    p = Paged(4, 90, kv_heads=kv_heads, dim=dim, kind=kind, marks=True)
    before = p.scores.cpu().double()
    q = queries(4, heads, dim)
    lengths = ints([1333, 0, 17, 1440])
    out = run(p, q, lengths, accumulate=True)
    want, added = attend_reference(p, q, lengths)
    close(out, want, p)
    off = (p.scores.cpu().double() - before - added).abs()
    assert (off <= added * 2.0 ** -14 + (before + added) * 2.0 ** -23).all(), float(off.max())
    untouched = added == 0
    assert torch.equal(p.scores.cpu()[untouched], before.float()[untouched])


def test_scores_of_several_rows_of_one_sequence_and_again():
    p = Paged(3, 6, marks=True)
    before = p.scores.cpu().double()
    q = queries(5, 4, 64)
    lengths, seqs = ints([50, 51, 20, 52, 9]), ints([2, 2, 0, 2, 7])
    call, out = attend_call(p.describe(), p, q, lengths, seqs=seqs, accumulate=True)
    for _ in range(3):
        call.launch(stream())
    torch.cuda.synchronize()
    want, added = attend_reference(p, q, lengths, seqs)
    close(out, want, p)
    off = (p.scores.cpu().double() - before - 3 * added).abs()
    assert (off <= added * 2.0 ** -12 + (before + 3 * added) * 2.0 ** -21).all()


def test_results_repeat_and_the_workspace_serves_calls_of_any_lengths():
    p = Paged(5, 130, kv_heads=2, dim=128, page=32, marks=True)
    q = queries(5, 6, 128)
    lengths = ints([1, 1, 1, 1, 1])
    call, out = attend_call(p.describe(), p, q, lengths, accumulate=True)
    seen = {}
    for n in ([4000, 3, 0, 2047, 1024], [1, 1, 1, 1, 1], [4160, 4160, 4160, 4160, 4160], [4000, 3, 0, 2047, 1024], [0, 0, 0, 0, 0], [4000, 3, 0, 2047, 1024]):
        lengths.copy_(ints(n))
        p.scores.zero_()
        call.launch(stream())
        torch.cuda.synchronize()
        close(out, attend_reference(p, q, lengths)[0], p)
        key = tuple(n)
        if key in seen:
            assert torch.equal(seen[key][0], out) and torch.equal(seen[key][1], p.scores)
        seen[key] = (out.clone(), p.scores.clone())


def test_a_pool_beyond_32_bits_of_offset():
    """Pages more than 2^31 elements into the pool."""
    p = Paged(1, 4, kv_heads=2, dim=64)
    base = 2 ** 31 // (2 * 16 * 64) + 5
    far = p.n_pages + base
    for name in ("k", "v"):
        pool = torch.empty((far, 2, 16, 64), dtype=torch.bfloat16, device="cuda")
        pool[base:] = getattr(p, name)
        setattr(p, name, pool)
    q = queries(1, 4, 64)
    lengths = ints([60])
    p.tables += base
    p.n_pages = far
    out = run(p, q, lengths)
    p.k, p.v = p.k[base:].clone(), p.v[base:].clone()
    p.tables -= base
    p.n_pages -= base
    close(out, attend_reference(p, q, lengths)[0], p)


def test_many_rows_and_another_stream():
    """More rows than a wavefront has lanes, some without tokens, on a stream of their own."""
    p = Paged(150, 3, kv_heads=2, dim=32)
    q = queries(150, 2, 32)
    lengths = ints([(7 * r) % 49 if r % 5 else 0 for r in range(150)])
    want = attend_reference(p, q, lengths)[0]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out = run(p, q, lengths)
    close(out, want, p)


@pytest.mark.parametrize("kind,track", [("bf16", False), ("int8", True), ("bf16", True)])
@pytest.mark.parametrize("rows,longest,heads,kv_heads,dim", [
    (16, 500, 8, 8, 64), (16, 700, 16, 8, 64), (17, 1000, 8, 8, 64), (40, 1000, 20, 10, 64), (16, 700, 8, 8, 128), (64, 760, 8, 8, 96), (33, 400, 12, 6, 256),
    (16, 1270, 8, 8, 64), (4, 5100, 34, 2, 64), (11, 2900, 8, 8, 128), (2, 20000, 3, 3, 64), (65, 1100, 4, 4, 64),
    (12, 2000, 4, 4, 192), (12, 2000, 2, 2, 80)])
def test_how_rows_are_cut(rows, longest, heads, kv_heads, dim, kind, track):
    """Rows that are as long as each other, spread, and with one of them far longer: not cut, cut at whole shares, cut anywhere; twice with one workspace."""
    p = Paged(rows, -(-longest // 16), kv_heads=kv_heads, dim=dim, kind=kind, marks=track, seed=rows)
    q = queries(rows, heads, dim, longest)
    for lengths in ([longest] * rows, [(r * 619 + 5) % (longest + 1) for r in range(rows)], [longest if r == rows // 2 else r for r in range(rows)]):
        lengths = ints(lengths)
        call, out = attend_call(p.describe(), p, q, lengths, accumulate=track)
        want = attend_reference(p, q, lengths)[0]
        for _ in range(2):
            out.fill_(float("nan"))
            call.launch(stream())
            torch.cuda.synchronize()
            close(out, want, p)


@pytest.mark.parametrize("heads,kv_heads,dim,rows", [(8, 1, 256, 1), (5, 1, 128, 2), (2, 1, 64, 1), (16, 1, 64, 3)])
def test_rows_that_many_workgroups_share(heads, kv_heads, dim, rows):
    """Up to 160 parts of one row: joined by clusters first; rows that begin and end inside a cluster."""
    p = Paged(rows, 2600, kv_heads=kv_heads, dim=dim)
    q = queries(rows, heads, dim)
    for n in ([41600, 9000, 41500], [4096, 41600, 300], [20000, 0, 30001]):
        lengths = ints(n[:rows])
        call, out = attend_call(p.describe(), p, q, lengths)
        want = attend_reference(p, q, lengths)[0]
        for _ in range(2):
            call.launch(stream())
            torch.cuda.synchronize()
            close(out, want, p)


@pytest.mark.parametrize("kind", ["bf16", "int8"])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_weights_enter_the_sum_with_all_their_bits(kind, dim):
    """Large terms that cancel, so that the result's own rounding to bf16 hides nothing.

    Keys are unit vectors, so a logit is one product: q * (scale * log2 e) with two roundings of 2^-24 of a factor of 2^-24 itself, 2^-22.4 of
    the logit, which is at most 0.5; a weight is off by ln 2 * (2 * 0.5 * 2^-22.4 + 2^-25) and exp2's last place, 2^-23: 2^-21.8 of it, twice that
    beside the total.  Products of 24 and 8 bits are exact; some ten additions at 2^-24: 2^-19.8 of sum p |v| in all, taken as 2^-19."""
    rows, heads, scale = 40, 4, 0.125
    p = Paged(rows, 1, kv_heads=heads, dim=dim, kind=kind)
    g = torch.Generator().manual_seed(dim)
    q = torch.zeros((rows, heads, dim))
    q[..., 0], q[..., 1:4] = 2.7, 1 + 1.6 * torch.rand((rows, heads, 3), generator=g)
    w = torch.exp(q[..., :4].double() * scale)
    w /= w.sum(dim=-1, keepdim=True)
    one = (1 + torch.rand((rows, heads, dim), generator=g)) * torch.where(torch.rand((rows, heads, dim), generator=g) < 0.5, -1, 1)
    v = torch.zeros((rows, heads, 4, dim), dtype=torch.float64)
    k, k_scale, v_scale = torch.zeros((rows, heads, 4, dim)), torch.full((rows, heads, 4), 2.0 ** -6), torch.ones((rows, heads, 4))
    if kind == "bf16":
        v[:, :, 1] = one.to(torch.bfloat16).double()
        for t in (2, 3):      # what is left, divided by this token's weight
            v[:, :, t] = (-(w[..., None] * v).sum(dim=2) / w[..., t, None]).float().to(torch.bfloat16).double()
        k[..., range(4), range(4)] = 1
        levels = v
    else:
        levels = torch.zeros_like(v)
        levels[:, :, 1] = levels[:, :, 2] = torch.round(one * 60).double()
        levels[:, :, 3] = -levels[:, :, 1]
        v_scale[..., 1:3] = 0.5 + torch.rand((rows, heads, 2), generator=g)
        v_scale[..., 3] = ((w[..., 1:3] * v_scale[..., 1:3].double()).sum(dim=-1) / w[..., 3]).float()
        v = levels * v_scale.double()[..., None]
        k[..., range(4), range(4)] = 64
    pages = p.tables[:, 0].cpu().long()
    for name, t, s in (("k", k, k_scale), ("v", levels, v_scale)):
        getattr(p, name)[pages.cuda(), :, :4] = t.to(getattr(p, name).dtype).cuda()
        if kind == "int8":
            getattr(p, name + "_scale")[pages.cuda(), :, :4] = s.cuda()
    lengths = ints([4] * rows)
    out = run(p, q.cuda(), lengths, scale=scale)
    want, size = (w[..., None] * v).sum(dim=2), (w[..., None] * v.abs()).sum(dim=2)
    assert (attend_reference(p, q, lengths, scale=scale)[0] - want).abs().max() < 2.0 ** -40
    assert (want.abs() < size * 2.0 ** -12).all()
    off = (out.cpu().double() - want).abs()
    assert (off <= want.abs() * 2.0 ** -8 + size * 2.0 ** -19).all(), float((off / size).max() * 2 ** 19)


def test_one_workspace_serves_calls_of_any_rows_and_heads():
    """Every row is cut between workgroups in every call, and what one call leaves in the workspace is not what the next one expects there."""
    p = Paged(16, 256, kv_heads=8, dim=64, marks=True)
    calls = []
    for rows, heads, track in [(4, 8, False), (16, 8, False), (1, 8, True), (16, 72, False), (7, 24, True), (16, 8, True)]:
        q = queries(rows, heads, 64, rows + heads)
        lengths = ints([4096 - 300 * (r % 3) for r in range(rows)])
        n = tq.Attend.workspace_bytes(p.describe(), q=ptr(q), lengths=ptr(lengths), rows=rows, heads=heads, scale=0.125, q_type=tq.TQ_FP32, accumulate=int(track))
        calls.append((rows, q, lengths, track, n, attend_reference(p, q, lengths)))
    ws = torch.zeros(max(c[4] for c in calls), dtype=torch.uint8, device="cuda")
    for _ in range(2):
        for rows, q, lengths, track, _, (want, added) in calls:
            p.scores.zero_()
            close(run(p, q, lengths, accumulate=track, workspace=ws), want, p)
            if track:
                assert ((p.scores.cpu().double() - added).abs() <= added * 2.0 ** -14 + added * 2.0 ** -23).all()


def agrees(out, want, vmax):
    """As close(), with infinities and NaN where the formula has them."""
    out = out.cpu().double()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(out), torch.isnan(want)) and torch.equal(torch.isinf(out), torch.isinf(want))
    assert torch.equal(out[torch.isinf(want)], want[torch.isinf(want)])
    off = (out - want).abs()[fine]
    assert (off <= want[fine].abs() * 2.0 ** -8 + vmax * 2.0 ** -14).all()


INF = float("inf")


@pytest.mark.parametrize("dim,length,rows,track", [(64, 40, 2, False), (80, 300, 3, True), (128, 2100, 2, False), (128, 9000, 1, True), (208, 700, 2, False),
                                                   (256, 20000, 1, False), (64, 41600, 1, True), (16, 77, 2, True)])
def test_infinities_within_a_length_do_what_the_formula_says(dim, length, rows, track):
    """A key of -inf (towards this query) takes its token's weight, one of +inf makes the row NaN; an infinite value reaches its own dim alone."""
    p = Paged(rows, -(-length // 16), kv_heads=4, dim=dim, marks=track, seed=dim)
    q = queries(rows, 8, dim, length)
    vmax = p.values("v").abs().max()
    some = sorted({0, 16, 17, length // 2, length - 1})
    for s in range(rows):
        for t in some:
            page, at = int(p.tables[s, t // 16]), t % 16
            for h in range(4):      # heads 2 h and 2 h + 1 may see the same key on two sides: one of them is NaN
                p.k[page, h, at, 3] = -INF if q[s, 2 * h, 3] > 0 else INF
        page = int(p.tables[s, some[2] // 16])
        p.v[page, 1, some[2] % 16, 5], p.v[page, 2, some[2] % 16, 6] = INF, -INF      # of a token without weight
        page = int(p.tables[s, (length - 2) // 16])
        p.v[page, 3, (length - 2) % 16, 7], p.v[page, 3, (length - 2) % 16, 8] = INF, -INF
    lengths = ints([length] * rows)
    before = p.scores.cpu().double() if track else None
    out = run(p, q, lengths, accumulate=track)
    want, added = attend_reference(p, q, lengths)
    assert torch.isfinite(want[:, 0]).all() and torch.isnan(want).any() and torch.isinf(want[:, 6]).any()
    agrees(out, want, vmax)
    if track:
        got, fine = p.scores.cpu().double(), torch.isfinite(added)
        assert torch.equal(torch.isnan(got), ~fine)
        assert ((got - before - added).abs()[fine] <= (added * 2.0 ** -14 + (before + added) * 2.0 ** -23)[fine]).all()


@pytest.mark.parametrize("kind", ["bf16", "int8"])
def test_queries_that_are_not_finite_stay_in_their_heads(kind):
    p = Paged(2, 20, kind=kind)
    q = queries(2, 8, 64)
    lengths = ints([310, 33])
    want = attend_reference(p, q, lengths)[0]
    q[0, 1, 5], q[0, 6, 0], q[1, 3, 63] = INF, float("nan"), -INF
    out = run(p, q, lengths)
    odd = torch.zeros((2, 8), dtype=torch.bool)
    odd[0, 1] = odd[0, 6] = odd[1, 3] = True
    assert torch.isnan(out.cpu()[odd]).all()
    off = (out.cpu().double() - want).abs()[~odd]
    assert (off <= want[~odd].abs() * 2.0 ** -8 + p.values("v").abs().max() * 2.0 ** -14).all()


@pytest.mark.parametrize("kind", ["bf16", "int8"])
def test_a_nan_value_reaches_the_result_whatever_its_weight(kind):
    """0 * NaN is NaN: a token whose weight is too small for a number is still there."""
    p = Paged(1, 5, kv_heads=1, dim=32, kind=kind)
    q = queries(1, 2, 32)
    q[0, 1] = q[0, 0]
    page, at = int(p.tables[0, 2]), 4
    if kind == "int8":
        p.k[page, 0, at], p.k_scale[page, 0, at] = torch.where(q[0, 0] > 0, -127, 127).to(torch.int8), 50.0
        p.v_scale[page, 0, at] = float("nan")
    else:
        p.k[page, 0, at], p.v[page, 0, at] = torch.where(q[0, 0] > 0, -6000.0, 6000.0).to(torch.bfloat16), float("nan")
    lengths = ints([70])
    assert torch.isnan(attend_reference(p, q, lengths)[0]).all()
    assert torch.isnan(run(p, q, lengths)).all()


def test_a_row_whose_logits_are_all_minus_infinity_gives_zeros():
    p = Paged(2, 40, marks=True)
    q = queries(2, 2, 64).abs()
    p.k[p.tables[0].long(), :, :, 9] = -INF
    lengths = ints([600, 600])
    before = p.scores[0].clone()
    out = run(p, q, lengths, accumulate=True)
    assert (out[0] == 0).all() and torch.equal(p.scores[0], before)
    close(out[1:], attend_reference(p, q, lengths)[0][1:], p)


@pytest.mark.parametrize("dim", [16, 80, 128, 208, 256])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_queries_at_any_address_of_their_type(dim, dtype):
    """Rows with odd strides, from addresses one after another; the last row ends where the buffer does."""
    p = Paged(3, 3, kv_heads=2, dim=dim, kind="int8" if dim == 80 else "bf16")
    lengths, stride = ints([40, 7, 48]), 4 * dim + 1
    for first in range(3):
        buf = queries(1, 1, first + 2 * stride + 4 * dim, first, dtype).view(-1)
        q = buf.as_strided((3, 4, dim), (stride, dim, 1), first)
        close(run(p, q, lengths, q_stride=stride), attend_reference(p, q, lengths)[0], p)


@pytest.mark.parametrize("rows,n,heads,kv_heads,dim", [(1, [41600], 3, 1, 64), (2, [20000, 9001], 2, 1, 128), (3, [41500, 300, 30001], 4, 2, 64), (1, [30000], 2, 1, 256),
                                                       (16, [1270 - 3 * r for r in range(16)], 4, 4, 64), (5, [5000, 2000, 257, 4097, 3333], 8, 8, 128), (40, [1000] * 40, 10, 10, 64)])
@pytest.mark.parametrize("kind", ["bf16", "int8"])
def test_every_token_at_a_cut_counts_once(rows, n, heads, kv_heads, dim, kind):
    """The first and last tokens of all stretches of 256, where shares, units and clusters are cut, have nearly all of the weight: the result without
    one of them, or with one twice, is beyond the tolerance, as the reference itself shows."""
    p = Paged(rows, -(-max(n) // 16), kv_heads=kv_heads, dim=dim, kind=kind, seed=rows)
    q = queries(rows, heads, dim, max(n))
    q[..., 0] = 8
    edges = [sorted({t for t in range(length) if t % 256 in (0, 255)} | {length - 1}) for length in n]
    for s in range(rows):
        t = torch.tensor(edges[s])
        pages = p.tables[s].cpu().long()[t // 16].cuda()
        if kind == "bf16":
            p.k[pages, :, (t % 16).cuda(), 0] = dim ** 0.5
        else:      # the other dims keep their levels: this one is the largest
            p.k[pages, :, (t % 16).cuda()] = 0
            p.k[pages, :, (t % 16).cuda(), 0] = 127
            p.k_scale[pages, :, (t % 16).cuda()] = dim ** 0.5 / 127
    lengths = ints(n)
    want = attend_reference(p, q, lengths)[0]
    close(run(p, q, lengths), want, p)
    keys, vals, group = p.values("k"), p.values("v"), heads // kv_heads
    bound = p.values("v").abs().max() * 2.0 ** -14
    for s in {0, rows - 1}:
        k, _ = p.of_sequence(keys, s, 0, n[s])
        v, _ = p.of_sequence(vals, s, 0, n[s])
        w = torch.softmax(q[s, :group].cpu().double() @ k.T / dim ** 0.5, dim=-1)
        assert w[:, edges[s]].sum(dim=1).min() > 0.5
        for t in edges[s][:: max(1, len(edges[s]) // 8)]:
            for wrong in (1 - w[:, t], 1 + w[:, t]):      # the total without this token, and with it twice
                other = (w @ v + (wrong - 1)[:, None] * v[t]) / wrong[:, None]
                assert ((other - want[s, :group]).abs() > want[s, :group].abs() * 2.0 ** -8 + bound).any()


@pytest.mark.parametrize("kind", ["bf16", "int8"])
@pytest.mark.parametrize("order", ["pthd", "tphd"])
def test_what_is_not_finite_in_pools_of_any_order_with_pages_that_are_not_there(kind, order):
    """bf16 queries, keys and values (or their scales) that are not finite in some tokens, two chunks of query heads, weights added up."""
    p = Paged(3, 60, kv_heads=2, dim=80, kind=kind, order=order, marks=True, table_stride=70, seed=3)
    p.tables[0, 5], p.tables[1, 0], p.tables[2, 59] = -1, p.n_pages, -1
    q = queries(3, 18, 80, dtype=torch.bfloat16).abs()
    vmax = p.values("v").abs().max()
    lengths = ints([950, 333, 960])
    for s, t in ((0, 17), (0, 400), (1, 300), (2, 940)):
        page, at = int(p.tables[s, t // 16]), t % 16
        if kind == "bf16":
            p.k[page, 0, at, 11] = -INF
            p.v[page, 1, at, 3] = INF
        elif s == 0:
            p.v_scale[page, 1, at] = float("nan")
        else:
            p.k_scale[page, 1, at] = float("nan")
    before = p.scores.cpu().double()
    out = run(p, q, lengths, accumulate=True)
    want, added = attend_reference(p, q, lengths)
    assert torch.isfinite(want[:, :9]).all() and not torch.isfinite(want[:, 9:]).all()
    agrees(out, want, vmax)
    got, fine = p.scores.cpu().double(), torch.isfinite(added)
    there = torch.zeros_like(fine)
    for s in range(3):
        for h in range(2):
            there[s, h, :int(lengths[s])] = p.of_sequence(p.values("k"), s, h, int(lengths[s]))[1]
    assert torch.equal(torch.isnan(got)[there], ~fine[there])
    fine &= there
    assert ((got - before - added).abs()[fine] <= (added * 2.0 ** -14 + (before + added) * 2.0 ** -23)[fine]).all()
