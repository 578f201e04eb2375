"""tq_attend_tree against the formula in 64 bits.

Tolerances as of tq_attend: a logit in units of log 2 is a sum of fp32 products of exact operands whose terms add up to some 2^5 in magnitude, off by at
most 2^5 * 2^-22, and a weight relatively as much; sums are fp32: 2^-15 of sum p |v| <= 2^-15 max |v|, taken twice; rounding the result to
bf16 adds 2^-8 of it."""
import pytest

torch = pytest.importorskip("torch")

import paper_2509_22951_amd as tq
from drafts import bits_of, ints, masks_of, random_parents, tree_call, tree_reference
from paged import Paged, attend_call, ptr, stream

pytestmark = pytest.mark.gpu


def queries(trees, nodes, heads, dim, seed=0, dtype=torch.float32):
    return torch.randn((trees, nodes, heads, dim), generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def close(out, want, p, scale=1.0):
    vmax = p.values("v").nan_to_num(0, 0, 0).abs().max()
    off = (out.cpu().double() - want).abs()
    assert (off <= want.abs() * 2.0 ** -8 + vmax * 2.0 ** -14 * scale).all(), float((off - want.abs() * 2.0 ** -8).max() / vmax)


def run(p, q, lengths, bits, **more):
    call, out = tree_call(p.describe(), q, lengths, masks_of(bits), **more)
    call.launch(stream())
    torch.cuda.synchronize()
    return out


@pytest.mark.parametrize("length", [0, 1, 15, 16, 17, 31, 33, 60, 63, 64, 65, 127, 128, 129, 500, 1023, 1025, 2000, 4100])
@pytest.mark.parametrize("kind", ["bf16", "int8"])
def test_lengths(length, kind):
    p = Paged(2, -(-length // 16) + 1, kind=kind, seed=length)
    bits = bits_of(random_parents(2, 11, length))
    q = queries(2, 11, 8, 64, length)
    lengths = ints([length, max(0, length - 7)])
    close(run(p, q, lengths, bits), tree_reference(p, q, lengths, bits), p)


@pytest.mark.parametrize("dim", [16, 32, 48, 64, 80, 96, 112, 128, 144, 192, 240, 256])
@pytest.mark.parametrize("kind", ["bf16", "int8"])
def test_head_dims(dim, kind):
    p = Paged(3, 6, dim=dim, page=32, kind=kind, seed=dim)
    bits = bits_of(random_parents(3, 9, dim))
    q = queries(3, 9, 6, dim, dim)
    lengths = ints([150, 7, 64])
    close(run(p, q, lengths, bits), tree_reference(p, q, lengths, bits), p)


@pytest.mark.parametrize("nodes", [1, 2, 3, 5, 7, 8, 15, 16, 17, 31, 33, 48, 63, 64])
@pytest.mark.parametrize("heads,kv_heads,kind", [(2, 2, "bf16"), (6, 2, "int8"), (8, 1, "bf16")])
def test_nodes(nodes, heads, kv_heads, kind):
    p = Paged(2, 24, kv_heads=kv_heads, kind=kind, seed=nodes)
    bits = bits_of(random_parents(2, nodes, nodes))
    q = queries(2, nodes, heads, 64, nodes)
    lengths = ints([300, 33])
    close(run(p, q, lengths, bits), tree_reference(p, q, lengths, bits), p)


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (3, 1), (9, 1), (16, 1), (24, 8), (20, 4), (34, 2), (71, 1)])
@pytest.mark.parametrize("kind,dim", [("bf16", 128), ("int8", 64)])
def test_groups_of_query_heads(heads, kv_heads, kind, dim):
    p = Paged(2, 7, kv_heads=kv_heads, dim=dim, kind=kind, seed=heads)
    bits = bits_of(random_parents(2, 12, heads))
    q = queries(2, 12, heads, dim, heads)
    lengths = ints([70, 33])
    close(run(p, q, lengths, bits), tree_reference(p, q, lengths, bits), p)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 1024])
@pytest.mark.parametrize("kind", ["bf16", "int8"])
def test_pages(page, kind):
    p = Paged(3, -(-1520 // page), page=page, kind=kind, seed=page)
    bits = bits_of(random_parents(3, 16, page))
    q = queries(3, 16, 4, 64, page)
    lengths = ints([1500, 1, 777])
    close(run(p, q, lengths, bits), tree_reference(p, q, lengths, bits), p)


@pytest.mark.parametrize("order", ["pthd", "hptd", "tphd"])
@pytest.mark.parametrize("kind", ["bf16", "int8"])
def test_pools_in_another_order_with_gaps(order, kind):
    p = Paged(2, 8, kv_heads=3, dim=80, kind=kind, order=order, table_stride=11)
    bits = bits_of(random_parents(2, 10))
    q = queries(2, 10, 6, 80)
    lengths = ints([90, 41])
    close(run(p, q, lengths, bits), tree_reference(p, q, lengths, bits), p)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dim", [64, 80])
def test_query_types_strides_and_addresses(dtype, dim):
    p = Paged(3, 5, dim=dim)
    bits = bits_of(random_parents(3, 6))
    buf = queries(18, 1, 9, dim, dtype=dtype).view(18, -1)
    q = buf.as_strided((3, 6, 8, dim), (6 * buf.stride(0), buf.stride(0), dim, 1), 3)
    out = torch.full((18, 8 * dim + 100), 7, dtype=torch.bfloat16, device="cuda")
    o = out.as_strided((3, 6, 8, dim), (6 * out.stride(0), out.stride(0), dim, 1), 1)
    lengths = ints([60, 3, 17])
    run(p, q, lengths, bits, out=o, q_stride=buf.stride(0), out_stride=out.stride(0))
    close(o, tree_reference(p, q, lengths, bits), p)
    assert (out[:, 0] == 7).all() and (out[:, 8 * dim + 1:] == 7).all()


def test_sizes_sequences_that_are_not_there_and_the_end_of_the_room():
    p = Paged(4, 3)                                   # 48 tokens of room
    bits = bits_of(random_parents(7, 8))
    q = queries(7, 8, 4, 64)
    lengths, seqs, sizes = ints([20, -5, 20, 20, 44, 99999, 48]), ints([0, 1, -1, 4, 3, 2, 0]), ints([5, 8, 8, 8, 8, 3, 99])
    lengths[6], seqs[6] = 0, 1                        # (two trees read one sequence: nothing is written there)
    out = run(p, q, lengths, bits, seqs=seqs, sizes=sizes)
    close(out, tree_reference(p, q, lengths, bits, sizes, seqs), p)
    assert (out[2:4] == 0).all() and (out[0, 5:] == 0).all() and (out[5, 3:] == 0).all() and (out[4, 4:].float().abs().sum() > 0)
    out = run(p, q, lengths, bits, seqs=seqs, sizes=ints([0, -3, 0, 0, 0, 0, 0]))
    assert (out == 0).all()


def test_masks_that_leave_nothing_that_see_anything_and_only_others():
    p = Paged(3, 8)
    bits = [[0] * 64, [(1 << 64) - 1] * 64, [(1 << 63) >> i for i in range(64)]]
    q = queries(3, 64, 4, 64)
    for n in ([0, 0, 0], [0, 17, 40], [33, 1, 0]):
        lengths = ints(n)
        out = run(p, q, lengths, bits)
        close(out, tree_reference(p, q, lengths, bits), p)
        if n[0] == 0:
            assert (out[0] == 0).all()


def test_a_chain_is_what_attend_gives_for_rising_lengths():
    p = Paged(2, 30, dim=128)
    nodes, lengths = 16, ints([400, 123])
    q = queries(2, nodes, 8, 128)
    out = run(p, q, lengths, bits_of([list(range(-1, nodes - 1))] * 2))
    rising = (lengths[:, None] + torch.arange(1, nodes + 1, device="cuda")[None, :]).to(torch.int32).view(-1)
    seqs = ints([0] * nodes + [1] * nodes)
    call, rows = attend_call(p.describe(), p, q.view(2 * nodes, 8, 128), rising, seqs=seqs)
    call.launch(stream())
    torch.cuda.synchronize()
    close(out.view(2 * nodes, 8, 128), rows.cpu().double(), p, scale=2)


@pytest.mark.parametrize("kind", ["bf16", "int8"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_what_a_node_does_not_attend_to_is_not_used(kind, bad):
    p = Paged(3, 5, kind=kind)
    bits = bits_of(random_parents(3, 8))
    q = queries(3, 8, 4, 64)
    lengths, sizes = ints([0, 21, 33]), ints([8, 6, 8])
    want = tree_reference(p, q, lengths, bits, sizes)
    for s, n in ((0, 8), (1, 27), (2, 41)):
        for slot in range(n, p.capacity):
            p.set_slot(s, slot, bad)
    spare = sorted(set(range(p.n_pages)) - set(p.tables.cpu().flatten().tolist()))
    for page in spare:
        (p.k if kind == "bf16" else p.k_scale)[page] = bad
        (p.v if kind == "bf16" else p.v_scale)[page] = bad
    out = run(p, q, lengths, bits, sizes=sizes)
    vmax = 8
    assert ((out.cpu().double() - want).abs() <= want.abs() * 2.0 ** -8 + vmax * 2.0 ** -14).all()
    # a node that holds it: only those that attend to it are touched
    p.set_slot(2, 33 + 5, bad)
    out, plain = run(p, q, lengths, bits, sizes=sizes).cpu().double(), tree_reference(p, q, lengths, bits, sizes)
    blind = [i for i in range(8) if not bits[2][i] >> 5 & 1]
    assert len(blind) >= 2 and torch.equal(torch.isnan(out), torch.isnan(plain))
    assert ((out[2, blind] - want[2, blind]).abs() <= want[2, blind].abs() * 2.0 ** -8 + vmax * 2.0 ** -14).all()
    assert torch.isfinite(out[:2]).all()


def test_pages_that_are_not_there_are_masked():
    for kind in ("bf16", "int8"):
        p = Paged(3, 5, kind=kind, spare_pages=1)
        p.tables[0, 1], p.tables[1, 0], p.tables[2] = -1, p.n_pages, 2 ** 30
        bits = bits_of(random_parents(3, 8))
        q = queries(3, 8, 4, 64)
        lengths = ints([55, 10, 40])
        out = run(p, q, lengths, bits)
        close(out, tree_reference(p, q, lengths, bits), p)
        assert (out[2] == 0).all()


@pytest.mark.parametrize("kind", ["bf16", "int8"])
@pytest.mark.parametrize("dim,length", [(64, 100), (128, 700)])
def test_infinities_that_are_attended_to_do_what_the_formula_says(kind, dim, length):
    """A key that gives -infinity takes its token's weight, one that gives +infinity or NaN makes the head NaN, an infinite value reaches its dim."""
    p = Paged(4, -(-length // 16) + 1, dim=dim, kind=kind, kv_heads=1, seed=dim)
    bits = bits_of(random_parents(4, 6))
    q = queries(4, 6, 3, dim, dim)
    q[1, 2, 0, 3] = float("inf")
    q[1, 3, 1, 0] = float("nan")
    at = [(int(p.tables[s, slot // 16]), slot % 16) for s, slot in ((0, 40), (2, 17), (3, length + 3))]
    if kind == "bf16":
        p.k[at[0][0], 0, at[0][1], 5] = float("-inf")
        p.v[at[1][0], 0, at[1][1], 9] = float("inf")
        p.v[at[2][0], 0, at[2][1], 2] = float("nan")
    else:
        p.k_scale[at[0][0], 0, at[0][1]] = float("inf")
        p.v_scale[at[1][0], 0, at[1][1]] = float("inf")
        p.v_scale[at[2][0], 0, at[2][1]] = float("nan")
    lengths = ints([length] * 4)
    out, want = run(p, q, lengths, bits).cpu().double(), tree_reference(p, q, lengths, bits)
    assert torch.equal(torch.isnan(out), torch.isnan(want))
    both = torch.isinf(want)
    assert torch.equal(both, torch.isinf(out)) and torch.equal(out[both], want[both])
    rest = torch.isfinite(want)
    assert ((out - want).abs()[rest] <= want.abs()[rest] * 2.0 ** -8 + 8 * 2.0 ** -14).all()


def test_large_logits_and_equal_ones():
    p = Paged(2, 20)
    bits = bits_of(random_parents(2, 16))
    lengths = ints([280, 100])
    q = queries(2, 16, 4, 64) * 30                   # logits of some hundreds: one token has nearly all the weight
    out, want = run(p, q, lengths, bits).cpu().double(), tree_reference(p, q, lengths, bits)
    # the logits' terms add up to 30 times as much: 2^-15 * 30, taken twice
    close(out, want, p, scale=30)
    close(run(p, q * 0, lengths, bits), tree_reference(p, q * 0, lengths, bits), p)


@pytest.mark.parametrize("kind", ["bf16", "int8"])
@pytest.mark.parametrize("trees,longest,nodes,heads,kv_heads,dim", [
    (16, 700, 4, 8, 8, 64), (5, 3000, 16, 6, 2, 128), (1, 20000, 7, 4, 2, 64), (1, 41600, 8, 8, 1, 256), (2, 9000, 64, 3, 1, 128), (40, 400, 3, 4, 2, 96), (70, 130, 5, 4, 2, 32),
    (3, 5000, 16, 16, 1, 192), (12, 2000, 13, 9, 3, 80)])
def test_how_trees_are_cut(trees, longest, nodes, heads, kv_heads, dim, kind):
    """Trees behind sequences as long as each other, spread, and with one far longer; twice with one workspace, and the same results."""
    p = Paged(trees, -(-(longest + nodes) // 16), kv_heads=kv_heads, dim=dim, kind=kind, seed=trees)
    q = queries(trees, nodes, heads, dim, longest)
    bits = bits_of(random_parents(trees, nodes, dim))
    for n in ([longest] * trees, [(r * 619 + 5) % (longest + 1) for r in range(trees)], [longest if r == trees // 2 else r for r in range(trees)]):
        lengths = ints(n)
        call, out = tree_call(p.describe(), q, lengths, masks_of(bits))
        want = tree_reference(p, q, lengths, bits)
        got = []
        for _ in range(2):
            out.fill_(float("nan"))
            call.launch(stream())
            torch.cuda.synchronize()
            close(out, want, p)
            got.append(out.clone())
        assert torch.equal(*got)


@pytest.mark.parametrize("kind", ["bf16", "int8"])
@pytest.mark.parametrize("trees,longest,nodes,heads,kv_heads,dim", [(70, 810, 5, 10, 5, 64), (131, 500, 3, 5, 5, 128), (200, 510, 4, 7, 7, 64), (67, 630, 17, 9, 3, 256)])
def test_more_trees_than_a_wavefront_has_lanes(trees, longest, nodes, heads, kv_heads, dim, kind):
    """Trees are looked at 64 at a time.  Sequences of several stages, and shares that begin in one 64 and end in the next, with parts that are joined behind them."""
    p = Paged(trees, -(-(longest + nodes) // 16), kv_heads=kv_heads, dim=dim, kind=kind, seed=trees)
    q = queries(trees, nodes, heads, dim, longest)
    bits = bits_of(random_parents(trees, nodes, dim))
    crossed = 0
    for n in ([longest] * trees, [(r * 619 + 5) % (longest + 1) for r in range(trees)], [longest if r % 64 in (0, 63) else r * 37 % 150 for r in range(trees)]):
        tokens = 32768 // (dim * (1 if kind == "int8" else 2))
        units = [max(1, -(-(length + nodes) // tokens)) for length in n]
        share = -(-sum(units) * kv_heads // 256)
        assert max(units) > 1 and share > 1
        crossed += bool(sum(units[:64]) * kv_heads % share or (trees > 128 and sum(units[:128]) * kv_heads % share))
        lengths = ints(n)
        call, out = tree_call(p.describe(), q, lengths, masks_of(bits))
        want = tree_reference(p, q, lengths, bits)
        got = []
        for _ in range(2):
            out.fill_(float("nan"))
            call.launch(stream())
            torch.cuda.synchronize()
            close(out, want, p)
            got.append(out.clone())
        assert torch.equal(*got)
    assert crossed      # (what the cut is made from: without a share across tree 64 or 128 this would show less)


def test_every_token_counts_once():
    """One token has nearly all of the weight, in turn at edges of tiles and of shares: left out or taken twice, the result would be another."""
    n, nodes, dim = 2600, 5, 64
    p = Paged(1, -(-(n + nodes) // 16), kv_heads=1, dim=dim)
    bits = bits_of(random_parents(1, nodes))
    q = torch.ones((1, nodes, 2, dim), device="cuda")
    lengths = ints([n])
    p.k.zero_()
    for slot in [0, 1, 15, 16, 31, 32, 63, 64, 127, 128, 255, 256, 257, 511, 512, 1023, 1024, 1279, 1280, 1535, 2047, 2048, 2303, 2304, n - 1, n, n + nodes - 1]:
        page, at = int(p.tables[0, slot // 16]), slot % 16
        p.k[page, 0, at] = 1.5                       # logit 12 beside zeros: a weight of 2600 e^-12 beside it is 1.6 %
        out, want = run(p, q, lengths, bits), tree_reference(p, q, lengths, bits)
        close(out, want, p)
        p.k[page, 0, at] = 0


@pytest.mark.parametrize("kind", ["bf16", "int8"])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_weights_enter_the_sum_with_all_their_bits(kind, dim):
    """Large terms that cancel, so that the result's own rounding to bf16 hides nothing: two tokens of equal logits, through keys in two dims with equal queries, and opposite
    values, and a third one with values of at most 1 beside their 60 to 120.  Equal weights leave nothing of the first two but the rounding of the fp32 sum; a weight that
    entered one of the terms with fewer bits than the other would leave more."""
    nodes, heads = 3, 2
    p = Paged(4, 2, kv_heads=1, dim=dim, kind=kind)
    g = torch.Generator().manual_seed(dim)
    q = torch.zeros((4, nodes, heads, dim))
    q[..., 0] = 0.3 + torch.rand((4, nodes, heads), generator=g)
    q[..., 1] = q[..., 0]                            # two dims with equal queries: keys (1, 0) and (0, 1) have equal logits
    v = torch.round((1 + torch.rand((4, dim), generator=g)) * 60)
    small = torch.round((torch.rand((4, dim), generator=g) - 0.5) * 2)
    for s in range(4):
        page = int(p.tables[s, 0])
        for slot, (key, value) in enumerate((((1, 0), v[s]), ((0, 1), -v[s]), ((0, 0), small[s]))):
            row = torch.zeros(dim)
            row[:2] = torch.tensor(key, dtype=torch.float32)
            p.k[page, 0, slot] = row.to(p.k.dtype).cuda()
            p.v[page, 0, slot] = value.to(p.v.dtype).cuda()
        if kind == "int8":
            p.k_scale[page, 0, :3], p.v_scale[page, 0, :3] = 1.0, 1.0
    lengths, sizes = ints([3] * 4), ints([3] * 4)
    bits = [[0] * nodes] * 4                         # the tree's own slots are not seen
    out, want = run(p, q.cuda(), lengths, bits, sizes=sizes, scale=1.0).cpu().double(), tree_reference(p, q.cuda(), lengths, bits, sizes, scale=1.0)
    size = v.double().abs()[:, None, None, :]
    # equal logits, equal weights: two equal products cancel but for the fp32 sum's rounding, 2^-23 of them
    assert ((out - want).abs() <= want.abs() * 2.0 ** -8 + size * 2.0 ** -22).all()


@pytest.mark.parametrize("kind", ["bf16", "int8"])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_nearly_equal_weights_of_opposite_values(kind, dim):
    """Logits 2^-7 apart at most, of 1 or 2: what is left of values v and -v is 2^-8 of them or less, and each bit of a weight below its eighth shows.

    A logit is off by 2^-22 (two fp32 roundings of it), a weight by that, by 2^-23 from the exponential function, by 2^-22 from its parts and by 2^-23 from the sum, both weights
    together by less than 2^-19 of v.  Parts of 16 bits in all would be up to 2^-16 off."""
    nodes, heads = 16, 3
    p = Paged(2, 2, kv_heads=1, dim=dim, kind=kind)
    g = torch.Generator().manual_seed(dim)
    q = torch.zeros((2, nodes, heads, dim))
    q[..., 0] = 1 + torch.rand((2, nodes, heads), generator=g)
    q[..., 1] = q[..., 0] + (torch.rand((2, nodes, heads), generator=g) - 0.5) * 2.0 ** -6
    v = torch.round((1 + torch.rand((2, dim), generator=g)) * 60)
    for s in range(2):
        page = int(p.tables[s, 0])
        for slot, value in enumerate((v[s], -v[s])):
            row = torch.zeros(dim)
            row[slot] = 1
            p.k[page, 0, slot] = row.to(p.k.dtype).cuda()
            p.v[page, 0, slot] = value.to(p.v.dtype).cuda()
        if kind == "int8":
            p.k_scale[page, 0, :2], p.v_scale[page, 0, :2] = 1.0, 1.0
    lengths, bits = ints([2, 2]), [[0] * nodes] * 2
    out, want = run(p, q.cuda(), lengths, bits, scale=1.0).cpu().double(), tree_reference(p, q.cuda(), lengths, bits, scale=1.0)
    assert ((out - want).abs() <= want.abs() * 2.0 ** -8 + v.double()[:, None, None, :] * 2.0 ** -19).all()


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("order", ["rising", "falling", "shuffled", "signs"])
def test_values_scales_of_any_size(order, dim):
    """8 bits, scales from 1e-30 to 1e30, beside weights about as different: off by 2^-14 of sum p |v|, as above, whatever the largest of the scales is."""
    n, nodes, heads = 700, 5, 6
    p = Paged(2, -(-(n + nodes) // 16), kv_heads=2, dim=dim, kind="int8", seed=dim)
    bits = bits_of(random_parents(2, nodes))
    q = queries(2, nodes, heads, dim, dim)
    size = 10.0 ** torch.linspace(-30, 30, n + nodes)
    if order == "falling":
        size = size.flip(0)
    if order in ("shuffled", "signs"):
        size = size[torch.randperm(n + nodes, generator=torch.Generator().manual_seed(dim))]
    if order == "signs":
        size[::2] *= -1
    for s in range(2):
        for slot in range(n + nodes):
            p.v_scale[int(p.tables[s, slot // 16]), :, slot % 16] = size[slot]
    lengths = ints([n, n // 2])
    out, want = run(p, q, lengths, bits).cpu().double(), tree_reference(p, q, lengths, bits)
    signed_v, p.v, p.v_scale = (p.v, p.v_scale), p.v.abs(), p.v_scale.abs()
    terms = tree_reference(p, q, lengths, bits)
    p.v, p.v_scale = signed_v
    assert torch.isfinite(out).all() and ((out - want).abs() <= want.abs() * 2.0 ** -8 + terms * 2.0 ** -14).all()


@pytest.mark.parametrize("kind", ["bf16", "int8"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("far", [1, 650])
@pytest.mark.parametrize("larger,gap", [(1.0, 0.36), (2.0 ** 13, 0.36), (2.0 ** 26, 0.36), (2.0 ** 34, 0.36), (2.0 ** 40, 0.36), (2.0 ** 100, 0.36), (1.0, 10.0), (1.0, 20.0), (1.0, 25.0), (1.0, 60.0),
                                        (2.0 ** 30, 40.0)])
def test_a_small_weight_where_the_larger_one_has_a_value_of_zero(larger, gap, far, dim, kind):
    """Two tokens, in one tile or in two wavefronts' shares.  The first has the larger weight times scale, and zeros in every other dim: what the second gives there is as good as anywhere, 2^-14 of it.

    Its logit, -gap, is off by six roundings to 24 bits: with a gap of 60, 87 in units of log 2, 2^7 * 6 * 2^-24 < 2^-14."""
    nodes, heads = 3, 2
    p = Paged(1, 44, kv_heads=1, dim=dim, kind=kind)
    q = torch.zeros((1, nodes, heads, dim), device="cuda")
    q[..., 0] = 1.0
    p.k.zero_(), p.v.zero_()
    p.k[..., 0] = -1 if kind == "int8" else -300.0     # the other tokens: a weight of e^-300, which is zero
    if kind == "int8":
        p.k_scale.fill_(300.0), p.v_scale.fill_(1.0)
    first = torch.tensor([127.0, 0.0] * (dim // 2))
    for slot, logit, size, values in ((0, 0.0, larger, first), (far, -gap, 1.0, torch.full((dim,), 101.0))):
        page, at = int(p.tables[0, slot // 16]), slot % 16
        if kind == "int8":
            p.k[page, 0, at, 0], p.k_scale[page, 0, at] = -1 if logit else 0, gap
            p.v[page, 0, at], p.v_scale[page, 0, at] = values.to(torch.int8).cuda(), size
        else:
            p.k[page, 0, at, 0], p.v[page, 0, at] = logit, (values * size).to(torch.bfloat16).cuda()
    lengths, bits = ints([far + 1]), [[0] * nodes]
    out, want = run(p, q, lengths, bits, scale=1.0).cpu().double(), tree_reference(p, q, lengths, bits, scale=1.0)
    assert (want[..., 1::2] > 0).all() and ((out - want).abs() <= want * (2.0 ** -8 + 2.0 ** -14)).all()      # (no value is negative: the terms add up to the result)


@pytest.mark.parametrize("size", [1.0, 2.0 ** -60, 2.0 ** -110])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_values_scales_that_are_all_small(size, dim):
    """8 bits.  Weights times scales end at 2^-133, half a step of which is 2^-24 of 2^-110: of 105 tokens, the largest with a weight of 1, 105 * 2^-24 of it, below 2^-17."""
    p = Paged(2, 8, dim=dim, kind="int8", seed=dim)
    p.v_scale.fill_(size)
    q, bits, lengths = queries(2, 5, 6, dim, 1), bits_of(random_parents(2, 5)), ints([100, 60])
    out, want = run(p, q, lengths, bits).cpu().double(), tree_reference(p, q, lengths, bits)
    p.v = p.v.abs()
    assert ((out - want).abs() <= want.abs() * 2.0 ** -8 + tree_reference(p, q, lengths, bits) * 2.0 ** -14 + 127 * size * 2.0 ** -17).all()


@pytest.mark.parametrize("kind", ["bf16", "int8"])
@pytest.mark.parametrize("dim", [64, 128])
def test_logits_that_rise_from_token_to_token(kind, dim):
    """The largest so far grows over and over, by 1 a token, in 8 bits with values' scales that fall as the weights rise."""
    n, nodes = 900, 3
    p = Paged(1, -(-(n + nodes) // 16), kv_heads=1, dim=dim, kind=kind, seed=dim)
    q = torch.zeros((1, nodes, 2, dim), device="cuda")
    q[..., 0] = 1.0
    bits = bits_of(random_parents(1, nodes))
    for slot in range(n + nodes):
        page, at = int(p.tables[0, slot // 16]), slot % 16
        p.k[page, 0, at, 0] = 1 if kind == "int8" else slot % 256
        if kind == "int8":
            p.k_scale[page, 0, at] = float(slot)
            p.v_scale[page, 0, at] = 2.0 ** max(-100, 40 - 1.4 * slot)
    lengths = ints([n])
    out, want = run(p, q, lengths, bits, scale=1.0).cpu().double(), tree_reference(p, q, lengths, bits, scale=1.0)
    signed_v, p.v, p.v_scale = (p.v, p.v_scale), p.v.abs(), p.v_scale
    terms = tree_reference(p, q, lengths, bits, scale=1.0)
    p.v, p.v_scale = signed_v
    # logits up to 2^10 in place of 2^5: 2^-10 of the terms, taken twice
    assert torch.isfinite(out).all() and ((out - want).abs() <= want.abs() * 2.0 ** -8 + terms * 2.0 ** -9).all()


def test_keys_scales_far_from_those_of_queries():
    """Logits of ordinary size from 8-bit keys of 1e30 and queries of 1e-30, all of them negative."""
    n, nodes, heads, dim = 200, 4, 3, 64
    p = Paged(1, -(-(n + nodes) // 16), kv_heads=1, dim=dim, kind="int8")
    p.k.copy_(-p.k.abs())
    bits = bits_of(random_parents(1, nodes))
    q = queries(1, nodes, heads, dim).abs()
    lengths = ints([n])
    for size in (2.0 ** 60, 2.0 ** 75, 2.0 ** 90, 2.0 ** 100):
        scale, p.k_scale = p.k_scale, p.k_scale * size
        close(run(p, q / size, lengths, bits), tree_reference(p, q / size, lengths, bits), p)
        p.k_scale = scale


def test_graphs_that_share_a_workspace():
    """Two calls of different trees captured into graphs of their own with one workspace, replayed in turn."""
    p = Paged(3, 60, dim=128, kind="int8")
    made, wants, graphs, shared = [], [], [], None
    for trees, nodes, lengths in ((3, 12, [900, 31, 333]), (1, 40, [700])):
        bits = bits_of(random_parents(trees, nodes))
        q = queries(trees, nodes, 8, 128, nodes)
        if shared is None:
            shared = torch.zeros(1 << 27, dtype=torch.uint8, device="cuda")
        made.append(tree_call(p.describe(), q, ints(lengths), masks_of(bits), workspace=shared))
        wants.append(tree_reference(p, q, ints(lengths), bits))
    for call, _ in made:
        call.launch(stream())
    torch.cuda.synchronize()
    for call, _ in made:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=torch.cuda.Stream()):
            call.launch(stream())
    for _ in range(3):
        for graph, (_, out), want in zip(graphs, made, wants):
            out.fill_(float("nan"))
            graph.replay()
        torch.cuda.synchronize()
        for (_, out), want in zip(made, wants):
            close(out, want, p)


def test_a_pool_beyond_32_bits_of_offset():
    p = Paged(1, 5, kv_heads=2, dim=64)
    base = 2 ** 31 // (2 * 16 * 64) + 5
    far = p.n_pages + base
    for name in ("k", "v"):
        pool = torch.empty((far, 2, 16, 64), dtype=torch.bfloat16, device="cuda")
        pool[base:] = getattr(p, name)
        setattr(p, name, pool)
    bits = bits_of(random_parents(1, 9))
    q = queries(1, 9, 4, 64)
    lengths = ints([60])
    p.tables += base
    p.n_pages = far
    out = run(p, q, lengths, bits)
    p.k, p.v = p.k[base:].clone(), p.v[base:].clone()
    p.tables -= base
    p.n_pages -= base
    close(out, tree_reference(p, q, lengths, bits), p)


def test_another_stream_two_calls_at_once_and_a_graph():
    p = Paged(3, 40, dim=128)
    bits = bits_of(random_parents(3, 12))
    qs = [queries(3, 12, 8, 128, s) for s in range(2)]
    lengths = ints([600, 31, 333])
    made = [tree_call(p.describe(), q, lengths, masks_of(bits)) for q in qs]
    wants = [tree_reference(p, q, lengths, bits) for q in qs]
    sides = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for side, (call, _) in zip(sides, made):
        with torch.cuda.stream(side):
            for _ in range(5):
                call.launch(stream())
    torch.cuda.synchronize()
    for (_, out), want in zip(made, wants):
        close(out, want, p)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        made[0][0].launch(stream())
    for step in range(3):
        lengths.copy_(ints([100 + step, 0, 600]))
        qs[0].mul_(0.9)
        made[0][1].fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        close(made[0][1], tree_reference(p, qs[0], lengths, bits), p)
