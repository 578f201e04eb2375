"""tq_cache_append_normed: the norm and the rotation against the formulas in 64 bits.

Tolerances.  The mean of squares is a sum of positive fp32 terms: two roundings each, ten additions, eps: 13 * 2^-24 of it, half of that beside
the square root, which is rounded, as are the division and the products with it and the weight: 11 * 2^-24 of a normed value; the rotation's
two products and sum add 4 * 2^-24 of |a| + |b|: 2^-20 of |a| + |b| in all.  Stored as bf16 2^-8 of the value more; in 8 bits half a step of the scale,
which is the largest value's 2^-20 and a rounding off, 127 * 2^-19 steps at most."""
import pytest

torch = pytest.importorskip("torch")

import paper_2509_22951_amd as tq
from drafts import ints
from paged import Paged, ptr, stream
from test_gpu_cache import angles, new_tokens, rotated, snapshot

pytestmark = pytest.mark.gpu


def normed(x, weight, eps):
    """[rows][heads][dim] -> 64 bits; weight: None, [dim] or [heads][dim]."""
    x = x.double()
    y = x / torch.sqrt(x.square().mean(dim=-1, keepdim=True) + eps)
    return y if weight is None else y * weight.double()


def launch(p, q, k, v, slots, cos, sin, rotary_dim, qw, kw, eps=1e-6, seqs=None, positions=None, adjacent=False, q16=False, in_place=False, gap=0, weight_gap=0):
    rows, heads, dim = q.shape

    def placed(t):
        buf = torch.zeros(rows, t.shape[1] * dim + gap, device="cuda")
        buf[:, : t.shape[1] * dim] = t.reshape(rows, -1)
        return buf

    def weights(w):
        if w is None:
            return None, 0
        if w.dim() == 1:
            return w.cuda(), 0
        buf = torch.full((w.shape[0], dim + weight_gap), 9, dtype=w.dtype, device="cuda")
        buf[:, :dim] = w
        return buf, dim + weight_gap

    qd, kd, vd, cd, sd = placed(q), placed(k), placed(v), cos.cuda(), sin.cuda()
    (qw, qs), (kw, ks) = weights(qw), weights(kw)
    kinds = {w.dtype for w in (qw, kw) if w is not None}
    norm = tq.HeadNorm(q_weight=ptr(qw), k_weight=ptr(kw), q_weight_stride=qs, k_weight_stride=ks, eps=eps,
                       weight_type=tq.TQ_BF16 if kinds == {torch.bfloat16} else tq.TQ_FP32)
    out = qd if in_place else torch.full((rows, heads * dim), 7, dtype=torch.bfloat16 if q16 else torch.float32, device="cuda")
    tq.CacheAppendNormed(p.describe(), norm, q=ptr(qd), k=ptr(kd), v=ptr(vd), q_out=ptr(out), seqs=ptr(seqs), slots=ptr(slots), positions=ptr(positions), cos=ptr(cd),
                         sin=ptr(sd), rows=rows, heads=heads, rotary_dim=rotary_dim, n_positions=cos.shape[0], q_stride=qd.stride(0), k_stride=kd.stride(0),
                         v_stride=vd.stride(0), q_out_stride=out.stride(0), q_out_type=tq.TQ_BF16 if q16 else tq.TQ_FP32, pairing=int(adjacent)).launch(stream())
    torch.cuda.synchronize()
    return out.cpu()[:, : heads * dim].reshape(rows, heads, dim)


def check(p, before, got_q, q, k, v, slots, cos, sin, rotary_dim, qw, kw, eps=1e-6, seqs=None, positions=None, adjacent=False):
    rows = q.shape[0]
    seqs = list(range(rows)) if seqs is None else seqs.tolist()
    slots = slots.tolist()
    at = torch.tensor(slots if positions is None else positions.tolist()) % cos.shape[0]
    want_q, mag_q = rotated(normed(q, qw, eps), cos[at], sin[at], rotary_dim, adjacent)
    want_k, mag_k = rotated(normed(k, kw, eps), cos[at], sin[at], rotary_dim, adjacent)
    more = 2.0 ** -8 * want_q.abs() if got_q.dtype == torch.bfloat16 else 0
    assert ((got_q.double() - want_q).abs() <= mag_q * 2.0 ** -20 + more).all()
    touched = torch.zeros(p.n_pages, p.page, dtype=torch.bool)
    table = p.tables.cpu()
    for r in range(rows):
        page, t = int(table[seqs[r], slots[r] // p.page]), slots[r] % p.page
        touched[page, t] = True
        for n, want, mag in (("k", want_k[r], mag_k[r]), ("v", v[r].double(), torch.zeros_like(mag_k[r]))):
            got = getattr(p, n)[page, :, t].cpu().double()
            if p.k_scale is None:
                assert ((got - want).abs() <= want.abs() * 2.0 ** -8 + mag * 2.0 ** -20).all()
            else:
                s, got_s = want.abs().amax(dim=1) / 127, getattr(p, n + "_scale")[page, :, t].cpu().double()
                assert ((got_s - s).abs() <= mag.amax(dim=1) / 127 * 2.0 ** -19 + s * 2.0 ** -22).all()
                assert ((got * got_s[:, None] - want).abs() <= s[:, None] * (0.5 + 127 * 2.0 ** -18)).all()
        if p.scores is not None:
            assert (p.scores[seqs[r], :, slots[r]] == 0).all() and (p.positions[seqs[r], :, slots[r]].cpu() == at[r]).all()
    rest = ~touched[:, None, :].expand(-1, p.kv_heads, -1)
    for n, was in zip(("k", "v"), before):
        assert torch.equal(getattr(p, n).cpu()[rest], was[rest])


@pytest.mark.parametrize("dim,rotary_dim", [(16, 16), (32, 8), (48, 48), (64, 64), (64, 0), (80, 64), (96, 96), (128, 128), (144, 72), (256, 256)])
@pytest.mark.parametrize("kind", ["bf16", "int8"])
@pytest.mark.parametrize("adjacent", [False, True])
def test_norm_rotation_cache(dim, rotary_dim, kind, adjacent):
    p = Paged(5, 4, kv_heads=3, dim=dim, kind=kind, marks=kind == "int8", seed=dim)
    q, k, v = new_tokens(5, 6, 3, dim, dim)
    g = torch.Generator().manual_seed(dim)
    qw, kw = 1 + 0.3 * torch.randn(dim, generator=g), 1 + 0.3 * torch.randn(dim, generator=g)
    if adjacent:
        qw, kw = qw.to(torch.bfloat16), kw.to(torch.bfloat16)
    cos, sin = angles(90, rotary_dim)
    slots = ints([0, 63, 17, 16, 5])
    before = snapshot(p)
    got = launch(p, 4 * q, 0.1 * k, v, slots, cos, sin, rotary_dim, qw, kw, adjacent=adjacent, q16=adjacent)
    check(p, before, got, 4 * q, 0.1 * k, v, slots, cos, sin, rotary_dim, qw, kw, adjacent=adjacent)


@pytest.mark.parametrize("per_head", [False, True])
@pytest.mark.parametrize("kind,order,dtype", [("bf16", "pthd", torch.float32), ("int8", "hptd", torch.bfloat16), ("bf16", "phtd", torch.bfloat16)])
def test_a_prompt_in_place_with_gaps_weights_of_each_head_and_positions(per_head, kind, order, dtype):
    p = Paged(2, 120, kv_heads=2, dim=96, kind=kind, order=order)
    rows = 1700                                    # several heads per group of lanes
    q, k, v = new_tokens(rows, 40, 2, 96, 3)
    g = torch.Generator().manual_seed(4)
    qw, kw = ((torch.randn((n, 96) if per_head else 96, generator=g)).to(dtype) for n in (40, 2))
    cos, sin = angles(4000, 96)
    seqs, slots, positions = ints([1] * rows), ints(list(range(rows))), ints([2 * r + 3 for r in range(rows)])
    before = snapshot(p)
    got = launch(p, q, k, v, slots, cos, sin, 96, qw, kw, seqs=seqs, positions=positions, in_place=True, gap=4, weight_gap=5)
    check(p, before, got, q, k, v, slots, cos, sin, 96, qw, kw, seqs=seqs, positions=positions)


def test_without_weights_it_is_the_append_of_normed_heads():
    p = Paged(4, 2, dim=64)
    q, k, v = new_tokens(4, 6, 2, 64)
    cos, sin = angles(40, 64)
    slots = ints([3, 0, 31, 16])
    before = snapshot(p)
    for qw, kw in ((None, None), (torch.rand(64), None), (None, torch.rand(2, 64))):
        got = launch(p, q, k, v, slots, cos, sin, 64, qw, kw, eps=0.25)
        check(p, before, got, q, k, v, slots, cos, sin, 64, qw, kw, eps=0.25)


def test_zero_heads_large_values_padding_and_what_is_not_finite():
    p = Paged(8, 2, dim=64, kv_heads=1)
    q, k, v = new_tokens(8, 2, 1, 64)
    q[0], k[0] = 0, 0
    q[1], k[1] = q[1] * 1e18, k[1] * 1e18
    q[2, 0, 5], k[2, 0, 7] = float("inf"), float("nan")
    cos, sin = angles(40, 0)
    slots = ints([0, 1, 2, 3, -1, 99999, 4, 5])     # two rows are padding
    seqs = ints([0, 1, 2, 3, 4, 5, 6, 9])           # and one more
    w = torch.ones(64)
    got = launch(p, q, k, v, slots, cos, sin, 0, w, w, seqs=seqs)
    assert (got[0] == 0).all() and (got[4] == 0).all() and (got[5] == 0).all() and (got[7] == 0).all()
    want = normed(q, None, 1e-6)
    assert ((got[1] - want[1]).abs() <= want[1].abs() * 2.0 ** -20).all() and torch.isfinite(got[1]).all()
    assert torch.isnan(got[2, 0, 5]) and (got[2, 0, :5] == 0).all() and torch.isfinite(got[2, 1]).all()
    assert torch.isnan(p.k[p.tables[2, 0].item(), 0, 2]).all()
    assert (launch(p, q, k, v, slots, cos, sin, 0, w, w, seqs=seqs, eps=0.0)[[4, 5, 7]] == 0).all()      # whatever eps


def test_captured_and_replayed():
    p = Paged(3, 4, dim=128, kind="int8")
    q, k, v = (x.cuda().view(3, -1) for x in new_tokens(3, 8, 2, 128))
    cos, sin = (x.cuda() for x in angles(64, 128))
    w, slots, out = torch.rand(128, device="cuda"), ints([0, 0, 0]), torch.empty_like(q)
    norm = tq.HeadNorm(q_weight=ptr(w), k_weight=ptr(w), eps=1e-5, weight_type=tq.TQ_FP32)
    made = tq.CacheAppendNormed(p.describe(), norm, q=ptr(q), k=ptr(k), v=ptr(v), q_out=ptr(out), slots=ptr(slots), cos=ptr(cos), sin=ptr(sin), rows=3, heads=8,
                                rotary_dim=128, n_positions=64, q_out_type=tq.TQ_FP32)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        made.launch(stream())
    for step in range(4):
        slots.copy_(ints([step, 20 + step, 63 - step]))
        q.mul_(1.5), k.add_(0.25)
        before = snapshot(p)
        graph.replay()
        torch.cuda.synchronize()
        check(p, before, out.cpu().view(3, 8, 128), q.cpu().view(3, 8, 128), k.cpu().view(3, 2, 128), v.cpu().view(3, 2, 128), slots, cos.cpu(), sin.cpu(), 128, w.cpu(), w.cpu(), eps=1e-5)
