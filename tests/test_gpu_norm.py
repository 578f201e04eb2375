"""tq_add_rms_norm against the formula in 64 bits.

Tolerances.  residual_out is one fp32 addition (and one rounding to bf16), which torch does alike: equal bits.  out: the sum of
squares has positive terms, at most 2^11 of them one after another in a thread, so it is within 2^11 * 2^-24 = 2^-13 in the very
worst case and its root within half of that; a few roundings of 2^-24 follow; rounding to bf16 adds 2^-8 of the value."""
import pytest

torch = pytest.importorskip("torch")

import paper_2509_22951_amd as tq
from paged import ptr, stream

pytestmark = pytest.mark.gpu

TYPES = {"fp32": (torch.float32, tq.TQ_FP32), "bf16": (torch.bfloat16, tq.TQ_BF16), "int8": (torch.int8, tq.TQ_INT8)}
EPS = 1e-5


def placed(t, gap, offset):
    """The same matrix with `gap` values behind every row, starting `offset` values into its buffer -> a view."""
    rows, cols = t.shape
    buf = torch.full((rows * (cols + gap) + offset,), 7, dtype=t.dtype, device="cuda")
    view = buf[offset:].view(rows, cols + gap)[:, :cols]
    view.copy_(t)
    return view


def inputs(rows, cols, residual, weight, seed=0):
    g = torch.Generator().manual_seed(seed)
    r = (torch.randn((rows, cols), generator=g) * 2).to(TYPES[residual][0])
    return r, torch.randn((rows, cols), generator=g) * 0.5, (1 + 0.2 * torch.randn(cols, generator=g)).to(TYPES[weight][0])


def normed(r, d, w, residual, weight, out, in_place=False, gap=0, offset=0, eps=EPS, want_residual=True):
    rows, cols = r.shape
    rd, wd = placed(r, gap, offset), w.cuda()
    dd = None if d is None else placed(d, gap, offset)
    ro = rd if in_place else placed(torch.zeros_like(r), gap, offset) if want_residual else None
    o = placed(torch.zeros((rows, cols), dtype=TYPES[out][0]), gap, offset)
    scale = torch.full((rows,), -1.0, device="cuda")
    strides = {n: cols + gap for n in ("residual_stride", "delta_stride", "residual_out_stride", "out_stride")} if gap else {}
    tq.AddNorm(residual=ptr(rd), delta=ptr(dd), weight=ptr(wd), residual_out=ptr(ro), out=ptr(o), out_scale=ptr(scale), rows=rows, cols=cols, eps=eps,
               residual_type=TYPES[residual][1], weight_type=TYPES[weight][1], out_type=TYPES[out][1], **strides).launch(stream())
    torch.cuda.synchronize()
    return ro, o, scale


def check(r, d, w, ro, o, scale, out, eps=EPS):
    if ro is not None:
        want = r.float() if d is None else r.float() + d
        assert torch.equal(ro.cpu(), want.to(r.dtype))
    h = r.double() if d is None else (r.float() + d).double()
    y = h / torch.sqrt(h.square().mean(dim=1, keepdim=True) + eps) * w.double()
    if out == "int8":
        s = y.abs().amax(dim=1) / 127
        assert torch.allclose(scale.cpu().double(), s, rtol=2.0 ** -13, atol=0)
        # half a step, and what the scale and the value are off, in steps: 127 * 2 * 2^-13
        off = (o.cpu().double() * scale.cpu().double()[:, None] - y).abs()
        assert (off <= s[:, None] * (0.5 + 127 * 2.0 ** -12) + 1e-300).all()
        assert (o.cpu().abs().amax(dim=1) == torch.where(s > 0, 127, 0)).all()
    else:
        assert ((o.cpu().double() - y).abs() <= y.abs() * (2.0 ** -8 + 2.0 ** -13)).all()


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 2048), (3, 63), (2, 64), (5, 257), (16, 2999), (7, 4096), (4, 5001), (3, 8192), (2, 16384), (1, 16388), (1, 20001),
                                       (1, 1 << 20), (300, 130)])
@pytest.mark.parametrize("residual,weight,out", [("fp32", "bf16", "bf16"), ("bf16", "fp32", "bf16"), ("fp32", "fp32", "int8"), ("bf16", "bf16", "int8")])
def test_norm(rows, cols, residual, weight, out):
    r, d, w = inputs(rows, cols, residual, weight, rows + cols)
    check(r, d, w, *normed(r, d, w, residual, weight, out), out)


@pytest.mark.parametrize("cols", [64, 2048, 2999, 6000, 20000])
@pytest.mark.parametrize("gap,offset", [(0, 1), (4, 0), (3, 0), (8, 4), (5, 3)])
def test_rows_with_gaps_and_any_alignment_in_place_and_without_delta(cols, gap, offset):
    for out in ("bf16", "int8"):
        r, d, w = inputs(4, cols, "fp32", "bf16", cols + gap)
        check(r, d, w, *normed(r, d, w, "fp32", "bf16", out, in_place=True, gap=gap, offset=offset), out)
        check(r, None, w, *normed(r, None, w, "fp32", "bf16", out, gap=gap, offset=offset, want_residual=False), out)


def test_gaps_between_rows_stay_as_they_are():
    r, d, w = inputs(5, 250, "fp32", "fp32")
    ro, o, _ = normed(r, d, w, "fp32", "fp32", "bf16", gap=6)
    for t in (ro, o):
        assert (t.as_strided((5, 6), (256, 1), t.storage_offset() + 250) == 7).all()


@pytest.mark.parametrize("cols", [100, 2048])
def test_zero_rows_large_values_and_rows_that_are_not_finite(cols):
    r, d, w = inputs(6, cols, "fp32", "fp32")
    r[0] = d[0] = 0
    r[1], d[1] = 1e18 * r[1], 0
    r[2], d[2] = 1e-18 * r[2], 0
    r[3, 5] = float("inf")
    r[4, cols - 1] = float("nan")
    for out in ("bf16", "int8"):
        ro, o, scale = normed(r, d, w, "fp32", "fp32", out)
        fine = [0, 1, 2, 5]
        check(r[fine], d[fine], w, ro[fine], o[fine], scale[fine], out)
        got = o.float() * scale[:, None] if out == "int8" else o.float()
        assert torch.isnan(got[4]).all()
        assert torch.isnan(got[3, 5]) and (torch.isnan(got[3]) | (got[3] == 0)).all()
        assert (o[0] == 0).all()


def test_no_rows_and_another_stream():
    tq.AddNorm(rows=0, cols=8, residual=0, out_type=tq.TQ_BF16).launch(stream())
    r, d, w = inputs(64, 2048, "fp32", "bf16")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        check(r, d, w, *normed(r, d, w, "fp32", "bf16", "bf16"), "bf16")
