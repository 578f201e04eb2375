"""What the calls between the products refuse, with which code: all of it decided on the host, before any launch (no GPU)."""
import pytest

import paper_2509_22951_amd as tq

A = 1 << 20      # an aligned address; nothing is launched
INVALID, UNSUPPORTED = -1, -3
CACHE = dict(k=A, v=A, tables=A, type=tq.TQ_BF16, n_pages=4, page_size=16, kv_heads=2, head_dim=64, n_seqs=2, seq_pages=2)
NORM = dict(residual=A, weight=A, out=2 * A, rows=2, cols=64, eps=1e-5, residual_type=tq.TQ_FP32, weight_type=tq.TQ_FP32, out_type=tq.TQ_BF16)
APPEND = dict(q=A, k=A, v=A, q_out=2 * A, slots=A, cos=A, sin=A, rows=2, heads=4, rotary_dim=64, n_positions=8, q_out_type=tq.TQ_FP32)
ATTEND = dict(q=A, out=2 * A, lengths=A, workspace=4 * A, workspace_bytes=1 << 40, rows=2, heads=4, scale=0.125, q_type=tq.TQ_FP32)
EVICT = dict(lengths=A, workspace=4 * A, workspace_bytes=1 << 40, keep=5)


def refused(code, call):
    with pytest.raises(tq.TqError) as e:
        call()
    assert e.value.code == code and len(str(e.value)) > 20
    return str(e.value)


@pytest.mark.parametrize("code,change", [
    (INVALID, dict(residual=0)), (INVALID, dict(weight=0)), (INVALID, dict(out=0)), (INVALID, dict(out_type=tq.TQ_INT8)), (UNSUPPORTED, dict(out_type=tq.TQ_FP32)),
    (UNSUPPORTED, dict(residual_type=tq.TQ_INT8)), (UNSUPPORTED, dict(weight_type=7)), (UNSUPPORTED, dict(cols=0)), (UNSUPPORTED, dict(cols=(1 << 20) + 1)),
    (INVALID, dict(residual_stride=63)), (INVALID, dict(out_stride=1)), (INVALID, dict(delta=A, delta_stride=63)), (INVALID, dict(residual=A + 2)),
    (INVALID, dict(out=A + 1)), (INVALID, dict(residual_out=A, residual_out_stride=80)), (INVALID, dict(eps=-1.0)), (INVALID, dict(eps=float("nan"))),
    (INVALID, dict(delta=A + 2)), (UNSUPPORTED, dict(rows=1 << 31)),
])
def test_norm_refuses(code, change):
    refused(code, lambda: tq.AddNorm(**{**NORM, **change}).launch())


@pytest.mark.parametrize("code,change", [
    (INVALID, dict(k=0)), (INVALID, dict(tables=0)), (UNSUPPORTED, dict(type=tq.TQ_FP32)), (INVALID, dict(type=tq.TQ_INT8)), (UNSUPPORTED, dict(page_size=8)),
    (UNSUPPORTED, dict(page_size=48)), (UNSUPPORTED, dict(page_size=2048)), (UNSUPPORTED, dict(head_dim=72)), (UNSUPPORTED, dict(head_dim=272)),
    (UNSUPPORTED, dict(head_dim=0)), (INVALID, dict(n_pages=0)), (INVALID, dict(n_seqs=0)), (INVALID, dict(seq_pages=0)), (INVALID, dict(kv_heads=0)),
    (UNSUPPORTED, dict(seq_pages=1 << 27)), (INVALID, dict(k=A + 8)), (INVALID, dict(page_stride=4096)), (INVALID, dict(page_stride=4096, head_stride=64, slot_stride=4)),
    (UNSUPPORTED, dict(page_stride=1 << 30, head_stride=64, slot_stride=1 << 26)), (INVALID, dict(table_stride=1)), (INVALID, dict(scores=A + 1)),
])
def test_every_call_refuses_a_cache_that_is_not_one(code, change):
    cache = tq.Cache(**{**CACHE, "scores": A, **change})
    refused(code, lambda: tq.CacheAppend(cache, **APPEND).launch())
    refused(code, lambda: tq.Attend(cache, **ATTEND).launch())
    refused(code, lambda: tq.CacheEvict(cache, **EVICT).launch())
    refused(code, lambda: tq.Attend.workspace_bytes(cache, **ATTEND))
    refused(code, lambda: tq.CacheEvict.workspace_bytes(cache, **EVICT))


@pytest.mark.parametrize("code,change", [
    (INVALID, dict(q=0)), (INVALID, dict(k=0)), (INVALID, dict(q_out=0)), (INVALID, dict(slots=0)), (INVALID, dict(cos=0)), (INVALID, dict(rows=3)),
    (INVALID, dict(heads=0)), (UNSUPPORTED, dict(rotary_dim=12)), (UNSUPPORTED, dict(rotary_dim=72)), (UNSUPPORTED, dict(q_out_type=tq.TQ_INT8)),
    (UNSUPPORTED, dict(pairing=2)), (INVALID, dict(q_stride=255)), (INVALID, dict(v_stride=127)), (INVALID, dict(q=A + 2)), (INVALID, dict(seqs=A + 1)),
    (INVALID, dict(q_out=A, q_out_type=tq.TQ_BF16)), (INVALID, dict(q_out=A, q_stride=512)),
])
def test_append_refuses(code, change):
    refused(code, lambda: tq.CacheAppend(tq.Cache(**CACHE), **{**APPEND, **change}).launch())


@pytest.mark.parametrize("code,change", [
    (INVALID, dict(q=0)), (INVALID, dict(out=0)), (INVALID, dict(lengths=0)), (INVALID, dict(workspace=0)), (INVALID, dict(rows=3)), (INVALID, dict(heads=3)),
    (INVALID, dict(heads=0)), (UNSUPPORTED, dict(q_type=tq.TQ_INT8)), (INVALID, dict(scale=0.0)), (INVALID, dict(scale=float("nan"))),
    (INVALID, dict(scale=float("inf"))), (INVALID, dict(accumulate=1)), (INVALID, dict(accumulate=2)), (INVALID, dict(workspace_bytes=8)),
    (INVALID, dict(workspace=A + 8)), (INVALID, dict(q=A + 2)), (INVALID, dict(q_stride=255)), (INVALID, dict(out_stride=100)),
])
def test_attend_refuses(code, change):
    refused(code, lambda: tq.Attend(tq.Cache(**CACHE), **{**ATTEND, **change}).launch())


@pytest.mark.parametrize("code,change,cache", [
    (INVALID, dict(lengths=0), {}), (INVALID, dict(workspace=0), {}), (INVALID, dict(keep=0), {}), (INVALID, dict(workspace_bytes=8), {}),
    (INVALID, dict(since=A), {}), (INVALID, dict(positions_out=A), {}), (INVALID, {}, dict(scores=0)), (INVALID, dict(scores_out=A + 2), {}),
])
def test_evict_refuses(code, change, cache):
    refused(code, lambda: tq.CacheEvict(tq.Cache(**{**CACHE, "scores": A, **cache}), **{**EVICT, **change}).launch())


def test_null_structures_unknown_fields_and_the_workspaces():
    lib = tq.load()
    c = tq.Cache(**CACHE, scores=A)
    assert lib.tq_add_rms_norm(None, None) == INVALID
    assert lib.tq_cache_append(c.address, None, None) == INVALID and lib.tq_cache_append(None, None, None) == INVALID
    assert lib.tq_attend(c.address, None, None) == INVALID and lib.tq_attend_workspace(c.address, None, None) == INVALID
    assert lib.tq_cache_evict(c.address, None, None) == INVALID and lib.tq_cache_evict_workspace(c.address, None, None) == INVALID
    with pytest.raises(TypeError, match="colums"):
        tq.AddNorm(**NORM, colums=3)
    need = tq.Attend.workspace_bytes(c, **ATTEND)
    assert 0 < need < tq.Attend.workspace_bytes(c, **{**ATTEND, "accumulate": 1})
    assert "needed" in refused(INVALID, lambda: tq.Attend(c, **{**ATTEND, "workspace_bytes": need - 1}).launch())
    need = tq.CacheEvict.workspace_bytes(c, **EVICT)
    assert "needed" in refused(INVALID, lambda: tq.CacheEvict(c, **{**EVICT, "workspace_bytes": need - 1}).launch())


def test_no_rows_are_no_work():
    tq.AddNorm(**{**NORM, "rows": 0}).launch()
    tq.CacheAppend(tq.Cache(**CACHE), **{**APPEND, "rows": 0}).launch()
    tq.Attend(tq.Cache(**CACHE), **{**ATTEND, "rows": 0}).launch()


@pytest.mark.parametrize("change", [
    dict(page_stride=16, head_stride=16, slot_stride=16), dict(page_stride=4096, head_stride=1024, slot_stride=56), dict(page_stride=4096, head_stride=48, slot_stride=128),
    dict(page_stride=32, head_stride=1024, slot_stride=64), dict(type=tq.TQ_INT8, k_scale=A, v_scale=A, page_stride=4096, head_stride=1024, slot_stride=48),
])
def test_every_call_refuses_keys_that_overlap(change):
    cache = tq.Cache(**{**CACHE, "scores": A, **change})
    for call in (lambda: tq.CacheAppend(cache, **APPEND).launch(), lambda: tq.Attend(cache, **ATTEND).launch(), lambda: tq.CacheEvict(cache, **EVICT).launch(),
                 lambda: tq.Attend.workspace_bytes(cache, **ATTEND), lambda: tq.CacheEvict.workspace_bytes(cache, **EVICT)):
        assert "smaller than" in refused(INVALID, call)


@pytest.mark.parametrize("change", [dict(page_stride=2048, head_stride=16, slot_stride=64, kv_heads=1), dict(page_stride=16, head_stride=1024, slot_stride=64, n_pages=1)])
def test_the_stride_between_heads_or_pages_of_which_there_is_one_is_free(change):
    assert tq.Attend.workspace_bytes(tq.Cache(**{**CACHE, **change}), **ATTEND) > 0


@pytest.mark.parametrize("rows,cols", [(1 << 22, 4096), (1 << 22, 1 << 20), (1 << 23, 2048), (1 << 26, 64)])
def test_norm_refuses_more_rows_than_a_launch_has_threads_for(rows, cols):
    assert "too many rows" in refused(UNSUPPORTED, lambda: tq.AddNorm(**{**NORM, "rows": rows, "cols": cols}).launch())


def test_append_refuses_more_rows_than_a_launch_has_threads_for():
    assert "too many rows" in refused(UNSUPPORTED, lambda: tq.CacheAppend(tq.Cache(**CACHE), **{**APPEND, "seqs": A, "rows": 1 << 24}).launch())
