"""What head norms, trees of drafted tokens and drawing refuse, with which code: all of it decided on the host, before any launch (no GPU)."""
import pytest

import paper_2509_22951_amd as tq
from test_host_refusals import A, APPEND, CACHE, INVALID, UNSUPPORTED, refused

NORM = dict(q_weight=A, k_weight=A, eps=1e-6, weight_type=tq.TQ_FP32)
TREE = dict(q=A, out=2 * A, lengths=A, masks=A, workspace=4 * A, workspace_bytes=1 << 40, trees=2, nodes=4, heads=4, scale=0.125, q_type=tq.TQ_FP32)
ACCEPT = dict(masks=A, lengths=A, drafted=A, sampled=A, path=2 * A, accepted=3 * A, next=4 * A, lengths_out=5 * A, trees=2, nodes=4)
SAMPLE = dict(logits=A, uniform=A, tokens=2 * A, workspace=4 * A, workspace_bytes=1 << 40, rows=2, vocab=100)


@pytest.mark.parametrize("code,change", [
    (INVALID, dict(eps=-1e-6)), (INVALID, dict(eps=float("nan"))), (INVALID, dict(eps=float("inf"))), (UNSUPPORTED, dict(weight_type=tq.TQ_INT8)), (INVALID, dict(q_weight=A + 2)),
    (INVALID, dict(k_weight=A + 1, weight_type=tq.TQ_BF16)), (INVALID, dict(q_weight_stride=63)), (INVALID, dict(k_weight_stride=1)),
])
def test_head_norm_refuses(code, change):
    refused(code, lambda: tq.CacheAppendNormed(tq.Cache(**CACHE), tq.HeadNorm(**{**NORM, **change}), **APPEND).launch())


@pytest.mark.parametrize("code,change", [
    (INVALID, dict(q=0)), (INVALID, dict(k=0)), (INVALID, dict(q_out=0)), (INVALID, dict(slots=0)), (INVALID, dict(cos=0)), (INVALID, dict(rows=3)),
    (INVALID, dict(heads=0)), (UNSUPPORTED, dict(rotary_dim=12)), (UNSUPPORTED, dict(q_out_type=tq.TQ_INT8)), (UNSUPPORTED, dict(pairing=2)), (INVALID, dict(q_stride=255)),
    (INVALID, dict(q=A + 2)), (INVALID, dict(q_out=A, q_out_type=tq.TQ_BF16)), (UNSUPPORTED, dict(seqs=A, rows=1 << 24)),
])
def test_the_append_with_a_norm_refuses_what_the_append_does(code, change):
    assert "tq_cache_append_normed" in refused(code, lambda: tq.CacheAppendNormed(tq.Cache(**CACHE), tq.HeadNorm(**NORM), **{**APPEND, **change}).launch())


@pytest.mark.parametrize("code,change", [
    (INVALID, dict(q=0)), (INVALID, dict(out=0)), (INVALID, dict(lengths=0)), (INVALID, dict(masks=0)), (INVALID, dict(workspace=0)), (INVALID, dict(trees=3)),
    (UNSUPPORTED, dict(trees=65536, seqs=A)), (UNSUPPORTED, dict(nodes=0)), (UNSUPPORTED, dict(nodes=65)), (INVALID, dict(heads=3)), (INVALID, dict(heads=0)),
    (UNSUPPORTED, dict(q_type=tq.TQ_INT8)), (INVALID, dict(scale=0.0)), (INVALID, dict(scale=float("nan"))), (INVALID, dict(scale=float("inf"))), (INVALID, dict(workspace_bytes=8)),
    (INVALID, dict(workspace=A + 8)), (INVALID, dict(q=A + 2)), (INVALID, dict(masks=A + 4)), (INVALID, dict(sizes=A + 2)), (INVALID, dict(q_stride=255)), (INVALID, dict(out_stride=100)),
])
def test_tree_attention_refuses(code, change):
    refused(code, lambda: tq.AttendTree(tq.Cache(**CACHE), **{**TREE, **change}).launch())


@pytest.mark.parametrize("code,change", [
    (INVALID, dict(masks=0)), (INVALID, dict(lengths=0)), (INVALID, dict(drafted=0)), (INVALID, dict(sampled=0)), (INVALID, dict(path=0)), (INVALID, dict(accepted=0)),
    (INVALID, dict(next=0)), (INVALID, dict(lengths_out=0)), (INVALID, dict(lengths_out=A)), (INVALID, dict(masks=A + 4)), (INVALID, dict(path=A + 2)), (UNSUPPORTED, dict(nodes=0)),
    (UNSUPPORTED, dict(nodes=65)), (UNSUPPORTED, dict(trees=65536, seqs=A)), (INVALID, dict(trees=3)),
])
def test_accept_refuses(code, change):
    refused(code, lambda: tq.TreeAccept([tq.Cache(**CACHE)], **{**ACCEPT, **change}).launch())


def test_accept_refuses_a_cache_that_is_there_twice():
    one, other_tables, other_pool = tq.Cache(**CACHE), tq.Cache(**{**CACHE, "tables": CACHE["tables"] + 4096}), tq.Cache(**{**CACHE, "k": CACHE["k"] + 4096})
    for caches in ([one, one], [other_pool, one, other_tables, tq.Cache(**CACHE)]):
        assert "twice" in refused(INVALID, lambda: tq.TreeAccept(caches, **ACCEPT).launch())
    tq.TreeAccept([one, other_tables, other_pool], **{**ACCEPT, "trees": 0}).launch()


@pytest.mark.parametrize("code,change", [
    (INVALID, dict(logits=0)), (INVALID, dict(uniform=0)), (INVALID, dict(tokens=0)), (INVALID, dict(workspace=0)), (INVALID, dict(workspace=A + 8)), (INVALID, dict(workspace_bytes=8)),
    (UNSUPPORTED, dict(vocab=0)), (UNSUPPORTED, dict(vocab=(1 << 20) + 1)), (UNSUPPORTED, dict(rows=65536)), (INVALID, dict(logits_stride=99)), (INVALID, dict(logits=A + 2)),
    (INVALID, dict(top_k=A + 1)), (INVALID, dict(temperature=A + 2)), (INVALID, dict(probs=A + 2)),
])
def test_sample_refuses(code, change):
    refused(code, lambda: tq.Sample(**{**SAMPLE, **change}).launch())


@pytest.mark.parametrize("code,change", [
    (INVALID, dict(k=0)), (UNSUPPORTED, dict(type=tq.TQ_FP32)), (INVALID, dict(type=tq.TQ_INT8)), (UNSUPPORTED, dict(page_size=48)), (UNSUPPORTED, dict(head_dim=72)),
    (INVALID, dict(n_pages=0)), (UNSUPPORTED, dict(seq_pages=1 << 27)), (INVALID, dict(k=A + 8)), (INVALID, dict(page_stride=4096)), (INVALID, dict(table_stride=1)),
])
def test_every_call_refuses_a_cache_that_is_not_one(code, change):
    cache = tq.Cache(**{**CACHE, **change})
    refused(code, lambda: tq.CacheAppendNormed(cache, tq.HeadNorm(**NORM), **APPEND).launch())
    refused(code, lambda: tq.AttendTree(cache, **TREE).launch())
    refused(code, lambda: tq.AttendTree.workspace_bytes(cache, **TREE))
    refused(code, lambda: tq.TreeAccept([tq.Cache(**CACHE), cache], **ACCEPT).launch())


def test_null_structures_no_work_and_the_workspaces():
    lib = tq.load()
    c = tq.Cache(**CACHE)
    append, norm = tq.CacheAppendNormed(c, tq.HeadNorm(**NORM), **{**APPEND, "rows": 0}), tq.HeadNorm(**NORM)
    append.launch()
    assert lib.tq_cache_append_normed(c.address, None, norm.address, None) == INVALID and lib.tq_cache_append_normed(None, None, norm.address, None) == INVALID
    assert lib.tq_cache_append_normed(c.address, append._at[1], None, None) == INVALID
    assert lib.tq_attend_tree(c.address, None, None) == INVALID and lib.tq_attend_tree_workspace(c.address, None, None) == INVALID
    assert lib.tq_tree_accept(1, None, None, None) == INVALID and lib.tq_sample(None, None) == INVALID and lib.tq_sample_workspace(None, None) == INVALID
    made = tq.TreeAccept([c], **ACCEPT)
    assert lib.tq_tree_accept(1, None, made._at[2], None) == INVALID and lib.tq_tree_accept(4097, made._at[1], made._at[2], None) == UNSUPPORTED
    tq.AttendTree(c, **{**TREE, "trees": 0}).launch()
    tq.TreeAccept([c], **{**ACCEPT, "trees": 0}).launch()
    tq.Sample(**{**SAMPLE, "rows": 0}).launch()
    need = tq.AttendTree.workspace_bytes(c, **TREE)
    assert "needed" in refused(INVALID, lambda: tq.AttendTree(c, **{**TREE, "workspace_bytes": need - 1}).launch())
    need = tq.Sample.workspace_bytes(**SAMPLE)
    assert "needed" in refused(INVALID, lambda: tq.Sample(**{**SAMPLE, "workspace_bytes": need - 1}).launch())


def test_drawing_asks_for_no_more_room_than_it_uses():
    """Lists of keys, 8 bytes a logit, only where something can be cut off and LDS may be too small; of rows that one workgroup draws from nothing else."""
    def need(rows, vocab, **more):
        return tq.Sample.workspace_bytes(**{**SAMPLE, "rows": rows, "vocab": vocab, **more})

    filters = dict(top_k=A, top_p=A)
    assert need(65535, 100, **filters) <= 256 and need(65535, 2048, **filters) <= 256 and need(65535, 4096) <= 256
    for only in (dict(top_k=A), dict(top_p=A), filters):
        assert 8 * 1000 * 2049 <= need(1000, 2049, **only) <= 8 * 1000 * 2049 + 512 and 8 * 64 * 128256 <= need(64, 128256, **only) <= 8 * 64 * (128256 + 4096)
    assert need(64, 128256, temperature=A, min_p=A) <= 8 * 64 * 4096
    assert need(1, 1) >= 16 and need(0, 128256) >= 16 and all(need(r + 1, v, **filters) >= need(r, v, **filters) for r in (1, 7) for v in (100, 4096, 4097, 1 << 20))
