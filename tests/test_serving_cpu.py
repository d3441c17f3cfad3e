"""What the batch-serving entry points refuse, before anything touches a GPU."""
import ctypes as C

import pytest

from paper_2502_12574_amd import binding as hb

A = 0x10000                                    # an aligned address that nobody follows
OFF = A + 8
B = A + 0x10000


def norm(**kw):
    a = dict(stream=None, x_dev=A, x_fp32=0, residual_dev=A, residual_fp32=0, weight_dev=A, n_rows=4, d=64, eps=1e-5,
             residual_out_dev=A, out_dev=B)
    a.update(kw)
    return hb.hi_add_rmsnorm(**a, check=False)


@pytest.mark.parametrize("kw,status", [
    (dict(x_dev=None), hb.HI_ERR_ARG), (dict(weight_dev=None), hb.HI_ERR_ARG), (dict(out_dev=None), hb.HI_ERR_ARG),
    (dict(x_dev=OFF), hb.HI_ERR_ARG), (dict(residual_dev=OFF), hb.HI_ERR_ARG), (dict(residual_out_dev=OFF), hb.HI_ERR_ARG),
    (dict(weight_dev=OFF), hb.HI_ERR_ARG), (dict(out_dev=OFF), hb.HI_ERR_ARG), (dict(n_rows=-1), hb.HI_ERR_ARG),
    (dict(d=0), hb.HI_ERR_ARG), (dict(x_fp32=2), hb.HI_ERR_ARG), (dict(residual_fp32=-1), hb.HI_ERR_ARG),
    (dict(eps=-1.0), hb.HI_ERR_ARG), (dict(eps=float("nan")), hb.HI_ERR_ARG), (dict(eps=float("inf")), hb.HI_ERR_ARG),
    (dict(x_fp32=1, out_dev=A, residual_dev=None, residual_out_dev=None), hb.HI_ERR_ARG),                                # an fp32 x and a bf16 output in one buffer
    (dict(d=60), hb.HI_ERR_UNSUPPORTED), (dict(d=16392), hb.HI_ERR_UNSUPPORTED), (dict(n_rows=0), hb.HI_OK),
    (dict(out_dev=A), hb.HI_ERR_ARG), (dict(out_dev=A, residual_out_dev=B), hb.HI_ERR_ARG),              # the residual's buffers
    (dict(n_rows=0, x_dev=None, residual_dev=None, residual_out_dev=None, out_dev=None), hb.HI_OK)])
def test_norm_refusals(kw, status):
    assert norm(**kw) == status


def linear(**kw):
    a = dict(stream=None, x_dev=A, codes_dev=A, scales_dev=A, zeros_dev=A, n_rows=3, n_in=256, n_out=128, x_heads=0, y_heads=0,
             y_dev=B)
    a.update(kw)
    return hb.hi_linear_quantized(**a, check=False)


@pytest.mark.parametrize("kw,status", [
    (dict(x_dev=None), hb.HI_ERR_ARG), (dict(codes_dev=None), hb.HI_ERR_ARG), (dict(scales_dev=None), hb.HI_ERR_ARG),
    (dict(zeros_dev=None), hb.HI_ERR_ARG), (dict(y_dev=None), hb.HI_ERR_ARG), (dict(x_dev=OFF), hb.HI_ERR_ARG),
    (dict(codes_dev=OFF), hb.HI_ERR_ARG), (dict(scales_dev=A + 1), hb.HI_ERR_ARG), (dict(y_dev=OFF), hb.HI_ERR_ARG),
    (dict(n_rows=-1), hb.HI_ERR_ARG), (dict(n_in=0), hb.HI_ERR_ARG), (dict(n_out=-16), hb.HI_ERR_ARG),
    (dict(n_in=(1 << 20) + 128), hb.HI_ERR_UNSUPPORTED), (dict(n_out=(1 << 24) + 16), hb.HI_ERR_UNSUPPORTED),
    (dict(x_heads=2), hb.HI_ERR_ARG), (dict(y_heads=-1), hb.HI_ERR_ARG), (dict(n_in=192), hb.HI_ERR_UNSUPPORTED),
    (dict(n_out=24), hb.HI_ERR_UNSUPPORTED), (dict(n_out=144, y_heads=1), hb.HI_ERR_UNSUPPORTED), (dict(n_rows=0), hb.HI_OK),
    (dict(y_dev=A), hb.HI_ERR_ARG), (dict(n_rows=0, x_dev=None, y_dev=None), hb.HI_OK)])
def test_linear_refusals(kw, status):
    assert linear(**kw) == status


@pytest.mark.parametrize("args,status", [
    ((None, 16, 128, A, A, A), hb.HI_ERR_ARG), ((A, 16, 128, None, A, A), hb.HI_ERR_ARG), ((A, 16, 128, A, None, A), hb.HI_ERR_ARG),
    ((A, 16, 128, A, A, None), hb.HI_ERR_ARG), ((OFF, 16, 128, A, A, A), hb.HI_ERR_ARG), ((A, 16, 128, OFF, A, A), hb.HI_ERR_ARG),
    ((A, 0, 128, A, A, A), hb.HI_ERR_ARG), ((A, 16, -128, A, A, A), hb.HI_ERR_ARG), ((A, 16, 100, A, A, A), hb.HI_ERR_UNSUPPORTED)])
def test_weight_quantize_refusals(args, status):
    assert hb.hi_weight_quantize(None, *args, check=False) == status


CACHE = dict(pages=A, scales=A, n_pages=9, n_kv_heads=2, page_rows=32, kv_bits=8)
BATCH = dict(page_table=A, past_lens=A, row_starts=A, n_seqs=2, table_pages=5, n_rows=7, max_rows=4)

SHARED = [
    (dict(pages=None), {}, hb.HI_ERR_ARG), (dict(scales=None), {}, hb.HI_ERR_ARG), (dict(pages=OFF), {}, hb.HI_ERR_ARG),
    (dict(scales=OFF), {}, hb.HI_ERR_ARG), (dict(n_pages=0), {}, hb.HI_ERR_ARG), (dict(n_kv_heads=0), {}, hb.HI_ERR_ARG),
    (dict(page_rows=8), {}, hb.HI_ERR_UNSUPPORTED), (dict(page_rows=48), {}, hb.HI_ERR_UNSUPPORTED),
    (dict(page_rows=2048), {}, hb.HI_ERR_UNSUPPORTED), (dict(kv_bits=4), {}, hb.HI_ERR_UNSUPPORTED),
    ({}, dict(page_table=None), hb.HI_ERR_ARG), ({}, dict(past_lens=None), hb.HI_ERR_ARG),
    ({}, dict(row_starts=None), hb.HI_ERR_ARG), ({}, dict(page_table=A + 2), hb.HI_ERR_ARG),
    ({}, dict(n_seqs=-1), hb.HI_ERR_ARG), ({}, dict(n_rows=-1), hb.HI_ERR_ARG), ({}, dict(table_pages=0), hb.HI_ERR_ARG),
    ({}, dict(max_rows=0), hb.HI_ERR_ARG), (dict(page_rows=1024), dict(table_pages=1 << 21), hb.HI_ERR_RANGE),
    (dict(page_rows=1024), dict(table_pages=(1 << 20) + 1), hb.HI_ERR_RANGE),
    ({}, dict(n_seqs=0, page_table=None, past_lens=None, row_starts=None), hb.HI_OK), ({}, dict(n_rows=0), hb.HI_OK)]


def structs(cache, batch):
    return hb.make_paged_cache(**{**CACHE, **cache}), hb.make_paged_batch(**{**BATCH, **batch})


def append(cache={}, batch={}, **kw):
    a = dict(q_in_dev=A, k_in_dev=A, v_in_dev=A, in_fp32=0, n_q_heads=4, rope_theta=1e4, q_scale=1.0, q_out_dev=A)
    a.update(kw)
    return hb.hi_paged_append(None, *structs(cache, batch), **a, check=False)


def attn(cache={}, batch={}, **kw):
    a = dict(q_dev=A, n_q_heads=4, q_prescaled=0, out_dev=B, workspace_dev=A)
    a.update(kw)
    return hb.hi_paged_attn(None, *structs(cache, batch), **a, check=False)


@pytest.mark.parametrize("cache,batch,status", SHARED)
def test_paged_cache_and_batch_refusals(cache, batch, status):
    assert append(cache, batch) == status
    assert attn(cache, batch) == status


@pytest.mark.parametrize("kw,status", [
    (dict(k_in_dev=None), hb.HI_ERR_ARG), (dict(v_in_dev=None), hb.HI_ERR_ARG), (dict(q_in_dev=None), hb.HI_ERR_ARG),
    (dict(q_out_dev=None), hb.HI_ERR_ARG), (dict(k_in_dev=OFF), hb.HI_ERR_ARG), (dict(q_out_dev=OFF), hb.HI_ERR_ARG),
    (dict(in_fp32=3), hb.HI_ERR_ARG), (dict(n_q_heads=0), hb.HI_ERR_ARG), (dict(rope_theta=-1.0), hb.HI_ERR_ARG),
    (dict(rope_theta=float("nan")), hb.HI_ERR_ARG), (dict(rope_theta=float("inf")), hb.HI_ERR_ARG),
    (dict(q_scale=0.0), hb.HI_ERR_ARG), (dict(q_scale=float("nan")), hb.HI_ERR_ARG),
    (dict(n_q_heads=0, q_in_dev=None), hb.HI_ERR_ARG), (dict(in_fp32=1), hb.HI_ERR_ARG)])    # fp32 queries in place of bf16 ones
def test_append_refusals(kw, status):
    assert append(**kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(q_dev=None), hb.HI_ERR_ARG), (dict(out_dev=None), hb.HI_ERR_ARG), (dict(workspace_dev=None), hb.HI_ERR_ARG),
    (dict(q_dev=OFF), hb.HI_ERR_ARG), (dict(workspace_dev=OFF), hb.HI_ERR_ARG), (dict(n_q_heads=3), hb.HI_ERR_ARG),
    (dict(n_q_heads=0), hb.HI_ERR_ARG), (dict(q_prescaled=2), hb.HI_ERR_ARG), (dict(n_q_heads=34), hb.HI_ERR_UNSUPPORTED),
    (dict(out_dev=A), hb.HI_ERR_ARG)])
def test_attention_refusals(kw, status):
    assert attn(**kw) == status


def test_null_structs_and_workspace_size():
    L, cache, batch = hb.lib(), *structs({}, {})
    assert L.hi_paged_attn(None, None, batch, A, 4, 0, A, A) == hb.HI_ERR_ARG
    assert L.hi_paged_append(None, cache, None, A, A, A, 0, 4, 0.0, 1.0, A) == hb.HI_ERR_ARG
    assert L.hi_paged_workspace_bytes(4, 2, None) == hb.HI_ERR_ARG
    n = C.c_int64()
    assert L.hi_paged_workspace_bytes(5, 2, C.byref(n)) == hb.HI_ERR_ARG
    assert L.hi_paged_workspace_bytes(34, 2, C.byref(n)) == hb.HI_ERR_UNSUPPORTED
    assert hb.hi_paged_workspace_bytes(32, 8) > 0
    with pytest.raises(hb.HiError):
        hb.hi_paged_workspace_bytes(5, 2)


def test_struct_layouts():
    assert C.sizeof(hb.hi_paged_cache) == 32 and hb.hi_paged_cache.n_pages.offset == 16
    assert C.sizeof(hb.hi_paged_batch) == 40 and hb.hi_paged_batch.max_rows.offset == 36


@pytest.mark.parametrize("cache,batch,kw", [
    # (bounds from the call's own sizes, before any launch) a short table and so many sequences that the blocks' starts count
    (dict(n_kv_heads=100), dict(n_seqs=1600000, n_rows=1600000, table_pages=1, max_rows=1), dict(n_q_heads=100)),
    (dict(kv_bits=16, n_kv_heads=100), dict(n_seqs=3000000, n_rows=3000000, table_pages=1, max_rows=1), dict(n_q_heads=100)),
    # a long table
    (dict(page_rows=1024), dict(n_seqs=100, n_rows=100, table_pages=1 << 19, max_rows=1), {}),
    (dict(page_rows=1024), dict(n_seqs=100, n_rows=1 << 20, table_pages=1 << 19, max_rows=1 << 20), {}),
    # more blocks than a launch has workgroups
    (dict(n_kv_heads=16), dict(n_seqs=1, n_rows=1 << 28, table_pages=1, max_rows=1 << 28), dict(n_q_heads=16)),
    (dict(n_kv_heads=65536), {}, dict(n_q_heads=65536))])
def test_attention_refuses_what_it_cannot_count(cache, batch, kw):
    assert attn(cache, batch, **kw) == hb.HI_ERR_RANGE


def test_a_step_without_rows_needs_no_buffers():
    for batch in (dict(n_rows=0), dict(n_seqs=0)):
        assert append({}, batch, q_in_dev=None, k_in_dev=None, v_in_dev=None, q_out_dev=None) == hb.HI_OK
        assert attn({}, batch, q_dev=None, out_dev=None) == hb.HI_OK
