"""Refusals of the serving loop's operators: every argument error is found on the host, with a text, before anything is launched (no GPU
needed); and the references that the GPU tests compare with."""
import ctypes as C

import numpy as np
import pytest

import serve_reference as ref
from paper_2510_27641_amd import binding as sa


def _set(a, kw):
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def _pages(**kw):
    a = sa.PagesArgs()
    a.page_table, a.B, a.page_size, a.max_pages_per_seq, a.num_pages = 0x10000, 4, 16, 32, 100
    a.free_pages, a.free_count, a.free_count_out, a.seq_lens, a.new_lens, a.lens_out = 0x20000, 0x30000, 0x30000, 0x40000, 0x50000, 0x40000
    a.slots, a.token_capacity = 0x60000, 64
    return _set(a, kw)


def _store(**kw):
    a = sa.StoreArgs()
    a.k, a.v, a.dtype, a.B, a.T, a.H_kv, a.d = 0x10000, 0x20000, sa.BF16, 1, 50, 8, 128
    a.stride_b, a.stride_t, a.stride_h = 0, 1024, 128
    a.k_cache, a.v_cache, a.num_pages, a.page_size = 0x30000, 0x40000, 20, 16
    a.cache_stride_page, a.cache_stride_h, a.cache_stride_n = 8 * 16 * 128, 16 * 128, 128
    a.slots, a.num_slots = 0x50000, 50
    return _set(a, kw)


def _prompt(paged=False, **kw):
    a = sa.PromptArgs()
    a.q, a.k, a.v, a.dtype = 0x10000, 0x20000, 0x30000, sa.BF16
    a.B, a.H_q, a.H_kv, a.d, a.total_q, a.total_kv = 3, 32, 8, 128, 5000, 5000
    a.q_stride_t, a.q_stride_h, a.kv_stride_n, a.kv_stride_h = 32 * 128, 128, 8 * 128, 128
    a.q_starts, a.out_lowp = 0x40000, 0x50000
    if paged:
        a.page_table, a.page_size, a.max_pages_per_seq, a.num_pages, a.seq_lens = 0x60000, 16, 100, 300, 0x70000
        a.kv_stride_page, a.kv_stride_h, a.kv_stride_n = 8 * 16 * 128, 16 * 128, 128
    return _set(a, kw)


def _tree(paged=False, **kw):
    a = sa.TreeArgs()
    a.q, a.k, a.v, a.k_new, a.v_new, a.dtype = 0x10000, 0x20000, 0x30000, 0x40000, 0x50000, sa.F16
    a.B, a.H_q, a.H_kv, a.T, a.d, a.n_max = 2, 16, 4, 20, 64, 512
    a.q_stride_b, a.q_stride_h, a.q_stride_t = 16 * 20 * 64, 20 * 64, 64
    a.kv_stride_b, a.kv_stride_h, a.kv_stride_n = 4 * 512 * 64, 512 * 64, 64
    a.tree_masks, a.out = 0x60000, 0x70000
    a.indices, a.counts, a.idx_stride_row, a.idx_capacity = 0x80000, 0x90000, 512, 512
    if paged:
        a.page_table, a.page_size, a.max_pages_per_seq, a.num_pages = 0xa0000, 16, 32, 70
        a.kv_stride_page, a.kv_stride_h = 4 * 16 * 64, 16 * 64
    return _set(a, kw)


@pytest.mark.parametrize("kw,status", [
    (dict(page_table=None), sa.EINVAL), (dict(free_pages=None), sa.EINVAL), (dict(free_count=None), sa.EINVAL), (dict(free_count_out=None), sa.EINVAL),
    (dict(seq_lens=None), sa.EINVAL), (dict(new_lens=None), sa.EINVAL), (dict(lens_out=None), sa.EINVAL), (dict(B=0), sa.EINVAL), (dict(num_pages=0), sa.EINVAL),
    (dict(max_pages_per_seq=-1), sa.EINVAL), (dict(token_capacity=0), sa.EINVAL), (dict(slots=None, positions=0x1000), sa.EINVAL),
    (dict(page_size=12), sa.ESHAPE), (dict(page_size=0), sa.ESHAPE), (dict(num_pages=1 << 27), sa.ESHAPE), (dict(max_pages_per_seq=1 << 27), sa.ESHAPE),
    (dict(B=1 << 27), sa.ESHAPE), ({}, sa.EWORKSPACE),
])
def test_pages_refusals(kw, status):
    a = _pages(**kw)
    assert sa.load().specattn_pages_update(C.byref(a), None, 0, None) == status and sa.last_error()


@pytest.mark.parametrize("kw,status", [
    (dict(k=None), sa.EINVAL), (dict(v_cache=None), sa.EINVAL), (dict(slots=None), sa.EINVAL), (dict(T=0), sa.EINVAL), (dict(num_slots=0), sa.EINVAL),
    (dict(page_size=0), sa.EINVAL), (dict(dtype=9), sa.EUNSUPPORTED), (dict(d=100), sa.EALIGN), (dict(k=0x10008), sa.EALIGN), (dict(stride_h=132), sa.EALIGN),
    (dict(cache_stride_n=-128), sa.ESHAPE), (dict(cache_stride_n=64), sa.ESHAPE), (dict(cache_stride_page=0), sa.ESHAPE), (dict(cache_stride_h=128), sa.ESHAPE),
    (dict(B=1 << 20, T=1 << 12), sa.ESHAPE), (dict(H_kv=1 << 20), sa.ESHAPE),
])
def test_store_refusals(kw, status):
    a = _store(**kw)
    assert sa.load().specattn_cache_store(C.byref(a), None) == status and sa.last_error()


@pytest.mark.parametrize("paged,kw,status", [
    (False, dict(q=None), sa.EINVAL), (False, dict(out_lowp=None), sa.EINVAL), (False, dict(q_starts=None), sa.EINVAL), (False, dict(B=0), sa.EINVAL),
    (False, dict(total_q=0), sa.EINVAL), (False, dict(total_kv=0), sa.EINVAL), (False, dict(dtype=sa.F32), sa.EUNSUPPORTED), (False, dict(H_q=30), sa.ESHAPE),
    (False, dict(d=96), sa.ESHAPE), (False, dict(kv_stride_n=64), sa.ESHAPE), (False, dict(q_stride_t=4100), sa.EALIGN), (False, dict(v=0x30008), sa.EALIGN),
    (False, dict(out=0x8), sa.EALIGN), (False, dict(total_q=1 << 26), sa.ESHAPE), (False, dict(total_kv=(1 << 30) + 1), sa.ESHAPE),
    (False, dict(seq_lens=0x1000), sa.EINVAL), (False, dict(B=1 << 22), sa.ESHAPE), (False, dict(B=(1 << 18) + 1), sa.ESHAPE),
    (False, dict(kv_stride_n=1 << 23), sa.ESHAPE), (True, dict(kv_stride_page=1 << 27), sa.ESHAPE),
    (True, dict(seq_lens=None), sa.EINVAL), (True, dict(kv_starts=0x1000), sa.EINVAL), (True, dict(page_size=24), sa.ESHAPE), (True, dict(num_pages=0), sa.EINVAL),
    (True, dict(kv_stride_page=0), sa.ESHAPE), (True, dict(kv_stride_page=12), sa.EALIGN), (True, dict(max_pages_per_seq=0), sa.ESHAPE),
    (True, dict(max_pages_per_seq=1 << 27), sa.ESHAPE), (True, dict(total_q=100), sa.EWORKSPACE),
])
def test_prompt_refusals(paged, kw, status):
    a = _prompt(paged, **kw)
    assert sa.load().specattn_prompt_attn(C.byref(a), None) == status and sa.last_error()
    if status != sa.EWORKSPACE:
        assert sa.specattn_prompt_workspace_size(a) == 0


@pytest.mark.parametrize("paged,kw,status", [
    (False, dict(q=None), sa.EINVAL), (False, dict(k_new=None), sa.EINVAL), (False, dict(tree_masks=None), sa.EINVAL), (False, dict(out=None), sa.EINVAL),
    (False, dict(indices=None), sa.EINVAL), (False, dict(indices=None, counts=None, indices_are_physical=1), sa.EINVAL), (False, dict(T=0), sa.EINVAL),
    (False, dict(T=65), sa.ESHAPE), (False, dict(dtype=sa.F32), sa.EUNSUPPORTED), (False, dict(H_q=18), sa.ESHAPE), (False, dict(d=32), sa.ESHAPE),
    (False, dict(H_q=1 << 13, T=64, H_kv=4), sa.ESHAPE), (False, dict(idx_capacity=0), sa.ESHAPE), (False, dict(idx_stride_row=5), sa.ESHAPE),
    (False, dict(chunk_size=12), sa.ESHAPE), (False, dict(chunk_size=16, indices=None, counts=None), sa.EUNSUPPORTED),
    (False, dict(idx_capacity=1 << 22, idx_stride_row=1 << 22, chunk_size=16), sa.ESHAPE), (False, dict(num_pages=3), sa.EINVAL),
    (False, dict(kv_stride_n=1 << 27), sa.ESHAPE), (True, dict(kv_stride_page=1 << 29), sa.ESHAPE),
    (False, dict(kv_stride_n=32), sa.ESHAPE), (False, dict(kv_stride_b=4), sa.EALIGN), (False, dict(k_new=0x40004), sa.EALIGN), (False, dict(q_stride_t=65), sa.EALIGN),
    (True, dict(chunk_size=16, indices_are_physical=1), sa.EUNSUPPORTED), (True, dict(page_size=10), sa.ESHAPE), (True, dict(max_pages_per_seq=8), sa.ESHAPE),
    (True, dict(num_pages=0), sa.EINVAL), (True, dict(kv_stride_page=-8), sa.ESHAPE), (True, {}, sa.EWORKSPACE), (False, {}, sa.EWORKSPACE),
])
def test_tree_refusals(paged, kw, status):
    a = _tree(paged, **kw)
    assert sa.load().specattn_tree_attn(C.byref(a), None) == status and sa.last_error()
    if status != sa.EWORKSPACE:
        assert sa.specattn_tree_workspace_size(a) == 0
    else:
        need = sa.specattn_tree_workspace_size(a)
        a.workspace, a.workspace_bytes = 0x100000, need - 1
        assert sa.load().specattn_tree_attn(C.byref(a), None) == sa.EWORKSPACE
        a.workspace, a.workspace_bytes = 0x100080, need
        assert sa.load().specattn_tree_attn(C.byref(a), None) == sa.EWORKSPACE


def test_null_structs():
    lib = sa.load()
    for call in (lambda: lib.specattn_pages_update(None, None, 0, None), lambda: lib.specattn_cache_store(None, None), lambda: lib.specattn_prompt_attn(None, None),
                 lambda: lib.specattn_tree_attn(None, None)):
        assert call() == sa.EINVAL and sa.last_error()
    assert lib.specattn_pages_workspace_size(None) == lib.specattn_prompt_workspace_size(None) == lib.specattn_tree_workspace_size(None) == 0


def test_reference_pages_by_hand():
    table = np.array([[7, 1, -1], [3, -1, -1], [0, 5, -1]], dtype=np.int32)
    got = ref.pages(table, np.array([2, 6, 4, -1, -1, -1, -1, -1], dtype=np.int32), 3, [8, 3, 5], [2, 12, 9], 4, 20)
    # sequence 0 returns page 1; sequence 1 takes 1 and then 4, sequence 2 takes 6
    assert got["table"].tolist() == [[7, 1, -1], [3, 1, 4], [0, 5, 6]] and got["count"] == 1 and got["free"].tolist()[:4] == [2, 6, 4, 1]
    assert got["starts"].tolist() == [0, 0, 9, 13] and got["slots"].tolist()[:13] == [15, 4, 5, 6, 7, 16, 17, 18, 19, 21, 22, 23, 24]
    assert got["slots"].tolist()[13:] == [-1] * 7 and got["owners"].tolist()[8:13] == [1, 2, 2, 2, 2]


def test_reference_attention_tolerances_catch_a_lost_key():
    rng = np.random.default_rng(0)
    q, k, v = rng.standard_normal((3, 64)), rng.standard_normal((50, 64)), rng.standard_normal((50, 64))
    seen = np.ones((3, 50), dtype=bool)
    out, lse, tol32, tol_low, tol_lse = ref.attend(q, k, v, seen, 0.125, "bf16")
    seen[:, 17] = False
    less, lse_less, *_ = ref.attend(q, k, v, seen, 0.125, "bf16")
    assert (np.abs(out - less) > tol_low).any(axis=1).all() and (np.abs(lse - lse_less) > tol_lse).all()
