"""Refusals of the operators around the 4-bit cache and of the eviction: every argument error is found on the host, with a text, before
anything is launched (no GPU needed)."""
import ctypes as C

import numpy as np
import pytest

import mx_reference as ref
from paper_2510_27641_amd import binding as sa


def _cache(paged=False, **kw):
    c = sa.MxCache()
    c.codes, c.scales = 0x10000, 0x20000
    c.B, c.H_kv, c.n_max, c.d = 2, 4, 512, 128
    c.codes_stride_b, c.codes_stride_h, c.codes_stride_n = 4 * 512 * 128, 512 * 128, 128
    c.scales_stride_b, c.scales_stride_h, c.scales_stride_n = 4 * 512 * 8, 512 * 8, 8
    if paged:
        c.page_table, c.page_size, c.max_pages_per_seq, c.num_pages = 0x30000, 16, 32, 100
        c.codes_stride_h, c.codes_stride_page, c.scales_stride_h, c.scales_stride_page = 16 * 128, 4 * 16 * 128, 16 * 8, 4 * 16 * 8
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _rows(cache, **kw):
    a = sa.MxRowsArgs()
    a.cache, a.k, a.v, a.dtype, a.T = cache, 0x40000, 0x50000, sa.BF16, 7
    a.stride_b, a.stride_h, a.stride_t = 4 * 7 * 128, 7 * 128, 128
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def _attn(cache, **kw):
    a = sa.MxAttnArgs()
    a.cache, a.q, a.dtype, a.H_q, a.T = cache, 0x40000, sa.BF16, 16, 5
    a.q_stride_b, a.q_stride_h, a.q_stride_t = 16 * 5 * 128, 5 * 128, 128
    a.indices, a.counts, a.idx_stride_row, a.idx_capacity = 0x50000, 0x60000, 512, 512
    a.out = 0x70000
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def _evict(**kw):
    a = sa.EvictArgs()
    a.probs, a.probs_stride_b, a.probs_stride_row = 0x10000, 8 * 3 * 512, 512
    a.B, a.H, a.n_max, a.H_draft, a.S = 2, 4, 512, 8, 3
    a.scores, a.positions, a.scores_out, a.positions_out = 0x20000, 0x30000, 0x20000, 0x30000
    a.row_stride_b, a.row_stride_h = 4 * 512, 512
    a.seq_lens, a.next_positions, a.decay, a.budget, a.sinks, a.recent = 0x40000, 0x50000, 0.9, 300, 4, 64
    a.move_src, a.move_dst, a.move_stride_row, a.move_capacity, a.move_counts, a.new_lens = 0x60000, 0x70000, 256, 212, 0x80000, 0x90000
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def _move(paged=False, plane=(), **kw):
    a = sa.MoveArgs()
    a.move_src, a.move_dst, a.move_counts, a.move_stride_row, a.move_capacity = 0x10000, 0x20000, 0x30000, 256, 212
    a.B, a.H, a.n_max, a.num_planes = 2, 4, 512, 2
    for p in (a.planes[0], a.planes[1]):
        p.data, p.row_bytes, p.H_kv = 0x40000, 256, 8
        p.stride_b, p.stride_h, p.stride_n = 8 * 512 * 256, 512 * 256, 256
    if paged:
        a.page_table, a.page_size, a.max_pages_per_seq = 0x50000, 16, 32
        for p in (a.planes[0], a.planes[1]):
            p.stride_page, p.num_pages = 8 * 16 * 256, 70
    for k, v in kw.items():
        setattr(a, k, v)
    for k, v in plane:
        setattr(a.planes[1], k, v)
    return a


BAD_CACHES = [
    (dict(codes=None), sa.EINVAL), (dict(scales=None), sa.EINVAL), (dict(B=0), sa.EINVAL), (dict(n_max=-1), sa.EINVAL), (dict(d=96), sa.ESHAPE),
    (dict(codes_stride_n=64), sa.ESHAPE), (dict(scales_stride_n=4), sa.ESHAPE), (dict(codes_stride_h=-128), sa.ESHAPE),
    (dict(codes_stride_n=136), sa.EALIGN), (dict(scales_stride_n=10), sa.EALIGN), (dict(codes=0x10008), sa.EALIGN), (dict(scales=0x20002), sa.EALIGN),
    (dict(codes_stride_b=24), sa.EALIGN), (dict(B=1 << 20, H_kv=1 << 10), sa.ESHAPE),
]
BAD_POOLS = [
    (dict(page_size=12), sa.ESHAPE), (dict(page_size=0), sa.ESHAPE), (dict(max_pages_per_seq=31), sa.ESHAPE), (dict(num_pages=0), sa.EINVAL),
    (dict(codes_stride_page=0), sa.ESHAPE), (dict(scales_stride_page=2), sa.EALIGN),
]


@pytest.mark.parametrize("paged,kw,status", [(False, *x) for x in BAD_CACHES] + [(True, *x) for x in BAD_POOLS])
def test_caches_are_refused_by_every_call(paged, kw, status):
    lib = sa.load()
    cache = _cache(paged, **kw)
    for fn, args in ((lib.specattn_mx_store, _rows(cache)), (lib.specattn_mx_load, _rows(cache)), (lib.specattn_mx_decode_attn, _attn(cache))):
        assert fn(C.byref(args), None) == status
        assert sa.last_error() != ""


@pytest.mark.parametrize("kw,status", [
    (dict(k=None), sa.EINVAL), (dict(v=None), sa.EINVAL), (dict(T=0), sa.EINVAL), (dict(dtype=9), sa.EUNSUPPORTED), (dict(k=0x40008), sa.EALIGN),
    (dict(stride_t=132), sa.EALIGN), (dict(stride_h=4), sa.EALIGN),
])
def test_rows_are_refused(kw, status):
    lib = sa.load()
    for fn in (lib.specattn_mx_store, lib.specattn_mx_load):
        assert fn(C.byref(_rows(_cache(), **kw)), None) == status
        assert sa.last_error() != ""
    assert lib.specattn_mx_store(None, None) == sa.EINVAL


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), sa.EINVAL), (dict(out=None), sa.EINVAL), (dict(counts=None), sa.EINVAL), (dict(indices=None), sa.EINVAL), (dict(H_q=0), sa.EINVAL),
    (dict(T=9), sa.ESHAPE), (dict(H_q=15), sa.ESHAPE), (dict(dtype=sa.F32), sa.EUNSUPPORTED), (dict(idx_capacity=0), sa.ESHAPE),
    (dict(idx_stride_row=511), sa.ESHAPE), (dict(chunk_size=3), sa.ESHAPE), (dict(chunk_size=2048), sa.ESHAPE),
    (dict(chunk_size=16, indices=None, counts=None), sa.EUNSUPPORTED), (dict(indices_are_physical=1, indices=None, counts=None), sa.ESHAPE),
    (dict(indices_are_physical=1), sa.ESHAPE), (dict(k_new=0x1000), sa.EINVAL), (dict(q=0x40008), sa.EALIGN), (dict(q_stride_t=4), sa.EALIGN),
    (dict(k_new=0x1000, v_new=0x2008), sa.EALIGN), (dict(idx_capacity=2 ** 30, idx_stride_row=2 ** 30, chunk_size=4), sa.ESHAPE),
    (dict(), sa.EWORKSPACE), (dict(workspace=0x1010, workspace_bytes=1 << 30), sa.EWORKSPACE), (dict(workspace=0x1000, workspace_bytes=256), sa.EWORKSPACE),
])
def test_attention_is_refused(kw, status):
    lib = sa.load()
    assert lib.specattn_mx_decode_attn(C.byref(_attn(_cache(), **kw)), None) == status
    assert sa.last_error() != ""


def test_attention_over_more_than_64_gib_is_refused():
    far = _cache(True, num_pages=1 << 24, codes_stride_page=1 << 14, scales_stride_page=1 << 10)
    assert sa.load().specattn_mx_decode_attn(C.byref(_attn(far)), None) == sa.ESHAPE and "64 GiB" in sa.last_error()
    wide = _cache(codes_stride_n=1 << 30)
    assert sa.load().specattn_mx_decode_attn(C.byref(_attn(wide)), None) == sa.ESHAPE


def test_workspace_sizes():
    assert sa.specattn_mx_workspace_size(_attn(_cache())) % 256 == 0
    assert 0 < sa.specattn_mx_workspace_size(_attn(_cache(), H_q=4, T=1)) < sa.specattn_mx_workspace_size(_attn(_cache(), H_q=64))
    assert sa.specattn_mx_workspace_size(_attn(_cache(), H_q=30)) == 0 and sa.specattn_mx_workspace_size(_attn(_cache(), T=9)) == 0
    assert sa.specattn_evict_workspace_size(_evict()) > 0 and sa.specattn_evict_workspace_size(_evict(B=0)) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(scores=None), sa.EINVAL), (dict(positions_out=None), sa.EINVAL), (dict(next_positions=None), sa.EINVAL), (dict(move_dst=None), sa.EINVAL),
    (dict(new_lens=None), sa.EINVAL), (dict(new_lens=0x40000), sa.EINVAL), (dict(B=0), sa.EINVAL), (dict(budget=0), sa.EINVAL),
    (dict(decay=1.5), sa.EINVAL), (dict(decay=float("nan")), sa.EINVAL), (dict(n_max=(1 << 19) + 1), sa.ESHAPE), (dict(H_draft=6), sa.ESHAPE),
    (dict(S=0), sa.EINVAL), (dict(probs_stride_row=500), sa.ESHAPE), (dict(row_stride_h=100), sa.ESHAPE), (dict(sinks=-1), sa.ESHAPE),
    (dict(sinks=200, recent=101), sa.ESHAPE), (dict(move_capacity=211), sa.ESHAPE), (dict(move_capacity=0, budget=512), sa.ESHAPE),
    (dict(move_stride_row=100), sa.ESHAPE), (dict(), sa.EWORKSPACE),
])
def test_eviction_is_refused(kw, status):
    lib = sa.load()
    assert lib.specattn_evict_select(C.byref(_evict(**kw)), None, 0, None) == status
    assert sa.last_error() != ""
    assert lib.specattn_evict_select(C.byref(_evict()), 0x1000, 256, None) == sa.EWORKSPACE


@pytest.mark.parametrize("paged,plane,kw,status", [
    (False, (), dict(move_src=None), sa.EINVAL), (False, (), dict(B=0), sa.EINVAL), (False, (), dict(move_capacity=513, move_stride_row=600), sa.ESHAPE),
    (False, (), dict(move_stride_row=100), sa.ESHAPE), (False, (), dict(num_planes=0), sa.ESHAPE), (False, (), dict(num_planes=9), sa.ESHAPE),
    (False, (("data", None),), {}, sa.EINVAL), (False, (("H_kv", 6),), {}, sa.ESHAPE), (False, (("row_bytes", 6),), {}, sa.ESHAPE),
    (False, (("row_bytes", 8196),), {}, sa.ESHAPE), (False, (("stride_n", 128),), {}, sa.ESHAPE), (False, (("stride_n", 264),), {}, sa.EALIGN),
    (False, (("data", 0x40004),), {}, sa.EALIGN), (True, (), dict(page_size=10), sa.ESHAPE), (True, (), dict(max_pages_per_seq=31), sa.ESHAPE),
    (True, (("num_pages", 0),), {}, sa.ESHAPE), (True, (("stride_page", 0),), {}, sa.ESHAPE), (True, (("stride_page", 24),), {}, sa.EALIGN),
])
def test_moves_are_refused(paged, plane, kw, status):
    assert sa.load().specattn_evict_move(C.byref(_move(paged, plane, **kw)), None) == status
    assert sa.last_error() != ""


def test_the_reference_quantiser_takes_the_nearest_value():
    """By trying all sixteen codes of every element."""
    rng = np.random.default_rng(0)
    x = (rng.standard_normal((50, 64)) * 2.0 ** rng.integers(-20, 20, size=(50, 1))).astype(np.float32)
    codes, scales = ref.quantise(x)
    got = ref.values(codes, scales)
    unit = np.repeat(2.0 ** (scales.astype(np.float64) - 127), 32, -1)
    every = np.concatenate((ref.GRID, -ref.GRID)) * unit[..., None]
    assert np.array_equal(np.abs(got - x), np.abs(every - x[..., None].astype(np.float64)).min(-1))
    assert ((np.abs(x).reshape(50, 2, 32).max(-1) / unit.reshape(50, 2, 32)[..., 0]) >= 4).all() and (np.abs(x) < 8 * unit).all()
    assert np.array_equal(ref.unpack(ref.pack(codes)), codes)


def test_the_reference_eviction_by_hand():
    scores = np.array([[[5.0, 1.0, 4.0, 1.0, 3.0, 2.0]]], dtype=np.float32)
    positions = np.array([[[0, 1, 2, 3, 4, 5]]], dtype=np.int32)
    s, p, moves, lens, _ = ref.evict(scores, positions, np.array([6]), np.array([6]), 3, 0, 1, 1.0)
    assert moves == [[(5, 1)]] and list(lens) == [3]           # slot 5 is the newest; 0 and 2 weigh most
    assert s.tolist() == [[[5.0, 2.0, 4.0, 0.0, 0.0, 0.0]]] and p.tolist() == [[[0, 5, 2, -1, -1, -1]]]
