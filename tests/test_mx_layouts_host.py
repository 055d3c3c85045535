"""Layouts that the calls around the 4-bit cache and the eviction refuse: a pool taken for a contiguous cache, rows that share bytes.  Found on the host, before
anything is launched (no GPU needed)."""
import ctypes as C

import pytest
import torch

from paper_2510_27641_amd import binding as sa
from test_mx_host import _attn, _cache, _evict, _move, _rows


def _refused(fn, args, status=sa.ESHAPE):
    assert fn(C.byref(args), None) == status
    assert sa.last_error() != ""


@pytest.mark.parametrize("kw", [dict(), dict(indices=None, counts=None), dict(chunk_size=16)])
def test_a_pool_without_a_page_table_takes_lists_of_pool_slots_alone(kw):
    lib = sa.load()
    codes, scales = torch.zeros((10, 4, 16, 128), dtype=torch.uint8), torch.zeros((10, 4, 16, 8), dtype=torch.uint8)
    for cache in (sa.mx_cache(codes, scales, B=2), _cache(num_pages=10, page_size=16, codes_stride_page=4 * 16 * 128, scales_stride_page=4 * 16 * 8)):
        for fn, args in ((lib.specattn_mx_store, _rows(cache)), (lib.specattn_mx_load, _rows(cache)), (lib.specattn_mx_decode_attn, _attn(cache, **kw))):
            _refused(fn, args, sa.EINVAL)
    # and lists of pool slots are taken (refused for their workspace, behind every other check)
    _refused(lib.specattn_mx_decode_attn, _attn(sa.mx_cache(codes, scales, B=2), indices_are_physical=1), sa.EWORKSPACE)


OVERLAPPING_CACHES = [
    (False, dict(codes_stride_b=0)), (False, dict(scales_stride_b=0)), (False, dict(codes_stride_h=0)), (False, dict(scales_stride_h=0)),
    (False, dict(codes_stride_b=4 * 512 * 128 - 16)), (False, dict(scales_stride_h=512 * 8 - 4)), (False, dict(codes_stride_h=64)),
    (True, dict(codes_stride_h=16 * 128 - 16)), (True, dict(scales_stride_h=0)), (True, dict(codes_stride_page=16 * 128)), (True, dict(scales_stride_page=8)),
]


@pytest.mark.parametrize("paged,kw", OVERLAPPING_CACHES)
def test_rows_do_not_go_into_a_cache_whose_rows_share_bytes(paged, kw):
    """Stores race there; reading such a cache (a prompt that all sequences share) is no fault."""
    lib = sa.load()
    cache = _cache(paged, **kw)
    _refused(lib.specattn_mx_store, _rows(cache))
    _refused(lib.specattn_mx_decode_attn, _attn(cache), sa.EWORKSPACE)


@pytest.mark.parametrize("kw", [dict(stride_b=0), dict(stride_h=0), dict(stride_t=0), dict(stride_t=64), dict(stride_h=6 * 128), dict(stride_b=-8 * 128), dict(stride_h=-120)])
def test_rows_do_not_come_out_into_rows_that_share_bytes(kw):
    _refused(sa.load().specattn_mx_load, _rows(_cache(), **kw))


def test_layouts_without_shared_bytes_are_taken():
    """Heads inside positions, pitched rows, dimensions of size 1 with any stride: refused for what is looked at behind the layout alone."""
    lib = sa.load()
    one = _cache(B=1, codes_stride_b=0, scales_stride_b=0, H_kv=1, codes_stride_h=0, scales_stride_h=0)
    inside = _cache(codes_stride_n=4 * 128, codes_stride_h=128, scales_stride_n=4 * 8, scales_stride_h=8)
    pitched = _cache(codes_stride_n=144, codes_stride_h=512 * 144, codes_stride_b=4 * 512 * 144)
    for cache in (one, inside, pitched, _cache(True)):
        for fn in (lib.specattn_mx_store, lib.specattn_mx_load):
            _refused(fn, _rows(cache, stride_b=7 * 8 * 128, stride_t=8 * 128, stride_h=128, k=0x40008), sa.EALIGN)
    # rows that are read may be the same for all
    _refused(lib.specattn_mx_store, _rows(_cache(), stride_b=0, stride_h=0, stride_t=0, v=0x40008), sa.EALIGN)


@pytest.mark.parametrize("T", [2 ** 30 + 1, 2 ** 31 - 40, 2 ** 31 - 1])
def test_more_rows_than_are_counted_in_31_bits_are_refused(T):
    """The kernels count rows of whole workgroups past the last one."""
    lib = sa.load()
    for fn in (lib.specattn_mx_store, lib.specattn_mx_load):
        _refused(fn, _rows(_cache(), T=T, stride_h=2 ** 31 * 128, stride_b=2 ** 33 * 128))


@pytest.mark.parametrize("paged,plane", [
    (False, (("stride_b", -8 * 512 * 256),)), (False, (("stride_h", -512 * 256),)), (True, (("stride_h", -16 * 256),)),
    (False, (("stride_b", 0),)), (False, (("stride_h", 0),)), (False, (("stride_h", 512 * 256 - 16),)), (True, (("stride_h", 16),)), (True, (("stride_page", 16 * 256),)),
])
def test_moves_are_refused_in_planes_that_run_backwards_or_whose_rows_share_bytes(paged, plane):
    _refused(sa.load().specattn_evict_move, _move(paged, plane))


@pytest.mark.parametrize("kw", [dict(row_stride_b=512), dict(row_stride_b=4 * 512 - 1), dict(row_stride_b=1000, row_stride_h=600)])
def test_score_rows_that_share_entries_are_refused(kw):
    lib = sa.load()
    _refused(lambda args, stream: lib.specattn_evict_select(args, None, 0, stream), _evict(**kw))


def test_score_rows_of_any_order_are_taken():
    lib = sa.load()
    for kw in (dict(row_stride_b=512, row_stride_h=2 * 512), dict(row_stride_b=600, row_stride_h=5000), dict(B=1, row_stride_b=512), dict(H=1, row_stride_h=512, row_stride_b=512)):
        _refused(lambda args, stream: lib.specattn_evict_select(args, None, 0, stream), _evict(**kw), sa.EWORKSPACE)


def test_more_work_than_a_launch_takes_is_refused():
    """A launch has fewer than 2^32 threads along each axis: what asks for more is refused before anything runs."""
    lib = sa.load()
    for fn in (lib.specattn_mx_store, lib.specattn_mx_load):
        _refused(fn, _rows(_cache(), T=2 ** 28 + 1, stride_h=2 ** 31 * 128, stride_b=2 ** 33 * 128))
        _refused(fn, _rows(_cache(), T=2 ** 28, stride_h=2 ** 31 * 128, stride_b=2 ** 33 * 128, k=0x40008), sa.EALIGN)
    select = lambda args, stream: lib.specattn_evict_select(args, None, 0, stream)  # noqa: E731
    _refused(select, _evict(B=2 ** 18, H=16, H_draft=16, S=1, row_stride_b=16 * 512))
    _refused(select, _evict(B=2 ** 18 - 1, H=16, H_draft=16, S=1, row_stride_b=16 * 512), sa.EWORKSPACE)
    assert sa.specattn_evict_workspace_size(_evict(B=2 ** 18, H=16)) == 0
