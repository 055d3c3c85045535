"""Layouts that the calls around the 4-bit cache and the eviction refuse: a pool taken for a contiguous cache.  Found on the host, before
anything is launched (no GPU needed)."""
import ctypes as C

import pytest
import torch

from paper_2510_27641_amd import binding as sa
from test_mx_host import _attn, _cache, _rows


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
