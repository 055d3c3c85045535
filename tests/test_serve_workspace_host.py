"""Workspace sizes of the serving loop's operators: 0 for everything that the call itself refuses (no GPU needed)."""
import pytest

import test_serve_host as host
from paper_2510_27641_amd import binding as sa

REFUSED = [
    dict(page_table=None), dict(free_pages=None), dict(free_count=None), dict(free_count_out=None), dict(seq_lens=None), dict(new_lens=None), dict(lens_out=None), dict(B=0),
    dict(num_pages=0), dict(max_pages_per_seq=-1), dict(token_capacity=0), dict(slots=None, positions=0x1000), dict(page_size=12), dict(page_size=0), dict(num_pages=1 << 27),
    dict(max_pages_per_seq=1 << 27), dict(B=1 << 27),
]


@pytest.mark.parametrize("kw", REFUSED)
def test_pages(kw):
    assert sa.specattn_pages_workspace_size(host._pages(**kw)) == 0


def test_pages_that_are_not_refused():
    assert sa.specattn_pages_workspace_size(host._pages()) > 0
    assert sa.specattn_pages_workspace_size(host._pages(slots=None, token_capacity=0)) > 0


def test_trees_that_are_not_cut_need_none():
    """Up to 448 positions: every unit is finished where it is computed."""
    for kw in (dict(idx_capacity=448), dict(indices=None, counts=None, n_max=448), dict(idx_capacity=28, chunk_size=16)):
        a = host._tree(**kw)
        assert sa.specattn_tree_workspace_size(a) == 0
    for kw in (dict(idx_capacity=449), dict(indices=None, counts=None, n_max=449), dict(idx_capacity=29, chunk_size=16)):
        assert sa.specattn_tree_workspace_size(host._tree(**kw)) > 0


def test_trees_of_many_units():
    """Two partial results of up to 256 rows for each of 256 workgroups (fewer on smaller devices), and 8 bytes for each unit of a launch, of which there are 2048 * 256 at most;
    not a partial result for every unit."""
    a = host._tree(B=2048, H_q=1024, H_kv=1, T=64, d=128, n_max=100000, indices=None, counts=None, kv_stride_n=128, q_stride_t=128)
    assert 0 < sa.specattn_tree_workspace_size(a) <= 2 * 256 * 256 * (128 + 2) * 4 + 2048 * 256 * 8 + 2 * 256
