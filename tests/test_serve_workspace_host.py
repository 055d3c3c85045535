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
