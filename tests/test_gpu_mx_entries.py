"""List entries outside the 4-bit cache: each is read as the nearest slot inside it."""
import numpy as np
import pytest
import torch

import mx_reference as ref
from paper_2510_27641_amd import binding as sa
from test_gpu_mx_attention import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [0, 16])
def test_chunk_numbers_far_outside(page, d):
    """Also numbers whose first position does not fit in 31 bits."""
    n, chunk, wild = 200, 16, [2 ** 27, 2 ** 28, 2 ** 28 + 3, 2 ** 31 - 1, 13, 10 ** 6, -1, -2 ** 31]
    c = Case(1, 4, 1, 2, d, n, page=page, seed=41)
    lists = np.array([[3, *wild, 7]], dtype=np.int32)
    at = lambda u: np.arange(16) if u < 0 else np.minimum(u * chunk + np.arange(chunk), n - 1)  # noqa: E731
    # (a negative number's positions lie below 0)
    kept = np.concatenate([np.zeros(16, dtype=np.int64) if u < 0 else at(int(u)) for u in lists[0].astype(np.int64)])
    c.check([[kept]], lists=lists, counts=np.array([10], dtype=np.int32), chunk=chunk)
