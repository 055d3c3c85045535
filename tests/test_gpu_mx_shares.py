"""Shares of the 4-bit attention that begin in one row and end in another, several rows on."""
import numpy as np
import pytest

from test_gpu_mx_attention import Case

pytestmark = pytest.mark.gpu

CUS, TILE, SEG_COST, LAUNCH = 256, 32, 10, 512


def _rows_of_shares(sizes, workgroups=2 * CUS):
    """How many rows with positions each share meets: rows lie on one line, each of its tiles behind SEG_COST, cut into equal shares."""
    tiles = -(-np.asarray(sizes) // TILE)
    cost = np.where(tiles > 0, tiles + SEG_COST, 0)
    size = max(1, -(-int(cost.sum()) // workgroups))
    ends = np.cumsum(cost)
    first, last = (ends - cost + SEG_COST) // size, (ends - 1) // size
    met = np.zeros(workgroups, dtype=int)
    for a, b, t in zip(first, last, tiles):
        if t:
            met[a:b + 1] += 1
    return met


@pytest.mark.parametrize("dtype,d,G,T,new", [("bf16", 128, 1, 1, False), ("f16", 64, 4, 5, True), ("bf16", 64, 8, 8, False)])
def test_a_share_over_many_rows(dtype, d, G, T, new):
    """Hundreds of short rows, every third one empty, between a few of 40000 positions (repeats of 200: lists may name a position again)."""
    B, H, n, long = 130, 3, 200, 40000
    rng = np.random.default_rng(G)
    sizes = rng.choice([0, 1, 20, 33], size=B * H, p=[0.34, 0.22, 0.22, 0.22])
    sizes[rng.permutation(B * H)[:12]] = long - rng.integers(0, 100, size=12)
    met = _rows_of_shares(sizes)
    assert B * H <= LAUNCH and (met >= 3).sum() > 20 and (met == 1).sum() > 20
    lists = rng.integers(0, n, size=(B * H, long), dtype=np.int32)
    c = Case(B, G * H, H, T, d, n, dtype, new=new, seed=51)
    kept = [[lists[b * H + h, :sizes[b * H + h]] for h in range(H)] for b in range(B)]
    c.check(kept, lists=lists, counts=sizes.astype(np.int32))
