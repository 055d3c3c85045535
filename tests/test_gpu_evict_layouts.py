"""Moves and attention rows in layouts other than the plain one."""
import numpy as np
import pytest
import torch

from paper_2510_27641_amd import binding as sa

pytestmark = pytest.mark.gpu


def test_moves_with_heads_inside_positions_pitched_rows_and_single_heads():
    rng = np.random.default_rng(2)
    B, H, n = 2, 3, 40
    src, dst = np.tile(np.arange(30, 40, dtype=np.int32), (B * H, 1)), np.stack([rng.permutation(30)[:10] for _ in range(B * H)]).astype(np.int32)
    moves = [torch.from_numpy(x).cuda() for x in (src, dst, np.full(B * H, 10, dtype=np.int32))]
    base = [torch.from_numpy(rng.integers(0, 255, size=shape, dtype=np.uint8)).cuda() for shape in ((B, n, H, 64), (B, H, n, 48), (B, H, n + 5, 16))]
    planes = [base[0].transpose(1, 2), base[1][..., :32], base[2][:, :, :n]]
    want = [x.clone() for x in base]
    for b in range(B):
        for h in range(H):
            for a, d in zip(src[b * H + h], dst[b * H + h]):
                want[0][b, d, h] = base[0][b, a, h]
                want[1][b, h, d, :32] = base[1][b, h, a, :32]
                want[2][b, h, d] = base[2][b, h, a]
    sa.specattn_evict_move(sa.move_args(*moves, planes, B=B))
    assert all(torch.equal(x, y) for x, y in zip(base, want))
