"""The weights of the 4-bit attention one by one against 64 bits."""
import numpy as np
import pytest
import torch

import mx_weights as W
from paper_2510_27641_amd import binding as sa

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("far", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d,n", [(64, 60), (128, 100)])
@pytest.mark.parametrize("B,H_q,H,T", [(2, 2, 2, 1), (2, 8, 2, 5), (1, 8, 1, 6), (1, 8, 1, 8), (70, 1, 1, 1), (35, 8, 2, 5), (70, 6, 1, 8), (70, 8, 1, 8)])
def test_every_weight(B, H_q, H, T, d, n, dtype, far):
    """One to four query tiles, up to 64 rows and more."""
    codes, scales, q = W.inputs(B, H_q, H, T, d, n, B + H_q + T, far)
    want, bound = W.want_and_bound(*W.scores_and_values(codes, scales, q))
    held = [torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), torch.from_numpy(q).to(dtype).cuda()]
    out = torch.full((B, H_q, T, d), float("nan"), device="cuda")
    args = sa.mx_attn_args(held[2], sa.mx_cache(*held[:2]), out=out, sm_scale=1.0)
    ws = sa.alloc_workspace(sa.specattn_mx_workspace_size(args))
    args.workspace, args.workspace_bytes = ws.data_ptr(), ws.numel()
    sa.specattn_mx_decode_attn(args)
    got = out.cpu().double().numpy()
    assert (got[..., n:] == 0).all()
    assert (np.abs(got[..., :n] - want) <= bound).all(), (np.abs(got[..., :n] - want) / bound).max()
