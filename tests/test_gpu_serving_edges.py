"""Attention over prompts and trees where rows see nothing, values are not finite or close to fp32's end, rows are long, and neighbours differ; against
masked attention in 64 bits."""
import numpy as np
import pytest
import torch

import serve_reference as ref
import test_gpu_prompt as prompts
import test_gpu_tree as trees
from paper_2510_27641_amd import binding as sa

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("rows", [90, 3100])
def test_a_query_that_sees_nothing_beside_values_that_are_not_finite(rows, bad):
    """100 queries over 90 keys: the first ten see none.  90 rows of keys make units of 128 query rows, 3100 of them units of 256, in one part each."""
    H_q, H_kv, d = 512, 256, 64
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = (torch.randn((n, h, d), generator=g, device="cuda").bfloat16() for n, h in ((100, H_q), (rows, H_kv), (rows, H_kv)))
    v[5] = bad                                                          # seen from query 15 on
    starts, kv_starts = (torch.tensor([0, n], dtype=torch.int32, device="cuda") for n in (100, 90))
    out, low, lse = torch.full((100, H_q, d), 7.0, device="cuda"), torch.full((100, H_q, d), 7.0, dtype=q.dtype, device="cuda"), torch.full((100, H_q), 7.0, device="cuda")
    for want in (dict(out=out), dict(out_lowp=low)):
        a = sa.prompt_args(q, k, v, starts, kv_starts=kv_starts, lse=lse, **want)
        assert sa.specattn_prompt_workspace_size(a) == 0
        sa.specattn_prompt_attn(a)
        torch.cuda.synchronize()
        assert (lse[:10] == -float("inf")).all() and torch.isfinite(lse[10:]).all()
        lse.fill_(7.0)
    assert (out[:10] == 0).all() and (low[:10] == 0).all()
    seen = np.arange(90)[None] < np.arange(100)[:, None] - 9
    for h in (0, 301):
        want, _, tol32, tol_low, _ = ref.attend(*(x[:n, i].double().cpu().numpy() for x, n, i in ((q, 100, h), (k, 90, h // 2), (v, 90, h // 2))), seen, d ** -0.5, "bf16")
        assert (np.abs(out[:15, h].cpu().numpy() - want[:15]) <= tol32[:15]).all() and (np.abs(low[:15, h].double().cpu().numpy() - want[:15]) <= tol_low[:15]).all()


@pytest.mark.parametrize("q_lens,kv_lens", [([3], [700]), ([3], [4100]), ([40], [4100]), ([200], [1000])])
def test_prompts_with_values_at_the_end_of_fp32(q_lens, kv_lens):
    """3e38 in every row, in one part or several, waves that share rows or not: an average stays what it is however the call is cut."""
    c = prompts.Case(q_lens, 4, 2, 128, kv_lens=kv_lens, page=16, seed=21)
    c.v[:] = (c.v.float().sign() * 3e38).to(c.v.dtype)
    c.v[:, :, :32] = 3e38
    c.check()


@pytest.mark.parametrize("G,T,n", [(1, 5, 300), (1, 5, 5000), (4, 26, 5000), (8, 30, 3000)])
def test_trees_with_values_at_the_end_of_fp32(G, T, n):
    c = trees.Case(1, 2 * G, 2, T, 128, n, seed=22)
    for x in (c.v, c.v_new):
        x[:] = (x.float().sign() * 3e38).to(x.dtype)
        x[..., :32] = 3e38
    c.check([[np.arange(n)] * 2])
