"""Trees of more rows than a launch takes, with units that are cut and joined in each of the launches; page updates of more sequences than are found in LDS."""
import numpy as np
import pytest
import torch

import serve_reference as ref
import test_gpu_pages as pages
import test_gpu_tree as trees
from paper_2510_27641_amd import binding as sa

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H_q,T", [(8, 2), (64, 33)])
def test_cut_rows_in_several_launches(H_q, T):
    """300 sequences by 8 kv heads over one cache of 6000 positions (no stride between sequences), of which most see a few and some most; twice, the second time
    over the first one's workspace."""
    B, H_kv, d, n = 300, 8, 64, 6000
    g, rng = torch.Generator(device="cuda").manual_seed(31), np.random.default_rng(31)
    new = lambda *s: torch.randn(s, generator=g, device="cuda").half()  # noqa: E731
    k, v, q, k_new, v_new = new(1, H_kv, n, d), new(1, H_kv, n, d), new(B, H_q, T, d), new(B, H_kv, T, d), new(B, H_kv, T, d)
    masks = trees.tree_masks(rng, B, T)
    lens = rng.integers(0, 60, B)
    far = np.array([0, 3, 100, 255, 256, 257, 280, 299])                # 256 is where the second launch begins
    lens[far] = [6000, 1500, 5999, 4000, 3000, 700, 2500, 6000]
    out, lse = torch.full((B, H_q, T, d), 7.0, device="cuda"), torch.full((B, H_q, T), 7.0, device="cuda")
    x = torch.from_numpy(masks.view(np.int64)).cuda(), torch.from_numpy(lens.astype(np.int32)).cuda()
    a = sa.tree_args(q, k.expand(B, -1, -1, -1), v.expand(B, -1, -1, -1), k_new, v_new, x[0], out=out, lse=lse, seq_lens=x[1])
    ws = sa.alloc_workspace(sa.specattn_tree_workspace_size(a))
    sa.set_workspace(a, ws)
    sa.specattn_tree_attn(a)
    torch.cuda.synchronize()
    first = out.clone()
    out.fill_(7.0)
    sa.specattn_tree_attn(a)
    torch.cuda.synchronize()
    assert torch.equal(out, first) and torch.isfinite(out).all()
    key, val = k[0].double().cpu().numpy(), v[0].double().cpu().numpy()
    for b in [*far, 1, 120, 254, 258, 298]:
        bits = np.array([[bool((int(masks[b, t]) >> u) & 1) for u in range(T)] for t in range(T)])
        seen = np.concatenate((np.ones((T, lens[b]), dtype=bool), bits), 1)
        for h in (0, H_q // 2, H_q - 1):
            at = h // (H_q // H_kv)
            kk, vv = (np.concatenate((old[at, :lens[b]], fresh[b, at].double().cpu().numpy())) for old, fresh in ((key, k_new), (val, v_new)))
            want, want_lse, tol, _, tol_lse = ref.attend(q[b, h].double().cpu().numpy(), kk, vv, seen, d ** -0.5, "f16")
            assert (np.abs(out[b, h].double().cpu().numpy() - want) <= tol).all(), (b, h)
            assert (np.abs(lse[b, h].double().cpu().numpy() - want_lse) <= tol_lse).all(), (b, h)


@pytest.mark.parametrize("B,capacity", [(4096, 30000), (4097, 30000), (5000, 9000)])
def test_updates_of_many_sequences(B, capacity):
    rng = np.random.default_rng(B)
    width, page = 6, 8
    s = pages.State(B, width, page, rng.integers(0, width * page // 2, B), pages=B * 3, seed=B)
    for _ in range(2):
        pick = rng.random(B)
        new = np.where(pick < 0.7, s.lens + rng.integers(0, 7, B), np.where(pick < 0.85, s.lens // 2, 0))
        s.update(np.minimum(new, width * page), capacity)


def test_trees_stay_inside_their_workspace():
    """Cut and joined in exactly the bytes that the size asks for; a call that is not cut runs without any."""
    c = trees.Case(30, 8, 2, 16, 64, 3000, seed=5)
    lens = np.random.default_rng(5).integers(1, 3000, 30).astype(np.int32)
    a = c.args(seq_lens=lens)
    need = sa.specattn_tree_workspace_size(a)
    ws = torch.full((need + (1 << 16),), 0xab, dtype=torch.uint8, device="cuda")
    sa.set_workspace(a, ws[:need])
    sa.specattn_tree_attn(a)
    torch.cuda.synchronize()
    assert (ws[need:] == 0xab).all() and not (ws[:need] == 0xab).all()
    c.compare([[np.arange(x)] * 2 for x in lens])
    c = trees.Case(3, 8, 2, 16, 64, 448, seed=6)
    a = c.args()
    a.workspace, a.workspace_bytes = None, 0
    sa.specattn_tree_attn(a)
    torch.cuda.synchronize()
    c.compare([[np.arange(448)] * 2] * 3)
