"""Moves and attention rows in layouts other than the plain one."""
import numpy as np
import pytest
import torch

import mx_reference as ref
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


@pytest.mark.parametrize("page", [0, 16])
def test_more_moves_than_a_workgroup_takes(page):
    """Rows of 257, 700 and 1100 moves, of none and of 256."""
    rng = np.random.default_rng(page)
    B, H, n, counts = 5, 2, 2400, [257, 700, 1100, 0, 256]
    cap = 1150
    src, dst = np.zeros((B * H, cap), dtype=np.int32), np.zeros((B * H, cap), dtype=np.int32)
    for r in range(B * H):
        m = counts[r // H]
        src[r, :m], dst[r, :m] = np.sort(1200 + rng.permutation(1200)[:m]), np.sort(rng.permutation(1200)[:m])
    moves = [torch.from_numpy(x).cuda() for x in (src, dst, np.repeat(counts, H).astype(np.int32))]
    per = n // page if page else 1
    slots, width = (B * per + 3, page) if page else (B, n)
    table = rng.permutation(slots)[:B * per].reshape(B, per).astype(np.int32) if page else None
    planes = [rng.integers(0, 1000, size=(slots, 2 * H, width, w), dtype=np.int32) for w in (32, 1, 2)]
    dev = [torch.from_numpy(x).cuda() for x in planes]
    held = None if table is None else torch.from_numpy(table).cuda()
    sa.specattn_evict_move(sa.move_args(*moves, dev, B=B, page_table=held, n_max=n))
    for before, after in zip(planes, dev):
        want = before.copy()
        for b in range(B):
            for kv in range(2 * H):
                a, d = src[b * H + kv // 2, :counts[b]], dst[b * H + kv // 2, :counts[b]]
                if page:
                    want[table[b, d // page], kv, d % page] = before[table[b, a // page], kv, a % page]
                else:
                    want[b, kv, d] = before[b, kv, a]
        assert np.array_equal(after.cpu().numpy(), want)


@pytest.mark.parametrize("n,pad", [(1000, 0), (1000, 24), (1000, 3), (1001, 7), (9000, 8), (9000, 1), (34000, 16), (34000, 5)])
def test_attention_rows_with_entries_behind_them(n, pad):
    """Rows of n entries with others behind them, which are NaN here, and sequences with rows in between: with and without whole 16 bytes."""
    rng = np.random.default_rng(n + pad)
    B, H, S, budget = 2, 2, 3, n // 2
    wide = torch.full((B, 2 * H + 1, S, n + pad), float("nan"), device="cuda")
    probs = rng.random((B, 2 * H, S, n), dtype=np.float32)
    wide[:, :2 * H, :, :n] = torch.from_numpy(probs).cuda()
    scores, positions = rng.random((B, H, n), dtype=np.float32), np.broadcast_to(np.arange(n, dtype=np.int32), (B, H, n)).copy()
    lens, nxt = np.array([n, n - 13]), np.array([n, n - 13])
    want = ref.evict(scores, positions, lens, nxt, budget, 4, 16, 0.8, probs)
    s, p = torch.from_numpy(scores).cuda(), torch.from_numpy(positions).cuda()
    src, dst = (torch.zeros((B * H, budget), dtype=torch.int32, device="cuda") for _ in range(2))
    moved, new_lens, flags = (torch.full((k,), -9, dtype=torch.int32, device="cuda") for k in (B * H, B, B * H))
    held = [torch.from_numpy(x.astype(np.int32)).cuda() for x in (lens, nxt)]
    args = sa.evict_args(wide[:, :2 * H, :, :n], s, p, held[1], budget, move_src=src, move_dst=dst, move_counts=moved, new_lens=new_lens, seq_lens=held[0],
                         sinks=4, recent=16, decay=0.8, row_flags=flags)
    sa.specattn_evict_select(args, sa.alloc_workspace(sa.specattn_evict_workspace_size(args)))
    s, p, a, d, m = (x.cpu().numpy() for x in (s, p, src, dst, moved))
    for b in range(B):
        assert np.array_equal(s[b, :, :lens[b]], want[0][b, :, :lens[b]]) and np.array_equal(p[b, :, :lens[b]], want[1][b, :, :lens[b]])
    assert [list(zip(a[r, :m[r]], d[r, :m[r]])) for r in range(B * H)] == want[2] and (flags == 0).all() and np.array_equal(new_lens.cpu().numpy(), want[3])
