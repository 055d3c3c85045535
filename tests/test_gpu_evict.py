"""Eviction: scores, kept slots and moves against the plain form, exactly; rows of any caches after the moves."""
import numpy as np
import pytest
import torch

import mx_reference as ref
from paper_2510_27641_amd import binding as sa

pytestmark = pytest.mark.gpu


def _dev(x):
    return None if x is None else torch.from_numpy(np.ascontiguousarray(x)).cuda()


def _select(scores, positions, lens, nxt, budget, *, sinks=0, recent=0, decay=1.0, probs=None, in_place=True, flags=True, seq_lens=True, pad=0):
    """Runs the call; returns what it wrote, with the moves as lists of pairs."""
    B, H, n = scores.shape
    wide_s, wide_p = torch.full((B, H, n + pad), 55.0, device="cuda"), torch.full((B, H, n + pad), 55, dtype=torch.int32, device="cuda")
    s, p = wide_s[..., :n], wide_p[..., :n]
    s.copy_(_dev(scores)); p.copy_(_dev(positions))
    so, po = (s, p) if in_place else (torch.full_like(wide_s, 77.0)[..., :n], torch.full_like(wide_p, 77)[..., :n])
    cap = max(1, min(budget, n - budget))
    src, dst = (torch.full((B * H, cap + 3), -9, dtype=torch.int32, device="cuda") for _ in range(2))
    moved, new_lens = torch.full((B * H,), -9, dtype=torch.int32, device="cuda"), torch.full((B,), -9, dtype=torch.int32, device="cuda")
    bits = torch.full((B * H,), -9, dtype=torch.int32, device="cuda") if flags else None
    held = [_dev(probs), _dev(lens.astype(np.int32)) if seq_lens else None, _dev(nxt.astype(np.int32))]
    args = sa.evict_args(held[0], s, p, held[2], budget, scores_out=so, positions_out=po, move_src=src[:, :cap], move_dst=dst[:, :cap],
                         move_counts=moved, new_lens=new_lens, seq_lens=held[1], sinks=sinks, recent=recent, decay=decay, row_flags=bits)
    ws = sa.alloc_workspace(sa.specattn_evict_workspace_size(args))
    ws.fill_(0xA5)
    sa.specattn_evict_select(args, ws)
    torch.cuda.synchronize()
    assert (wide_s[..., n:] == 55).all() and (wide_p[..., n:] == 55).all()
    assert (src[:, cap:] == -9).all() and (dst[:, cap:] == -9).all()
    m = moved.cpu().numpy()
    a, b = src.cpu().numpy(), dst.cpu().numpy()
    return (so.cpu().numpy(), po.cpu().numpy(), [list(zip(a[r, :m[r]], b[r, :m[r]])) for r in range(B * H)], new_lens.cpu().numpy(),
            None if bits is None else bits.cpu().numpy()), (src[:, :cap], dst[:, :cap], moved)


def _check(scores, positions, lens, nxt, budget, in_place=True, **kw):
    given = {k: kw[k] for k in ("sinks", "recent", "decay", "probs") if k in kw}
    want = ref.evict(scores, positions, lens, nxt, budget, given.get("sinks", 0), given.get("recent", 0), given.get("decay", 1.0), given.get("probs"))
    got, moves = _select(scores, positions, lens, nxt, budget, in_place=in_place, **kw)
    inside = np.arange(scores.shape[2]) < lens[:, None, None]
    for g, w, before in ((got[0], want[0], scores if in_place else 77.0), (got[1], want[1], positions if in_place else 77)):
        assert np.array_equal(np.where(inside, g, 0), np.where(inside, w, 0), equal_nan=True)
        assert np.array_equal(np.where(inside, 0, g), np.where(inside, 0, np.broadcast_to(before, g.shape)), equal_nan=True)
    assert got[2] == want[2] and np.array_equal(got[3], want[3])
    if got[4] is not None:
        assert np.array_equal(got[4], want[4])
    return moves


def _state(rng, B, H, n, lens, ties=False):
    scores = rng.integers(0, 4, size=(B, H, n)).astype(np.float32) if ties else rng.random((B, H, n), dtype=np.float32) ** 8
    positions = np.stack([np.stack([rng.permutation(n) for _ in range(H)]) for _ in range(B)]).astype(np.int32)
    return scores, positions, np.asarray(lens), np.full(B, n)


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("n,budget", [(1, 1), (2, 1), (63, 20), (64, 64), (65, 64), (1000, 1), (1000, 999), (1025, 300), (5000, 2500), (40000, 39995)])
def test_sizes(n, budget, in_place):
    rng = np.random.default_rng(n)
    B, H = 2, 3
    state = _state(rng, B, H, n, [n, max(0, n - 7)])
    _check(*state, budget, in_place, probs=rng.random((B, H, 2, n), dtype=np.float32), decay=0.9, pad=5)


@pytest.mark.parametrize("H,H_draft,S", [(1, 1, 1), (1, 8, 3), (4, 4, 5), (4, 16, 2), (2, 6, 1)])
def test_members(H, H_draft, S):
    rng = np.random.default_rng(H_draft)
    state = _state(rng, 3, H, 777, [777, 500, 100])
    _check(*state, 300, probs=rng.random((3, H_draft, S, 777), dtype=np.float32), decay=0.97, sinks=4, recent=32)


def test_without_rows_lengths_and_flags():
    rng = np.random.default_rng(4)
    state = _state(rng, 2, 2, 300, [300, 300])
    _check(*state, 100, flags=False, seq_lens=False, sinks=1, recent=99)


@pytest.mark.parametrize("budget", [1, 37, 500, 999])
def test_ties(budget):
    """Four values in all: the lowest slots stay."""
    rng = np.random.default_rng(budget)
    _check(*_state(rng, 2, 2, 1000, [1000, 640], ties=True), budget)
    scores, positions, lens, nxt = _state(rng, 1, 1, 1000, [1000])
    _check(np.full_like(scores, 0.25), positions, lens, nxt, budget)
    _check(np.zeros_like(scores), positions, lens, nxt, budget, sinks=1, recent=0)
    _check(np.where(rng.random(scores.shape) < 0.5, 0.0, -0.0).astype(np.float32), positions, lens, nxt, budget)


def test_more_protected_tokens_than_the_budget_and_none():
    rng = np.random.default_rng(6)
    scores, positions, lens, nxt = _state(rng, 1, 2, 200, [200])
    _check(scores, np.full_like(positions, 2), lens, nxt, 50, sinks=3)                 # all equal: the lowest slots stay
    _check(scores, positions, lens, nxt + 1000, 50, recent=50)                         # nobody is that recent
    _check(scores, positions, lens, np.full(1, -2 ** 31), 50, recent=50)               # everybody is


def test_nan_infinities_and_negative_scores():
    rng = np.random.default_rng(7)
    scores, positions, lens, nxt = _state(rng, 2, 2, 400, [400, 300])
    scores -= np.float32(0.01)
    scores[0, 0, 5:9] = [np.nan, np.inf, -np.inf, np.nan]
    scores[1, 1, 350] = np.nan                                                          # behind the row: not looked at
    scores[1, 0, :200] = np.nan
    _check(scores, positions, lens, nxt, 150, sinks=3)
    _check(scores, positions, lens, nxt, 399, sinks=3, recent=20)


def test_empty_rows():
    rng = np.random.default_rng(8)
    _check(*_state(rng, 3, 2, 100, [0, 100, 0]), 30, probs=rng.random((3, 2, 1, 100), dtype=np.float32))


def test_rows_of_one_bit_pattern_apart():
    """Keys that agree in their first 22 bits, so that the last pass decides."""
    bits = np.uint32(0x3f800000) + np.random.default_rng(9).permutation(1000).astype(np.uint32)
    scores = bits.view(np.float32).reshape(1, 1, 1000)
    positions = np.arange(1000, dtype=np.int32).reshape(1, 1, 1000)
    _check(scores, positions, np.array([1000]), np.array([1000]), 333)


@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("H,H_kv", [(1, 1), (1, 4), (4, 4), (2, 4)])
def test_moves(H, H_kv, page):
    """Rows of 4, 8, 12, 16, 128, 256 and 260 bytes, for one choice per head and shared ones."""
    rng = np.random.default_rng(H * 10 + H_kv + page)
    B, n, budget = 3, 500, 200
    state = _state(rng, B, H, n, [500, 350, 60])
    moves = _check(*state, budget)
    pairs, _ = _select(*state, budget)[0][2], None
    per = -(-n // page) if page else 1
    slots, width = (B * per + 4, page) if page else (B, n)
    table = rng.permutation(slots)[:B * per].reshape(B, per).astype(np.int32) if page else None
    shapes = [(1, np.int32), (2, np.int32), (3, np.int32), (4, np.int32), (128, np.uint8), (128, np.int16), (65, np.float32)]
    planes = [rng.integers(0, 100, size=(slots, H_kv, width, w)).astype(t) for w, t in shapes]
    dev, t = [_dev(x) for x in planes], _dev(table)
    sa.specattn_evict_move(sa.move_args(*moves, dev, B=B, page_table=t, n_max=n))
    for before, after in zip(planes, dev):
        want = before.copy()
        for b in range(B):
            for kv in range(H_kv):
                for a, d in pairs[b * H + kv // (H_kv // H)]:
                    if page:
                        want[table[b, d // page], kv, d % page] = before[table[b, a // page], kv, a % page]
                    else:
                        want[b, kv, d] = before[b, kv, a]
        assert np.array_equal(after.cpu().numpy(), want)


def test_moves_that_lead_outside_are_left_out():
    n = 64
    src = torch.tensor([[10, 64, 12, -1, 14, 20]], dtype=torch.int32, device="cuda")
    dst = torch.tensor([[1, 2, 70, 4, 5, 6]], dtype=torch.int32, device="cuda")
    plane = torch.arange(n, dtype=torch.int32, device="cuda").repeat_interleave(4).view(4, 1, 16, 4).clone()
    before = plane.clone().view(n, 4)
    table = torch.tensor([[0, 1, 2, 3]], dtype=torch.int32, device="cuda")
    count = torch.tensor([100], dtype=torch.int32, device="cuda")                       # more than the lists hold
    sa.specattn_evict_move(sa.move_args(src, dst, count, [plane], B=1, page_table=table, n_max=n))
    want = before.clone()
    for a, d in ((10, 1), (14, 5), (20, 6)):
        want[d] = before[a]
    assert torch.equal(plane.view(n, 4), want)
    table[0, 0] = 4                                                                     # beyond the pool: nothing may move there
    plane.copy_(before.view(4, 1, 16, 4))
    sa.specattn_evict_move(sa.move_args(src, dst, count, [plane], B=1, page_table=table, n_max=n))
    assert torch.equal(plane.view(n, 4), before)


@pytest.mark.parametrize("B,H,n,budget", [(3, 1, 33000, 20000), (2, 1, 70001, 69990), (1, 2, 100000, 3), (65, 1, 9000, 8000), (2, 40, 20000, 1000)])
def test_long_rows(B, H, n, budget):
    """Rows that one workgroup holds and rows that are cut up, on both sides of the lines between them; ties across the cuts."""
    rng = np.random.default_rng(n)
    scores = np.round(rng.random((B, H, n), dtype=np.float32) * 3000) / 64
    positions = np.broadcast_to(np.arange(n, dtype=np.int32), (B, H, n)).copy()
    lens = np.maximum(0, n - np.arange(B) * (n // 3 + 11))
    probs = (np.round(rng.random((B, H, 1, n), dtype=np.float32) * 4) / 64).astype(np.float32)
    _check(scores, positions, lens, np.full(B, n), budget, probs=probs, sinks=min(2, budget), recent=min(40, budget - min(2, budget)))


@pytest.mark.parametrize("value", [0.0, 1.5])
def test_one_value_throughout_a_long_row(value):
    n = 50000
    scores, positions = np.full((1, 1, n), value, dtype=np.float32), np.arange(n, dtype=np.int32).reshape(1, 1, n)
    scores[0, 0, 40000] = np.nan
    _check(scores, positions, np.array([n]), np.array([n]), 20000, sinks=4, recent=64)
    _check(scores, positions, np.array([n]), np.array([n]), 20000, in_place=False)
