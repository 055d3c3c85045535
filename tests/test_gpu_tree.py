"""Attention of trees of drafted tokens over the cache, against masked attention in 64 bits."""
import numpy as np
import pytest
import torch

import serve_reference as ref
from paper_2510_27641_amd import binding as sa

pytestmark = pytest.mark.gpu


def tree_masks(rng, B, T):
    m = np.zeros((B, T), dtype=np.uint64)
    for b in range(B):
        for t in range(T):
            above = 0 if t == 0 else m[b, rng.integers(0, t)]
            m[b, t] = np.uint64(above) | np.uint64(1) << np.uint64(t)
    return m


class Case:
    def __init__(self, B, H_q, H_kv, T, d, n, dtype="bf16", *, page=0, seed=0, pitch=0):
        g, rng = torch.Generator().manual_seed(seed), np.random.default_rng(seed)
        self.B, self.H_q, self.H_kv, self.T, self.d, self.n, self.dtype, self.page = B, H_q, H_kv, T, d, n, dtype, page
        dt = ref.DT[dtype]
        per = -(-n // page) if page else 1
        pages, width = (B * per + 2, page) if page else (B, n)
        new = lambda *s: torch.randn(s, generator=g).to(dt)  # noqa: E731
        self.k, self.v = new(pages, H_kv, width, d + pitch), new(pages, H_kv, width, d + pitch)
        self.q, self.k_new, self.v_new = new(B, H_q, T, d), new(B, H_kv, T, d), new(B, H_kv, T, d)
        self.table = rng.permutation(pages)[:B * per].reshape(B, per).astype(np.int32) if page else None
        self.masks = tree_masks(rng, B, T)

    def rows(self, b, h, pos):
        if self.table is None:
            return self.k[b, h, pos, :self.d].double().numpy(), self.v[b, h, pos, :self.d].double().numpy()
        page = self.table[b][pos // self.page]
        return tuple(x[page, h, pos % self.page, :self.d].double().numpy() for x in (self.k, self.v))

    def args(self, *, lists=None, counts=None, seq_lens=None, nodes=None, chunk=0, want=("out", "low", "lse"), scale=0.0, physical=False):
        dev = lambda x: None if x is None else torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
        shape = tuple(self.q.shape)
        self.out = torch.full(shape, float("nan"), device="cuda") if "out" in want else None
        self.low = torch.full(shape, float("nan"), dtype=self.q.dtype, device="cuda") if "low" in want else None
        self.lse = torch.full(shape[:3], float("nan"), device="cuda") if "lse" in want else None
        self.keep = dict(q=self.q.cuda(), k=self.k.cuda(), v=self.v.cuda(), k_new=self.k_new.cuda(), v_new=self.v_new.cuda(), masks=dev(self.masks.view(np.int64)),
                         lists=dev(lists), counts=dev(counts), lens=dev(seq_lens), nodes=dev(nodes), table=None if physical else dev(self.table))
        x = self.keep
        a = sa.tree_args(x["q"], x["k"][..., :self.d], x["v"][..., :self.d], x["k_new"], x["v_new"], x["masks"], out=self.out, out_lowp=self.low, lse=self.lse,
                         indices=x["lists"], counts=x["counts"], seq_lens=x["lens"], node_counts=x["nodes"], chunk_size=chunk, page_table=x["table"],
                         n_max=self.n, sm_scale=scale, indices_are_physical=physical)
        self.ws = sa.alloc_workspace(sa.specattn_tree_workspace_size(a))
        sa.set_workspace(a, self.ws)
        return a

    def compare(self, kept, nodes=None, scale=0.0, skip=None):
        """kept[b][h]: positions that the row's list stands for."""
        G, T = self.H_q // self.H_kv, self.T
        scale = scale or self.d ** -0.5
        got = [None if x is None else x.cpu().double().numpy() for x in (self.out, self.low, self.lse)]
        for b in range(self.B):
            m = T if nodes is None else min(max(int(nodes[b]), 0), T)
            bits = np.array([[(int(self.masks[b, t]) >> u) & 1 and u < m for u in range(T)] for t in range(T)], dtype=bool)
            for h in range(self.H_q):
                key, val = self.rows(b, h // G, np.asarray(kept[b][h // G], dtype=np.int64))
                k = np.concatenate((key, self.k_new[b, h // G].double().numpy()))
                v = np.concatenate((val, self.v_new[b, h // G].double().numpy()))
                seen = np.concatenate((np.ones((T, len(key)), dtype=bool), bits), 1)
                seen[m:] = False
                if skip is not None:
                    seen[skip] = False
                out, lse, tol32, tol_low, tol_lse = ref.attend(self.q[b, h].double().numpy(), k, v, seen, scale, self.dtype)
                rows = np.ones(T, dtype=bool) if skip is None else ~skip
                for x, tol in ((got[0], tol32), (got[1], tol_low)):
                    if x is not None:
                        assert (np.abs(x[b, h] - out) <= tol)[rows].all(), (b, h, np.nanmax((np.abs(x[b, h] - out) / (tol + 1e-30))[rows]))
                if got[2] is not None:
                    some = np.isfinite(lse)
                    assert np.array_equal(some[rows], np.isfinite(got[2][b, h])[rows]) and (got[2][b, h][rows & ~some] == -np.inf).all()
                    some &= rows
                    assert (np.abs(got[2][b, h][some] - lse[some]) <= tol_lse[some]).all()

    def check(self, kept, **kw):
        a = self.args(**kw)
        sa.specattn_tree_attn(a)
        torch.cuda.synchronize()
        self.compare(kept, kw.get("nodes"), kw.get("scale", 0.0))
        return a


def make_lists(rng, B, H, n, fraction, capacity=None):
    kept = [[np.sort(rng.permutation(n)[:int(round(n * fraction * (0.5 + rng.random())))]) for _ in range(H)] for _ in range(B)]
    cap = capacity or max(1, max(len(x) for row in kept for x in row))
    lists, counts = np.full((B * H, cap), 2 ** 31 - 1, dtype=np.int32), np.zeros(B * H, dtype=np.int32)
    for r, x in enumerate(x for row in kept for x in row):
        lists[r, :len(x)], counts[r] = x, len(x)
    return kept, lists, counts


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H_q,H_kv,T", [(1, 1, 1), (4, 4, 7), (8, 2, 5), (8, 2, 13), (10, 2, 16), (8, 1, 9), (8, 1, 26), (8, 2, 64), (3, 1, 61)])
def test_lists(dtype, d, H_q, H_kv, T):
    """Query rows for one wave, two, four, and more than a workgroup takes."""
    c = Case(2, H_q, H_kv, T, d, 333, dtype, seed=H_q * 100 + T)
    kept, lists, counts = make_lists(np.random.default_rng(1), 2, H_kv, 333, 0.5)
    c.check(kept, lists=lists, counts=counts)


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 513])
@pytest.mark.parametrize("G,T", [(1, 3), (4, 12), (4, 30)])
def test_dense_lengths(n, G, T):
    c = Case(1, 2 * G, 2, T, 128, n, seed=n)
    c.check([[np.arange(n)] * 2])


@pytest.mark.parametrize("page", [0, 16, 4])
@pytest.mark.parametrize("G,T", [(2, 4), (4, 16), (5, 33)])
def test_ragged_dense_with_empty_rows(page, G, T):
    c = Case(6, 2 * G, 2, T, 128, 200, "f16", page=page, seed=3)
    lens = np.array([0, 1, 200, 37, 250, 0], dtype=np.int32)            # the fifth is cut to the cache
    nodes = np.array([T, 1, 3, T + 5, 0, 0], dtype=np.int32)            # the last has nothing at all
    c.check([[np.arange(min(x, 200))] * 2 for x in lens], seq_lens=lens, nodes=nodes)


@pytest.mark.parametrize("chunk", [2, 16, 64])
@pytest.mark.parametrize("page", [0, 16])
def test_chunk_lists(chunk, page):
    rng = np.random.default_rng(chunk)
    c = Case(3, 8, 2, 11, 128, 301, page=page, seed=chunk)
    lens = np.array([301, 150, 7], dtype=np.int32)
    kept, rows = [], []
    for b in range(3):
        units = -(-int(lens[b]) // chunk)
        per = []
        for _ in range(2):
            use = np.sort(rng.permutation(units)[:max(1, units // 2)])
            use = np.union1d(use, [units - 1])                          # the last chunk ends inside itself
            rows.append(use)
            per.append(np.concatenate([np.arange(u * chunk, min((u + 1) * chunk, lens[b])) for u in use]))
        kept.append(per)
    lists, counts = np.full((6, max(map(len, rows)) + 3), -9, dtype=np.int32), np.zeros(6, dtype=np.int32)
    for r, x in enumerate(rows):
        lists[r, :len(x)], counts[r] = x, len(x)
    c.check(kept, lists=lists, counts=counts, seq_lens=lens, chunk=chunk)


def test_physical_lists():
    c = Case(2, 8, 2, 10, 64, 320, "f16", page=16, seed=5)
    kept, lists, counts = make_lists(np.random.default_rng(2), 2, 2, 320, 0.4)
    for r in range(4):
        x = lists[r, :counts[r]]
        lists[r, :counts[r]] = c.table[r // 2][x // 16] * 16 + x % 16
    c.check(kept, lists=lists, counts=counts, physical=True)


def test_pitched_rows_and_scale():
    c = Case(2, 4, 2, 9, 128, 150, seed=6, pitch=24)
    c.check([[np.arange(150)] * 2] * 2, scale=0.3)


@pytest.mark.parametrize("want", [("out",), ("low",), ("low", "lse")])
def test_outputs_on_their_own(want):
    c = Case(2, 8, 2, 20, 128, 400, seed=7)
    c.check([[np.arange(400)] * 2] * 2, want=want)


def test_counts_beyond_the_capacity():
    c = Case(1, 4, 2, 5, 128, 100, seed=8)
    kept, lists, counts = make_lists(np.random.default_rng(3), 1, 2, 100, 0.5, capacity=80)
    lists[:] = np.sort(np.stack([np.random.default_rng(i).permutation(100)[:80] for i in range(2)]), 1)
    c.check([[lists[0], lists[1]]], lists=lists, counts=np.array([1000, 80], dtype=np.int32))


def test_masks_that_are_no_trees():
    """Nodes that see nothing of the tree, everything, or other nodes alone; bits of nodes that are not there."""
    c = Case(2, 4, 2, 40, 128, 90, seed=9)
    rng = np.random.default_rng(4)
    c.masks = rng.integers(0, 2 ** 63, (2, 40)).astype(np.uint64) * np.uint64(2)
    c.masks[0, 0] = 0
    c.masks[0, 1] = np.uint64(2 ** 64 - 1)
    kept = [[np.arange(90)] * 2, [np.arange(0)] * 2]
    c.check(kept, seq_lens=np.array([90, 0], dtype=np.int32), nodes=np.array([40, 22], dtype=np.int32))


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("G,T", [(1, 7), (4, 16), (8, 30)])
def test_hidden_nodes_have_no_effect(bad, G, T):
    """A node's infinite keys and values reach its descendants alone; rows behind the last node and unlisted positions reach nobody."""
    c = Case(1, 2 * G, 2, T, 128, 100, seed=10)
    c.k_new[0, :, 3], c.v_new[0, :, 3] = bad, bad
    c.k_new[0, :, T - 1], c.v_new[0, :, T - 1], c.q[0, :, T - 1] = float("nan"), float("nan"), float("nan")
    c.k[0, :, 50:], c.v[0, :, 50:] = bad, bad
    nodes = np.array([T - 1], dtype=np.int32)
    a = c.args(seq_lens=np.array([50], dtype=np.int32), nodes=nodes)
    sa.specattn_tree_attn(a)
    torch.cuda.synchronize()
    below = np.array([bool((int(c.masks[0, t]) >> 3) & 1) and t < T - 1 for t in range(T)])
    c.compare([[np.arange(50)] * 2], nodes, skip=below)
    assert not np.isfinite(c.out.cpu().numpy()[0][:, below]).all(axis=2).any()


@pytest.mark.parametrize("cached", [0, 40, 2000])
@pytest.mark.parametrize("G,T", [(1, 7), (4, 20), (8, 30)])
def test_a_key_that_is_no_number_shows(cached, G, T):
    """Rows that see the node are NaN, also where its score is the only one of a wave or of a share; the others have nothing of it."""
    c = Case(1, 2 * G, 2, T, 64, max(cached, 1), seed=12)
    c.k_new[0, :, 0] = float("nan")
    c.masks[0, 2] = np.uint64(4)                              # a second root
    for t in range(3, T):
        c.masks[0, t] = np.uint64(1) << np.uint64(t) | np.uint64(t % 2) | np.uint64(2) * np.uint64(t % 3 == 0)
    a = c.args(seq_lens=np.array([cached], dtype=np.int32))
    sa.specattn_tree_attn(a)
    torch.cuda.synchronize()
    sees = np.array([bool(int(c.masks[0, t]) & 1) for t in range(T)])
    assert sees[:2].all() and not sees[2]
    c.compare([[np.arange(cached)] * 2], skip=sees)
    for x in (c.out, c.low, c.lse):
        assert torch.isnan(x[0][:, torch.from_numpy(sees).cuda()]).all()


def test_many_rows():
    """More rows of sequences and kv heads than a launch takes."""
    c = Case(300, 8, 8, 2, 64, 40, "f16", seed=11)
    lens = np.random.default_rng(5).integers(0, 41, 300).astype(np.int32)
    a = c.args(seq_lens=lens)
    sa.specattn_tree_attn(a)
    torch.cuda.synchronize()
    got = c.out.cpu()
    for b0 in (0, 250, 280):
        d = Case(300, 8, 8, 2, 64, 40, "f16", seed=11)
        d.B = 20
        for name in ("q", "k", "v", "k_new", "v_new"):
            setattr(d, name, getattr(c, name)[b0:b0 + 20])
        d.masks, d.out, d.low, d.lse = c.masks[b0:b0 + 20], got[b0:b0 + 20], None, None
        d.compare([[np.arange(x)] * 8 for x in lens[b0:b0 + 20]])


def test_wild_entries_stay_inside():
    c = Case(1, 8, 2, 12, 128, 160, page=16, seed=12)
    lists = np.array([[-5, 3, 10 ** 9, 40], [0, 159, 160, 2 ** 31 - 1]], dtype=np.int32)
    for physical in (False, True):
        a = c.args(lists=lists, counts=np.array([4, 4], dtype=np.int32), physical=physical)
        sa.specattn_tree_attn(a)
        torch.cuda.synchronize()
        assert torch.isfinite(c.out).all()
    c.check([[[0, 3, 159, 40], [0, 159, 159, 159]]], lists=lists, counts=np.array([4, 4], dtype=np.int32))
    c.table[0, 3] = -1
    a = c.args(lists=lists, counts=np.array([4, 4], dtype=np.int32), chunk=16)
    sa.specattn_tree_attn(a)
    torch.cuda.synchronize()


def test_long_rows_are_cut_and_joined_in_order():
    """A row over many workgroups beside short ones; the same bits every time, eager and replayed."""
    c = Case(3, 8, 2, 20, 128, 5000, seed=13)
    lens = np.array([5000, 3, 1200], dtype=np.int32)
    a = c.check([[np.arange(x)] * 2 for x in lens], seq_lens=lens)
    first = c.out.clone()
    sa.specattn_init()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        sa.specattn_tree_attn(a)
    for _ in range(3):
        c.out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.out, first)
        c.out.zero_()
        sa.specattn_tree_attn(a, stream=torch.cuda.Stream())
        torch.cuda.synchronize()
        assert torch.equal(c.out, first)


@pytest.mark.parametrize("B,H_q,T,n,seed", [(30, 2, 3, 3000, 4), (30, 2, 3, 3000, 5), (48, 2, 3, 2500, 6), (48, 2, 3, 2500, 11), (12, 16, 33, 2000, 1)])
def test_cuts_in_many_ragged_rows(B, H_q, T, n, seed):
    """Cuts that are moved to a unit's ends in one place and left in another: the joining takes every share of a unit, and no other unit's."""
    lens = np.random.default_rng(seed).integers(1, n, B).astype(np.int32)
    c = Case(B, H_q, 2, T, 64, n, seed=seed)
    c.check([[np.arange(x)] * 2 for x in lens], seq_lens=lens)


def test_a_chain_is_the_causal_decode_attention():
    """Masks 0 .. t: what specattn_sparse_decode_attn computes with new tokens."""
    c = Case(2, 16, 4, 5, 128, 700, seed=14)
    c.masks[:] = (np.uint64(2) << np.arange(5, dtype=np.uint64)) - np.uint64(1)
    kept, lists, counts = make_lists(np.random.default_rng(6), 2, 4, 700, 0.3)
    c.check(kept, lists=lists, counts=counts)
    out, lse = torch.empty_like(c.out), torch.empty_like(c.lse)
    x = c.keep
    b = sa.attn_args(x["q"], x["k"], x["v"], out=out, lse=lse, indices=x["lists"], counts=x["counts"], k_new=x["k_new"], v_new=x["v_new"])
    ws = sa.alloc_workspace(sa.specattn_workspace_size(None, b))
    sa.set_workspace(b, ws)
    sa.specattn_sparse_decode_attn(b)
    torch.cuda.synchronize()
    c.out, c.lse, c.low = out, lse, None
    c.compare(kept)
