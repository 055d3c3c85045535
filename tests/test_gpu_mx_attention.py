"""Decode attention over the 4-bit cache against masked attention in 64 bits on the values the cache stands for."""
import numpy as np
import pytest
import torch

import mx_reference as ref
from paper_2510_27641_amd import binding as sa

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f16": torch.float16}


class Case:
    """A cache of random codes under scales around 1, queries, and what a call over them gives."""

    def __init__(self, B, H_q, H_kv, T, d, n, dtype="bf16", *, page=0, new=False, seed=0, spread=3, pitch=0):
        rng = np.random.default_rng(seed)
        self.B, self.H_q, self.H_kv, self.T, self.d, self.n, self.page = B, H_q, H_kv, T, d, n, page
        per = -(-n // page) if page else 1
        slots, width = (B * per + 2, page) if page else (B, n)
        self.codes = rng.integers(0, 256, size=(slots, H_kv, width, d), dtype=np.uint8)
        self.scales = rng.integers(125 - spread, 126 + spread, size=(slots, H_kv, width, d // 16), dtype=np.uint8)
        self.table = rng.permutation(slots)[:B * per].reshape(B, per).astype(np.int32) if page else None
        g = torch.Generator().manual_seed(seed + 1)
        self.q = torch.randn((B, H_q, T, d), generator=g).to(DT[dtype])
        self.k_new = torch.randn((B, H_kv, T, d), generator=g).to(DT[dtype]) if new else None
        self.v_new = torch.randn((B, H_kv, T, d), generator=g).to(DT[dtype]) if new else None

    def rows(self):
        k, v = ref.cache_values(self.codes, self.scales)
        if self.table is None:
            return k, v
        return tuple(np.stack([np.concatenate([x[p] for p in row], 1)[:, :self.n] for row in self.table]) for x in (k, v))

    def run(self, *, kept=None, lists=None, counts=None, seq_lens=None, chunk=0, lowp=True, **kw):
        B, H_q, T, d = self.q.shape
        out = torch.full((B, H_q, T, d), float("nan"), device="cuda")
        low = torch.full((B, H_q, T, d), float("nan"), dtype=self.q.dtype, device="cuda") if lowp else None
        lse = torch.full((B, H_q, T), float("nan"), device="cuda")
        dev = lambda x: None if x is None else torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
        self.keep = dev(self.codes), dev(self.scales), dev(self.table), dev(lists), dev(counts), dev(seq_lens), self.q.cuda()
        new = [None if x is None else x.cuda() for x in (self.k_new, self.v_new)]
        codes, scales, table, lists, counts, seq_lens, q = self.keep
        cache = sa.mx_cache(codes, scales, page_table=table, n_max=self.n)
        args = sa.mx_attn_args(q, cache, out=out, out_lowp=low, lse=lse, indices=lists, counts=counts, seq_lens=seq_lens, chunk_size=chunk,
                               k_new=new[0], v_new=new[1], **kw)
        ws = sa.alloc_workspace(sa.specattn_mx_workspace_size(args))
        args.workspace, args.workspace_bytes = ws.data_ptr(), ws.numel()
        sa.specattn_mx_decode_attn(args)
        torch.cuda.synchronize()
        if low is not None:
            assert torch.allclose(low, out.to(low.dtype), rtol=0, atol=0, equal_nan=True)
        return out.cpu().double().numpy(), lse.cpu().double().numpy()

    def check(self, kept, *, scale=None, **kw):
        got, lse = self.run(sm_scale=0.0 if scale is None else scale, **kw)
        k, v = self.rows()
        new = [None if x is None else x.double().numpy() for x in (self.k_new, self.v_new)]
        want, want_lse, tol = ref.attention(self.q.double().numpy(), k, v, kept, self.d ** -0.5 if scale is None else scale, *new)
        assert (np.abs(got - want) <= tol[..., None] + 1e-30).all(), np.max(np.abs(got - want) / (tol[..., None] + 1e-30))
        some = np.isfinite(want_lse)
        assert np.array_equal(some, np.isfinite(lse)) and (lse[~some] == -np.inf).all() and (got[~some] == 0).all()
        # the log-sum is off by what the scores and the sum of weights are off
        assert (np.abs(lse - want_lse)[some] <= tol[some] / max(np.abs(v).max(), 1e-30) + 2.0 ** -22 * (np.abs(want_lse[some]) + 32)).all()
        return got


def _lists(rng, B, H, n, fraction, capacity=None):
    kept = [[np.sort(rng.permutation(n)[:int(round(n * fraction))]) for _ in range(H)] for _ in range(B)]
    cap = capacity or max(1, max(len(x) for row in kept for x in row))
    lists, counts = np.full((B * H, cap), -7, dtype=np.int32), np.zeros(B * H, dtype=np.int32)
    for r, x in enumerate(x for row in kept for x in row):
        lists[r, :len(x)], counts[r] = x, len(x)
    return kept, lists, counts


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H_q,H_kv,T", [(1, 1, 1), (4, 4, 3), (8, 2, 5), (10, 2, 4), (16, 2, 5), (8, 1, 8)])
def test_lists(dtype, d, H_q, H_kv, T):
    """One to four query tiles, groups that are no power of two."""
    c = Case(2, H_q, H_kv, T, d, 333, dtype, seed=H_q * 10 + T)
    kept, lists, counts = _lists(np.random.default_rng(1), 2, H_kv, 333, 0.37)
    c.check(kept, lists=lists, counts=counts)


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 255, 256, 257, 513])
@pytest.mark.parametrize("d", [64, 128])
def test_dense_lengths(n, d):
    c = Case(1, 8, 2, 3, d, n, seed=n)
    c.check([[np.arange(n)] * 2])


@pytest.mark.parametrize("new", [False, True])
@pytest.mark.parametrize("page", [0, 16, 4])
def test_ragged_dense_with_empty_rows(page, new):
    c = Case(5, 8, 2, 4, 128, 200, "f16", page=page, new=new, seed=3)
    lens = np.array([0, 1, 200, 37, 250], dtype=np.int32)      # the last is cut to the cache
    c.check([[np.arange(min(x, 200))] * 2 for x in lens], seq_lens=lens)
    lens = np.array([0, 0, -3, 0, 0], dtype=np.int32)
    c.check([[np.arange(0)] * 2] * 5, seq_lens=lens)


@pytest.mark.parametrize("new", [False, True])
@pytest.mark.parametrize("d,page", [(128, 0), (128, 16), (64, 16)])
def test_lists_of_very_different_lengths(d, page, new):
    """Rows without any position between rows of one and of thousands, so that shares cross many rows."""
    B, H, n = 3, 4, 4000
    c = Case(B, 8, H, 2, d, n, page=page, new=new, seed=11)
    rng = np.random.default_rng(5)
    sizes = [0, 4000, 1, 0, 0, 31, 2500, 32, 0, 33, 5, 0]
    kept = [[np.sort(rng.permutation(n)[:sizes[b * H + h]]) for h in range(H)] for b in range(B)]
    lists, counts = np.full((B * H, n), 10 ** 9, dtype=np.int32), np.array(sizes, dtype=np.int32)
    for r in range(B * H):
        lists[r, :sizes[r]] = kept[r // H][r % H]
    c.check(kept, lists=lists, counts=counts)


@pytest.mark.parametrize("dtype,d,page", [("bf16", 128, 0), ("f16", 128, 16), ("bf16", 64, 16), ("f16", 64, 0)])
@pytest.mark.parametrize("G,T", [(1, 1), (4, 5), (5, 8), (8, 8)])
def test_more_than_64_rows(dtype, d, page, G, T):
    """One to four query tiles where workgroups take stretches of the rows' tiles: rows of nothing, of one position, of many."""
    B, H, n = 10, 7, 700
    c = Case(B, G * H, H, T, d, n, dtype, page=page, new=(T == 5), seed=G + T)
    rng = np.random.default_rng(G * T)
    kept = [[np.sort(rng.permutation(n)[:rng.choice([0, 1, 31, 33, 200, 700])]) for _ in range(H)] for _ in range(B)]
    lists, counts = np.full((B * H, n), -1, dtype=np.int32), np.zeros(B * H, dtype=np.int32)
    for r in range(B * H):
        x = kept[r // H][r % H]
        lists[r, :len(x)], counts[r] = x, len(x)
    c.check(kept, lists=lists, counts=counts)


@pytest.mark.parametrize("chunk", [2, 16, 128])
@pytest.mark.parametrize("page", [0, 16])
def test_chunk_lists(chunk, page):
    B, H, n = 2, 2, 777
    c = Case(B, 8, H, 5, 128, n, page=page, seed=chunk)
    rng = np.random.default_rng(chunk)
    lens = np.array([777, 300], dtype=np.int32)
    kept, lists, counts = [], np.full((B * H, -(-n // chunk)), -1, dtype=np.int32), np.zeros(B * H, dtype=np.int32)
    for b in range(B):
        units = -(-int(lens[b]) // chunk)
        kept.append([])
        for h in range(H):
            u = np.unique(np.append(rng.permutation(units)[:max(1, units // 3)], units - 1))
            lists[b * H + h, :len(u)], counts[b * H + h] = u, len(u)
            pos = (u[:, None] * chunk + np.arange(chunk)).ravel()
            kept[b].append(pos[pos < lens[b]])
    c.check(kept, lists=lists, counts=counts, seq_lens=lens, chunk=chunk)


def test_counts_beyond_the_capacity_and_list_strides():
    c = Case(1, 4, 2, 2, 128, 100, seed=21)
    kept, lists, counts = _lists(np.random.default_rng(2), 1, 2, 100, 0.5, capacity=50)
    wide = np.full((2, 77), 99, dtype=np.int32)
    wide[:, :50] = lists
    idx, cnt, q = torch.from_numpy(wide).cuda(), torch.from_numpy(counts).cuda(), c.q.cuda()
    codes, scales = torch.from_numpy(c.codes).cuda(), torch.from_numpy(c.scales).cuda()
    k, v = c.rows()
    for cap in (50, 20):
        out = torch.empty((1, 4, 2, 128), device="cuda")
        args = sa.mx_attn_args(q, sa.mx_cache(codes, scales), out=out, indices=idx[:, :cap], counts=cnt)
        assert args.idx_stride_row == 77 and args.idx_capacity == cap
        ws = sa.alloc_workspace(sa.specattn_mx_workspace_size(args))
        args.workspace, args.workspace_bytes = ws.data_ptr(), ws.numel()
        sa.specattn_mx_decode_attn(args)
        want, _, tol = ref.attention(c.q.double().numpy(), k, v, [[x[:cap] for x in kept[0]]], 128 ** -0.5)
        assert (np.abs(out.cpu().double().numpy() - want) <= tol[..., None]).all()


def test_pool_slots():
    """Lists of pool slots, without a page table."""
    B, H, page, d = 2, 2, 16, 128
    c = Case(B, 4, H, 2, d, 64, page=page, seed=8)
    rng = np.random.default_rng(8)
    kept, lists, counts = _lists(rng, B, H, 64, 0.6)
    slots = lists.copy()
    for r in range(B * H):
        pos = lists[r, :counts[r]]
        slots[r, :counts[r]] = c.table[r // H][pos // page] * page + pos % page
    k, v = c.rows()
    want, _, tol = ref.attention(c.q.double().numpy(), k, v, kept, d ** -0.5)
    codes, scales, q = torch.from_numpy(c.codes).cuda(), torch.from_numpy(c.scales).cuda(), c.q.cuda()
    out, idx, cnt = torch.empty((B, 4, 2, d), device="cuda"), torch.from_numpy(slots).cuda(), torch.from_numpy(counts).cuda()
    args = sa.mx_attn_args(q, sa.mx_cache(codes, scales, B=B), out=out, indices=idx, counts=cnt, indices_are_physical=True)
    ws = sa.alloc_workspace(sa.specattn_mx_workspace_size(args))
    args.workspace, args.workspace_bytes = ws.data_ptr(), ws.numel()
    sa.specattn_mx_decode_attn(args)
    assert (np.abs(out.cpu().double().numpy() - want) <= tol[..., None]).all()


@pytest.mark.parametrize("H_q,T", [(40, 2), (24, 8), (9, 8)])
def test_more_than_64_query_rows(H_q, T):
    c = Case(1, H_q, 1, T, 128, 150, seed=H_q)
    kept, lists, counts = _lists(np.random.default_rng(4), 1, 1, 150, 0.5)
    c.check(kept, lists=lists, counts=counts)


def test_more_rows_than_a_launch_takes():
    c = Case(300, 4, 4, 1, 64, 40, seed=6, new=True)
    lens = np.random.default_rng(0).integers(0, 41, size=300).astype(np.int32)
    c.check([[np.arange(x)] * 4 for x in lens], seq_lens=lens)


def test_far_scales_and_large_scores():
    """Blocks that differ by 2^40 in scale, scores of several hundred, and a scale of the caller's own."""
    c = Case(1, 4, 1, 3, 128, 300, seed=13, spread=20)
    c.scales[..., :4] = np.clip(c.scales[..., :4], 105, 132)
    c.check([[np.arange(300)]], scale=0.05)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128])
def test_key_blocks_of_any_scale_and_rows_of_zeros(dtype, d):
    """Blocks of a key 2^120 apart, the smallest scale there is, and positions without any key, the last one among them, behind which a
    tile is masked."""
    c = Case(1, 4, 1, 3, d, 45, dtype, seed=15)
    c.scales[..., :d // 32] = np.random.default_rng(15).choice([0, 1, 60, 100, 112, 120, 124], size=(1, 1, 45, d // 32))
    for at in (3, 20, 44):
        c.codes[0, 0, at, :d // 2], c.scales[0, 0, at, :d // 32] = 0, 0
    c.check([[np.arange(45)]])
    c.scales[..., :d // 32] = 0
    c.check([[np.arange(45)]])


@pytest.mark.parametrize("d", [64, 128])
def test_fp16_queries_below_the_normal_numbers(d):
    """Queries of a few units of 2^-24 against keys large enough for them to matter, single blocks of which lie 2^-12 lower."""
    c = Case(2, 8, 2, 4, d, 90, "f16", seed=37, spread=1)
    c.q = (c.q.float() * 2.0 ** -18).half()
    assert (c.q.abs() < 2.0 ** -14).all() and (c.q != 0).any()
    c.scales[..., :d // 32] += 17
    c.scales[..., 1] -= 12
    c.check([[np.arange(90)] * 2] * 2)


def test_nan_keys_with_fp16_queries():
    c = Case(1, 4, 2, 2, 128, 70, "f16", seed=19)
    c.scales[0, 1, 69, 3] = 255
    got, lse = c.run()
    k, v = c.rows()
    want, _, tol = ref.attention(c.q.double().numpy(), np.nan_to_num(k), v, [[np.arange(70)] * 2], 128 ** -0.5)
    assert (np.abs(got - want) <= tol[..., None])[:, :2].all() and np.isnan(got[0, 2:]).all() and np.isnan(lse[0, 2:]).all()


def test_a_sink_of_almost_all_weight():
    """One position 25 binary orders above the others: their small weights have to come through."""
    c = Case(1, 2, 1, 1, 128, 5000, "f16", seed=17)
    c.scales[:] = 122
    q = c.q.double().numpy()[0, 0, 0]
    code, scale = ref.quantise(q[None])
    c.codes[0, 0, 0, :64], c.scales[0, 0, 0, :4] = ref.pack(code)[0], scale[0]
    c.codes[0, 0, 0, 64:] = 0
    c.check([[np.arange(5000)]], scale=0.12)


def test_nan_blocks_count_only_where_they_are_attended_to():
    c = Case(1, 4, 2, 2, 128, 100, seed=19)
    c.scales[0, 0, 50, 5] = 255                                # a value block of head 0: columns 32 .. 63
    c.scales[0, 1, 60, 1] = 255                                # a key block of head 1
    kept = [[np.setdiff1d(np.arange(100), [50, 60])] * 2]
    lists = np.tile(kept[0][0].astype(np.int32), (2, 1))
    k, v = c.rows()
    got, _ = c.run(lists=lists, counts=np.full(2, 98, dtype=np.int32))
    want, _, tol = ref.attention(c.q.double().numpy(), np.nan_to_num(k), np.nan_to_num(v), kept, 128 ** -0.5)
    assert (np.abs(got - want) <= tol[..., None]).all()
    got, lse = c.run()                                         # every position
    assert np.isnan(got[0, :2, :, 32:64]).all() and np.isfinite(got[0, :2, :, :32]).all() and np.isfinite(got[0, :2, :, 64:]).all()
    assert np.isfinite(lse[0, :2]).all() and np.isnan(got[0, 2:]).all() and np.isnan(lse[0, 2:]).all()


def test_entries_outside_the_cache_stay_inside_it():
    """Wrong list entries and pages are read somewhere inside the cache: finite results, and other rows as they should be."""
    c = Case(2, 4, 2, 2, 128, 96, page=16, seed=23)
    kept, lists, counts = _lists(np.random.default_rng(6), 2, 2, 96, 0.5)
    lists[0, 3], lists[0, 9] = -5, 2 ** 31 - 1
    c.table[0, 1], c.table[0, 2] = -4, 10 ** 6
    got, _ = c.run(lists=lists, counts=counts)
    c.table[0, 1:3] = 0
    k, v = c.rows()
    want, _, tol = ref.attention(c.q.double().numpy(), k, v, kept, 128 ** -0.5)
    assert np.isfinite(got).all() and (np.abs(got[1] - want[1]) <= tol[1, ..., None]).all()


def test_repeated_calls_are_bit_identical():
    c = Case(3, 8, 2, 5, 128, 3000, seed=29)
    kept, lists, counts = _lists(np.random.default_rng(7), 3, 2, 3000, 0.4)
    first = c.run(lists=lists, counts=counts)
    for _ in range(3):
        again = c.run(lists=lists, counts=counts)
        assert np.array_equal(first[0], again[0]) and np.array_equal(first[1], again[1])


def test_outputs_are_optional_and_strided_queries():
    c = Case(2, 6, 2, 3, 128, 90, seed=31)
    base = torch.zeros((2, 3, 18, 128), dtype=torch.bfloat16, device="cuda")
    base[:, :, :6] = c.q.cuda().transpose(1, 2)
    q = base[:, :, :6].transpose(1, 2)                         # as a packed projection leaves them
    codes, scales = torch.from_numpy(c.codes).cuda(), torch.from_numpy(c.scales).cuda()
    k, v = c.rows()
    want, _, tol = ref.attention(c.q.double().numpy(), k, v, [[np.arange(90)] * 2] * 2, 128 ** -0.5)
    out, low = torch.empty((2, 6, 3, 128), device="cuda"), torch.empty((2, 6, 3, 128), dtype=torch.bfloat16, device="cuda")
    for kw in (dict(out=out), dict(out_lowp=low)):
        args = sa.mx_attn_args(q, sa.mx_cache(codes, scales), **kw)
        ws = sa.alloc_workspace(sa.specattn_mx_workspace_size(args))
        args.workspace, args.workspace_bytes = ws.data_ptr(), ws.numel()
        sa.specattn_mx_decode_attn(args)
    assert (np.abs(out.cpu().double().numpy() - want) <= tol[..., None]).all()
    # half a step of bf16 on top
    assert (np.abs(low.cpu().double().numpy() - want) <= tol[..., None] * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(want)).all()
