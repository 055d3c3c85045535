"""Page tables, free pages and slots of new tokens, and rows into those slots, against lists."""
import numpy as np
import pytest
import torch

import serve_reference as ref
from paper_2510_27641_amd import binding as sa

pytestmark = pytest.mark.gpu

dev = lambda x: torch.from_numpy(np.ascontiguousarray(np.asarray(x, dtype=np.int32))).cuda()  # noqa: E731


class State:
    def __init__(self, B, width, page, lens, pages=None, seed=0):
        rng = np.random.default_rng(seed)
        self.B, self.page = B, page
        self.lens = np.asarray(lens, dtype=np.int32)
        have = -(-np.clip(self.lens, 0, width * page).astype(np.int64) // page)
        pages = int(have.sum()) + 5 if pages is None else pages
        order = rng.permutation(pages).astype(np.int32)
        self.table = np.full((B, width), -3, dtype=np.int32)
        at = 0
        for b in range(B):
            self.table[b, :have[b]] = order[at:at + have[b]]
            at += have[b]
        self.free = np.full(pages, -3, dtype=np.int32)
        self.count = pages - at
        self.free[:self.count] = order[at:]

    def update(self, new, capacity, *, in_place=False):
        x = dict(table=dev(self.table), free=dev(self.free), count=dev([self.count]), lens=dev(self.lens), new=dev(new))
        filled = lambda n: torch.full((n,), -7, dtype=torch.int32, device="cuda")  # noqa: E731
        lens_out, count_out = (x["lens"], x["count"]) if in_place else (filled(self.B), filled(1))
        starts, flags = filled(self.B + 1), filled(self.B)
        slots, places, owners = (filled(capacity) for _ in range(3)) if capacity else (None, None, None)
        a = sa.pages_args(x["table"], self.page, x["free"], x["count"], x["lens"], x["new"], lens_out=lens_out, free_count_out=count_out, token_starts=starts,
                          slots=slots, positions=places, owners=owners, row_flags=flags)
        ws = sa.alloc_workspace(sa.specattn_pages_workspace_size(a))
        sa.specattn_pages_update(a, ws)
        torch.cuda.synchronize()
        want = ref.pages(self.table, self.free, self.count, self.lens, np.asarray(new), self.page, capacity or None)
        got = dict(table=x["table"], free=x["free"], count=count_out, lens=lens_out, starts=starts, flags=flags)
        if capacity:
            got.update(slots=slots, positions=places, owners=owners)
        for name, t in got.items():
            assert np.array_equal(t.cpu().numpy().reshape(-1), np.asarray(want[name]).reshape(-1)), name
        self.table, self.free, self.count, self.lens = want["table"], want["free"], want["count"], want["lens"]
        return want


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B,page,capacity", [(1, 16, 40), (5, 4, 100), (64, 16, 600), (700, 1, 5000), (1024, 16, 8192), (1025, 16, 2000), (2500, 2, 30000), (40, 16, 20000)])
def test_steps(B, page, capacity, in_place):
    """Several updates in a row; sequences grow, shrink and end, and new ones come in their places."""
    rng = np.random.default_rng(B)
    width = max(4, 200 // page)
    s = State(B, width, page, rng.integers(0, width * page // 2, B), pages=B * width // 2 + 9, seed=B)
    for _ in range(4):
        pick = rng.random(B)
        new = np.where(pick < 0.6, s.lens + rng.integers(0, 9, B), np.where(pick < 0.8, s.lens // 2, np.where(pick < 0.9, 0, s.lens + rng.integers(0, 60, B))))
        s.update(np.minimum(new, width * page), capacity, in_place=in_place)


def test_pages_that_have_just_come_back_are_taken():
    s = State(3, 8, 4, [32, 5, 0], pages=10)
    assert s.count == 0
    want = s.update([3, 5, 20], 64)
    assert want["lens"].tolist() == [3, 5, 20] and want["count"] == 2


def test_short_of_pages():
    """From the first sequence on that does not get its pages none gets any, and those that need none go on."""
    s = State(6, 8, 4, [4, 4, 4, 3, 4, 4], pages=9)
    want = s.update([8, 12, 24, 4, 8, 4], 64)
    assert want["flags"].tolist() == [0, 0, 4, 0, 4, 0] and want["lens"].tolist() == [8, 12, 4, 4, 4, 4]


def test_short_of_slots():
    s = State(4, 8, 4, [0, 1, 2, 3], pages=30)
    assert s.update([5, 6, 3, 4], 10)["flags"].tolist() == [0, 0, 4, 4]
    assert s.update([0, 0, 0, 0], 10)["tokens"] == 0


def test_lengths_out_of_range():
    s = State(5, 4, 4, [3, -1, 17, 9, 16], pages=30)
    assert s.update([20, 4, 4, -2, 16], 64)["flags"].tolist() == [4, 1, 1, 1, 0]


def test_without_slots():
    s = State(9, 50, 16, np.arange(9) * 20)
    s.update(np.arange(9)[::-1] * 20, 0)


def test_long_prompts():
    """Sums that pass 32 bits where nobody has the pages for them."""
    s = State(5, 1 << 20, 1024, [0] * 5, pages=70)
    top = (1 << 30) - 1
    assert s.update([top, top, 60000, top, 5000], 70000)["flags"].tolist() == [4, 4, 4, 4, 4]
    assert s.update([60000, 0, 0, 5000, 0], 70000)["tokens"] == 65000


def test_captured():
    """A step in place, replayed: the state moves on from replay to replay as it does from call to call."""
    rng = np.random.default_rng(1)
    B, width, page, capacity = 50, 40, 16, 400
    s = State(B, width, page, rng.integers(1, 100, B), pages=900)
    x = dict(table=dev(s.table), free=dev(s.free), count=dev([s.count]), lens=dev(s.lens), new=dev(s.lens))
    slots = dev(np.zeros(capacity))
    a = sa.pages_args(x["table"], page, x["free"], x["count"], x["lens"], x["new"], slots=slots)
    ws = sa.alloc_workspace(sa.specattn_pages_workspace_size(a))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        sa.specattn_pages_update(a, ws)
    for _ in range(4):
        new = np.where(rng.random(B) < 0.8, s.lens + rng.integers(0, 9, B), s.lens // 3).astype(np.int32)
        x["new"].copy_(dev(new))
        g.replay()
        torch.cuda.synchronize()
        want = ref.pages(s.table, s.free, s.count, s.lens, new, page, capacity)
        s.table, s.free, s.count, s.lens = want["table"], want["free"], want["count"], want["lens"]
        for name, t in (("table", x["table"]), ("free", x["free"]), ("count", x["count"]), ("lens", x["lens"]), ("slots", slots)):
            assert np.array_equal(t.cpu().numpy().reshape(-1), np.asarray(want[name]).reshape(-1)), name


# ---- rows into slots --------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("H,d,page", [(1, 8, 16), (8, 128, 16), (3, 64, 1), (5, 72, 7), (2, 520, 4)])
def test_packed_rows(dtype, H, d, page):
    rng = np.random.default_rng(d)
    N, pages = 333, 90 if page > 4 else 500
    joint = torch.randn((N, 2 * H + 1, d)).to(ref.DT[dtype]).cuda()
    k, v = joint[:, :H], joint[:, H + 1:]
    pool = [torch.full((pages, H, page, d), 7.0, dtype=k.dtype, device="cuda") for _ in range(2)]
    M = min(N, pages * page)
    slots = rng.permutation(pages * page)[:M].astype(np.int32)
    slots[::5] = -1
    slots[3], slots[4] = pages * page, 2 ** 31 - 1
    sa.specattn_cache_store(sa.store_args(k, v, *pool, dev(slots)))
    torch.cuda.synchronize()
    for rows, got in ((k, pool[0]), (v, pool[1])):
        want = torch.full((pages, page, H, d), 7.0, dtype=k.dtype).view(-1, H, d)
        for i, s in enumerate(slots):
            if 0 <= s < pages * page:
                want[s] = rows[i].cpu()
        assert torch.equal(got.cpu(), want.view(pages, page, H, d).transpose(1, 2))


@pytest.mark.parametrize("contiguous", [False, True])
def test_nodes_by_their_numbers(contiguous):
    """Accepted nodes of trees, some of them twice; numbers that do not exist are left out; a contiguous cache is a pool of sequences."""
    B, H, T, d, n = 4, 2, 9, 64, 37
    k, v = torch.randn((B, H, T, d)).bfloat16().cuda(), torch.randn((B, H, T, d)).bfloat16().cuda()
    pages, page = (B, n) if contiguous else (10, 16)
    pool = [torch.zeros((pages, H, page, d), dtype=k.dtype, device="cuda") for _ in range(2)]
    slots, rows = np.array([5, 36, 37, 80, 81, 147, 3], dtype=np.int32), np.array([0, 35, 12, 12, -1, 36, 20], dtype=np.int32)
    sa.specattn_cache_store(sa.store_args(k, v, *pool, dev(slots), rows=dev(rows)))
    torch.cuda.synchronize()
    for src, got in ((k, pool[0]), (v, pool[1])):
        want = torch.zeros((pages, H, page, d), dtype=k.dtype)
        for s, r in zip(slots, rows):
            if 0 <= r < B * T and s < pages * page:
                want[s // page, :, s % page] = src[r // T, :, r % T].cpu()
        assert torch.equal(got.cpu(), want)


def test_far_slots():
    """A pool beyond 4 GiB."""
    pool = [torch.zeros((70000, 2, 128, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    k = torch.randn((3, 2, 128)).bfloat16().cuda()
    slots = dev([70000 * 128 - 1, 40000 * 128 + 5, 0])
    sa.specattn_cache_store(sa.store_args(k, -k, *pool, slots))
    torch.cuda.synchronize()
    for i, (p, o) in enumerate(((69999, 127), (40000, 5), (0, 0))):
        assert torch.equal(pool[0][p, :, o], k[i]) and torch.equal(pool[1][p, :, o], -k[i])
    assert int((pool[0] != 0).sum(dtype=torch.int64)) == int((k != 0).sum())
