"""Causal attention over packed prompts and behind a prefix in pages, against masked attention in 64 bits."""
import numpy as np
import pytest
import torch

import serve_reference as ref
from paper_2510_27641_amd import binding as sa

pytestmark = pytest.mark.gpu


class Case:
    """Packed sequences; kv_lens given: keys and values of their own (packed, or in pages)."""

    def __init__(self, q_lens, H_q, H_kv, d, dtype="bf16", *, kv_lens=None, page=0, fused=False, seed=0, gap=0):
        g = torch.Generator().manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.q_lens, self.H_q, self.H_kv, self.d, self.dtype, self.page = list(q_lens), H_q, H_kv, d, dtype, page
        self.kv_lens = list(q_lens if kv_lens is None else kv_lens)
        B, dt = len(self.q_lens), ref.DT[dtype]
        self.starts = gap + np.concatenate(([0], np.cumsum(self.q_lens))).astype(np.int32)
        rows = int(self.starts[-1]) + gap
        self.own_kv = kv_lens is not None
        self.kv_starts = np.concatenate(([0], np.cumsum(self.kv_lens))).astype(np.int32)
        kv_rows = int(self.kv_starts[-1]) if self.own_kv else rows
        if fused:
            joint = torch.randn((rows, H_q + 2 * H_kv, d), generator=g).to(dt)
            self.q, self.k, self.v = joint[:, :H_q], joint[:, H_q:H_q + H_kv], joint[:, H_q + H_kv:]
        else:
            self.q = torch.randn((rows, H_q, d), generator=g).to(dt)
            self.k, self.v = (torch.randn((max(kv_rows, 1), H_kv, d), generator=g).to(dt) for _ in range(2))
        self.table = None
        if page:
            per = max(1, max(-(-n // page) for n in self.kv_lens))
            self.pool_pages = B * per + 2
            self.table = rng.permutation(self.pool_pages)[:B * per].reshape(B, per).astype(np.int32)

    def kv(self, b):
        """[n, H_kv, d] keys and values of sequence b."""
        s, n = (self.kv_starts if self.own_kv else self.starts)[b], self.kv_lens[b]
        return self.k[s:s + n], self.v[s:s + n]

    def args(self, want=("out", "low", "lse"), scale=0.0):
        dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
        q = torch.empty_strided(self.q.shape, self.q.stride(), dtype=self.q.dtype, device="cuda").copy_(self.q)
        if self.q._base is not None:                                    # views of one projection stay so
            joint = self.q._base.cuda()
            q, k, v = joint[:, :self.H_q], joint[:, self.H_q:self.H_q + self.H_kv], joint[:, self.H_q + self.H_kv:]
        elif self.page:
            pools = [torch.full((self.pool_pages, self.H_kv, self.page, self.d), float("nan"), dtype=self.q.dtype) for _ in range(2)]
            for b, n in enumerate(self.kv_lens):
                for x, pool in zip(self.kv(b), pools):
                    for p in range(-(-n // self.page)):
                        piece = x[p * self.page:(p + 1) * self.page].transpose(0, 1)
                        pool[self.table[b, p], :, :piece.shape[1]] = piece
            k, v = (p.cuda() for p in pools)
        else:
            k, v = self.k.cuda(), self.v.cuda()
        shape = tuple(self.q.shape)
        self.out = torch.full(shape, 7.0, device="cuda") if "out" in want else None
        self.low = torch.full(shape, 7.0, dtype=self.q.dtype, device="cuda") if "low" in want else None
        self.lse = torch.full(shape[:2], 7.0, device="cuda") if "lse" in want else None
        self.keep = [q, k, v, dev(self.starts), dev(self.kv_starts), None if self.table is None else dev(self.table), dev(np.array(self.kv_lens, dtype=np.int32))]
        kw = {}
        if self.page:
            kw = dict(page_table=self.keep[5], seq_lens=self.keep[6])
        elif self.own_kv:
            kw = dict(kv_starts=self.keep[4])
        a = sa.prompt_args(q, k, v, self.keep[3], out=self.out, out_lowp=self.low, lse=self.lse, sm_scale=scale, **kw)
        self.ws = sa.alloc_workspace(sa.specattn_prompt_workspace_size(a))
        sa.set_workspace(a, self.ws)
        return a

    def expected(self, scale=0.0):
        G = self.H_q // self.H_kv
        scale = scale or self.d ** -0.5
        for b, (m, n) in enumerate(zip(self.q_lens, self.kv_lens)):
            rows = slice(self.starts[b], self.starts[b] + m)
            k, v = (x.double().numpy() for x in self.kv(b))
            seen = np.arange(n)[None] < (n - m + np.arange(m)[:, None] + 1)
            for h in range(self.H_q):
                yield rows, h, ref.attend(self.q[rows, h].double().numpy(), k[:, h // G], v[:, h // G], seen, scale, self.dtype)

    def check(self, scale=0.0, want=("out", "low", "lse")):
        a = self.args(want, scale)
        sa.specattn_prompt_attn(a)
        torch.cuda.synchronize()
        self.compare(scale)
        outside = np.ones(self.q.shape[0], dtype=bool)
        outside[self.starts[0]:self.starts[-1]] = False
        for x in (self.out, self.low, self.lse):
            assert x is None or (x.cpu()[torch.from_numpy(outside)] == 7.0).all()
        return a

    def compare(self, scale=0.0):
        got = [None if x is None else x.cpu().double().numpy() for x in (self.out, self.low, self.lse)]
        for rows, h, (out, lse, tol32, tol_low, tol_lse) in self.expected(scale):
            if got[0] is not None:
                assert (np.abs(got[0][rows, h] - out) <= tol32).all(), np.nanmax(np.abs(got[0][rows, h] - out) / (tol32 + 1e-30))
            if got[1] is not None:
                assert (np.abs(got[1][rows, h] - out) <= tol_low).all(), np.nanmax(np.abs(got[1][rows, h] - out) / (tol_low + 1e-30))
            if got[2] is not None:
                some = np.isfinite(lse)
                mine = got[2][rows, h]
                assert np.array_equal(some, np.isfinite(mine)) and (mine[~some] == -np.inf).all()
                assert (np.abs(mine[some] - lse[some]) <= tol_lse[some]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H_q,H_kv", [(1, 1), (4, 4), (4, 1), (10, 2), (24, 2)])
def test_ragged(dtype, d, H_q, H_kv):
    Case([1, 33, 0, 70, 17, 129], H_q, H_kv, d, dtype, seed=H_q).check()


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 257, 700])
def test_lengths(n):
    Case([n], 2, 1, 128, "bf16", seed=n).check()
    Case([n], 3, 3, 64, "f16", seed=n).check()


@pytest.mark.parametrize("want", [("out",), ("low",), ("low", "lse"), ("out", "lse")])
def test_outputs_on_their_own(want):
    Case([100, 5], 4, 2, 128, seed=3).check(want=want)


@pytest.mark.parametrize("page", [0, 1, 4, 16, 128])
@pytest.mark.parametrize("d,dtype", [(128, "bf16"), (64, "f16")])
def test_behind_a_prefix(page, d, dtype):
    """More keys than queries, as many, and fewer (the first queries then see nothing), none at all; single tokens."""
    Case([5, 1, 40, 64, 9, 3], 8, 2, d, dtype, kv_lens=[205, 333, 40, 65, 4, 0], page=page, seed=page).check()


@pytest.mark.parametrize("H_q,H_kv", [(8, 8), (8, 1), (40, 1)])
def test_single_tokens(H_q, H_kv):
    """One token to a sequence: few query rows per kv head, waves over positions."""
    Case([1] * 9, H_q, H_kv, 128, kv_lens=[1, 2, 127, 128, 129, 500, 31, 64, 0], page=16, seed=H_q).check()


def test_views_of_one_projection_and_rows_around():
    Case([37, 130], 8, 2, 128, fused=True, gap=3, seed=1).check(scale=0.21)


def test_many_sequences():
    """More sequences than threads look at in one go."""
    rng = np.random.default_rng(0)
    Case(rng.integers(0, 4, 600), 2, 1, 64, "f16", seed=2).check()


def test_parts_of_long_sequences():
    """Few query rows over many keys: the keys are cut into parts."""
    c = Case([3, 20], 4, 1, 128, kv_lens=[4100, 2050], page=16, seed=4)
    assert sa.specattn_prompt_workspace_size(c.args()) > 0
    c.check()
    Case([600], 1, 1, 64, "f16", seed=5).check()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f16", 64)])
def test_hidden_values_have_no_effect(bad, dtype, d):
    """Keys and values that a causal mask hides, rows of other sequences, pages' unused rows: queries ahead of them stay exact."""
    c = Case([90, 40], 4, 2, d, dtype, seed=6)
    for x in (c.k, c.v):
        x[70] = bad                                                     # seen by queries 70 .. 89 of the first sequence
    a = c.args()
    sa.specattn_prompt_attn(a)
    got = c.out.cpu().double().numpy(), c.low.cpu().double().numpy(), c.lse.cpu().double().numpy()
    for rows, h, (out, lse, tol32, tol_low, tol_lse) in c.expected():
        some = np.ones(out.shape[0], dtype=bool)
        if rows.start == 0:
            some[70:] = False
            assert not np.isfinite(got[0][70:90, h]).all(axis=1).any()
        assert (np.abs(got[0][rows, h] - out) <= tol32)[some].all() and (np.abs(got[1][rows, h] - out) <= tol_low)[some].all()
        assert (np.abs(got[2][rows, h] - lse) <= tol_lse)[some].all()


@pytest.mark.parametrize("q_lens,H_q,kv_lens", [([5], 2, None), ([70, 3], 2, None), ([9], 2, [1200]), ([300], 8, None)])
def test_a_key_that_is_no_number_shows(q_lens, H_q, kv_lens):
    """Queries that see it are NaN, the first of which may see nothing else."""
    c = Case(q_lens, H_q, 2, 64, "bf16", kv_lens=kv_lens, seed=13)
    c.k[0] = float("nan")
    sa.specattn_prompt_attn(c.args())
    torch.cuda.synchronize()
    n = q_lens[0]
    for x in (c.out, c.low, c.lse):
        assert torch.isnan(x[:n]).all() and torch.isfinite(x[n:]).all()


def test_large_values_and_scores():
    """Values whose unnormalised sums pass fp32, and scores far apart."""
    c = Case([80], 2, 1, 128, seed=7)
    c.v[:] = (c.v.float().sign() * 1.5e38).to(c.v.dtype)
    c.k *= 12
    c.check(want=("out", "lse"))


def test_wild_lengths_stay_inside():
    """Starts and lengths beyond what there is are cut to it, pages outside the pool read the nearest one."""
    c = Case([20, 30], 4, 2, 128, kv_lens=[64, 64], page=16, seed=8)
    a = c.args()
    c.keep[3].copy_(torch.tensor([0, 20, 10 ** 6]))
    c.keep[6].copy_(torch.tensor([2 ** 31 - 1, 64]))
    c.keep[5][1, 2] = 10 ** 8
    c.keep[5][1, 3] = -5
    sa.specattn_prompt_attn(a)
    torch.cuda.synchronize()


def test_captured_and_on_another_stream():
    """Replays with eager work between them, and calls on two streams at once with workspaces of their own."""
    c, e = Case([3, 150], 8, 2, 128, kv_lens=[2100, 700], page=16, seed=9), Case([300, 2], 4, 4, 64, "f16", seed=10)
    a, b = c.args(), e.args()
    sa.specattn_init()
    sa.specattn_prompt_attn(a)
    sa.specattn_prompt_attn(b)
    torch.cuda.synchronize()
    eager = c.out.clone(), e.out.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        sa.specattn_prompt_attn(a)
        sa.specattn_prompt_attn(b)
    for _ in range(3):
        c.out.zero_()
        e.out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.out, eager[0]) and torch.equal(e.out, eager[1])
        sa.specattn_prompt_attn(b)
        torch.cuda.synchronize()
    s = torch.cuda.Stream(), torch.cuda.Stream()
    c.out.zero_()
    e.out.zero_()
    torch.cuda.synchronize()
    sa.specattn_prompt_attn(a, stream=s[0])
    sa.specattn_prompt_attn(b, stream=s[1])
    torch.cuda.synchronize()
    assert torch.equal(c.out, eager[0]) and torch.equal(e.out, eager[1])
