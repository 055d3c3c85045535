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


def not_finite(v, at, d):
    """Infinities of either sign, both in one column, and a NaN, in the rows `at` of v [..., rows, d]."""
    inf = float("inf")
    for i, (row, column, x) in enumerate(zip(at * 2, (3, d - 3, 17, 17, 40, 3), (inf, -inf, inf, -inf, float("nan"), inf))):
        v[..., row, column] = x


def compare_not_finite(got, q, k, v, seen, scale, dtype, low):
    """Elements that are infinite or NaN where they have to be, and as near as others elsewhere."""
    out, _, tol32, tol_low, _ = ref.attend(q, k, np.where(np.isfinite(v), v, 0.0), seen, scale, dtype)
    for i in range(seen.shape[0]):
        rows = v[seen[i]]
        plus, minus, nan = ((x[:, None] if x.ndim == 1 else x).any(0) for x in (rows == np.inf, rows == -np.inf, np.isnan(rows)))
        out[i] = np.where(nan | (plus & minus), np.nan, np.where(plus, np.inf, np.where(minus, -np.inf, out[i])))
    finite = np.isfinite(out)
    assert np.array_equal(np.isnan(got), np.isnan(out)) and np.array_equal(got[np.isinf(out)], out[np.isinf(out)])
    assert (np.abs(got - out)[finite] <= (tol_low if low else tol32)[finite]).all()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f16", 64), ("f16", 128)])
@pytest.mark.parametrize("q_lens,kv_lens,page", [([90], [90], 0), ([300, 7], [400, 64], 16), ([4, 2], [900, 130], 16), ([30], [2000], 0), ([130], [3000], 0)])
def test_prompts_over_values_that_are_not_finite(q_lens, kv_lens, page, dtype, d):
    """Seen by some queries, hidden from others of the same tile, and far behind them all."""
    c = prompts.Case(q_lens, 8, 2, d, dtype, kv_lens=kv_lens, page=page, seed=23)
    n, m = kv_lens[0], q_lens[0]
    not_finite(c.v.transpose(0, 1), [n // 3, n - m // 2 - 1, n - 1], d)
    for want in (("out",), ("low",)):
        sa.specattn_prompt_attn(c.args(want))
        torch.cuda.synchronize()
        got = (c.out if want == ("out",) else c.low).double().cpu().numpy()
        for b in range(len(q_lens)):
            k, v = (x.double().numpy() for x in c.kv(b))
            rows = slice(c.starts[b], c.starts[b + 1])
            seen = np.arange(kv_lens[b])[None] < (kv_lens[b] - q_lens[b] + np.arange(q_lens[b])[:, None] + 1)
            for h in range(8):
                compare_not_finite(got[rows, h], c.q[rows, h].double().numpy(), k[:, h // 4], v[:, h // 4], seen, d ** -0.5, dtype, want == ("low",))


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f16", 64)])
@pytest.mark.parametrize("G,T,n", [(1, 6, 200), (4, 20, 90), (4, 20, 3000), (8, 33, 900)])
def test_trees_over_values_that_are_not_finite(G, T, n, dtype, d):
    c = trees.Case(1, 2 * G, 2, T, d, n, dtype, page=16, seed=24)
    not_finite(c.v_new, [1, T // 2, T - 1], d)
    for column, at in ((5, n // 4), (d - 1, n - 1)):
        c.v[c.table[0][at // 16], :, at % 16, column] = float("inf")
    bits = np.array([[bool((int(c.masks[0, t]) >> u) & 1) for u in range(T)] for t in range(T)])
    seen = np.concatenate((np.ones((T, n), dtype=bool), bits), 1)
    for want in (("out",), ("low",)):
        sa.specattn_tree_attn(c.args(want=want))
        torch.cuda.synchronize()
        got = (c.out if want == ("out",) else c.low).double().cpu().numpy()
        for h in range(2 * G):
            key, val = c.rows(0, h // G, np.arange(n))
            k, v = np.concatenate((key, c.k_new[0, h // G].double().numpy())), np.concatenate((val, c.v_new[0, h // G].double().numpy()))
            compare_not_finite(got[0, h], c.q[0, h].double().numpy(), k, v, seen, d ** -0.5, dtype, want == ("low",))


def test_an_infinity_that_every_query_sees_costs_no_multiple_of_the_rows():
    """What is computed once more is computed for all rows of a wave together: a row after the other took 200 times the plain call."""
    n = 2048
    g = torch.Generator(device="cuda").manual_seed(2)
    q, k, v = (torch.randn((n, h, 128), generator=g, device="cuda").bfloat16() for h in (8, 2, 2))
    starts, out = torch.tensor([0, n], dtype=torch.int32, device="cuda"), torch.empty_like(q)
    a = sa.prompt_args(q, k, v, starts, out_lowp=out)
    ws = sa.alloc_workspace(sa.specattn_prompt_workspace_size(a))
    sa.set_workspace(a, ws)

    def took():
        least = float("inf")
        for _ in range(4):
            one, two = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            one.record()
            sa.specattn_prompt_attn(a)
            two.record()
            torch.cuda.synchronize()
            least = min(least, one.elapsed_time(two))
        return least

    plain = took()
    v[0, :, 9] = float("inf")
    spoiled = took()
    print("plain", plain, "ms, with an infinity", spoiled, "ms")
    assert (out[..., 9] == float("inf")).all() and torch.isfinite(out[..., :9]).all() and torch.isfinite(out[..., 10:]).all()
    assert spoiled < 30 * plain


@pytest.mark.parametrize("n", [5000, 1 << 18])
@pytest.mark.parametrize("tree", [False, True])
def test_long_sums_of_equal_weights(tree, n):
    """A first key and n - 1 equal ones behind it, in one part (256 kv heads): the total is off by what its weights are (2^-21 of them, and as much for the
    argument), not by a step of itself for each of them; 2^-22 of the result for the logarithm."""
    H, d, scale = 256, 64, float(np.log(2.0))
    k, v = torch.zeros((n, 1, d), device="cuda").bfloat16(), torch.ones((n, 1, d), device="cuda").bfloat16()
    k[1:, :, 0] = -0.5
    lse = torch.empty((1, H), device="cuda")
    if tree:
        q = torch.zeros((1, H, 1, d), device="cuda").bfloat16()
        q[..., 0] = 1
        out, new = torch.empty((1, H, 1, d), device="cuda"), torch.zeros((1, H, 1, d), device="cuda").bfloat16()
        k, v = (x.transpose(0, 1)[None].expand(1, H, n, d) for x in (k, v))
        a = sa.tree_args(q, k, v, new, new, torch.zeros((1, 1), dtype=torch.int64, device="cuda"), out=out, lse=lse[..., None], sm_scale=scale)
        ws = sa.alloc_workspace(sa.specattn_tree_workspace_size(a))
        sa.set_workspace(a, ws)
        sa.specattn_tree_attn(a)
    else:
        q = torch.zeros((1, H, d), device="cuda").bfloat16()
        q[..., 0] = 1
        out = torch.empty((1, H, d), device="cuda")
        kw = dict(kv_starts=torch.tensor([0, n], dtype=torch.int32, device="cuda"))
        a = sa.prompt_args(q, k.expand(n, H, d), v.expand(n, H, d), torch.tensor([0, 1], dtype=torch.int32, device="cuda"), out=out, lse=lse, sm_scale=scale, **kw)
        assert sa.specattn_prompt_workspace_size(a) == 0
        sa.specattn_prompt_attn(a)
    torch.cuda.synchronize()
    want = np.log(1 + (n - 1) * np.exp(-0.5 * np.float64(np.float32(scale))))
    off = (lse.double().cpu() - want).abs().max().item()
    print("lse", want, "off by", off, "out off by", (out.double() - 1).abs().max().item())
    assert off <= 2.0 ** -20 + 2.0 ** -22 * want
    # (products are added up sixteen positions at a time: half a step of the sum for each sixteen)
    assert (out.double() - 1).abs().max().item() <= 2 * (n / 16 + 32) * 2.0 ** -24 + 2.0 ** -16


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f16", 128), ("f16", 64)])
@pytest.mark.parametrize("q_len,H_q,kv_len", [(100, 2, 100), (300, 8, 700), (20, 2, 1500)])
def test_prompts_do_not_depend_on_what_they_do_not_see(q_len, H_q, kv_len, dtype, d):
    """Other keys, values and queries behind a place: the queries ahead of it keep their bits."""
    c = prompts.Case([q_len], H_q, 1, d, dtype, kv_lens=[kv_len], seed=25)
    c.k *= 4
    sa.specattn_prompt_attn(c.args())
    torch.cuda.synchronize()
    first = c.out.clone(), c.low.clone(), c.lse.clone()
    for cut in (q_len // 2, q_len // 5):
        x = prompts.Case([q_len], H_q, 1, d, dtype, kv_lens=[kv_len], seed=26)
        for name in ("q", "k", "v"):
            at = cut + (kv_len - q_len if name != "q" else 0)
            getattr(x, name)[:at] = getattr(c, name)[:at]
            getattr(x, name)[at:] *= 6
        sa.specattn_prompt_attn(x.args())
        torch.cuda.synchronize()
        for got, was in zip((x.out, x.low, x.lse), first):
            assert torch.equal(got[:cut], was[:cut])


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f16", 128), ("f16", 64)])
@pytest.mark.parametrize("G,T,n", [(1, 9, 100), (4, 20, 3000), (8, 33, 300)])
def test_trees_do_not_depend_on_what_they_do_not_see(G, T, n, dtype, d):
    """Nodes that are not there, and nodes that others do not descend from: their queries, keys and values leave the others' bits alone."""
    c = trees.Case(1, 2 * G, 2, T, d, n, dtype, seed=27)
    for x in (c.k, c.k_new):
        x *= 4
    c.masks[0] = [np.uint64(1) << np.uint64(t) | np.uint64(1) << np.uint64(t % 2) for t in range(T)]      # two roots, leaves of either
    nodes = np.array([T - 2], dtype=np.int32)
    sa.specattn_tree_attn(c.args(nodes=nodes))
    torch.cuda.synchronize()
    first = c.out.clone(), c.low.clone(), c.lse.clone()
    odd = torch.arange(T) % 2 == 1
    odd[T - 2:] = True
    g = torch.Generator().manual_seed(28)
    for x in (c.q, c.k_new, c.v_new):
        x[:, :, odd] = (torch.randn(x[:, :, odd].shape, generator=g) * 6).to(x.dtype)
    sa.specattn_tree_attn(c.args(nodes=nodes))
    torch.cuda.synchronize()
    for got, was in zip((c.out, c.low, c.lse), first):
        assert torch.equal(got[:, :, ~odd.cuda()], was[:, :, ~odd.cuda()])


@pytest.mark.parametrize("size", [1e30, 1e31, 1e32, 1e33, 1e34, 1e36])
def test_values_on_either_side_of_where_rows_are_mended(size):
    """Unnormalised sums from 2^100 on: as they are, mended in some parts of a row or in some rows, mended in all."""
    c = prompts.Case([3, 40], 4, 2, 128, kv_lens=[4100, 900], page=16, seed=29)
    c.v[:] = (c.v.float() * size).to(c.v.dtype)
    c.v[:2000] *= 0.01
    c.check()
    c = trees.Case(2, 8, 2, 20, 128, 3000, seed=30)
    c.v[:] = (c.v.float() * size).to(c.v.dtype)
    c.v[:, :, 1000:] *= 0.01
    c.v_new[:] = (c.v_new.float() * size).to(c.v_new.dtype)
    c.check([[np.arange(3000)] * 2] * 2)
