"""Attention over values as large as the cache and the new tokens hold them: the result lies among them."""
import numpy as np
import pytest
import torch

from test_gpu_mx_attention import Case

pytestmark = pytest.mark.gpu

LARGEST = 252                                                  # the largest scale byte that rows get: values up to 1.5 * 2^127


def _large(c, low):
    d = c.d
    c.scales[..., d // 32:] = np.random.default_rng(c.n).integers(low, LARGEST + 1, size=c.scales[..., d // 32:].shape, dtype=np.uint8)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d,H_q,H,T,n", [(128, 4, 1, 3, 1), (128, 4, 2, 5, 70), (64, 4, 1, 3, 2000), (128, 8, 1, 8, 3000), (128, 2, 1, 1, 9000)])
def test_up_to_64_rows(dtype, d, H_q, H, T, n):
    c = Case(2, H_q, H, T, d, n, dtype, seed=n)
    _large(c, 244)
    c.check([[np.arange(n)] * H] * 2, lowp=False)


@pytest.mark.parametrize("dtype,d,G,T", [("bf16", 128, 1, 1), ("f16", 64, 4, 5), ("bf16", 128, 8, 8)])
def test_more_than_64_rows(dtype, d, G, T):
    c = Case(70, G, 1, T, d, 200, dtype, seed=G)
    _large(c, 244)
    lens = np.random.default_rng(G).integers(0, 201, size=70).astype(np.int32)
    c.check([[np.arange(x)] for x in lens], seq_lens=lens, lowp=False)


@pytest.mark.parametrize("n", [0, 1, 40, 5000])
def test_new_tokens(n):
    """bf16 as large as 2^127, equal ones and ones of either sign."""
    c = Case(2, 8, 2, 8, 128, max(n, 1), "bf16", seed=n, new=True)
    _large(c, 250)
    c.k_new.mul_(0.1)
    c.v_new = (torch.where(torch.arange(128) % 3 == 0, c.v_new.sign(), torch.ones(())) * 2.0 ** 127 * 1.5).bfloat16()
    lens = np.array([n, 0], dtype=np.int32)
    c.check([[np.arange(x)] * 2 for x in lens], seq_lens=lens, lowp=False)


def test_equal_values_throughout():
    """The sum of 9000 equal values would need 14 binary orders more than one."""
    c = Case(1, 4, 1, 2, 128, 9000, "bf16", seed=3)
    c.codes[..., 64:], c.scales[..., 4:] = 0x77, LARGEST
    got = c.check([[np.arange(9000)]], lowp=False)
    assert (np.abs(got / (1.5 * 2.0 ** 127) - 1) <= 2.0 ** -18).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_small_values(dtype):
    """And as small as 2^-122.  Scaling by a power of two changes nothing but where fp32 ends: what lies below 2^-126 is rounded to
    2^-149.  That happens to a wave's state, to its share of a workgroup's and to that one's share of the result: with eight waves and three
    workgroups to a row, each half a step and none counted more than twice, less than 8 steps.  Sums of so changed terms may round the other
    way, each by one step of at most 2^-23 of the largest value: eight additions in a workgroup and three of its like, and the products before them."""
    c = Case(2, 8, 2, 4, 128, 600, dtype, seed=5)
    c.scales[..., 4:] -= 116
    got, _ = c.run(lowp=False)
    c.scales[..., 4:] += 116
    plain, _ = c.run(lowp=False)
    largest = 6 * 2.0 ** (c.scales[..., 4:].max() - 127.0)
    assert (np.abs(got - plain * 2.0 ** -116) <= 2.0 ** -146 + 24 * 2.0 ** -23 * largest * 2.0 ** -116).all()


@pytest.mark.parametrize("T", [1, 3, 8])
def test_infinite_new_values_stay_with_the_queries_that_see_them(T):
    """Query t sees new tokens 0 .. t: an infinity in the last is the last query's, and an infinity there, not a NaN."""
    c = Case(1, 4, 2, T, 128, 60, "bf16", seed=T, new=True)
    c.v_new[0, 0, T - 1, 5], c.v_new[0, 1, T - 1, 9] = float("inf"), float("-inf")
    got, lse = c.run(lowp=False)
    assert (got[0, :2, T - 1, 5] == np.inf).all() and (got[0, 2:, T - 1, 9] == -np.inf).all() and np.isfinite(lse).all()
    got[0, :2, T - 1, 5] = got[0, 2:, T - 1, 9] = 0
    assert np.isfinite(got).all()
