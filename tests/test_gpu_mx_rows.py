"""Rows into the 4-bit cache and back: codes, scales and values bit for bit against the plain form, which has one answer."""
import numpy as np
import pytest
import torch

import mx_reference as ref
from paper_2510_27641_amd import binding as sa

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _pools(B, H, n, d, page=0, seed=0, spare=3):
    """A cache full of 0xA5, its page table (or None)."""
    if page == 0:
        return torch.full((B, H, n, d), 0xA5, dtype=torch.uint8, device="cuda"), torch.full((B, H, n, d // 16), 0xA5, dtype=torch.uint8, device="cuda"), None
    per = -(-n // page)
    table = torch.from_numpy(np.random.default_rng(seed).permutation(B * per + spare)[:B * per].reshape(B, per).astype(np.int32)).cuda()
    return (torch.full((B * per + spare, H, page, d), 0xA5, dtype=torch.uint8, device="cuda"),
            torch.full((B * per + spare, H, page, d // 16), 0xA5, dtype=torch.uint8, device="cuda"), table)


def _expected(k, v, codes0, scales0, table, starts, counts, n):
    """The cache after the rows went in."""
    codes, scales = codes0.cpu().numpy().copy(), scales0.cpu().numpy().copy()
    page = codes.shape[2]
    k, v = k.double().cpu().numpy(), v.double().cpu().numpy()
    (ck, sk), (cv, sv) = ref.quantise(k), ref.quantise(v)
    rows, marks = np.concatenate((ref.pack(ck), ref.pack(cv)), -1), np.concatenate((sk, sv), -1)
    for b in range(k.shape[0]):
        for t in range(counts[b]):
            slot = starts[b] + t
            if not 0 <= slot < n:
                continue
            if table is None:
                codes[b, :, slot], scales[b, :, slot] = rows[b, :, t], marks[b, :, t]
            else:
                p = int(table[b, slot // page])
                if 0 <= p < codes.shape[0]:
                    codes[p, :, slot % page], scales[p, :, slot % page] = rows[b, :, t], marks[b, :, t]
    return codes, scales


def _round_trip(k, v, n, *, page=0, starts=None, counts=None, seed=0, mend=None):
    B, H, T, d = k.shape
    codes, scales, table = _pools(B, H, n, d, page, seed)
    if mend is not None:
        mend(table)
    s = None if starts is None else torch.tensor(starts, dtype=torch.int32, device="cuda")
    c = None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda")
    starts, counts = starts or [0] * B, [min(max(x, 0), T) for x in (counts or [T] * B)]
    want = _expected(k, v, codes, scales, table, starts, counts, n)
    cache = sa.mx_cache(codes, scales, page_table=table, n_max=n)
    sa.specattn_mx_store(sa.mx_rows_args(cache, k, v, starts=s, counts=c))
    assert np.array_equal(codes.cpu().numpy(), want[0]) and np.array_equal(scales.cpu().numpy(), want[1])
    back_k, back_v = torch.full_like(k, 7.0), torch.full_like(v, 7.0)
    sa.specattn_mx_load(sa.mx_rows_args(cache, back_k, back_v, starts=s, counts=c))
    full_k, full_v = ref.cache_values(want[0], want[1])
    for got, full in ((back_k, full_k), (back_v, full_v)):
        held = torch.full(k.shape, 7.0, dtype=torch.float64)
        for b in range(B):
            for t in range(counts[b]):
                slot = starts[b] + t
                if not 0 <= slot < n:
                    continue
                p = b if table is None else int(table[b, slot // page])
                if 0 <= p < full.shape[0]:
                    held[b, :, t] = torch.from_numpy(full[p, :, slot if table is None else slot % page])
        held = held.float().to(k.dtype)                        # (a value of the cache is exact in fp32)
        assert torch.equal(got.cpu().nan_to_num(12345.0), held.nan_to_num(12345.0)) and torch.equal(got.cpu().isnan(), held.isnan())


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,H,T,n", [(1, 1, 1, 1), (2, 3, 5, 9), (3, 2, 33, 70), (1, 8, 200, 200)])
def test_contiguous(dtype, d, B, H, T, n):
    g = torch.Generator().manual_seed(B * 100 + T)
    k, v = ((s * torch.randn((B, H, T, d), generator=g)).to(DT[dtype]).cuda() for s in (3.0, 0.01))
    _round_trip(k, v, n)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,page", [(128, 16), (64, 16), (128, 1), (64, 64)])
def test_paged_ragged(dtype, d, page):
    g = torch.Generator().manual_seed(page)
    k, v = (torch.randn((4, 3, 40, d), generator=g).to(DT[dtype]).cuda() for _ in range(2))
    _round_trip(k, v, 100, page=page, starts=[0, 13, 60, 99], counts=[40, 0, 17, 1], seed=5)


def test_rows_outside_the_cache_are_left_out():
    g = torch.Generator().manual_seed(3)
    k, v = (torch.randn((4, 2, 12, 128), generator=g).bfloat16().cuda() for _ in range(2))
    _round_trip(k, v, 50, starts=[-5, 45, 50, 2 ** 31 - 3], counts=[12, 99, 12, 12])

    def mend(table):
        table[0, 0], table[1, 1], table[2, 2] = -1, 10 ** 6, table.max() + 100
    _round_trip(k, v, 50, page=16, starts=[10, 10, 30, 45], counts=[12, 12, 12, 12], mend=mend)


def test_every_bf16_value_and_the_ends_of_the_range():
    """Every finite bf16 in a block with a given largest magnitude, blocks of zeros, of the smallest and the largest numbers, with an
    infinity, with a NaN."""
    words = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).float()
    x = words.reshape(-1, 32).clone()                          # neighbours share a block: every exponent is a block's largest
    mixed = words[torch.randperm(65536, generator=torch.Generator().manual_seed(1))].reshape(-1, 32)
    mixed = torch.where(mixed.abs() < 100.0, mixed, torch.rand(mixed.shape, generator=torch.Generator().manual_seed(2)) * 16 - 8)
    rows = torch.cat((x, mixed, torch.zeros(8, 32))).reshape(-1, 128)
    rows[-1, 32:64] = -0.0
    k = rows[None, None].contiguous()
    _round_trip(k.bfloat16().cuda(), k.flip(2).contiguous().bfloat16().cuda(), rows.shape[0])
    f = torch.cat((torch.full((32,), 2.0 ** -149), torch.full((32,), torch.finfo(torch.float32).max), torch.tensor([float("nan")] * 1 + [1.0] * 31), torch.tensor([1.0] * 31 + [-float("inf")])))
    g = torch.cat((torch.linspace(-7.999999, 7.999999, 32), torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.9999] * 4), torch.linspace(0, 2.0 ** -126, 32), torch.logspace(-30, 30, 32)))
    f, g = f.reshape(1, 1, 1, 128).cuda(), g.reshape(1, 1, 1, 128).cuda()
    _round_trip(f, g, 1)


def test_strided_rows_and_cache():
    """Rows as a projection leaves them ([B, T, H, d]) and a cache that interleaves heads."""
    B, H, T, d = 2, 4, 9, 128
    base = torch.randn((B, T, 3 * H, d), generator=torch.Generator().manual_seed(9)).half().cuda()
    k, v = base[:, :, :H].transpose(1, 2), base[:, :, H:2 * H].transpose(1, 2)
    codes = torch.zeros((B, 20, H, d), dtype=torch.uint8, device="cuda")
    scales = torch.zeros((B, 20, H, d // 16), dtype=torch.uint8, device="cuda")
    cache = sa.mx_cache(codes.transpose(1, 2), scales.transpose(1, 2))
    starts = torch.tensor([3, 11], dtype=torch.int32, device="cuda")
    sa.specattn_mx_store(sa.mx_rows_args(cache, k, v, starts=starts))
    want = _expected(k, v, torch.zeros((B, H, 20, d), dtype=torch.uint8), torch.zeros((B, H, 20, d // 16), dtype=torch.uint8), None, [3, 11], [T, T], 20)
    assert np.array_equal(codes.transpose(1, 2).cpu().numpy(), want[0]) and np.array_equal(scales.transpose(1, 2).cpu().numpy(), want[1])
    back = torch.zeros_like(base)
    sa.specattn_mx_load(sa.mx_rows_args(cache, back[:, :, :H].transpose(1, 2), back[:, :, H:2 * H].transpose(1, 2), starts=starts))
    assert torch.equal(back[:, :, 2 * H:], torch.zeros_like(back[:, :, 2 * H:]))
    full_k, _ = ref.cache_values(*want)
    assert torch.equal(back[1, :, :H].transpose(0, 1).double().cpu(), torch.from_numpy(full_k[1, :, 11:20]))


def test_load_of_any_bytes():
    """All codes under all scale bytes, read as fp32, and as fp16 where small values round and large ones become infinite."""
    codes = np.tile(np.arange(256, dtype=np.uint8), 128).reshape(1, 1, 256, 128)
    scales = np.repeat(np.arange(256, dtype=np.uint8), 8).reshape(1, 1, 256, 8)
    held_codes, held_scales = torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda()
    cache = sa.mx_cache(held_codes, held_scales)
    want = ref.cache_values(codes, scales)
    for dtype in (torch.float32, torch.float16, torch.bfloat16):
        k, v = (torch.zeros((1, 1, 256, 128), dtype=dtype, device="cuda") for _ in range(2))
        sa.specattn_mx_load(sa.mx_rows_args(cache, k, v))
        for got, full in ((k, want[0]), (v, want[1])):
            held = torch.from_numpy(full).float().to(dtype)
            assert torch.equal(got.cpu().nan_to_num(12345.0), held.nan_to_num(12345.0)) and torch.equal(got.cpu().isnan(), held.isnan())
