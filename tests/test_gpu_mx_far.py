"""4-bit caches in pitched layouts and in ones that reach beyond 4 GiB: rows in, attention over them, rows out, rows moved."""
import numpy as np
import pytest
import torch

import mx_reference as ref
from paper_2510_27641_amd import binding as sa

pytestmark = pytest.mark.gpu

GIB = 1 << 30


def _views(kind, B, H, n, d):
    """Codes and scales of one layout, and a page table (or None)."""
    def strided(shape, strides):
        size = sum((s - 1) * t for s, t in zip(shape, strides)) + 1
        return torch.empty(size, dtype=torch.uint8, device="cuda").as_strided(shape, strides)
    if kind == "one record":                                   # codes and scales of a position side by side, heads inside positions
        pitch = d + 16
        base = torch.full((B, n, H, pitch), 0xA5, dtype=torch.uint8, device="cuda")
        return base[..., :d].transpose(1, 2), base[..., d:d + d // 16].transpose(1, 2), None
    if kind == "heads far apart":
        return strided((B, H, n, d), (2 * d * n, 5 * GIB, 2 * d, 1)), strided((B, H, n, d // 16), (n * 16, 4 * GIB + 16, 16, 1)), None
    if kind == "positions far apart":
        far = (5 * GIB // n) // 16 * 16
        return strided((B, H, n, d), (n * far, d, far, 1)), strided((B, H, n, d // 16), (n * far // 16 * 4, d // 16, far // 16 * 4, 1)), None
    pages = 700                                                # a pool of 10.5 GiB, its pages 15 MiB apart
    table = torch.from_numpy(np.random.default_rng(3).permutation(pages - 1)[:B * (-(-n // 16))].reshape(B, -1).astype(np.int32)).cuda()
    table[0, 0] = pages - 1
    return strided((pages, H, 16, d), (15 << 20, 16 * d, d, 1)), strided((pages, H, 16, d // 16), (7 << 20, 16 * (d // 16), d // 16, 1)), table


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kind", ["one record", "heads far apart", "positions far apart", "pages far apart"])
def test_layouts(kind, d, dtype):
    B, H, n, T = 2, 2, 150, 3
    codes, scales, table = _views(kind, B, H, n, d)
    cache = sa.mx_cache(codes, scales, page_table=table, n_max=n)
    g = torch.Generator().manual_seed(d)
    k, v = (torch.randn((B, H, n, d), generator=g).to(dtype).cuda() for _ in range(2))
    sa.specattn_mx_store(sa.mx_rows_args(cache, k, v))
    want = [torch.from_numpy(ref.values(*ref.quantise(x.double().cpu().numpy()))) for x in (k, v)]
    back = [torch.zeros_like(k) for _ in range(2)]
    sa.specattn_mx_load(sa.mx_rows_args(cache, *back))
    assert all(torch.equal(x.double().cpu(), w) for x, w in zip(back, want))
    q = torch.randn((B, 4, T, d), generator=g).to(dtype).cuda()
    lists = torch.stack([torch.randperm(n, generator=g)[:90].sort().values for _ in range(B * H)]).int()
    out = torch.empty((B, 4, T, d), device="cuda")
    held = [lists.cuda(), torch.full((B * H,), 90, dtype=torch.int32, device="cuda")]
    for kept, kw in ((lists.view(B, H, 90).numpy(), dict(indices=held[0], counts=held[1])), ([[np.arange(n)] * H] * B, {})):
        args = sa.mx_attn_args(q, cache, out=out, **kw)
        ws = sa.alloc_workspace(sa.specattn_mx_workspace_size(args))
        args.workspace, args.workspace_bytes = ws.data_ptr(), ws.numel()
        sa.specattn_mx_decode_attn(args)
        expect, _, tol = ref.attention(q.double().cpu().numpy(), *(w.numpy() for w in want), kept, d ** -0.5)
        assert (np.abs(out.cpu().double().numpy() - expect) <= tol[..., None]).all()
    src, dst = (torch.tensor([x] * (B * H), dtype=torch.int32, device="cuda") for x in ([140, 149, 120], [3, 0, 77]))
    sa.specattn_evict_move(sa.move_args(src, dst, torch.full((B * H,), 3, dtype=torch.int32, device="cuda"), [codes, scales], B=B, page_table=table, n_max=n))
    sa.specattn_mx_load(sa.mx_rows_args(cache, *back))
    for x, w in zip(back, want):
        moved = w.clone()
        moved[:, :, [3, 0, 77]] = w[:, :, [140, 149, 120]]
        assert torch.equal(x.double().cpu(), moved)


def test_pool_slots_beyond_4_gib():
    H, d, T, pages = 2, 128, 2, 700
    codes, scales, _ = _views("pages far apart", 1, H, 100, d)
    slots = torch.tensor([0, 17, 5000, pages * 16 - 1, pages * 16 - 16, 8000], dtype=torch.int32)
    g = torch.Generator().manual_seed(1)
    k, v = (torch.randn((1, H, 6, d), generator=g).bfloat16() for _ in range(2))
    (ck, sk), (cv, sv) = (ref.quantise(x.double().numpy()) for x in (k, v))
    for i, s in enumerate(slots.tolist()):
        codes[s // 16, :, s % 16] = torch.from_numpy(np.concatenate((ref.pack(ck[0, :, i]), ref.pack(cv[0, :, i])), -1)).cuda()
        scales[s // 16, :, s % 16] = torch.from_numpy(np.concatenate((sk[0, :, i], sv[0, :, i]), -1)).cuda()
    q, out = torch.randn((1, 4, T, d), generator=g).bfloat16().cuda(), torch.empty((1, 4, T, d), device="cuda")
    lists, counts = slots.repeat(H, 1).cuda(), torch.full((H,), 6, dtype=torch.int32, device="cuda")
    args = sa.mx_attn_args(q, sa.mx_cache(codes, scales, B=1), out=out, indices=lists, counts=counts, indices_are_physical=True)
    ws = sa.alloc_workspace(sa.specattn_mx_workspace_size(args))
    args.workspace, args.workspace_bytes = ws.data_ptr(), ws.numel()
    sa.specattn_mx_decode_attn(args)
    expect, _, tol = ref.attention(q.double().cpu().numpy(), ref.values(ck, sk), ref.values(cv, sv), [[np.arange(6)] * H], d ** -0.5)
    assert (np.abs(out.cpu().double().numpy() - expect) <= tol[..., None]).all()
