"""The operators of the 4-bit cache together, as a decoder calls them: a prompt goes in, attention rows choose positions, the attention
reads them, slots are evicted, new tokens come behind what stayed; eager and captured in a graph."""
import numpy as np
import pytest
import torch

import mx_reference as ref
from paper_2510_27641_amd import binding as sa

pytestmark = pytest.mark.gpu

B, H_q, H, T, D, N, PAGE = 2, 8, 2, 3, 128, 160, 16
BUDGET = 96


class Decoder:
    """Buffers of one layer, and one step over them."""

    def __init__(self, seed=0):
        g = torch.Generator().manual_seed(seed)
        per = N // PAGE
        self.table = torch.randperm(B * per, generator=g).int().view(B, per).cuda()
        self.codes = torch.zeros((B * per, H, PAGE, D), dtype=torch.uint8, device="cuda")
        self.scales = torch.zeros((B * per, H, PAGE, D // 16), dtype=torch.uint8, device="cuda")
        self.cache = sa.mx_cache(self.codes, self.scales, page_table=self.table)
        self.lens = torch.tensor([120, 70], dtype=torch.int32, device="cuda")
        self.next = self.lens.clone()
        self.new_lens, self.accepted = torch.zeros_like(self.lens), torch.tensor([T, 2], dtype=torch.int32, device="cuda")
        self.scores = torch.zeros((B, H, N), device="cuda")
        self.positions = torch.arange(N, dtype=torch.int32, device="cuda").expand(B, H, N).contiguous()
        self.prompt = [torch.randn((B, H, 120, D), generator=g).bfloat16().cuda() for _ in range(2)]
        self.q = torch.randn((B, H_q, T, D), generator=g).bfloat16().cuda()
        self.new = [torch.randn((B, H, T, D), generator=g).bfloat16().cuda() for _ in range(2)]
        self.probs = torch.rand((B, H, 1, N), generator=g).pow(6).cuda()
        self.lists, self.counts = torch.zeros((B * H, N), dtype=torch.int32, device="cuda"), torch.zeros(B * H, dtype=torch.int32, device="cuda")
        self.out, self.lse = torch.zeros((B, H_q, T, D), device="cuda"), torch.zeros((B, H_q, T), device="cuda")
        cap = max(BUDGET, N - BUDGET)
        self.src, self.dst = (torch.zeros((B * H, cap), dtype=torch.int32, device="cuda") for _ in range(2))
        self.moved = torch.zeros(B * H, dtype=torch.int32, device="cuda")
        self.select = sa.select_args(self.probs[:, :, 0], 0.9, indices=self.lists, counts=self.counts, seq_lens=self.lens)
        self.attn = sa.mx_attn_args(self.q, self.cache, out=self.out, lse=self.lse, indices=self.lists, counts=self.counts, k_new=self.new[0], v_new=self.new[1])
        self.ws = sa.alloc_workspace(sa.specattn_mx_workspace_size(self.attn))
        self.attn.workspace, self.attn.workspace_bytes = self.ws.data_ptr(), self.ws.numel()
        self.evict = sa.evict_args(self.probs, self.scores, self.positions, self.next, BUDGET, move_src=self.src, move_dst=self.dst, move_counts=self.moved,
                                   new_lens=self.new_lens, seq_lens=self.lens, sinks=2, recent=8, decay=0.9)
        self.ews = sa.alloc_workspace(sa.specattn_evict_workspace_size(self.evict))
        self.move = sa.move_args(self.src, self.dst, self.moved, [self.codes, self.scales], B=B, page_table=self.table)
        self.append = sa.mx_rows_args(self.cache, *self.new, starts=self.new_lens, counts=self.accepted)

    def fill(self):
        sa.specattn_mx_store(sa.mx_rows_args(self.cache, *self.prompt, counts=self.lens))

    def step(self):
        sa.specattn_topp_select(self.select)
        sa.specattn_mx_decode_attn(self.attn)
        sa.specattn_evict_select(self.evict, self.ews)
        sa.specattn_evict_move(self.move)
        sa.specattn_mx_store(self.append)

    def state(self):
        return [x.clone() for x in (self.codes, self.scales, self.scores, self.positions, self.new_lens, self.out, self.lse, self.counts, self.moved)]

    def slots(self):
        """Codes and scales [B, H, N, .] in slot order."""
        return [torch.cat([x[p] for p in self.table.view(-1).long()], 1).view(H, B, N, -1).transpose(0, 1).cpu().numpy() for x in (self.codes, self.scales)]


def test_a_step_against_the_plain_forms():
    dec = Decoder()
    dec.fill()
    codes, scales = dec.slots()
    lens = dec.lens.cpu().numpy()
    for x, at in zip(dec.prompt, (0, 1)):
        want = ref.quantise(x.double().cpu().numpy())
        for b in range(B):
            assert np.array_equal(codes[b, :, :lens[b], at * D // 2:(at + 1) * D // 2], ref.pack(want[0])[b, :, :lens[b]])
            assert np.array_equal(scales[b, :, :lens[b], at * 4:(at + 1) * 4], want[1][b, :, :lens[b]])
    dec.step()
    torch.cuda.synchronize()
    lists, counts = dec.lists.cpu().numpy(), dec.counts.cpu().numpy()
    kept = [[lists[b * H + h, :counts[b * H + h]] for h in range(H)] for b in range(B)]
    assert all(0 < len(x) < lens[b] for b in range(B) for x in kept[b])
    k, v = ref.cache_values(codes, scales)
    want, want_lse, tol = ref.attention(dec.q.double().cpu().numpy(), k, v, kept, D ** -0.5, *(x.double().cpu().numpy() for x in dec.new))
    assert (np.abs(dec.out.cpu().double().numpy() - want) <= tol[..., None]).all()
    s, p, moves, new_lens, _ = ref.evict(np.zeros((B, H, N), np.float32), np.tile(np.arange(N, dtype=np.int32), (B, H, 1)), lens, lens, BUDGET, 2, 8, 0.9, dec.probs.cpu().numpy())
    inside = np.arange(N) < lens[:, None, None]
    assert np.array_equal(np.where(inside, s, 0), np.where(inside, dec.scores.cpu().numpy(), 0)) and np.array_equal(np.where(inside, p, 0), np.where(inside, dec.positions.cpu().numpy(), 0))
    assert np.array_equal(dec.new_lens.cpu().numpy(), new_lens) and list(new_lens) == [BUDGET, 70] and len(moves[0]) > 0
    after = dec.slots()
    new = [ref.quantise(x.double().cpu().numpy()) for x in dec.new]
    rows = [np.concatenate((ref.pack(new[0][0]), ref.pack(new[1][0])), -1), np.concatenate((new[0][1], new[1][1]), -1)]
    for got, full, fresh in zip(after, (codes, scales), rows):
        for b in range(B):
            for h in range(H):
                one = full[b, h].copy()
                for a, d in moves[b * H + h]:
                    one[d] = full[b, h, a]
                for t in range(int(dec.accepted[b])):
                    one[new_lens[b] + t] = fresh[b, h, t]
                assert np.array_equal(got[b, h], one)


def test_a_captured_step_equals_the_eager_one():
    """Replayed three times with eager work between; every replay starts from the same cache and has to end in the same state."""
    dec = Decoder(3)
    dec.fill()
    start = [x.clone() for x in (dec.codes, dec.scales, dec.scores, dec.positions)]

    def reset():
        for x, y in zip((dec.codes, dec.scales, dec.scores, dec.positions), start):
            x.copy_(y)
        dec.out.fill_(float("nan"))
        dec.ws.fill_(0xA5)
        dec.ews.fill_(0x5A)
    reset()
    dec.step()
    torch.cuda.synchronize()
    want = dec.state()
    reset()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        dec.step()
    torch.cuda.current_stream().wait_stream(side)
    for _ in range(3):
        reset()
        graph.replay()
        torch.cuda.synchronize()
        for got, w in zip(dec.state(), want):
            assert torch.equal(got, w)
        other = Decoder(4)                                     # other eager work in between
        other.fill()
        other.step()
        torch.cuda.synchronize()


def test_two_streams_with_their_own_workspaces():
    a, b = Decoder(5), Decoder(6)
    want = []
    for dec in (a, b):
        dec.fill()
        dec.step()
        torch.cuda.synchronize()
        want.append(dec.state())
    a, b = Decoder(5), Decoder(6)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for dec, stream in zip((a, b), streams):
        with torch.cuda.stream(stream):
            dec.fill()
            dec.step()
    torch.cuda.synchronize()
    for dec, w in zip((a, b), want):
        for x, y in zip(dec.state(), w):
            assert torch.equal(x, y)
