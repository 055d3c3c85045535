"""A 4-bit cache at its budget over many steps: attention rows come in, slots leave, accepted tokens come behind what stayed and are entered with
their places in the text.  After every step each slot has to hold the token that positions names, whatever moved where; eager and captured."""
import numpy as np
import pytest
import torch

import mx_reference as ref
from paper_2510_27641_amd import binding as sa

pytestmark = pytest.mark.gpu

D, PAGE, T, SINKS, RECENT = 128, 16, 3, 2, 6


class Sequences:
    """Buffers of one layer.  Every step reads its own attention rows, new rows and accepted counts from the fixed ones."""

    def __init__(self, B, H, N, budget, prompt, seed):
        self.B, self.H, self.N, self.budget = B, H, N, budget
        g = torch.Generator().manual_seed(seed)
        per = N // PAGE
        self.table = torch.randperm(B * per, generator=g).int().view(B, per).cuda()
        self.codes, self.scales = (torch.zeros((B * per, H, PAGE, w), dtype=torch.uint8, device="cuda") for w in (D, D // 16))
        self.cache = sa.mx_cache(self.codes, self.scales, page_table=self.table)
        self.text = [torch.randn((B, H, 400, D), generator=g).bfloat16().cuda() for _ in range(2)]       # the rows of every token there will be
        self.lens = torch.tensor(prompt, dtype=torch.int32, device="cuda")
        self.next, self.new_lens, self.accepted = self.lens.clone(), torch.zeros_like(self.lens), torch.zeros_like(self.lens)
        self.scores = torch.zeros((B, H, N), device="cuda")
        self.positions = torch.where(torch.arange(N, device="cuda") < self.lens[:, None, None], torch.arange(N, device="cuda"), -1).int().expand(B, H, N).contiguous()
        self.probs = torch.zeros((B, H, 1, N), device="cuda")
        self.new = [torch.zeros((B, H, T, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        cap = max(1, min(budget, N - budget))
        self.src, self.dst = (torch.zeros((B * H, cap), dtype=torch.int32, device="cuda") for _ in range(2))
        self.moved = torch.zeros(B * H, dtype=torch.int32, device="cuda")
        self.evict = sa.evict_args(self.probs, self.scores, self.positions, self.next, budget, move_src=self.src, move_dst=self.dst, move_counts=self.moved,
                                   new_lens=self.new_lens, seq_lens=self.lens, sinks=SINKS, recent=RECENT, decay=0.9)
        self.ws = sa.alloc_workspace(sa.specattn_evict_workspace_size(self.evict))
        self.move = sa.move_args(self.src, self.dst, self.moved, [self.codes, self.scales], B=B, page_table=self.table)
        self.append = sa.mx_rows_args(self.cache, *self.new, starts=self.new_lens, counts=self.accepted)
        sa.specattn_mx_store(sa.mx_rows_args(self.cache, *(x[:, :, :max(prompt)].contiguous() for x in self.text), counts=self.lens))

    def feed(self, rng):
        """What the models give: attention rows, the accepted tokens and their rows."""
        self.probs.copy_(torch.from_numpy((rng.random((self.B, self.H, 1, self.N)) ** 6).astype(np.float32)))
        self.accepted.copy_(torch.from_numpy(rng.integers(0, T + 1, size=self.B).astype(np.int32)))
        for b, at in enumerate(self.next.tolist()):
            for x, y in zip(self.new, self.text):
                x[b].copy_(y[b, :, at:at + T])

    def step(self):
        sa.specattn_evict_select(self.evict, self.ws)
        sa.specattn_evict_move(self.move)
        sa.specattn_mx_store(self.append)
        # the appended tokens are entered with their places in the text
        ahead = torch.arange(self.N, device="cuda", dtype=torch.int32) - self.new_lens[:, None]
        fresh = ((ahead >= 0) & (ahead < self.accepted[:, None]))[:, None]
        self.positions.copy_(torch.where(fresh, (self.next[:, None] + ahead)[:, None], self.positions))
        self.scores.masked_fill_(fresh, 0.25)
        torch.add(self.new_lens, self.accepted, out=self.lens)
        self.next += self.accepted

    def state(self):
        return [x.clone() for x in (self.codes, self.scales, self.scores, self.positions, self.lens, self.next, self.moved)]

    def slots(self):
        return [torch.cat([x[p] for p in self.table.view(-1).long()], 1).view(self.H, self.B, self.N, -1).transpose(0, 1).cpu().numpy() for x in (self.codes, self.scales)]


def test_slots_hold_the_tokens_that_positions_names():
    seq = Sequences(3, 2, 64, 48, [60, 20, 48], 1)
    rows = [np.concatenate(x, -1) for x in zip(*((ref.pack(c), s) for c, s in (ref.quantise(x.double().cpu().numpy()) for x in seq.text)))]
    rng, dropped = np.random.default_rng(2), 0
    for _ in range(25):
        seq.feed(rng)
        before = [x.cpu().numpy().copy() for x in (seq.scores, seq.positions, seq.lens, seq.next, seq.probs, seq.accepted)]
        seq.step()
        torch.cuda.synchronize()
        s, p, moves, new_lens, _ = ref.evict(*before[:4], seq.budget, SINKS, RECENT, 0.9, before[4])
        lens, positions, scores = (x.cpu().numpy() for x in (seq.lens, seq.positions, seq.scores))
        assert np.array_equal(lens, new_lens + before[5]) and seq.moved.tolist() == [len(m) for m in moves]
        codes, scales = seq.slots()
        for b in range(seq.B):
            dropped += int(before[2][b] - new_lens[b])
            for h in range(seq.H):
                held = positions[b, h, :lens[b]]
                assert np.array_equal(held[:new_lens[b]], p[b, h, :new_lens[b]]) and np.array_equal(scores[b, h, :new_lens[b]], s[b, h, :new_lens[b]])
                assert np.array_equal(held[new_lens[b]:], before[3][b] + np.arange(before[5][b])) and (positions[b, h, lens[b]:] == -1).all()
                # nobody twice, the first and the last tokens always among them
                assert len(set(held)) == len(held) and set(range(SINKS)) <= set(held) and set(range(int(seq.next[b]) - RECENT, int(seq.next[b]))) <= set(held)
                assert np.array_equal(codes[b, h, :lens[b]], rows[0][b, h, held]) and np.array_equal(scales[b, h, :lens[b]], rows[1][b, h, held])
    assert dropped > 50


def test_captured_steps_equal_eager_ones():
    """One captured step replayed over twelve, eager work of another object between them."""
    a, b = Sequences(2, 2, 64, 48, [64, 30], 5), Sequences(2, 2, 64, 48, [64, 30], 5)
    first = Sequences(2, 2, 64, 48, [64, 30], 6)                # (loads every kernel before the capture)
    first.feed(np.random.default_rng(0))
    first.step()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    b.feed(np.random.default_rng(7))
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        b.step()
    rng = [np.random.default_rng(3), np.random.default_rng(3)]
    for _ in range(12):
        a.feed(rng[0])
        b.feed(rng[1])
        a.step()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(a.state(), b.state()):
            assert torch.equal(x, y)
        first.feed(rng[0].spawn(1)[0])
        first.step()
        torch.cuda.synchronize()
