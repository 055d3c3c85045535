"""The serving loop as it is used: prompts take pages and go in, are attended to, trees of drafted tokens are verified over what the selection kept, the
accepted nodes stay, sequences end and others come in their place; eager, and with a verify step replayed from a graph."""
import numpy as np
import pytest
import torch

import serve_reference as ref
from paper_2510_27641_amd import binding as sa
from test_gpu_tree import tree_masks

pytestmark = pytest.mark.gpu

PAGE, H_Q, H_KV, D, T = 16, 8, 2, 128, 12


class Server:
    """Device state of a loop over B sequences, and what it should hold: every sequence's keys and values, token by token."""

    def __init__(self, B=4, width=24, dtype="bf16"):
        i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
        self.B, self.dt, self.dtype, pages = B, ref.DT[dtype], dtype, B * width - 20
        self.table, self.free, self.count = i32(B, width), torch.randperm(pages, dtype=torch.int32).cuda(), torch.tensor([pages], dtype=torch.int32, device="cuda")
        self.lens, self.new = i32(B), i32(B)
        self.capacity = 600
        self.slots, self.starts, self.flags = i32(self.capacity), i32(B + 1), i32(B)
        self.pool = [torch.full((pages, H_KV, PAGE, D), float("nan"), dtype=self.dt, device="cuda") for _ in range(2)]
        self.args = sa.pages_args(self.table, PAGE, self.free, self.count, self.lens, self.new, slots=self.slots, token_starts=self.starts, row_flags=self.flags)
        self.ws = sa.alloc_workspace(sa.specattn_pages_workspace_size(self.args))
        self.held = [([], []) for _ in range(B)]

    def grow(self, new):
        self.new.copy_(torch.tensor(new, dtype=torch.int32))
        sa.specattn_pages_update(self.args, self.ws)
        assert not self.flags.any() and self.lens.tolist() == list(new)

    def rows(self, b):
        return [torch.stack(x).double().cpu().numpy() for x in self.held[b]]

    def prompt(self, new, seed):
        """new[b] tokens come to sequence b, behind what it holds."""
        g = torch.Generator(device="cuda").manual_seed(seed)
        total = sum(new)
        q, k, v = (torch.randn((total, h, D), generator=g, device="cuda").to(self.dt) for h in (H_Q, H_KV, H_KV))
        before = self.lens.tolist()
        self.grow([x + n for x, n in zip(before, new)])
        sa.specattn_cache_store(sa.store_args(k, v, *self.pool, self.slots[:total].contiguous()))
        at = 0
        for b, n in enumerate(new):
            self.held[b][0].extend(k[at:at + n])
            self.held[b][1].extend(v[at:at + n])
            at += n
        out, lse = torch.full((total, H_Q, D), float("nan"), device="cuda"), torch.full((total, H_Q), float("nan"), device="cuda")
        a = sa.prompt_args(q, *self.pool, self.starts, page_table=self.table, seq_lens=self.lens, out=out, lse=lse)
        ws = sa.alloc_workspace(sa.specattn_prompt_workspace_size(a))
        sa.set_workspace(a, ws)
        sa.specattn_prompt_attn(a)
        torch.cuda.synchronize()
        at = 0
        for b, n in enumerate(new):
            if n == 0:
                continue
            key, val = self.rows(b)
            seen = np.arange(len(key))[None] < (before[b] + np.arange(n)[:, None] + 1)
            for h in range(H_Q):
                want, want_lse, tol, _, tol_lse = ref.attend(q[at:at + n, h].double().cpu().numpy(), key[:, h // (H_Q // H_KV)], val[:, h // (H_Q // H_KV)], seen, D ** -0.5, self.dtype)
                assert (np.abs(out[at:at + n, h].cpu().numpy() - want) <= tol).all() and (np.abs(lse[at:at + n, h].cpu().numpy() - want_lse) <= tol_lse).all()
            at += n

    def draft(self, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.q = torch.randn((self.B, H_Q, T, D), generator=g, device="cuda").to(self.dt)
        self.k_new, self.v_new = (torch.randn((self.B, H_KV, T, D), generator=g, device="cuda").to(self.dt) for _ in range(2))
        self.masks = tree_masks(rng, self.B, T)
        n = self.table.shape[1] * PAGE
        probs = torch.rand((self.B, H_KV, n), generator=g, device="cuda") ** 6
        self.probs = probs
        return rng

    def verify(self, state):
        """Selection and attention of the trees; `state` holds the buffers, which a graph keeps."""
        sa.specattn_topp_select(state["sel"])
        sa.specattn_tree_attn(state["tree"])

    def verify_state(self):
        n = self.table.shape[1] * PAGE
        s = dict(indices=torch.empty((self.B * H_KV, n), dtype=torch.int32, device="cuda"), counts=torch.empty(self.B * H_KV, dtype=torch.int32, device="cuda"),
                 out=torch.empty((self.B, H_Q, T, D), device="cuda"), lse=torch.empty((self.B, H_Q, T), device="cuda"), masks=torch.from_numpy(self.masks.view(np.int64)).cuda())
        s["sel"] = sa.select_args(self.probs, 0.8, indices=s["indices"], counts=s["counts"], seq_lens=self.lens)
        s["tree"] = sa.tree_args(self.q, *self.pool, self.k_new, self.v_new, s["masks"], out=s["out"], lse=s["lse"], indices=s["indices"], counts=s["counts"],
                                 seq_lens=self.lens, page_table=self.table)
        s["ws"] = sa.alloc_workspace(sa.specattn_tree_workspace_size(s["tree"]))
        sa.set_workspace(s["tree"], s["ws"])
        return s

    def check_verify(self, s):
        torch.cuda.synchronize()
        counts, lists = s["counts"].tolist(), s["indices"].cpu().numpy()
        for b in range(self.B):
            if not self.held[b][0]:
                continue
            key, val = self.rows(b)
            bits = np.array([[bool((int(self.masks[b, t]) >> u) & 1) for u in range(T)] for t in range(T)])
            for h in range(H_Q):
                r = b * H_KV + h // (H_Q // H_KV)
                pos = lists[r, :counts[r]]
                k = np.concatenate((key[pos, h // (H_Q // H_KV)], self.k_new[b, h // (H_Q // H_KV)].double().cpu().numpy()))
                v = np.concatenate((val[pos, h // (H_Q // H_KV)], self.v_new[b, h // (H_Q // H_KV)].double().cpu().numpy()))
                seen = np.concatenate((np.ones((T, len(pos)), dtype=bool), bits), 1)
                want, want_lse, tol, _, tol_lse = ref.attend(self.q[b, h].double().cpu().numpy(), k, v, seen, D ** -0.5, self.dtype)
                assert (np.abs(s["out"][b, h].cpu().numpy() - want) <= tol).all() and (np.abs(s["lse"][b, h].cpu().numpy() - want_lse) <= tol_lse).all()

    def accept(self, rng):
        """A path of each tree, as long as it happens to be, becomes part of its sequence."""
        picked, new = [], self.lens.tolist()
        for b in range(self.B):
            t = int(rng.integers(0, T))
            path = [u for u in range(T) if (int(self.masks[b, t]) >> u) & 1]
            picked += [b * T + u for u in path]
            new[b] += len(path)
            for u in path:
                self.held[b][0].append(self.k_new[b, :, u].clone())
                self.held[b][1].append(self.v_new[b, :, u].clone())
        self.grow(new)
        rows = torch.full((self.capacity,), -1, dtype=torch.int32, device="cuda")
        rows[:len(picked)] = torch.tensor(picked, dtype=torch.int32)
        sa.specattn_cache_store(sa.store_args(self.k_new, self.v_new, *self.pool, self.slots, rows=rows))      # the whole map: -1 is left out

    def check_cache(self):
        torch.cuda.synchronize()
        table, used = self.table.cpu().long(), []
        for b, n in enumerate(self.lens.tolist()):
            assert n == len(self.held[b][0])
            if n == 0:
                continue
            pages = table[b, :-(-n // PAGE)]
            used += pages.tolist()
            for pool, want in zip(self.pool, self.held[b]):
                got = pool[pages.cuda()].transpose(1, 2).reshape(-1, H_KV, D)[:n]
                assert torch.equal(got, torch.stack(want))
        free = self.free.tolist()[:int(self.count)]
        assert sorted(used + free) == list(range(self.free.numel()))       # no page is lost, none is there twice


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_loop(dtype):
    s = Server(dtype=dtype)
    s.prompt([70, 1, 33, 16], 1)
    s.check_cache()
    for step in range(3):
        rng = s.draft(10 + step)
        state = s.verify_state()
        s.verify(state)
        s.check_verify(state)
        s.accept(rng)
        s.check_cache()
    s.grow([s.lens.tolist()[0], 0, 0, s.lens.tolist()[3]])                # two end,
    s.held[1], s.held[2] = ([], []), ([], [])
    s.prompt([5, 100, 17, 0], 2)                                          # others come, one goes on
    s.check_cache()


def test_verify_step_from_a_graph():
    s = Server()
    s.prompt([50, 40, 90, 130], 3)
    rng = s.draft(20)
    state = s.verify_state()
    sa.specattn_init()
    s.verify(state)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.verify(state)
    buffers = [s.q, s.k_new, s.v_new, s.probs]
    for step in range(3):
        state["out"].zero_()
        g.replay()
        s.check_verify(state)
        s.accept(rng)
        s.check_cache()
        rng = s.draft(21 + step)                                          # new drafts into the buffers that the graph reads
        for old, name in zip(buffers, ("q", "k_new", "v_new", "probs")):
            old.copy_(getattr(s, name))
            setattr(s, name, old)
        state["masks"].copy_(torch.from_numpy(s.masks.view(np.int64)))


def test_two_attention_calls_at_once():
    """Prompts and trees on two streams, each with its own workspace, over one cache."""
    s = Server()
    s.prompt([200, 60, 10, 31], 4)
    s.draft(30)
    state = s.verify_state()
    s.verify(state)
    q = torch.randn((301, H_Q, D), device="cuda").to(s.dt)
    out = torch.empty((301, H_Q, D), device="cuda")
    a = sa.prompt_args(q, *s.pool, s.starts, page_table=s.table, seq_lens=s.lens, out=out)
    ws = sa.alloc_workspace(sa.specattn_prompt_workspace_size(a))
    sa.set_workspace(a, ws)
    sa.specattn_prompt_attn(a)
    torch.cuda.synchronize()
    want = state["out"].clone(), out.clone()
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        state["out"].zero_()
        out.zero_()
        torch.cuda.synchronize()
        sa.specattn_tree_attn(state["tree"], stream=one)
        sa.specattn_prompt_attn(a, stream=two)
        torch.cuda.synchronize()
        assert torch.equal(state["out"], want[0]) and torch.equal(out, want[1])
