"""The operators of a serving loop in pages, as cases that can be timed and checked: prompts come in, trees of drafted tokens are
verified, the accepted tokens stay.

A case is a dict of plain values.  Its `kind` names the operator:

  pages    page tables, free pages and the slots of new tokens, from the lengths that the sequences have and are to have
  store    rows of keys and values into the slots of a cache
  prompt   causal attention over packed prompts of different lengths, alone or behind a prefix that the cache holds in pages
  tree     attention of a tree of drafted tokens over the cache (index lists, chunk lists or every position) and over the nodes
           that each of them descends from

With `own` false, `run` computes an operator from elementary torch operations; with `own` true it calls this library.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ELEM_BYTES = {"f32": 4, "bf16": 2, "f16": 2}
PAGE = 16


def _pages(name, mode, B, n, T):
    """mode "step": up to T tokens come to most of B sequences of up to n tokens, some shrink, some end; "admit": up to T tokens of
    prompts come in, an eighth of the sequences runs on."""
    return dict(name=name, kind="pages", mode=mode, B=B, n=n, T=T)


def _store(name, dtype, d, H_kv, B, T, n, *, nodes=False):
    """nodes: some of the T rows of each sequence, by an index; otherwise packed rows, up to T a sequence."""
    return dict(name=name, kind="store", dtype=dtype, d=d, H_kv=H_kv, B=B, T=T, n=n, nodes=nodes)


def _prompt(name, dtype, d, H_q, H_kv, B, n, *, prefix=0, ragged=False):
    """prefix: most positions that the cache (in pages) holds ahead of a sequence's new tokens."""
    return dict(name=name, kind="prompt", dtype=dtype, d=d, H_q=H_q, H_kv=H_kv, B=B, n=n, prefix=prefix, ragged=ragged)


def _tree(name, dtype, d, H_q, H_kv, B, T, n, *, kept=0.25, chunk=1, paged=False, ragged=False):
    """kept 0: no list, every position of a sequence."""
    return dict(name=name, kind="tree", dtype=dtype, d=d, H_q=H_q, H_kv=H_kv, B=B, T=T, n=n, kept=kept, chunk=chunk, paged=paged, ragged=ragged)


def listed():
    return [
        # A verify step of 64 sequences: one to eight tokens more each, a few shrink or end.
        _pages("pages_step", "step", 64, 8192, 8),
        # Prompts of up to 4096 tokens come in, 256 at once.
        _pages("pages_admit", "admit", 256, 8192, 4096),
        # The accepted nodes of 64 drafted trees go into the cache.
        _store("store_accepted", "bf16", 128, 8, 64, 16, 4096, nodes=True),
        # Packed prompts of up to 4096 tokens go into the pages, 32 at once.
        _store("store_prompts", "f16", 128, 8, 32, 4096, 4096),
        # The smallest prompt: a question of 37 tokens to a small model; launches and latency only.
        _prompt("prompt_tiny", "f16", 64, 8, 8, 1, 37),
        # A batch of 24 questions of very different lengths, up to 2048 tokens.
        _prompt("prompt_packed", "bf16", 128, 32, 8, 24, 2048, ragged=True),
        # Pieces of 512 tokens of four long prompts, behind up to 16384 positions in pages; eight query heads to a kv head.
        _prompt("prompt_piece", "f16", 128, 64, 8, 4, 512, prefix=16384),
        # One document of 32768 tokens.
        _prompt("prompt_long", "bf16", 128, 32, 8, 1, 32768),
        # The smallest tree: seven nodes over a context of 1024.
        _tree("tree_tiny", "f16", 64, 8, 8, 1, 7, 1024, kept=0.2),
        # One layer of an interactive session: 26 nodes, one sequence of 8192 positions, a third of them selected.
        _tree("tree_single_8k", "bf16", 128, 32, 8, 1, 26, 8192, kept=0.33),
        # One layer of a verify step: a batch of 8 at 32768 positions, a quarter of them selected, 16 nodes.
        _tree("tree_step_32k", "bf16", 128, 32, 8, 8, 16, 32768, kept=0.23),
        # Wide trees of 64 nodes, eight query heads to a kv head, over 16 sequences in pages, selected in chunks.
        _tree("tree_wide_paged", "f16", 128, 64, 8, 16, 64, 16384, kept=0.4, chunk=16, paged=True, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_once(rng):
    pick = rng.random()
    dtype = rng.choice(["bf16", "f16"])
    d = rng.choice([64, 128, 128])
    if pick < 0.10:
        return _pages("", "step", _log_int(rng, 1, 512), _log_int(rng, 64, 32768), rng.randint(1, 64))
    if pick < 0.20:
        n = _log_int(rng, 64, 16384)
        return _pages("", "admit", _log_int(rng, 1, 512), n, _log_int(rng, 1, n))
    if pick < 0.28:
        return _store("", rng.choice(["bf16", "f16", "f32"]), d, rng.choice([1, 4, 8]), _log_int(rng, 1, 256), rng.randint(1, 64), _log_int(rng, 64, 4096), nodes=True)
    if pick < 0.36:
        n = _log_int(rng, 16, 4096)
        return _store("", rng.choice(["bf16", "f16", "f32"]), d, rng.choice([1, 4, 8]), _log_int(rng, 1, 32), _log_int(rng, 1, n), n)
    H_kv = rng.choice([1, 2, 4, 8])
    H_q = H_kv * rng.choice([1, 2, 4, 5, 8])
    if pick < 0.50:                                            # one prompt
        return _prompt("", dtype, d, H_q, H_kv, 1, _log_int(rng, 1, 16384))
    if pick < 0.60:                                            # packed prompts
        return _prompt("", dtype, d, H_q, H_kv, _log_int(rng, 2, 64), _log_int(rng, 4, 4096), ragged=True)
    if pick < 0.70:                                            # pieces behind a prefix, single tokens among them
        return _prompt("", dtype, d, H_q, H_kv, _log_int(rng, 1, 16), _log_int(rng, 1, 1024), prefix=_log_int(rng, 1, 16384), ragged=rng.random() < 0.5)
    if pick < 0.85:                                            # trees over lists of positions
        return _tree("", dtype, d, H_q, H_kv, rng.randint(1, 12), rng.randint(1, 64), _log_int(rng, 100, 32768), kept=round(rng.uniform(0.05, 0.9), 2))
    if pick < 0.93:                                            # over chunk lists
        return _tree("", dtype, d, H_q, H_kv, rng.randint(1, 8), rng.randint(2, 64), _log_int(rng, 500, 32768), kept=round(rng.uniform(0.2, 0.8), 2),
                     chunk=rng.choice([8, 16, 32]), paged=rng.random() < 0.5, ragged=rng.random() < 0.5)
    return _tree("", dtype, d, H_q, H_kv, _log_int(rng, 1, 32), rng.randint(1, 64), _log_int(rng, 1, 16384), kept=0.0, paged=rng.random() < 0.5, ragged=True)


def draw(rng):
    most = {}
    for c in listed():
        w = work(c)
        most["bytes"], most["flops"] = max(most.get("bytes", 0), w["bytes"]), max(most.get("flops", 0), w["flops"])
    while True:
        case = _draw_once(rng)
        w = work(case)
        if w["bytes"] <= most["bytes"] and w["flops"] <= most["flops"]:
            del case["name"]
            return case


# ------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------
def _spread(case, seed=None):
    """Lengths of the sequences: all n, or spread evenly (by their logarithm) from a 64th of n up to n, in an order that the seed sets."""
    B, n = case["B"], case["n"]
    if not case.get("ragged"):
        return np.full(B, n, dtype=np.int64)
    lens = np.exp(np.linspace(math.log(max(1.0, n / 64)), math.log(n), B)).round().astype(np.int64) if B > 1 else np.array([n], dtype=np.int64)
    return lens if seed is None else np.random.default_rng(seed).permutation(lens)


def _prefixes(case):
    """Positions in the cache ahead of the new tokens, sequence by sequence."""
    B, most = case["B"], case["prefix"]
    return np.linspace(most / B, most, B).round().astype(np.int64) if most else np.zeros(B, dtype=np.int64)


def _page_lens(case, seed):
    """What the sequences of a `pages` case have and are to have."""
    B, n, T = case["B"], case["n"], case["T"]
    rng = np.random.default_rng(seed)
    now, new = rng.integers(1, max(2, n - T), B), None
    pick = rng.random(B)
    if case["mode"] == "step":
        grown = now + rng.integers(1, T + 1, B)
        new = np.where(pick < 0.85, grown, np.where(pick < 0.93, np.maximum(now - rng.integers(0, T + 1, B), 0), np.where(pick < 0.97, 0, now)))
    else:
        now = np.where(pick < 0.125, now, 0)
        new = now + np.where(pick < 0.125, 1, rng.integers((T + 1) // 2, T + 1, B))
    return now.astype(np.int64), np.minimum(new, _width(case) * PAGE).astype(np.int64)


def _width(case):
    return -(-(case["n"] + case["T"]) // PAGE)


def _int32(x):
    return torch.from_numpy(np.ascontiguousarray(x).astype(np.int32)).cuda()


def _prepare_pages(case, seed, gen):
    B, width = case["B"], _width(case)
    now, new = _page_lens(case, seed)
    have = -(-now // PAGE)
    pages = B * width
    order = np.random.default_rng(seed + 1).permutation(pages)
    table = np.full((B, width), -1, dtype=np.int64)
    first = np.concatenate(([0], np.cumsum(have)))
    for b in range(B):
        table[b, :have[b]] = order[first[b]:first[b + 1]]
    free = np.full(pages, -1, dtype=np.int64)
    free[:pages - first[-1]] = order[first[-1]:]
    capacity = B * case["T"]
    out = {k: torch.full((size,), -7, dtype=torch.int32, device="cuda")
           for k, size in (("lens", B), ("free_left", 1), ("token_starts", B + 1), ("slots", capacity), ("places", capacity), ("owners", capacity), ("flags", B))}
    return {"case": case, "calls": {}, "table": _int32(table), "free": _int32(free), "free_count": _int32([pages - first[-1]]), "now": _int32(now),
            "new": _int32(new), "pages": pages, **out}


def _store_counts(case, seed=None):
    """Rows of each sequence that go into the cache."""
    B, T = case["B"], case["T"]
    counts = np.linspace(1, min(T, 6) if case["nodes"] else T, B).round().astype(np.int64)
    return counts if seed is None else np.random.default_rng(seed).permutation(counts)


def _normal(gen, shape, dtype):
    return torch.randn(shape, generator=gen, device="cuda").to(DTYPES[dtype])


def _prepare_store(case, seed, gen):
    B, T, H, d = case["B"], case["T"], case["H_kv"], case["d"]
    counts = _store_counts(case, seed)
    rows, pages = int(counts.sum()), B * (case["n"] // PAGE + 2)
    rng = np.random.default_rng(seed + 1)
    table = rng.permutation(pages).reshape(B, -1)
    slots, picked = [], []
    for b in range(B):
        start = int(rng.integers(0, max(1, table.shape[1] * PAGE - counts[b])))
        at = start + np.arange(counts[b])
        slots.append(table[b][at // PAGE] * PAGE + at % PAGE)
        picked.append(b * T + np.sort(rng.permutation(T)[:counts[b]]))
    shape = (B, H, T, d) if case["nodes"] else (rows, H, d)
    pool = [torch.zeros((pages, H, PAGE, d), dtype=DTYPES[case["dtype"]], device="cuda") for _ in range(2)]
    return {"case": case, "calls": {}, "k": _normal(gen, shape, case["dtype"]), "v": _normal(gen, shape, case["dtype"]), "k_pool": pool[0], "v_pool": pool[1],
            "slots": _int32(np.concatenate(slots)), "rows": _int32(np.concatenate(picked)) if case["nodes"] else None}


def _sink(q, k, first):
    """An attention sink: queries share a direction, to which the keys at `first` (a list of indexes into k) are turned."""
    d = q.shape[-1]
    q += 4.0 / math.sqrt(d)
    for at in first:
        k[at] = 1.5


def _prepare_prompt(case, seed, gen):
    B, H_q, H, d = case["B"], case["H_q"], case["H_kv"], case["d"]
    lens, prefix = _spread(case, seed), _prefixes(case)
    starts = np.concatenate(([0], np.cumsum(lens)))
    total, width = int(starts[-1]), (H_q + 2 * H) * d
    joint = _normal(gen, (total, width), case["dtype"])        # queries, keys and values as one projection leaves them
    q, k, v = joint[:, :H_q * d].view(total, H_q, d), joint[:, H_q * d:(H_q + H) * d].view(total, H, d), joint[:, (H_q + H) * d:].view(total, H, d)
    table = None
    if case["prefix"]:
        per = -(-(prefix + lens) // PAGE)
        pages, widest = int(per.sum()) + 3, int(per.max())
        order = np.random.default_rng(seed + 1).permutation(pages)
        first = np.concatenate(([0], np.cumsum(per)))
        rows = np.zeros((B, widest), dtype=np.int64)
        for b in range(B):
            rows[b, :per[b]] = order[first[b]:first[b + 1]]
        table = _int32(rows)
        k, v = _normal(gen, (pages, H, PAGE, d), case["dtype"]), _normal(gen, (pages, H, PAGE, d), case["dtype"])
        _sink(q, k, [(int(p), slice(None), 0) for p in rows[:, 0]])
    else:
        _sink(q, k, [int(s) for s in starts[:-1]])
    return {"case": case, "calls": {}, "q": q, "k": k, "v": v, "starts": _int32(starts), "table": table, "lens": _int32(prefix + lens),
            "sizes": [int(x) for x in lens], "seen": [int(x) for x in prefix + lens],
            "out": torch.empty((total, H_q, d), dtype=DTYPES[case["dtype"]], device="cuda"), "lse": torch.empty((total, H_q), device="cuda")}


def _tree_masks(rng, B, T):
    """Trees in which each node hangs below an earlier one (often the one just ahead); bit u of word t: node t descends from node u or is u."""
    masks = np.zeros((B, T), dtype=np.uint64)
    for b in range(B):
        for t in range(T):
            above = 0 if t == 0 else masks[b, t - 1 if rng.random() < 0.5 else rng.integers(0, t)]
            masks[b, t] = np.uint64(above) | (np.uint64(1) << np.uint64(t))
    return torch.from_numpy(masks.view(np.int64)).cuda()


def _prepare_tree(case, seed, gen):
    B, H_q, H, T, d, n, chunk, dtype = (case[k] for k in ("B", "H_q", "H_kv", "T", "d", "n", "chunk", "dtype"))
    lens = _spread(case, seed)
    rng = np.random.default_rng(seed + 2)
    table, shape = None, (B, H, n, d)
    if case["paged"]:
        per = -(-n // PAGE)
        table, shape = _int32(rng.permutation(B * per).reshape(B, per)), (B * per, H, PAGE, d)
    q, k, v = _normal(gen, (B, H_q, T, d), dtype), _normal(gen, shape, dtype), _normal(gen, shape, dtype)
    _sink(q, k, [(int(p), slice(None), 0) for p in table[:, 0].tolist()] if case["paged"] else [(slice(None), slice(None), 0)])
    lists = counts = None
    if case["kept"]:
        units = -(-torch.from_numpy(lens).cuda() // chunk).repeat_interleave(H)
        most = int(units.max())
        chance = torch.rand((B * H, most), generator=gen, device="cuda") < case["kept"]
        chance[:, 0] = True
        chance &= torch.arange(most, device="cuda") < units.view(-1, 1)
        counts = chance.sum(1).int()
        lists = torch.argsort((~chance).byte(), dim=1, stable=True)[:, :int(counts.max())].int().contiguous()
        lists[torch.arange(lists.shape[1], device="cuda") >= counts.view(-1, 1)] = -7
    return {"case": case, "calls": {}, "q": q, "k": k, "v": v, "k_new": _normal(gen, (B, H, T, d), dtype), "v_new": _normal(gen, (B, H, T, d), dtype),
            "masks": _tree_masks(rng, B, T), "table": table, "lens": _int32(lens), "lists": lists, "counts": counts,
            "out": torch.empty((B, H_q, T, d), dtype=DTYPES[dtype], device="cuda"), "lse": torch.empty((B, H_q, T), device="cuda")}


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return {"pages": _prepare_pages, "store": _prepare_store, "prompt": _prepare_prompt, "tree": _prepare_tree}[case["kind"]](case, seed, gen)


# ------------------------------------------------------------------------------------------
# the plain forms
# ------------------------------------------------------------------------------------------
def _pages_result(s):
    return {k: s[k] for k in ("table", "free", "lens", "free_left", "token_starts", "slots", "places", "owners", "flags")}


def _plain_pages(s):
    now, new, table, free = s["now"].long(), s["new"].long(), s["table"], s["free"]
    B, width = table.shape
    have, need = (now + PAGE - 1) // PAGE, (new + PAGE - 1) // PAGE
    gives = torch.where(new < now, have - need, 0)             # pages that a sequence returns, and asks for
    asks = torch.where(new > now, need - have, 0)
    count = s["free_count"].long()
    stack = count + gives.sum()
    fits = (asks == 0) | (asks.cumsum(0) <= stack)
    tokens = torch.where((new > now) & fits, new - now, 0)
    capacity = s["slots"].numel()
    grows = (tokens > 0) & (tokens.cumsum(0) <= capacity)
    refused = (new > now) & ~grows
    # returned pages go onto the stack in the order of the sequences and of their pages
    column = torch.arange(width, device="cuda")
    back = (new < now).view(-1, 1) & (column >= need.view(-1, 1)) & (column < have.view(-1, 1))
    rank = count + back.flatten().cumsum(0).view(B, width) - 1
    held = torch.cat((free, free.new_zeros(1)))                # (one place more, for what goes nowhere)
    held.scatter_(0, torch.where(back, rank, free.numel()).flatten(), table.flatten())
    free.copy_(held[:-1])
    # new pages come off its top in the same order
    taken = grows.view(-1, 1) & (column >= have.view(-1, 1)) & (column < need.view(-1, 1))
    order = stack - taken.flatten().cumsum(0).view(B, width)
    table.copy_(torch.where(taken, free[order.clamp(min=0)], table))
    s["free_left"].copy_(stack - taken.sum())
    s["lens"].copy_(torch.where(refused, now, new))
    s["flags"].copy_(torch.where(refused, 4, 0))
    ends = torch.where(grows, tokens, 0).cumsum(0)
    s["token_starts"].copy_(torch.cat((ends.new_zeros(1), ends)))
    i = torch.arange(capacity, device="cuda")
    owner = torch.searchsorted(ends, i, right=True)
    some = owner < B
    owner = owner.clamp(max=B - 1)
    place = now[owner] + i - s["token_starts"].long()[owner]
    slot = table[owner, (place // PAGE).clamp(max=width - 1)].long() * PAGE + place % PAGE
    for name, x in (("slots", slot), ("places", place), ("owners", owner)):
        s[name].copy_(torch.where(some, x, -1))
    return _pages_result(s)


def _plain_store(s):
    case = s["case"]
    slots = s["slots"].long()
    for rows, pool in ((s["k"], s["k_pool"]), (s["v"], s["v_pool"])):
        if case["nodes"]:
            rows = rows[s["rows"].long() // case["T"], :, s["rows"].long() % case["T"]]
        pool[slots // PAGE, :, slots % PAGE] = rows
    return {"k": s["k_pool"], "v": s["v_pool"]}


def _cached(pool, table_row, size):
    """Positions 0 .. size - 1 of a sequence: [H, size, d]."""
    pages = pool[table_row[:-(-size // PAGE)].long()]
    return pages.transpose(0, 1).flatten(1, 2)[:, :size]


def _plain_prompt(s):
    case = s["case"]
    H_q, H, d = case["H_q"], case["H_kv"], case["d"]
    G, row = H_q // H, 0
    for b, (size, seen) in enumerate(zip(s["sizes"], s["seen"])):
        q = s["q"][row:row + size].float()
        if s["table"] is None:
            k, v = (x[row:row + size].float().transpose(0, 1).contiguous() for x in (s["k"], s["v"]))
        else:
            k, v = (_cached(x, s["table"][b], seen).float().contiguous() for x in (s["k"], s["v"]))
        step = max(1, min(size, (1 << 28) // (seen * G)))       # rows of scores that are held at a time
        for i in range(0, size, step):
            m = min(step, size - i)
            last = seen - size + i + m                         # (later keys are seen by none of these rows)
            hidden = torch.arange(last, device="cuda") > (seen - size + i + torch.arange(m, device="cuda")).repeat_interleave(G).view(-1, 1)
            for h in range(H):
                x = q[i:i + m, h * G:(h + 1) * G].reshape(m * G, d) @ k[h, :last].t().contiguous()
                x = (x / math.sqrt(d)).masked_fill_(hidden, -math.inf)
                top = x.amax(-1, keepdim=True)
                w = x.sub_(top).exp_()
                total = w.sum(-1, keepdim=True)
                s["out"][row + i:row + i + m, h * G:(h + 1) * G] = ((w @ v[h, :last]) / total).view(m, G, d)
                s["lse"][row + i:row + i + m, h * G:(h + 1) * G] = (top + total.log()).view(m, G)
        row += size
    return {"out": s["out"], "lse": s["lse"]}


def _plain_tree(s):
    case = s["case"]
    B, H_q, H, T, d, n, chunk = (case[k] for k in ("B", "H_q", "H_kv", "T", "d", "n", "chunk"))
    G = H_q // H
    node = torch.arange(T, device="cuda")
    for b in range(B):
        hidden = ((s["masks"][b].view(T, 1) >> node) & 1) == 0
        for h in range(H):
            if case["kept"]:
                units = s["lists"][b * H + h].long()
                pos = (units.view(-1, 1) * chunk + torch.arange(chunk, device="cuda")).flatten()
                gone = (torch.arange(pos.numel(), device="cuda") // chunk >= s["counts"][b * H + h]) | (pos >= s["lens"][b])
            else:
                pos = torch.arange(n, device="cuda")
                gone = pos >= s["lens"][b]
            pos = torch.where(gone, 0, pos)
            if s["table"] is None:
                k, v = s["k"][b, h, pos], s["v"][b, h, pos]
            else:
                page = s["table"][b].long()[pos // PAGE]
                k, v = s["k"][page, h, pos % PAGE], s["v"][page, h, pos % PAGE]
            k, v = torch.cat((k, s["k_new"][b, h])).float(), torch.cat((v, s["v_new"][b, h])).float()
            x = (s["q"][b, h * G:(h + 1) * G].reshape(G * T, d).float() @ k.t().contiguous()) / math.sqrt(d)
            x = x.masked_fill(torch.cat((gone.expand(G * T, -1), hidden.repeat(G, 1)), 1), -math.inf)
            top = x.amax(-1, keepdim=True)
            w = (x - top).exp()
            total = w.sum(-1, keepdim=True)
            s["out"][b, h * G:(h + 1) * G] = ((w @ v) / total).view(G, T, d)
            s["lse"][b, h * G:(h + 1) * G] = (top + total.log()).view(G, T)
    return {"out": s["out"], "lse": s["lse"]}


# ------------------------------------------------------------------------------------------
# this library
# ------------------------------------------------------------------------------------------
def _own_pages(s):
    from paper_2510_27641_amd import binding as sa
    calls = s["calls"]
    if not calls:                                              # what a server sets up once
        calls["args"] = sa.pages_args(s["table"], PAGE, s["free"], s["free_count"], s["now"], s["new"], lens_out=s["lens"], free_count_out=s["free_left"],
                                      token_starts=s["token_starts"], slots=s["slots"], positions=s["places"], owners=s["owners"], row_flags=s["flags"])
        calls["ws"] = sa.alloc_workspace(sa.specattn_pages_workspace_size(calls["args"]))
    sa.specattn_pages_update(calls["args"], calls["ws"])
    return _pages_result(s)


def _own_store(s):
    from paper_2510_27641_amd import binding as sa
    calls = s["calls"]
    if not calls:
        calls["args"] = sa.store_args(s["k"], s["v"], s["k_pool"], s["v_pool"], s["slots"], rows=s["rows"])
    sa.specattn_cache_store(calls["args"])
    return {"k": s["k_pool"], "v": s["v_pool"]}


def _own_prompt(s):
    from paper_2510_27641_amd import binding as sa
    calls = s["calls"]
    if not calls:
        paged = {} if s["table"] is None else {"page_table": s["table"], "seq_lens": s["lens"]}
        calls["args"] = sa.prompt_args(s["q"], s["k"], s["v"], s["starts"], out_lowp=s["out"], lse=s["lse"], **paged)
        calls["ws"] = sa.alloc_workspace(sa.specattn_prompt_workspace_size(calls["args"]))
        sa.set_workspace(calls["args"], calls["ws"])
    sa.specattn_prompt_attn(calls["args"])
    return {"out": s["out"], "lse": s["lse"]}


def _own_tree(s):
    from paper_2510_27641_amd import binding as sa
    case, calls = s["case"], s["calls"]
    if not calls:
        calls["args"] = sa.tree_args(s["q"], s["k"], s["v"], s["k_new"], s["v_new"], s["masks"], out_lowp=s["out"], lse=s["lse"], indices=s["lists"],
                                     counts=s["counts"], seq_lens=s["lens"], chunk_size=case["chunk"], page_table=s["table"], page_size=PAGE, n_max=case["n"])
        calls["ws"] = sa.alloc_workspace(sa.specattn_tree_workspace_size(calls["args"]))
        sa.set_workspace(calls["args"], calls["ws"])
    sa.specattn_tree_attn(calls["args"])
    return {"out": s["out"], "lse": s["lse"]}


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"pages": _own_pages, "store": _own_store, "prompt": _own_prompt, "tree": _own_tree}[kind](state)
    return {"pages": _plain_pages, "store": _plain_store, "prompt": _plain_prompt, "tree": _plain_tree}[kind](state)


# ------------------------------------------------------------------------------------------
# what a pass cannot do without
# ------------------------------------------------------------------------------------------
def work(case):
    B = case["B"]
    if case["kind"] == "pages":
        now, new = _page_lens(case, 0)
        moved, tokens = np.abs(-(-now // PAGE) + (-new // PAGE)).sum(), np.maximum(new - now, 0).sum()
        return {"bytes": float(20 * B + 8 * moved + 12 * B * case["T"]), "flops": float(tokens + B)}
    d, H, e = case["d"], case["H_kv"], ELEM_BYTES[case["dtype"]]
    if case["kind"] == "store":
        rows = int(_store_counts(case).sum())
        return {"bytes": float(rows * (4 * H * d * e + (8 if case["nodes"] else 4))), "flops": float(rows)}
    H_q = case["H_q"]
    if case["kind"] == "prompt":
        lens, prefix = _spread(case), np.sort(_prefixes(case))
        pairs = float((lens * prefix + lens * (lens + 1) // 2).sum())
        rows = int(lens.sum())
        return {"bytes": float(rows * H_q * (2 * d * e + 4) + int((lens + prefix).sum()) * 2 * H * d * e), "flops": 4.0 * pairs * H_q * d}
    T = case["T"]
    seen = float(_spread(case).sum()) * H * (case["kept"] or 1.0)
    listed_bytes = 4 * seen / case["chunk"] if case["kept"] else 0
    rows = B * H_q * T
    return {"bytes": seen * 2 * d * e + listed_bytes + rows * (2 * d * e + 4) + B * T * (2 * H * d * e + 8), "flops": 4.0 * (seen + B * H * T) * (H_q // H) * T * d}


# ------------------------------------------------------------------------------------------
# the same in 64 bits, from the definitions
# ------------------------------------------------------------------------------------------
def _exact_pages(s):
    """Sequence by sequence, with lists."""
    case = s["case"]
    now, new, table = s["now"].tolist(), s["new"].tolist(), s["table"].tolist()
    stack, size = s["free"].tolist()[:int(s["free_count"])], s["free"].numel()
    held = s["free"].tolist()
    for b, (a, z) in enumerate(zip(now, new)):
        stack += table[b][-(-z // PAGE):-(-a // PAGE)] if z < a else []
    held[:len(stack)] = stack
    lens, flags, starts, room, asked = [], [], [0], case["B"] * case["T"], 0
    slots, places, owners = [], [], []
    available, tokens = len(stack), 0
    for b, (a, z) in enumerate(zip(now, new)):
        wanted = max(0, -(-z // PAGE) - -(-a // PAGE))
        asked += wanted
        fits = wanted == 0 or asked <= available
        if z > a and fits:
            tokens += z - a
            fits = tokens <= room
        if z > a and fits:
            for page in range(-(-a // PAGE), -(-z // PAGE)):
                table[b][page] = stack.pop()
            for place in range(a, z):
                slots.append(table[b][place // PAGE] * PAGE + place % PAGE)
                places.append(place)
                owners.append(b)
        lens.append(z if fits else a)
        flags.append(0 if fits else 4)
        starts.append(len(slots))
    fill = [-1] * (room - len(slots))
    out = {"table": table, "free": held[:size], "lens": lens, "free_left": [len(stack)], "token_starts": starts, "slots": slots + fill,
           "places": places + fill, "owners": owners + fill, "flags": flags}
    return {k: torch.tensor(x, dtype=torch.int32, device="cuda") for k, x in out.items()}


def _exact_store(s):
    case = s["case"]
    out = {}
    for name in ("k", "v"):
        pool, rows = s[name + "_pool"].double(), s[name].double()
        flat = pool.transpose(1, 2).reshape(-1, case["H_kv"], case["d"])
        if case["nodes"]:
            rows = rows.transpose(1, 2).reshape(-1, case["H_kv"], case["d"])[s["rows"].long()]
        flat[s["slots"].long()] = rows
        out[name] = flat.view(pool.shape[0], PAGE, case["H_kv"], case["d"]).transpose(1, 2).contiguous()
    return out


def _exact_prompt(s):
    case = s["case"]
    H_q, H, d = case["H_q"], case["H_kv"], case["d"]
    out, lse = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda"), torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    ends = np.cumsum(s["sizes"])
    for b, (end, seen) in enumerate(zip(ends.tolist(), s["seen"])):
        begin = end - s["sizes"][b]
        ahead = seen - s["sizes"][b]
        for h in range(H_q):
            if s["table"] is None:
                key, val = s["k"][begin:end, h // (H_q // H)].double(), s["v"][begin:end, h // (H_q // H)].double()
            else:
                at = torch.arange(seen, device="cuda")
                page = s["table"][b].long()[at // PAGE]
                key, val = s["k"][page, h // (H_q // H), at % PAGE].double(), s["v"][page, h // (H_q // H), at % PAGE].double()
            turned = key.t().contiguous()
            for i in range(begin, end, 4096):
                j = min(end, i + 4096)
                most = ahead + j - begin
                x = torch.mm(s["q"][i:j, h].double(), turned[:, :most]) * d ** -0.5
                x += torch.triu(torch.full((j - i, most), -math.inf, dtype=torch.float64, device="cuda"), diagonal=ahead + i - begin + 1)
                z = torch.logsumexp(x, 1)
                lse[i:j, h] = z
                out[i:j, h] = torch.mm((x - z[:, None]).exp(), val[:most])
    return {"out": out, "lse": lse}


def _exact_tree(s):
    case = s["case"]
    B, H_q, H, T, d = (case[k] for k in ("B", "H_q", "H_kv", "T", "d"))
    out, lse = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda"), torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    words = s["masks"].cpu().numpy().view(np.uint64)
    bits = torch.from_numpy(np.unpackbits(words.view(np.uint8).reshape(B, T, 8), axis=2, bitorder="little")[:, :, :T].astype(bool)).cuda()
    for b in range(B):
        for r in range(H):
            use = torch.arange(int(s["lens"][b]), device="cuda")
            if case["kept"]:
                units = s["lists"][b * H + r, :int(s["counts"][b * H + r])].long()
                spread = (units[:, None] * case["chunk"] + torch.arange(case["chunk"], device="cuda")).flatten()
                use = spread[spread < use.numel()]
            if s["table"] is None:
                key, val = s["k"][b, r][use], s["v"][b, r][use]
            else:
                page = s["table"][b].long()[use // PAGE]
                key, val = s["k"][page, r, use % PAGE], s["v"][page, r, use % PAGE]
            key, val = torch.cat((key, s["k_new"][b, r])).double(), torch.cat((val, s["v_new"][b, r])).double()
            turned = key.t().contiguous()
            for g in range(H_q // H):
                x = torch.mm(s["q"][b, r * (H_q // H) + g].double(), turned) * d ** -0.5
                x[:, use.numel():] += torch.where(bits[b], 0.0, -math.inf)
                z = torch.logsumexp(x, 1)
                lse[b, r * (H_q // H) + g] = z
                out[b, r * (H_q // H) + g] = torch.mm((x - z[:, None]).exp(), val)
    return {"out": out, "lse": lse}


def exact(case, seed):
    state = prepare(case, seed)
    return {"pages": _exact_pages, "store": _exact_store, "prompt": _exact_prompt, "tree": _exact_tree}[case["kind"]](state)
