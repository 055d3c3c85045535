"""Plain forms in 64 bits of the operators of the serving loop, and how far a kernel may be from them.

Rounding to a type is off by at most u = eps / 2 of the value (bf16 2^-8, fp16 2^-11, fp32 2^-24).  For an output element with normalised weights w
and values v let A = sum w |v|.
  scores   d exact products added up in fp32 and scaled: off by at most (d + 4) 2^-24 S, S = scale * the largest sum |q| |k| that the row sees
  weights  2^x and its argument: 2^-21 more; each rounded to the element type (u) or held in two parts (u^2); with fp16 also 2^-37 of
           the largest weight, n times
  sums     n terms in fp32, in the output and in the total that divides it
  output   rounded to its type
so |out - exact| <= A * (2 e + p + 2 (n + 8) 2^-24) + n 2^-37 max |v| + u |out|, e = (d + 4) 2^-24 S + 2^-21, and |lse - exact| <= e + (n + 8) 2^-24 + 2^-22 |lse|.
"""
import numpy as np
import torch

DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
HALF_STEP = {k: torch.finfo(t).eps / 2 for k, t in DT.items()}


def attend(q, k, v, seen, scale, dtype):
    """q [m,d], k, v [n,d], seen [m,n] bool, all float64 numpy -> out, lse, and the tolerances (fp32 out, out in dtype, lse).  Rows of k and v that a
    query does not see have no part in it, whatever they hold."""
    m, n = seen.shape
    out, lse = np.zeros((m, v.shape[1])), np.full(m, -np.inf)
    tol32, tol_low, tol_lse = np.zeros_like(out), np.zeros_like(out), np.zeros(m)
    u = HALF_STEP[dtype]
    for i in range(m):
        at = seen[i].nonzero()[0]
        if at.size == 0:
            continue
        x = k[at] @ q[i] * scale
        top = x.max()
        w = np.exp(x - top)
        total = w.sum()
        w /= total
        lse[i] = top + np.log(total)
        out[i] = w @ v[at]
        a = w @ np.abs(v[at])
        e = (q.shape[1] + 4) * 2.0 ** -24 * scale * (np.abs(k[at]) @ np.abs(q[i])).max() + 2.0 ** -21
        sums = 2 * (at.size + 8) * 2.0 ** -24
        lost = at.size * 2.0 ** -37 * np.abs(v[at]).max()
        tol32[i] = a * (2 * e + u * u + sums) + lost + 2.0 ** -24 * np.abs(out[i])
        tol_low[i] = (a * (2 * e + u + sums) + lost) * (1 + u) + u * np.abs(out[i]) + torch.finfo(DT[dtype]).smallest_normal * u
        tol_lse[i] = e + sums + 2.0 ** -22 * abs(lse[i])
    return out, lse, tol32, tol_low, tol_lse


def pages(table, free, count, now, new, page_size, capacity):
    """specattn_pages_update with lists; returns what it leaves (numpy) and how many new tokens there are."""
    table, free = table.copy(), free.copy()
    B, width = table.shape
    reach = width * page_size
    up = lambda x: -(-x // page_size)  # noqa: E731
    flags = [1 if a < 0 or a > reach or z < 0 else 4 if z > reach else 0 for a, z in zip(now, new)]
    stack = list(free[:count])
    for b in range(B):
        if not flags[b] and new[b] < now[b]:
            stack += list(table[b, up(new[b]):up(now[b])])
    free[:len(stack)] = stack
    available, asked, came, done = len(stack), 0, 0, 0
    lens, starts, slots, places, owners = [], [0], [], [], []
    for b in range(B):
        a, z = int(now[b]), int(new[b])
        if not flags[b] and z > a:
            want = up(z) - up(a)
            asked += want
            if want and asked > available:
                flags[b] |= 4
            else:
                came += z - a
                if capacity is not None and came > capacity:
                    flags[b] |= 4
        if not flags[b] and z > a:
            for p in range(up(a), up(z)):
                table[b, p] = stack.pop()
            for at in range(a, z):
                slots.append(table[b, at // page_size] * page_size + at % page_size)
                places.append(at)
                owners.append(b)
            done += z - a
        lens.append(a if flags[b] else z)
        starts.append(done)
    pad = lambda x: np.array(x + [-1] * ((capacity or len(x)) - len(x)), dtype=np.int32)  # noqa: E731
    return dict(table=table, free=free, count=len(stack), lens=np.array(lens, dtype=np.int32), starts=np.array(starts, dtype=np.int32),
                slots=pad(slots), positions=pad(places), owners=pad(owners), flags=np.array(flags, dtype=np.int32), tokens=done)
