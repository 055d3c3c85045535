"""Plain numpy forms, in 64 bits, of the operators around the 4-bit cache and of the eviction: what their tests compare
against.  Written from the definitions; shares nothing with the library."""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantise(x):
    """Codes [..., d] (one per element, 0..15) and scale bytes [..., d/32] of rows x [..., d]."""
    x = np.asarray(x, dtype=np.float64)
    blocks = x.reshape(*x.shape[:-1], -1, 32)
    top = np.abs(blocks).max(-1)
    bad = ~np.isfinite(blocks).all(-1)
    safe = np.where(bad | (top == 0), 1.0, top)
    e = np.clip(np.frexp(safe)[1] - 1 - 2, -127, 125)
    e = np.where(top == 0, -127, e)
    y = np.where(bad[..., None], 0.0, blocks) * 2.0 ** (-e[..., None].astype(np.float64))
    a = np.abs(y)
    low = np.clip(np.searchsorted(GRID, a, side="right") - 1, 0, 6)
    below, above = GRID[low], GRID[low + 1]
    up = (a - below > above - a) | ((a - below == above - a) & (low % 2 == 1))
    code = low + up + 8 * np.signbit(y)
    code = np.where(bad[..., None], 0, code)
    return code.reshape(x.shape).astype(np.uint8), np.where(bad, 255, e + 127).astype(np.uint8)


def pack(codes):
    return codes[..., 0::2] | (codes[..., 1::2] << 4)


def unpack(words):
    return np.stack((words & 15, words >> 4), -1).reshape(*words.shape[:-1], -1)


def values(codes, scales):
    """Values in 64 bits of codes [..., d] and scale bytes [..., d/32]."""
    v = np.where(codes & 8, -1.0, 1.0) * GRID[codes & 7]
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return v * np.repeat(s, 32, -1)


def cache_values(codes, scales):
    """Keys and values of a cache [..., d] / [..., d/16] as the library lays it out."""
    d = codes.shape[-1]
    c = unpack(codes)
    return values(c[..., :d], scales[..., :d // 32]), values(c[..., d:], scales[..., d // 32:])


def attention(q, k, v, kept, scale, k_new=None, v_new=None):
    """out [B,H_q,T,d], lse [B,H_q,T] and a bound on the fp32 error of out: q [B,H_q,T,d], k, v [B,H_kv,n,d] and a list kept[b][h]
    of positions (in any order, repeats count)."""
    B, H_q, T, d = q.shape
    H = k.shape[1]
    G = H_q // H
    out, lse, tol = np.zeros(q.shape), np.full(q.shape[:3], -np.inf), np.zeros(q.shape[:3])
    for b in range(B):
        for hq in range(H_q):
            h = hq // G
            at = np.asarray(kept[b][h], dtype=np.int64)
            for t in range(T):
                kk, vv = k[b, h, at], v[b, h, at]
                if k_new is not None:
                    kk, vv = np.concatenate((kk, k_new[b, h, :t + 1])), np.concatenate((vv, v_new[b, h, :t + 1]))
                if len(kk) == 0:
                    continue
                s = (kk @ q[b, hq, t]) * scale
                m = s.max()
                w = np.exp(s - m)
                out[b, hq, t] = (w @ vv) / w.sum()
                lse[b, hq, t] = m + np.log(w.sum())
                # Per score: d products summed, each addition off by at most 2^-23 of the sum of magnitudes; two more roundings and
                # the reference's subtraction, relative to the score in units of log2; the exponential and its parts 2^-22.
                mags = (np.abs(kk) @ np.abs(q[b, hq, t])) * scale
                score = (d + 4) * 2.0 ** -23 * mags.max() + 4 * 2.0 ** -23 * 1.5 * np.abs(s).max() + 2.0 ** -22
                # Weights off by that factor each way (numerator and sum), then as many additions as positions in either sum.
                tol[b, hq, t] = (2 * score + 2 * (len(kk) + 64) * 2.0 ** -23) * np.abs(vv).max()
    return out, lse, tol


def evict(scores, positions, lens, nxt, budget, sinks, recent, decay, probs=None):
    """New scores and positions, the moves [(src, dst), ...] per row, new lengths, NaN flags."""
    B, H, n = scores.shape
    scores, positions = scores.copy(), positions.copy()
    moves, flags = [], np.zeros(B * H, dtype=np.int64)
    for b in range(B):
        for h in range(H):
            size = int(lens[b])
            K = min(size, budget)
            acc = decay * scores[b, h, :size].astype(np.float64)
            if probs is not None:
                share = probs.shape[1] // H
                for x in range(h * share, (h + 1) * share):
                    for s in range(probs.shape[2]):
                        acc = acc + probs[b, x, s, :size].astype(np.float64)
            new = acc.astype(np.float32)
            flags[b * H + h] = np.isnan(new).any()
            at = positions[b, h, :size].astype(np.int64)
            stays = (at < sinks) | (at >= int(nxt[b]) - recent)
            order = sorted(range(size), key=lambda j: (not stays[j], bool(np.isnan(new[j])), 0.0 if np.isnan(new[j]) or stays[j] else -float(new[j]), j))
            kept = np.zeros(size, dtype=bool)
            kept[order[:K]] = True
            dst = [j for j in range(K) if not kept[j]]
            src = [j for j in range(K, size) if kept[j]]
            assert len(src) == len(dst)
            moves.append(list(zip(src, dst)))
            at = at.copy()
            for a, d in moves[-1]:
                new[d], at[d] = new[a], at[a]
            new[K:], at[K:] = 0.0, -1
            scores[b, h, :size], positions[b, h, :size] = new, at
    return scores, positions, moves, np.minimum(lens, budget), flags
