"""CPU oracle of the 8-bit key/value cache, in float64 numpy: written from the definitions in include/nsattn.h.

A cache's keys or values are `codes` [B,H,N,D] (the numbers that the 8-bit codes stand for) and `scale` [B,H,N/block].
"""
import math

import numpy as np

LIMIT = {"i8": 127.0, "e4m3": 448.0}


def nearest(y, code):
    """The numbers that the nearest codes (ties to even) of y stand for."""
    if code == "i8":
        return np.rint(y)
    with np.errstate(divide="ignore"):
        e = np.floor(np.log2(np.abs(y)))
    step = np.exp2(np.maximum(e, -6.0) - 3.0)
    return np.rint(y / step) * step


def scale_for(most, code):
    if not math.isfinite(most):
        return math.nan
    s = 2.0 ** -100
    if most > LIMIT[code] * s:
        s = 2.0 ** (math.floor(math.log2(most / LIMIT[code])) - 1)
        while most > LIMIT[code] * s:
            s *= 2.0
    return s


def values(codes, scale):
    B, H, N, D = codes.shape
    return (codes.reshape(B, H, scale.shape[2], -1, D) * scale[..., None, None]).reshape(B, H, N, D)


def append(codes, scale, x, start, counts, code):
    """x [B,H,T,D] enters codes and scale in place."""
    B, H, N, D = codes.shape
    block = N // scale.shape[2]
    for b in range(B):
        at = min(max(int(start[b]), 0), N)
        end = min(at + min(max(int(counts[b]), 0), x.shape[2]), N)
        for j in range(at // block, -(-end // block)):
            lo, hi = max(at, j * block), min(end, (j + 1) * block)
            if lo >= hi:
                continue
            for h in range(H):
                new = x[b, h, lo - at:hi - at]
                s = scale_for(np.abs(new).max() if np.isfinite(new).all() else math.inf, code)
                if at > j * block:
                    old = scale[b, h, j]
                    if math.isnan(old) or (not math.isnan(s) and np.abs(new).max() <= LIMIT[code] * old):
                        s = old
                    if s > old:
                        codes[b, h, j * block:at] = nearest(codes[b, h, j * block:at] * (old / s), code)
                codes[b, h, lo:hi] = 0.0 if math.isnan(s) else nearest(new / s, code)
                scale[b, h, j] = s


def attend(q, k, v, lengths, counts, scale, causal):
    """out [B,Hq,T,D], lse [B,Hq,T], weights [B,H,N] (this call's), and three sizes that bound rounding errors:
    the sum of |p v| like out, the largest scale * sum |q k| of each row like lse, and the sum of |v| over a row's keys like out."""
    B, Hq, T, D = q.shape
    H, N = k.shape[1], k.shape[2]
    G = Hq // H
    out, spread, volume = (np.zeros((B, Hq, T, D)) for _ in range(3))
    lse, reach = np.full((B, Hq, T), -np.inf), np.zeros((B, Hq, T))
    weights = np.zeros((B, H, N))
    for b in range(B):
        n, c = min(max(int(lengths[b]), 0), N), min(max(int(counts[b]), 0), T)
        if n == 0 or c == 0:
            continue
        seen = np.arange(n)[None] <= n - c + np.arange(c)[:, None] if causal else np.ones((c, n), bool)
        some = seen.any(1)
        for hq in range(Hq):
            h = hq // G
            z = np.where(seen, scale * (q[b, hq, :c] @ k[b, h, :n].T), -np.inf)
            most = np.where(some, z.max(1), 0.0)
            p = np.exp(z - most[:, None])
            total = np.where(some, p.sum(1), 1.0)
            p /= total[:, None]
            out[b, hq, :c] = p @ v[b, h, :n]
            spread[b, hq, :c] = p @ np.abs(v[b, h, :n])
            volume[b, hq, :c] = seen @ np.abs(v[b, h, :n])
            reach[b, hq, :c] = (np.abs(scale) * (np.abs(q[b, hq, :c]) @ np.abs(k[b, h, :n]).T) * seen).max(1)
            lse[b, hq, :c] = np.where(some, most + np.log(total), -np.inf)
            weights[b, h, :n] += p.sum(0)
    return out, lse, weights, spread, reach, volume


def select(weights, length, keep, n_global, n_recent):
    """Positions that stay, ascending, of one sequence and head."""
    n = min(max(int(length), 0), len(weights))
    if n <= keep:
        return np.arange(n)
    ranked = range(n_global, n - n_recent)
    order = sorted(ranked, key=lambda i: (0 if math.isnan(weights[i]) else 1, 0.0 if math.isnan(weights[i]) else -weights[i], i))
    chosen = order[:keep - n_global - n_recent]
    return np.array(sorted([*range(n_global), *chosen, *range(n - n_recent, n)]), dtype=np.int64)


def move(codes, scale, kept, block, code):
    """Codes [len(kept) rounded up to blocks, D] and scales of the kept tokens of one sequence and head; codes [N,D], scale [N/block]."""
    blocks = -(-len(kept) // block)
    to, to_scale = np.zeros((blocks * block, codes.shape[1])), np.zeros(blocks)
    for j in range(blocks):
        at = kept[j * block:(j + 1) * block]
        x = codes[at] * scale[at // block][:, None]
        s = to_scale[j] = scale_for(np.abs(x).max() if np.isfinite(x).all() else math.inf, code)
        if not math.isnan(s):
            to[j * block:j * block + len(at)] = nearest(x / s, code)
    return to, to_scale
