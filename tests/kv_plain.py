"""The key / value cache and its attention from their definitions, numpy fp64:
codes channel by channel, blocks packed bit by bit, softmax row by row."""
import numpy as np
import torch

TOP = {torch.float16: 65504.0, torch.bfloat16: float(torch.finfo(torch.bfloat16).max)}


def groups(lay):
    out, at = [], 0
    for g in range(lay.n_groups):
        out.append((at, lay.count[g], lay.bits[g]))
        at += lay.count[g]
    return out


def codes(lay, head, x, dtype):
    """One row x[D] (fp64) -> per group (scale, codes in packed order)."""
    res = []
    for at, count, n in groups(lay):
        ch = lay.perm_host[head][at:at + count]
        r = x[ch].copy()
        nan = np.isnan(r)
        r[nan] = 0.0
        r = np.clip(r, -TOP[dtype], TOP[dtype])
        s = np.abs(r).max()
        half = 2.0 ** (n - 1)
        j = np.zeros(count) if s == 0 else np.clip(np.rint(r * half / s), -half, half - 1)   # rint: half to even
        res.append((s, j.astype(np.int64)))
    return res


def pack(j, n):
    """Codes (two's complement) -> bytes of whole 32-code blocks."""
    nb = -(-len(j) // 32)
    u = np.zeros(32 * nb, dtype=np.int64)
    u[:len(j)] = np.asarray(j) & ((1 << n) - 1)
    out = np.zeros(4 * n * nb, dtype=np.uint8)
    per = 8 // n
    for i, c in enumerate(u):
        blk, p = divmod(i, 32)
        t, b = divmod(p, 4)
        out[4 * n * blk + 4 * (t // per) + b] |= np.uint8((int(c) << (n * (t % per))) & 0xFF)
    return out


def row_bytes(lay, head, x, dtype):
    parts = [pack(j, n) for (s, j), (_, _, n) in zip(codes(lay, head, x, dtype), groups(lay))]
    out = np.concatenate(parts)
    return np.concatenate([out, np.zeros(-len(out) % 16, dtype=np.uint8)]), [s for s, _ in codes(lay, head, x, dtype)]


def values(lay, x, dtype):
    """What the cache holds of rows x[..][heads][D] (fp64), fp64."""
    out = np.zeros_like(x)
    flat, o = x.reshape(-1, *x.shape[-2:]), out.reshape(-1, *x.shape[-2:])
    for g, (at, count, n) in enumerate(groups(lay)):
        for h in range(x.shape[-2]):
            ch = lay.perm_host[h][at:at + count]
            r = np.clip(np.where(np.isnan(flat[:, h, ch]), 0.0, flat[:, h, ch]), -TOP[dtype], TOP[dtype])
            s = np.abs(r).max(axis=-1, keepdims=True)
            half = 2.0 ** (n - 1)
            j = np.clip(np.rint(r * half / np.where(s > 0, s, 1.0)), -half, half - 1)
            o[:, h, ch] = np.where(s > 0, j * s / half, 0.0)
    return out


def attend(q, k, v, lens, mask, group, scale):
    """q [B][T][Hq][D]; k, v: per sequence [len + T][heads][D] (fp64).  Returns the
    outputs and, per output, the sum of p |v| and the bounds' other terms."""
    B, T, Hq, _ = q.shape
    o = np.zeros((B, T, Hq, v[0].shape[-1] if v else 0))
    mag, dscore, total = np.zeros_like(o), np.zeros((B, T, Hq, 1)), np.ones((B, T, Hq, 1))
    for b in range(B):
        n = int(lens[b])
        if n < 0:
            continue
        for t in range(T):
            see = np.ones(n + T, dtype=bool)
            see[n:] = (np.arange(T) <= t) if mask is None else mask[b, t]
            if not see.any():
                continue
            for h in range(Hq):
                kh, vh = k[b][see, h // group], v[b][see, h // group]
                s = kh @ q[b, t, h] * scale
                p = np.exp(s - s.max())
                total[b, t, h] = p.sum()
                p /= p.sum()
                o[b, t, h] = p @ vh
                mag[b, t, h] = p @ np.abs(vh)
                dscore[b, t, h] = abs(scale) * np.abs(q[b, t, h]).sum() * np.abs(kh).max()
    return o, mag, dscore, total


def tolerance(ref, mag, dscore, total, n_seen, v_max, dtype):
    """|error| allowed of an output.

    Weights are rounded to fp16 (2^-11 each, and 2^-25 of the largest weight
    times the largest value scale, doubled by its rounding up to a power of
    two, where they are subnormal); scores carry at most 2^-21 of the summed
    magnitudes (codes are held with an offset that doubles them, fp32 sums of at
    most 256 products); exp2 and the sums 2^-19; the output is rounded once."""
    half_ulp = 2.0 ** -11 if dtype == torch.float16 else 2.0 ** -8
    sub = 2.0 ** -24 * v_max * n_seen / total
    return mag * (2.0 ** -11 + 2.0 ** -20 * dscore + 2.0 ** -19) + sub + half_ulp * np.abs(ref) + 2.0 ** -24
