"""A step over packed prompts from its definitions: the plan with lists, one
sequence after the other; norms, rotations and attention in numpy fp64."""
import math
from fractions import Fraction

import numpy as np
import torch

TWO_PI = Fraction("6.2831853071795864769252867665590057683943387987502")
HALF_STEP = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
LEAST = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -126}      # half a step of subnormals; bf16: fp32's


def plan(page, table, free, n_free, lengths, targets, cap):
    """Lists in, lists out: starts, positions, slots, lengths, table, free, count."""
    table, free, W = [list(r) for r in table], list(free), len(table[0]) if len(table) else 0
    pages = lambda n: -(-max(n, 0) // page)
    back = [p for b, (n, t) in enumerate(zip(lengths, targets)) for p in table[b][pages(t):min(pages(n), W)]]
    pool, starts, positions, slots, after, waiting = free[:n_free] + back[::-1], [0], [], [], [], False
    for b, (n, t) in enumerate(zip(lengths, targets)):
        old, goal = max(n, 0), max(t, 0)
        has, to = min(pages(n), W), pages(t)
        end = starts[-1] + max(goal - old, 0)
        served = True
        if goal > old:
            served = to <= W and end <= cap
            if served and to > has:
                waiting = waiting or to - has > len(pool)
                served = not waiting
                if served:
                    for i in range(has, to):
                        table[b][i] = pool.pop()
        after.append(max(t, -1) if served else n)
        live = range(starts[-1], min(end, cap)) if starts[-1] < cap else range(0)
        for i, _ in enumerate(live):
            p = old + i
            positions.append(p)
            slots.append(table[b][p // page] * page + p % page if served else -1)
        starts.append(end)
    free[:len(pool)] = pool
    positions += [0] * (cap - len(positions))
    slots += [-1] * (cap - len(slots))
    return [min(s, cap) for s in starts], positions, slots, after, table, free, len(pool)


def angles(frequencies, positions):
    """Angles [n][pairs] modulo a turn: exact products, reduced exactly."""
    return np.array([[float(Fraction(f) * int(t) % TWO_PI) for f in frequencies] for t in positions]).reshape(len(positions), -1)


def rotate(x, frequencies, positions, interleaved=False, gain=None, eps=0.0, magnitude=1.0):
    """x [n][heads][D] fp64; returns the turned rows and, per channel, the summed
    magnitudes of what makes it."""
    x = np.asarray(x, dtype=np.float64)
    if gain is not None:
        x = x / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps) * np.asarray(gain, dtype=np.float64)
    out, mag = x.copy(), np.abs(x)
    half = len(frequencies)
    if half:
        ang = angles(frequencies, positions)[:, None]
        c, s = np.cos(ang) * magnitude, np.sin(ang) * magnitude
        i, j = (np.arange(0, 2 * half, 2), np.arange(1, 2 * half, 2)) if interleaved else (np.arange(half), np.arange(half, 2 * half))
        a, b = x[..., i], x[..., j]
        out[..., i], out[..., j] = a * c - b * s, b * c + a * s
        mag[..., i] = mag[..., j] = (np.abs(a) + np.abs(b)) * abs(magnitude)
    return out, mag


def rotate_tolerance(ref, mag, dtype):
    """One rounding of the output; in fp32 before it: the sum of at most 256 squares
    (13 roundings on a lane's way, halved by the root), the root (2^-22), four
    products, and cosines and sines off by 2^-22 (an angle held in 24 bits of half a
    turn, 2^-23.3 radians, and the functions' own 2^-24): below 2^-20 of the summed
    magnitudes."""
    return HALF_STEP[dtype] * np.abs(ref) + (1 + HALF_STEP[dtype]) * 2.0 ** -20 * mag + LEAST[dtype]


def attend(q, k, v, starts, causal, scale):
    """q [n][Hq][D], k, v [n][Hk][..] torch fp64.  Returns outputs and, for the
    tolerance, sum of p |v|, the largest summed magnitudes of a score, and of a row the
    softmax sum and the largest |v| that it sees."""
    n, Hq, _ = q.shape
    G = Hq // k.shape[1]
    o = torch.zeros(n, Hq, v.shape[2], dtype=torch.float64, device=q.device)
    mag, dscore = torch.zeros_like(o), torch.zeros(n, Hq, 1, dtype=torch.float64, device=q.device)
    total, v_max = torch.ones_like(dscore), torch.zeros_like(dscore)
    for s, e in zip(starts[:-1], starts[1:]):
        if e <= s:
            continue
        hide = torch.ones(e - s, e - s, dtype=torch.bool, device=q.device).triu(1) if causal else None
        for h in range(k.shape[1]):
            hq = slice(h * G, (h + 1) * G)
            x, y, z = q[s:e, hq].transpose(0, 1), k[s:e, h], v[s:e, h]
            sc, big = x @ y.T * scale, x.abs() @ y.abs().T * scale
            if causal:
                sc, big = sc.masked_fill(hide, -math.inf), big.masked_fill(hide, 0)
            p = torch.exp(sc - sc.amax(-1, keepdim=True))
            l = p.sum(-1, keepdim=True)
            o[s:e, hq] = (p / l @ z).transpose(0, 1)
            mag[s:e, hq] = (p / l @ z.abs()).transpose(0, 1)
            dscore[s:e, hq] = big.amax(-1, keepdim=True).transpose(0, 1)
            total[s:e, hq] = l.transpose(0, 1)
            top = z.abs().amax(-1, keepdim=True)
            v_max[s:e, hq] = (torch.cummax(top, 0).values if causal else top.amax().expand(e - s, 1))[:, None]
    return o, mag, dscore, total, v_max


def attend_tolerance(ref, mag, dscore, total, v_max, n, dtype):
    """|error| allowed: weights are rounded to the type (half a step each; fp16: or 2^-33 of
    the row's largest weight where they are subnormal, n of them at most); scores carry
    2^-21 of the summed magnitudes of their products (sums of at most 256 in fp32), which
    the exponential doubles over row and sum; exponentials and sums 2^-19; one rounding."""
    half = HALF_STEP[dtype]
    sub = 2.0 ** -33 * n * v_max / total if dtype == torch.float16 else 0.0
    return (1 + half) * (mag * (half + 2.0 ** -20 * dscore + 2.0 ** -19) + sub) + half * ref.abs() + LEAST[dtype]
