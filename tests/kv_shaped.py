"""A cached sequence whose scores and value scales are chosen token by token."""
import numpy as np
import torch

import kv_plain as plain
import test_gpu_kv_attend as base


def problem(sq, seed, shape, context, T, group, dtype, score, size, page=16):
    """One sequence of `context` tokens and a chain of T.  The queries of a key
    head are one vector u and token t's key is score[t] u / |u|^2, so its score at
    scale 1 is about score[t].  size[g][t]: log2 of the values' magnitude in group
    g, -inf: exact zeros."""
    p = base.Problem(sq, seed, shape, [context], T, group, page, dtype)
    rng, c, n = p.rng, p.cache, context + T
    heads, D, Dv = shape[:3]
    u = rng.choice([-1.0, 1.0], (heads, D))
    p.q = torch.from_numpy(np.broadcast_to(np.repeat(u, group, 0), (1, T, heads * group, D)).copy()).to(dtype)
    k = torch.from_numpy(np.asarray(score)[:n, None, None] * u[None] / D).to(dtype)
    v = rng.choice([-1.0, 1.0], (n, heads, Dv)) * rng.uniform(0.5, 1.0, (n, heads, Dv))
    for (at, count, _), log2 in zip(plain.groups(c.v), size):
        for h in range(heads):
            ch = c.v.perm_host[h][at:at + count]
            v[:, h, ch] *= np.exp2(np.asarray(log2)[:n, None])
    v = torch.from_numpy(v).to(dtype)
    assert torch.isfinite(v).all()
    pos = np.arange(n)
    table = p.table[0].cpu().numpy()
    slots = torch.from_numpy(table[pos // page].astype(np.int64) * page + pos % page).cuda()
    sq.kv_write(c, k.cuda(), v.cuda(), slots)
    p.k, p.v = [plain.values(c.k, k.double().numpy(), dtype)], [plain.values(c.v, v.double().numpy(), dtype)]
    p.slots = slots
    return p


def check_rows(p, out, mask, scale):
    """Outputs against their definition in fp64, with a bound that knows only what
    the row sees.

    As kv_plain.tolerance, but for the weights that are subnormal in fp16: a row's
    weights times value scales are held relative to a power of two at most twice
    the largest of them (per value group), and rounded by 2^-25 of it, so by 2^-24
    of the largest product, per token.  Weights below 2^-126 of the largest count
    as 0, which loses that much of a value scale."""
    c, dtype = p.cache, p.cache.dtype
    got = out.double().cpu().numpy()
    assert np.isfinite(got).all()
    q = p.q.double().numpy()
    o, mag, dscore, total = plain.attend(q, p.k, p.v, p.lens, mask, p.group, scale)
    sub = np.zeros_like(o)
    scales, table = c.v_scales.double().cpu().numpy(), p.table.cpu().numpy()
    for b in range(p.B):
        n = int(p.lens[b])
        if n < 0:
            continue
        pos = np.arange(n + p.T)
        s = scales[table[b, pos // c.page_size], :, pos % c.page_size]       # [token][head][group]
        for t in range(p.T):
            see = np.ones(n + p.T, dtype=bool)
            see[n:] = (np.arange(p.T) <= t) if mask is None else mask[b, t]
            if not see.any():
                continue
            for h in range(q.shape[2]):
                kv = h // p.group
                x = p.k[b][see, kv] @ q[b, t, h] * scale
                w = np.exp(x - x.max())
                for g, (at, count, _) in enumerate(plain.groups(c.v)):
                    ch = c.v.perm_host[kv][at:at + count]
                    most, big = (w * s[see, kv, g]).max(), s[see, kv, g].max()
                    sub[b, t, h, ch] = (2.0 ** -24 * most + 2.0 ** -126 * big) * see.sum() / w.sum()
    half_ulp, floor = (2.0 ** -11, 2.0 ** -25) if dtype == torch.float16 else (2.0 ** -8, 2.0 ** -134)
    tol = mag * (2.0 ** -11 + 2.0 ** -20 * dscore + 2.0 ** -19) + sub + half_ulp * np.abs(o) + floor
    err = np.abs(got - o)
    assert (err <= tol).all(), (float((err / tol).max()), np.unravel_index((err / tol).argmax(), err.shape))
