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
