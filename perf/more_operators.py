"""A step over packed prompts and new tokens, in front of a paged key / value cache, as cases that can be timed.

A server holds sequences whose tokens stand in the pages of a cache.  Before a layer runs, it works out
where the step's tokens go; in each layer, queries and keys are normalised and turned by their
positions, and whole prompts attend to themselves before their keys and values are put away.  A case's
"kind" says which call one pass makes:

  plan    kv_plan: from each sequence's length and the length it is to have, the pages it takes or
          gives back, and the slots and positions of the step's tokens
  rotate  rotate_heads: the norm of every query and key head and the rotation by the token's position
  attend  prompt_attend: attention of packed prompts over their own keys and values, grouped heads

`own` selects the library's kernels; otherwise the same is computed with elementary torch operations
in 32 bits (angles in 64).
"""
import math
import random

import torch

own = False

DT = {"f16": torch.float16, "bf16": torch.bfloat16}


# ---- cases --------------------------------------------------------------------

def _case(kind, name=None, **kw):
    base = {
        # B sequences; the first `grow` of each hundred append tokens, the next `cut` give some back, the
        # next `leave` go; new: most tokens that one appends; ctx: most tokens it has; pad: tokens that the
        # step's buffers hold beyond the planned ones; scarce: the pool has too few pages for all
        "plan": dict(B=8, grow=100, cut=0, leave=0, new=1, ctx=1000, page=64, pad=0, scarce=False),
        # rot: channels that are turned (from the first on); base: of the frequencies; far: largest
        # position; factor, low, high, length: frequencies scaled for long contexts (length 0: all by
        # factor, else by their wavelengths); fused: q and k are slices of one projection's output
        "rotate": dict(dtype="f16", heads=8, G=4, D=128, rot=128, interleaved=False, norm=True, base=10000.0, factor=1.0,
                       low=1.0, high=4.0, length=0, far=4096, fused=False),
        # B prompts of up to `len` tokens; spread: how far below it they go
        "attend": dict(dtype="f16", heads=8, G=4, D=128, Dv=128, B=1, spread=0.0, causal=True, pad=0),
    }[kind]
    c = dict(kind=kind, **base)
    c.update(kw)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # a decoding step of a small batch: latency
        _case("plan", "plan_8_decoding"),
        # a step of a busy server: most of 1000 sequences append a token or a piece of a prompt, some give
        # back drafts that were not accepted, some leave; the buffers are padded to a fixed size
        _case("plan", "plan_1000_mixed", B=1000, grow=85, cut=10, leave=5, new=40, ctx=8000, page=16, pad=777),
        # prompts of a batch are admitted
        _case("plan", "plan_32_prompts", B=32, new=4000, ctx=0, page=64),
        # the new tokens of eight sequences, norm and rotation: latency
        _case("rotate", "rotate_8_tokens", n=8),
        # an odd piece of a prompt: 80 channels of which 32 are turned, neighbours in pairs, slices of a
        # fused projection, no norm
        _case("rotate", "rotate_1001x80_part", n=1001, heads=12, G=1, D=80, rot=32, interleaved=True, norm=False, fused=True),
        # a batch of prompts at far positions of a long context, frequencies scaled by their wavelengths
        _case("rotate", "rotate_16384_long_bf16", n=16384, dtype="bf16", fused=True, base=500000.0, factor=8.0, length=8192,
              far=1000000),
        # one short question: latency
        _case("attend", "attend_97", len=97),
        # prompts of an odd model without powers of two
        _case("attend", "attend_3x1501x80", B=3, len=1501, spread=0.5, heads=4, G=5, D=80, Dv=80),
        # many short ones, no shared heads, in a buffer of a fixed size
        _case("attend", "attend_200_short", B=200, len=200, spread=1.0, heads=12, G=1, D=64, Dv=64, pad=333),
        # wide heads, all of the prompt seen
        _case("attend", "attend_2x4001x256", B=2, len=4001, heads=4, G=2, D=256, Dv=256, causal=False, dtype="bf16"),
        # the prompts of a serving batch
        _case("attend", "attend_16_ragged_bf16", B=16, len=4096, spread=0.9, dtype="bf16"),
        # a long document
        _case("attend", "attend_16384_bf16", len=16384, dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    if case["kind"] == "plan":
        return sum(_news(case)) + 16 * case["B"]
    if case["kind"] == "rotate":
        return case["n"] * case["heads"] * (case["G"] + 1) * case["D"]
    # pairs of whole blocks, as the plain form computes them, and rows
    return sum(L * (L + 512) for L in _lengths(case)) * case["heads"] * case["G"] * (case["D"] + case["Dv"])


def draw(rng):
    while True:
        kind = rng.choice(["plan", "rotate", "attend", "attend"])
        dtype, heads, G = rng.choice(["f16", "bf16"]), rng.choice([1, 2, 4, 5, 8, 12]), rng.choice([1, 2, 3, 4, 5, 8])
        D = rng.choice([40, 64, 64, 80, 96, 128, 128, 128, 192, 256])
        if kind == "plan":
            leave = rng.choice([0, 0, 5, 20])
            cut = rng.choice([0, 10, 40])
            c = _case(kind, B=_log_int(rng, 1, 1024), grow=100 - cut - leave, cut=cut, leave=leave, new=_log_int(rng, 1, 8192),
                      ctx=rng.choice([0, _log_int(rng, 1, 16384)]), page=rng.choice([16, 32, 64, 128, 256]),
                      pad=rng.choice([0, _log_int(rng, 1, 2000)]), scarce=rng.random() < 0.25)
        elif kind == "rotate":
            rot = D if rng.random() < 0.6 else 2 * rng.randint(1, D // 2)
            length = rng.choice([0, 4096, 8192])
            c = _case(kind, n=_log_int(rng, 1, 32768), dtype=dtype, heads=heads, G=G, D=D, rot=rot,
                      interleaved=rng.random() < 0.4, norm=rng.random() < 0.7, base=rng.choice([10000.0, 500000.0, 1000000.0]),
                      factor=rng.choice([1.0, 2.0, 8.0, 32.0]), length=length, far=_log_int(rng, 100, 1000000),
                      fused=rng.random() < 0.5)
        else:
            c = _case(kind, dtype=dtype, heads=heads, G=G, D=D, Dv=D if rng.random() < 0.8 else rng.choice([64, 128]),
                      B=_log_int(rng, 1, 200), len=_log_int(rng, 1, 16384), spread=rng.choice([0.0, 0.5, 1.0]),
                      causal=rng.random() < 0.8, pad=rng.choice([0, 0, _log_int(rng, 1, 500)]))
        if _cost(c) <= max(_cost(x) for x in listed() if x["kind"] == kind):
            return c


def _lengths(case):
    """Tokens of each prompt, from the longest down by `spread`, in an order that mixes them; some may be empty."""
    B, n, s = case["B"], case["len"], case["spread"]
    return [int(n * (1.0 - s * (((7 * b) % B) / max(B - 1, 1)))) for b in range(B)]


def _steps(case):
    """(length, length to have) of each sequence of a plan."""
    out = []
    for b in range(case["B"]):
        r = random.Random(1000003 * b + 17)
        ctx = r.randint(0, case["ctx"]) if case["ctx"] else 0
        which = (37 * b) % 100
        if which < case["grow"]:
            new = r.randint(1, case["new"]) if case["new"] > 40 or b % 10 == 3 else 1
            out.append((-1 if ctx == 0 else ctx, ctx + new))
        elif which < case["grow"] + case["cut"]:
            out.append((ctx, ctx - r.randint(0, min(ctx, 20))))
        else:
            out.append((ctx, -1))
    return out


def _news(case):
    return [max(max(t, 0) - max(n, 0), 0) for n, t in _steps(case)]


def _ceil(a, b):
    return -(-a // b)


def work(case):
    if case["kind"] == "plan":
        page, news, steps = case["page"], _news(case), _steps(case)
        tokens = sum(news) + case["pad"]
        moved = sum(abs(_ceil(max(t, 0), page) - _ceil(max(n, 0), page)) for n, t in steps)
        # lengths read and written; slots and positions; a page moved is read from one place and written to another
        return {"bytes": 16.0 * case["B"] + 12.0 * tokens + 8.0 * moved, "flops": 4.0 * tokens + 20.0 * case["B"]}
    if case["kind"] == "rotate":
        rows = case["n"] * case["heads"] * (case["G"] + 1)
        return {"bytes": 4.0 * rows * case["D"] + 4.0 * case["n"] + 8.0 * case["D"] * case["norm"] + 4.0 * case["rot"],
                "flops": rows * (3.0 * case["rot"] + 4.0 * case["D"] * case["norm"])}
    lens = _lengths(case)
    pairs = sum(L * (L + 1) // 2 if case["causal"] else L * L for L in lens)
    Hq = case["heads"] * case["G"]
    return {"bytes": 2.0 * sum(lens) * (Hq + case["heads"]) * (case["D"] + case["Dv"]) + 4.0 * (case["B"] + 1),
            "flops": 2.0 * pairs * Hq * (case["D"] + case["Dv"])}


# ---- inputs -------------------------------------------------------------------

def _rows(gen, shape, dtype):
    """Rows [..][channels] as a model makes them: some larger than others."""
    x = torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)
    x *= torch.exp(0.3 * torch.randn(*shape[:-1], 1, generator=gen, device="cuda"))
    return x.to(dtype)


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed * 7919 + 29)
    if case["kind"] == "plan":
        B, page, steps = case["B"], case["page"], _steps(case)
        has = [_ceil(max(n, 0), page) for n, _ in steps]
        to = [_ceil(max(t, 0), page) for _, t in steps]
        width = max(max(has), max(to), 1) + 2
        grown = sum(max(t - h, 0) for h, t in zip(has, to))
        back = sum(max(h - t, 0) for h, t in zip(has, to))
        n_free = max(grown // 2 - back, 1) if case["scarce"] else grown + 5
        n_pages = sum(has) + n_free
        pages = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
        table = torch.full((B, width), -1, dtype=torch.int32)
        at = 0
        host = pages.cpu()
        for b in range(B):
            table[b, :has[b]] = host[at:at + has[b]]
            at += has[b]
        free = torch.full((n_pages,), -1, dtype=torch.int32)
        free[:n_free] = host[at:]
        return {"n_pages": n_pages, "table": table.cuda(), "free": free.cuda(), "n_free": n_free,
                "lengths": torch.tensor([n for n, _ in steps], dtype=torch.int32, device="cuda"),
                "targets": torch.tensor([t for _, t in steps], dtype=torch.int32, device="cuda"),
                "cap": sum(_news(case)) + case["pad"]}
    dtype, heads, Hq = DT[case["dtype"]], case["heads"], case["heads"] * case["G"]
    if case["kind"] == "rotate":
        n, D = case["n"], case["D"]
        x = {"positions": torch.randint(0, case["far"] + 1, (n,), generator=gen, device="cuda", dtype=torch.int32)}
        if case["fused"]:
            # one projection's output holds [queries | keys | values]
            qkv = _rows(gen, (n, Hq + 2 * heads, D), dtype)
            x["q"], x["k"] = qkv[:, :Hq], qkv[:, Hq:Hq + heads]
        else:
            x["q"], x["k"] = _rows(gen, (n, Hq, D), dtype), _rows(gen, (n, heads, D), dtype)
        for s in ("q_gain", "k_gain"):
            x[s] = 1.0 + 0.2 * torch.randn(D, generator=gen, device="cuda") if case["norm"] else None
        return x
    lens = _lengths(case)
    n = sum(lens) + case["pad"]
    q, k = _rows(gen, (n, Hq, case["D"]), dtype), _rows(gen, (n, heads, case["D"]), dtype)
    # values are a slice of the projection's output, behind its keys
    kv = _rows(gen, (n, heads * (case["D"] + case["Dv"])), dtype)
    v = kv[:, heads * case["D"]:].unflatten(1, (heads, case["Dv"]))
    starts = [0]
    for L in lens:
        starts.append(starts[-1] + L)
    return {"q": q, "k": k, "v": v, "starts": torch.tensor(starts, dtype=torch.int32, device="cuda"),
            "out": torch.zeros(n, Hq, case["Dv"], dtype=dtype, device="cuda")}


def _frequencies(case):
    """Radians a position of each turned pair."""
    out = []
    for i in range(case["rot"] // 2):
        f = case["base"] ** (-2.0 * i / case["rot"])
        if case["length"] == 0:
            f /= case["factor"]
        else:
            # turns over the original length: few are slowed down, many kept, between them blended
            turns = case["length"] * f / (2.0 * math.pi)
            keep = min(max((turns - case["low"]) / (case["high"] - case["low"]), 0.0), 1.0)
            f = keep * f + (1.0 - keep) * f / case["factor"]
        out.append(f)
    return out


def prepare(case, seed):
    st = _inputs(case, seed)
    st["case"] = case
    if case["kind"] == "plan":
        st["count"] = torch.tensor([st["n_free"], 0], dtype=torch.int32, device="cuda")
        st["left"] = torch.zeros(2, dtype=torch.int32, device="cuda")
    if case["kind"] == "rotate":
        st["freq"] = torch.tensor(_frequencies(case), dtype=torch.float64, device="cuda")
    if own:
        from paper_2311_14114_gb300 import soniq as sq
        if case["kind"] == "plan":
            pages = sq.KVPages(st["n_pages"], case["page"], case["B"], st["table"].shape[1])
            pages.table.copy_(st.pop("table"))
            pages.free.copy_(st.pop("free"))
            pages.count.copy_(st.pop("count"))
            st["pages"] = pages
        elif case["kind"] == "rotate":
            scaling = ("linear", case["factor"]) if case["length"] == 0 else \
                ("wavelength", case["factor"], case["low"], case["high"], case["length"])
            st["rotary"] = sq.Rotary(case["rot"], base=case["base"], interleaved=case["interleaved"], scaling=scaling)
    return st


# ---- the plain form -----------------------------------------------------------

def _plan(case, st):
    page, W, cap, n_pages = case["page"], st["table"].shape[1], st["cap"], st["n_pages"]
    L, target = st["lengths"].long(), st["targets"].long()
    table, free, n_free = st["table"].long(), st["free"].long(), st["count"][0].long()
    old, goal = L.clamp(min=0), target.clamp(min=0)
    new = (goal - old).clamp(min=0)
    has, to = ((old + page - 1) // page).clamp(max=W), (goal + page - 1) // page
    end = torch.cumsum(new, 0)
    back = (has - to).clamp(min=0)
    fits = (to <= W) & (end <= cap)
    need = torch.where(fits, (to - has).clamp(min=0), 0)
    upto, gone = torch.cumsum(need, 0), torch.cumsum(back, 0)
    n_back = gone[-1]
    served = (new == 0) | fits & ((need == 0) | (upto <= n_free + n_back))
    taken = torch.where(served, torch.where(need > 0, upto, 0), 0).amax()
    # pages that are given back, in the order of sequences and tokens; then those of the pool from its end
    i = torch.arange(n_pages, device="cuda")
    seq = torch.searchsorted(gone, i, right=True).clamp(max=case["B"] - 1)
    released = table[seq, (to[seq] + i - (gone - back)[seq]).clamp(0, W - 1)]
    given = torch.where(i < n_back, released, free[(n_free - 1 - (i - n_back)).clamp(0, n_pages - 1)])
    col = torch.arange(W, device="cuda")
    mine = (upto - need)[:, None] + col - has[:, None]
    grows = (served & (need > 0))[:, None] & (col >= has[:, None]) & (col < to[:, None])
    table = torch.where(grows, given[mine.clamp(0, n_pages - 1)], table)
    stays = (i >= n_free) & (i < n_free + n_back - taken)
    free = torch.where(stays, released[(n_free + n_back - 1 - i).clamp(0, n_pages - 1)], free)
    t = torch.arange(cap, device="cuda")
    seq = torch.searchsorted(end, t, right=True)
    live = seq < case["B"]
    seq = seq.clamp(max=case["B"] - 1)
    pos = torch.where(live, old[seq] + t - (end - new)[seq], 0)
    slot = table[seq, (pos // page).clamp(max=W - 1)] * page + pos % page
    slot = torch.where(live & served[seq], slot, -1)
    lengths = torch.where(served, torch.where(target < 0, -1, target), L)
    starts = torch.cat([end.new_zeros(1), end]).clamp(max=cap)
    left = n_free + n_back - taken
    return [starts.int(), pos.int(), slot, lengths.int(), table.int(), free.int(), left.int().view(1)]


def _rotate(case, st):
    out, rot = [], case["rot"]
    turn = st["positions"].double()[:, None] * st["freq"]
    cos, sin = torch.cos(turn).float()[:, None], torch.sin(turn).float()[:, None]
    for x, gain in ((st["q"], st["q_gain"]), (st["k"], st["k_gain"])):
        y = x.float()
        if gain is not None:
            y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + 1e-6) * gain
        if case["interleaved"]:
            a, b = y[..., 0:rot:2], y[..., 1:rot:2]
            z = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
        else:
            a, b = y[..., :rot // 2], y[..., rot // 2:rot]
            z = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
        out.append(torch.cat([z, y[..., rot:]], -1).to(x.dtype))
    return out


def _attend(case, st):
    G, D = case["G"], case["D"]
    out = st["out"]
    at = 0
    for L in _lengths(case):
        if L == 0:
            continue
        k = st["k"][at:at + L].float().permute(1, 2, 0)[:, None]
        v = st["v"][at:at + L].float().transpose(0, 1)[:, None]
        for t0 in range(0, L, 512):
            t1 = min(t0 + 512, L)
            to = t1 if case["causal"] else L
            q = st["q"][at + t0:at + t1].float().unflatten(1, (case["heads"], G)).permute(1, 2, 0, 3)
            s = torch.matmul(q, k[..., :to]) / math.sqrt(D)
            if case["causal"]:
                s.masked_fill_(torch.arange(to, device="cuda") > torch.arange(t0, t1, device="cuda")[:, None], -math.inf)
            p = torch.exp(s - s.amax(-1, keepdim=True))
            o = torch.matmul(p, v[:, :, :to]) / p.sum(-1, keepdim=True)
            out[at + t0:at + t1] = o.permute(2, 0, 1, 3).flatten(1, 2).to(out.dtype)
        at += L
    return [out]


# ---- one pass -----------------------------------------------------------------

def run(st):
    case = st["case"]
    if own:
        from paper_2311_14114_gb300 import soniq as sq
        if case["kind"] == "plan":
            # the pool's count goes to another place, so that the same step can be planned again
            step = sq.kv_plan(st["pages"], st["lengths"], st["targets"], st["cap"], count_out=st["left"])
            return [step.starts, step.positions, step.slots, step.lengths, st["pages"].table, st["pages"].free, st["left"][:1]]
        if case["kind"] == "rotate":
            return list(sq.rotate_heads(st["rotary"], st["q"], st["k"], st["positions"], q_gain=st["q_gain"],
                                        k_gain=st["k_gain"], eps=1e-6))
        return [sq.prompt_attend(st["q"], st["k"], st["v"], st["starts"], causal=case["causal"], out=st["out"])]
    return {"plan": _plan, "rotate": _rotate, "attend": _attend}[case["kind"]](case, st)


# ---- the definition in 64 bits ------------------------------------------------

def _exact_rotate(case, x):
    out, half = [], case["rot"] // 2
    pair = torch.arange(half, dtype=torch.float64, device="cuda")
    f = torch.pow(torch.tensor(case["base"], dtype=torch.float64, device="cuda"), -pair / half)
    slow = f / case["factor"]
    if case["length"] == 0:
        f = slow
    else:
        longest = case["length"] / case["low"]
        shortest = case["length"] / case["high"]
        wave = 2 * math.pi / f
        blend = (case["length"] / wave - case["low"]) / (case["high"] - case["low"])
        f = torch.where(wave < shortest, f, torch.where(wave > longest, slow, blend * f + (1 - blend) * slow))
    angle = x["positions"].to(torch.float64)[:, None, None] * f
    turn = torch.polar(torch.ones_like(angle), angle)
    for t, gain in ((x["q"], x["q_gain"]), (x["k"], x["k_gain"])):
        y = t.to(torch.float64)
        if gain is not None:
            y = y / torch.sqrt(y.pow(2).sum(-1, keepdim=True) / case["D"] + 1e-6) * gain.to(torch.float64)
        turned, rest = y[..., :2 * half], y[..., 2 * half:]
        shape = (half, 2) if case["interleaved"] else (2, half)
        axis = -1 if case["interleaved"] else -2
        a, b = turned.unflatten(-1, shape).unbind(axis)
        z = torch.complex(a, b) * turn
        out.append(torch.cat([torch.stack([z.real, z.imag], axis).flatten(-2), rest], -1))
    return out


def _exact_attend(case, x):
    Hq, G, D = case["heads"] * case["G"], case["G"], case["D"]
    o = torch.zeros(x["q"].shape[0], Hq, case["Dv"], dtype=torch.float64, device="cuda")
    starts = x["starts"].tolist()
    for a, z in zip(starts[:-1], starts[1:]):
        for h in range(case["heads"]):
            k, v = x["k"][a:z, h].to(torch.float64), x["v"][a:z, h].to(torch.float64)
            for t0 in range(a, z, 1024):
                t1 = min(t0 + 1024, z)
                upto = (t1 if case["causal"] else z) - a
                q = x["q"][t0:t1, h * G:(h + 1) * G].to(torch.float64)
                s = torch.einsum("tgd,ld->tgl", q, k[:upto]) * D ** -0.5
                if case["causal"]:
                    late = torch.arange(upto, device="cuda")[None, :] + a > torch.arange(t0, t1, device="cuda")[:, None]
                    s = s.masked_fill(late[:, None, :], -math.inf)
                o[t0:t1, h * G:(h + 1) * G] = torch.einsum("tgl,ld->tgd", torch.softmax(s, -1), v[:upto])
    return [o]


def _exact_plan(case, x):
    """One sequence after the other, with lists."""
    page, lengths, targets = case["page"], x["lengths"].tolist(), x["targets"].tolist()
    table, free = x["table"].tolist(), x["free"].tolist()
    pool, back = free[:x["n_free"]], []
    for b, (n, t) in enumerate(zip(lengths, targets)):
        back += table[b][_ceil(max(t, 0), page):_ceil(max(n, 0), page)]
    pool += reversed(back)
    starts, positions, slots, after, waiting = [0], [], [], [], False
    for b, (n, t) in enumerate(zip(lengths, targets)):
        old, goal = max(n, 0), max(t, 0)
        has, to = _ceil(old, page), _ceil(goal, page)
        room = True
        if to > has:
            waiting = waiting or to - has > len(pool)
            room = not waiting
            if room:
                for i in range(has, to):
                    table[b][i] = pool.pop()
        after.append(max(t, -1) if room else n)
        starts.append(starts[-1] + max(goal - old, 0))
        positions += range(old, goal)
        slots += [table[b][p // page] * page + p % page if room else -1 for p in range(old, goal)]
    free[:len(pool)] = pool
    positions += [0] * case["pad"]
    slots += [-1] * case["pad"]
    lists = (starts, positions, slots, after, table, free, [len(pool)])
    return [torch.tensor(y, dtype=torch.int64 if y is slots else torch.int32, device="cuda") for y in lists]


def exact(case, seed):
    x = _inputs(case, seed)
    return {"plan": _exact_plan, "rotate": _exact_rotate, "attend": _exact_attend}[case["kind"]](case, x)
