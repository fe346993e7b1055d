"""A quantized key / value cache and the attention that reads it, as cases that can be timed.

Every key and value row (one token, one head) is held as SONIQ codes: the head's channels are split
in two precision groups, each with one max-abs scale, and code = the nearest level j / 2^(n-1) of
x / scale (n bits, half to even).  Rows live in pages of `page` tokens that a sequence finds through
its page table.  A case's "kind" says which calls one pass makes:

  store    kv_write of n tokens' keys and values into their slots, and kv_read of the same slots
  load     kv_read of the slots of a prefix that is in the cache
  attend   kv_attend: T drafted tokens of each sequence (T = 1: plain decoding; no mask: a chain, as
           for a piece of a prompt) over the cached context and over the drafts their mask shows,
           which are in the cache behind the context

`own` selects the library's kernels; otherwise the same is computed with elementary torch operations
in 32 bits.
"""
import math
import random

import torch

own = False

DT = {"f16": torch.float16, "bf16": torch.bfloat16}


# ---- cases --------------------------------------------------------------------

def _case(kind, name=None, **kw):
    # D, Dv: channels of a key / value head; k, v: (channels in the high group, low bits, high bits)
    c = dict(kind=kind, dtype="f16", heads=8, D=128, Dv=128, k_hi=32, k_lo_bits=4, k_hi_bits=8, v_hi=0, v_lo_bits=4,
             v_hi_bits=8, page=64)
    c.update(kw)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # the new tokens of eight sequences in one decoding step, written by one layer: latency
        _case("store", "store_8_tokens", n=8, page=16),
        # an odd piece of a prompt, 80 channels split 67 / 13, so groups end inside their 32-code blocks
        _case("store", "store_1001x80", n=1001, heads=12, D=80, Dv=80, k_hi=13, k_lo_bits=2, k_hi_bits=8, v_hi=5,
              v_lo_bits=4, v_hi_bits=8, page=16),
        # the prompts of a batch, keys and values as slices of the fused projection's output
        _case("store", "store_16384_fused_bf16", n=16384, dtype="bf16", fused=32),
        # a short shared prefix read back for a dense prompt kernel
        _case("load", "load_777", n=777, page=32),
        # a long one
        _case("load", "load_65536_bf16", n=65536, dtype="bf16", k_hi=16),
        # the first tokens of an answer to a short question: latency
        _case("attend", "one_token_ctx97", B=1, T=1, G=4, ctx=97, page=16),
        # one long document, decoded alone: all SMs share one sequence
        _case("attend", "one_token_ctx131071", B=1, T=1, G=4, ctx=131071),
        # a serving batch with lengths from a few hundred tokens up
        _case("attend", "batch64_ctx8192_bf16", B=64, T=1, G=8, ctx=8192, ragged=True, dtype="bf16", k_hi=16),
        # a small drafted tree without shared heads, odd sizes
        _case("attend", "tree13_mha_ctx1501", B=3, T=13, G=1, heads=12, D=64, Dv=64, k_hi=8, ctx=1501, ragged=True,
              page=32, tree=True),
        # drafted trees of a batch: 96 rows to a key head
        _case("attend", "tree24_batch16_ctx4096", B=16, T=24, G=4, ctx=4096, ragged=True, tree=True, dtype="bf16"),
        # wide trees over long contexts: 512 rows to a key head
        _case("attend", "tree64_ctx16384", B=4, T=64, G=8, ctx=16384, heads=4, tree=True, k_hi=0),
        # a piece of two prompts, each token seeing the ones before it
        _case("attend", "chunk512_ctx3500", B=2, T=512, G=4, ctx=3500, page=128),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    """Cached channels read or written, and products: what the cost of a pass grows with."""
    if case["kind"] != "attend":
        return case["n"] * case["heads"] * (case["D"] + case["Dv"]), 0
    L = sum(_lengths(case)) + case["B"] * case["T"]
    peak = (max(_lengths(case)) + case["T"]) * case["B"]
    return peak * case["heads"] * (case["D"] + case["Dv"]), L * case["T"] * case["G"] * case["heads"] * (case["D"] + case["Dv"])


def _most():
    costs = [_cost(c) for c in listed()]
    return max(c[0] for c in costs), max(c[1] for c in costs)


def draw(rng):
    most = _most()
    while True:
        D = rng.choice([40, 64, 64, 80, 96, 128, 128, 128, 192, 256])
        Dv = D if rng.random() < 0.8 else rng.choice([64, 128])
        lo, hi = rng.choice([(4, 8), (4, 8), (4, 8), (2, 8), (2, 4), (8, 8)])
        vlo, vhi = rng.choice([(4, 8), (4, 8), (2, 4), (8, 8)])
        # 256 channels fill the row's code space, so their groups end on whole blocks
        k_hi = rng.choice([0, 32, 64]) if D == 256 else rng.choice([0, 0, 8, 13, 16, 32])
        v_hi = rng.choice([0, 0, 32]) if Dv == 256 else rng.choice([0, 0, 0, 5, 16])
        kw = dict(dtype=rng.choice(["f16", "bf16"]), heads=rng.choice([1, 2, 4, 5, 8, 12]), D=D, Dv=Dv, k_hi=k_hi,
                  k_lo_bits=lo, k_hi_bits=hi, v_hi=v_hi, v_lo_bits=vlo, v_hi_bits=vhi, page=rng.choice([16, 32, 64, 128]))
        kind = rng.choices(["store", "load", "one", "tree", "chunk"], [2, 1, 3, 3, 1])[0]
        if kind in ("store", "load"):
            if kind == "store" and rng.random() < 0.4:
                kw["fused"] = kw["heads"] * rng.choice([1, 4, 8])
            c = _case(kind, n=_log_int(rng, 1, 65536), **kw)
        else:
            T = {"one": 1, "tree": _log_int(rng, 2, 64), "chunk": _log_int(rng, 65, 1024)}[kind]
            c = _case("attend", B=_log_int(rng, 1, 64) if kind != "chunk" else rng.randint(1, 4), T=T,
                      G=rng.choice([1, 2, 4, 5, 8]), ctx=_log_int(rng, 1, 131072) if kind == "one" else _log_int(rng, 1, 16384),
                      ragged=rng.random() < 0.6, tree=kind == "tree", **kw)
        cost = _cost(c)
        if cost[0] <= most[0] and cost[1] <= most[1]:
            return c


def _lengths(case):
    """Context tokens of each sequence; ragged ones spread from the full length down to a tenth of it."""
    B, ctx = case["B"], case["ctx"]
    if not case.get("ragged"):
        return [ctx] * B
    return [int(ctx * (1.0 - 0.9 * ((b * 7) % B) / B)) for b in range(B)]


def _groups(case, side):
    """(channels, bits) of the one or two groups of a key ('k') or value ('v') row."""
    D = case["D"] if side == "k" else case["Dv"]
    n_hi = case[side + "_hi"]
    g = [(D - n_hi, case[side + "_lo_bits"])]
    return g + [(n_hi, case[side + "_hi_bits"])] if n_hi else g


def _pad32(n):
    return -(-n // 32) * 32


def _row_bytes(case, side):
    return -(-sum(_pad32(c) * b // 8 for c, b in _groups(case, side)) // 16) * 16


def work(case):
    """Logical codes and scales of a row, each read or written once."""
    row = {s: sum(c * b / 8.0 + 2 for c, b in _groups(case, s)) for s in "kv"}
    packed = (row["k"] + row["v"]) * case["heads"]
    plain = 2.0 * (case["D"] + case["Dv"]) * case["heads"]
    if case["kind"] == "store":
        # read the inputs, write codes; read codes, write the values they stand for
        return {"bytes": case["n"] * (2 * plain + 2 * packed + 16), "flops": case["n"] * case["heads"] * 8.0 * (case["D"] + case["Dv"])}
    if case["kind"] == "load":
        return {"bytes": case["n"] * (plain + packed + 8), "flops": case["n"] * case["heads"] * 2.0 * (case["D"] + case["Dv"])}
    B, T, lens = case["B"], case["T"], _lengths(case)
    Hq = case["heads"] * case["G"]
    seen = T * (T + 1) // 2 if not case.get("tree") else None
    pairs = 0.0
    for L in lens:
        # a drafted token sees the context, itself and its ancestors: of T drafts about log2(T) + 1
        pairs += T * L + (seen if seen is not None else T * min(T, math.log2(T) + 1.0))
    return {"bytes": (sum(lens) + B * T) * packed + 2.0 * B * T * Hq * (case["D"] + case["Dv"]) + 4.0 * B
            + (B * T * T if case.get("tree") else 0) + 4.0 * sum(-(-(L + T) // case["page"]) for L in lens),
            "flops": 2.0 * pairs * Hq * (case["D"] + case["Dv"])}


# ---- inputs -------------------------------------------------------------------

def _rows(gen, lead, heads, D, high, dtype):
    """Rows as a model makes them: [*lead][heads][D], some tokens larger than others, outlier channels."""
    x = torch.randn(*lead, heads, D, generator=gen, device="cuda", dtype=torch.float32)
    x *= torch.exp(0.3 * torch.randn(*lead, heads, 1, generator=gen, device="cuda"))
    x *= 1.0 + 5.0 * high.to(torch.float32)
    return x.to(dtype)


def _high_channels(rng, heads, D, n_hi):
    high = torch.zeros(heads, D, dtype=torch.bool)
    for h in range(heads):
        high[h, rng.sample(range(D), n_hi)] = True
    return high


def _inputs(case, seed):
    rng = random.Random(seed * 7919 + 17)
    gen = torch.Generator(device="cuda").manual_seed(seed * 7919 + 17)
    dtype = DT[case["dtype"]]
    heads, page = case["heads"], case["page"]
    x = {"high_k": _high_channels(rng, heads, case["D"], case["k_hi"]).cuda(),
         "high_v": _high_channels(rng, heads, case["Dv"], case["v_hi"]).cuda()}
    if case["kind"] != "attend":
        n = case["n"]
        # slots of n tokens: whole pages in any order, the last one partly filled
        used = -(-n // page)
        x["n_pages"] = used + 3
        pages = torch.randperm(x["n_pages"], generator=gen, device="cuda")[:used]
        slots = (pages[:, None] * page + torch.arange(page, device="cuda")[None, :]).reshape(-1)[:n]
        x["slots"] = slots.to(torch.int64).contiguous()
        k = _rows(gen, (n,), heads, case["D"], x["high_k"], dtype)
        v = _rows(gen, (n,), heads, case["Dv"], x["high_v"], dtype)
        if case.get("fused"):
            # one projection's output holds [queries | keys | values]
            nq, nk = case["fused"] * case["D"], heads * case["D"]
            qkv = torch.zeros(n, nq + nk + heads * case["Dv"], dtype=dtype, device="cuda")
            qkv[:, nq:nq + nk] = k.reshape(n, -1)
            qkv[:, nq + nk:] = v.reshape(n, -1)
            k = qkv[:, nq:nq + nk].view(n, heads, case["D"])
            v = qkv[:, nq + nk:].view(n, heads, case["Dv"])
        x["k"], x["v"] = k, v
        return x
    B, T, lens = case["B"], case["T"], _lengths(case)
    need = [-(-(L + T) // page) for L in lens]
    x["n_pages"] = sum(need) + 3
    order = torch.randperm(x["n_pages"], generator=gen, device="cuda").to(torch.int32)
    table = torch.full((B, max(need)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b in range(B):
        table[b, :need[b]] = order[at:at + need[b]]
        at += need[b]
    x["table"], x["lens"] = table, torch.tensor(lens, dtype=torch.int32, device="cuda")
    # page-major rows [n_pages][page][heads][D]
    x["k"] = _rows(gen, (x["n_pages"], page), heads, case["D"], x["high_k"], dtype)
    x["v"] = _rows(gen, (x["n_pages"], page), heads, case["Dv"], x["high_v"], dtype)
    x["q"] = torch.randn(B, T, heads * case["G"], case["D"], generator=gen, device="cuda", dtype=torch.float32).to(dtype)
    x["mask"] = None
    if case.get("tree"):
        # a random tree for each sequence: a draft's parent is the context (-1) or an earlier draft
        mask = torch.zeros(B, T, T, dtype=torch.bool)
        for b in range(B):
            for i in range(T):
                parent = rng.randint(-1, i - 1)
                if parent >= 0:
                    mask[b, i] = mask[b, parent]
                mask[b, i, i] = True
        x["mask"] = mask.cuda()
    return x


def prepare(case, seed):
    x = _inputs(case, seed)
    heads, page, n_pages, dtype = case["heads"], case["page"], x["n_pages"], DT[case["dtype"]]
    st = {"case": case, "n_pages": n_pages}
    for s in "kv":
        # low channels first, each group in ascending order
        st["perm_" + s] = torch.sort(x["high_" + s].to(torch.int32), dim=1, stable=True).indices.to(torch.int32)
        rb = _row_bytes(case, s)
        st["codes_" + s] = torch.zeros(n_pages, heads, page, rb, dtype=torch.uint8, device="cuda")
        st["scales_" + s] = torch.zeros(n_pages, heads, page, len(_groups(case, s)), dtype=dtype, device="cuda")
    if case["kind"] == "store":
        st["k"], st["v"] = x["k"], x["v"]
    else:
        for s in "kv":
            if case["kind"] == "attend":
                codes, scales = _quantize(case, s, x[s], st["perm_" + s])
                st["codes_" + s].copy_(codes.transpose(1, 2))
                st["scales_" + s].copy_(scales.transpose(1, 2))
            else:
                _put(case, st, s, x["slots"], x[s])
    for name in ("slots", "table", "lens", "q", "mask"):
        if name in x:
            st[name] = x[name]
    if own:
        from paper_2311_14114_gb300 import soniq as sq
        lay = {}
        for s in "kv":
            g = _groups(case, s)
            lay[s] = sq.KVLayout(st["perm_" + s].cpu(), [c for c, _ in g], [b for _, b in g])
        cache = sq.KVCache(lay["k"], lay["v"], n_pages=n_pages, page_size=page, dtype=dtype)
        for s in "kv":
            getattr(cache, s + "_codes").copy_(st.pop("codes_" + s))
            getattr(cache, s + "_scales").copy_(st.pop("scales_" + s))
        st["cache"] = cache
    return st


# ---- the plain form -----------------------------------------------------------

def _pack(codes, bits):
    """[..][32 k] integer codes -> [..][4 bits k] bytes: blocks of 32 codes as little-endian words (soniq.h)."""
    lead = codes.shape[:-1]
    c = (codes & ((1 << bits) - 1)).to(torch.uint8)
    if bits == 8:
        return c
    if bits == 4:
        c = c.view(*lead, -1, 2, 4)
        return (c[..., 0, :] | (c[..., 1, :] << 4)).reshape(*lead, -1)
    c = c.view(*lead, -1, 4, 4)
    return (c[..., 0, :] | (c[..., 1, :] << 2) | (c[..., 2, :] << 4) | (c[..., 3, :] << 6)).reshape(*lead, -1)


def _unpack(b, bits):
    """The signed codes of _pack's bytes, fp32."""
    lead = b.shape[:-1]
    if bits == 8:
        u = b
    elif bits == 4:
        b = b.view(*lead, -1, 1, 4)
        u = torch.cat([b & 15, b >> 4], dim=-2).reshape(*lead, -1)
    else:
        b = b.view(*lead, -1, 1, 4)
        u = torch.cat([b & 3, (b >> 2) & 3, (b >> 4) & 3, b >> 6], dim=-2).reshape(*lead, -1)
    half = 1 << (bits - 1)
    return (u ^ half).to(torch.float32) - half


def _quantize(case, side, x, perm):
    """Rows [..][heads][D] -> packed codes [..][heads][row bytes] and scales [..][heads][groups]."""
    x = x.to(torch.float32)
    top = torch.finfo(DT[case["dtype"]]).max
    x = torch.nan_to_num(x, nan=0.0, posinf=top, neginf=-top)
    idx = perm.to(torch.int64).expand(*x.shape)
    x = torch.gather(x, -1, idx)
    out, scales, at = [], [], 0
    for count, bits in _groups(case, side):
        g = x[..., at:at + count]
        at += count
        s = g.abs().amax(-1, keepdim=True)
        half = float(1 << (bits - 1))
        j = torch.round(g / torch.where(s > 0, s, 1.0) * half).clamp(-half, half - 1).to(torch.int16)
        j = torch.nn.functional.pad(j, (0, _pad32(count) - count))
        out.append(_pack(j, bits))
        scales.append(s)
    codes = torch.cat(out, -1)
    codes = torch.nn.functional.pad(codes, (0, _row_bytes(case, side) - codes.shape[-1]))
    return codes, torch.cat(scales, -1).to(DT[case["dtype"]])


def _values(case, side, codes, scales, perm):
    """Packed rows [..][heads or broadcast][..] -> fp32 values in the channels' own order."""
    out, byte = [], 0
    for g, (count, bits) in enumerate(_groups(case, side)):
        nb = _pad32(count) * bits // 8
        j = _unpack(codes[..., byte:byte + nb].contiguous(), bits)[..., :count]
        byte += nb
        out.append(j * (scales[..., g:g + 1].to(torch.float32) / float(1 << (bits - 1))))
    x = torch.cat(out, -1)
    inverse = torch.argsort(perm.to(torch.int64), dim=-1)
    return torch.gather(x, -1, inverse.expand(*x.shape))


def _put(case, st, side, slots, x):
    codes, scales = _quantize(case, side, x, st["perm_" + side])
    page, at = slots // case["page"], slots % case["page"]
    st["codes_" + side][page, :, at] = codes
    st["scales_" + side][page, :, at] = scales


def _get(case, st, side, slots):
    page, at = slots // case["page"], slots % case["page"]
    x = _values(case, side, st["codes_" + side][page, :, at], st["scales_" + side][page, :, at], st["perm_" + side])
    return x.to(DT[case["dtype"]])


def _attend(case, st):
    B, T, G, heads, page = case["B"], case["T"], case["G"], case["heads"], case["page"]
    table = st["table"].clamp(min=0).to(torch.int64)
    kv = {}
    for s in "kv":
        # [B][pages][heads][page][..] -> [B][heads][tokens][channels]
        codes, scales = (st[n + s][table].transpose(1, 2).flatten(2, 3) for n in ("codes_", "scales_"))
        kv[s] = _values(case, s, codes, scales, st["perm_" + s][:, None, :])
    L = kv["k"].shape[2]
    q = st["q"].to(torch.float32).view(B, T, heads, G, case["D"]).permute(0, 2, 1, 3, 4).reshape(B, heads, T * G, case["D"])
    scores = torch.matmul(q, kv["k"].transpose(2, 3)).view(B, heads, T, G, L) / math.sqrt(case["D"])
    pos = torch.arange(L, device="cuda")
    lens = st["lens"].to(torch.int64)
    draft = pos[None, :] - lens[:, None]                                     # [B][L]: which draft a position holds
    if st["mask"] is None:
        seen = draft[:, None, :] <= torch.arange(T, device="cuda")[None, :, None]
    else:
        seen = torch.gather(st["mask"], 2, draft.clamp(0, T - 1)[:, None, :].expand(B, T, L))
        seen = seen & (draft < T)[:, None, :] | (draft < 0)[:, None, :]
    scores = scores.masked_fill(~seen[:, None, :, None, :], -math.inf)
    m = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(m == -math.inf, 0.0, m))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total > 0, total, 1.0)
    # values behind the last draft are not read
    v = kv["v"].masked_fill((draft >= T)[:, None, :, None], 0.0)
    o = torch.matmul(p.view(B, heads, T * G, L), v)
    o = o.view(B, heads, T, G, case["Dv"]).permute(0, 2, 1, 3, 4).reshape(B, T, heads * G, case["Dv"])
    return o.to(DT[case["dtype"]])


# ---- one pass -----------------------------------------------------------------

def run(st):
    case = st["case"]
    if own:
        from paper_2311_14114_gb300 import soniq as sq
        cache = st["cache"]
        if case["kind"] == "attend":
            return [sq.kv_attend(cache, st["q"], st["table"], st["lens"], mask=st["mask"])]
        if case["kind"] == "store":
            sq.kv_write(cache, st["k"], st["v"], st["slots"])
        return list(sq.kv_read(cache, st["slots"]))
    if case["kind"] == "attend":
        return [_attend(case, st)]
    if case["kind"] == "store":
        _put(case, st, "k", st["slots"], st["k"])
        _put(case, st, "v", st["slots"], st["v"])
    return [_get(case, st, "k", st["slots"]), _get(case, st, "v", st["slots"])]


# ---- the definition in 64 bits ------------------------------------------------

def _exact_rows(x, high, lo_bits, hi_bits):
    """What a cache holds of rows [..][heads][D], fp64: channel by channel, no packing and no permutation."""
    x = x.to(torch.float64)
    out = torch.zeros_like(x)
    for members, bits in ((~high, lo_bits), (high, hi_bits)):
        if not bool(members.any()):
            continue
        mag = torch.where(members, x.abs(), 0.0).max(dim=-1, keepdim=True).values
        levels = 2.0 ** (bits - 1)
        j = torch.round(x * levels / mag.clamp(min=1e-300))
        j = torch.minimum(torch.maximum(j, torch.full_like(j, -levels)), torch.full_like(j, levels - 1))
        out = torch.where(members & (mag > 0), j * mag / levels, out)
    return out


def exact(case, seed):
    x = _inputs(case, seed)
    if case["kind"] != "attend":
        return [_exact_rows(x["k"], x["high_k"], case["k_lo_bits"], case["k_hi_bits"]),
                _exact_rows(x["v"], x["high_v"], case["v_lo_bits"], case["v_hi_bits"])]
    B, T, G, heads = case["B"], case["T"], case["G"], case["heads"]
    o = torch.zeros(B, T, heads * G, case["Dv"], dtype=torch.float64, device="cuda")
    for b, L in enumerate(_lengths(case)):
        pages = x["table"][b, :-(-(L + T) // case["page"])].to(torch.int64)
        k = _exact_rows(x["k"][pages].flatten(0, 1)[:L + T], x["high_k"], case["k_lo_bits"], case["k_hi_bits"])
        v = _exact_rows(x["v"][pages].flatten(0, 1)[:L + T], x["high_v"], case["v_lo_bits"], case["v_hi_bits"])
        see = torch.ones(T, L + T, dtype=torch.bool, device="cuda")
        see[:, L:] = torch.ones(T, T, device="cuda").tril().bool() if x["mask"] is None else x["mask"][b]
        for h in range(heads):
            for t0 in range(0, T, 128):
                q = x["q"][b, t0:t0 + 128, h * G:(h + 1) * G].to(torch.float64)
                s = torch.einsum("tgd,ld->tgl", q, k[:, h]) * case["D"] ** -0.5
                s = s.masked_fill(~see[t0:t0 + 128, None, :], -math.inf)
                o[b, t0:t0 + 128, h * G:(h + 1) * G] = torch.einsum("tgl,ld->tgd", torch.softmax(s, -1), v[:, h])
    return [o]
