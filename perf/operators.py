"""The work that the operators of a 4-bit key-value cache and of its eviction are measured on.

A latent key-value row (576 bf16: 512 latent features, then 64 rotary ones) is held in 400 bytes: the latent part as 4-bit floats
(sign, two exponent bits, one fraction bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6) with one power of two per 128 features, the rotary part as it is.

  codes   bytes 0..255: feature f in the low (f even) or high (f odd) half of byte f / 2
  rotary  bytes 256..383: 64 bf16
  scales  bytes 384..387: biased exponents (127 + e, value = code * 2^e) of features 128 j .. 128 j + 127; 388..399 are zero

Each case is one operator, or the calls that make one operator in use: rows written and read back, attention over the selected rows,
the weight that each position received, and the choice and the move of the rows that stay.  `own` picks the framework's calls; the
plain forms are elementary torch operations in 32 bits.  Sizes are those of this repository's configurations (32 query heads,
k = 2048, contexts from 10K to 200K, index keys of 128 bf16) or generic.
"""
import math
import random

import torch

own = False

LAT, ROPE, ROW, BLOCK, HEADS, K = 512, 64, 400, 128, 32, 2048
MIN_E, MAX_E = -100, 100
SCALE = 1.0 / 24.0


def listed():
    rows = [
        # online serving: every sequence of a ragged batch appends one token to its pages and a layer reads it back
        ("append_one_token", dict(op="rows", B=40, T=1, Lk=49152, low=1, page=64)),
        # one piece of a chunked prefill lands behind a cached prefix
        ("append_chunk", dict(op="rows", B=1, T=701, Lk=41701, low=0, page=0)),
        # the longest prompt of the configurations is laid down at once
        ("append_prompt", dict(op="rows", B=1, T=131072, Lk=131072, low=0, page=0)),
        # one user's chat: a single request, one token
        ("attn_one_10k", dict(op="attn", B=1, T=1, Lk=10007, H=HEADS, k=K, low=0, page=0)),
        # online serving with the cache filled: ragged lengths behind a page table, some shorter than k
        ("attn_paged_800k", dict(op="attn", B=40, T=1, Lk=49152, H=HEADS, k=K, low=1, page=64)),
        # a drafted token beside the current one, a model of 20 heads that selects an odd number of rows
        ("attn_draft", dict(op="attn", B=12, T=2, Lk=30011, H=20, k=1021, low=0, page=0)),
        # a long prompt
        ("attn_prompt_32k", dict(op="attn", B=1, T=32768, Lk=32768, H=HEADS, k=K, low=0, page=0)),
        # a full batch of decode steps adds what each position received
        ("weight_decode_64k", dict(op="weight", B=32, T=1, Lk=65536, H=HEADS, k=K, low=0, page=0)),
        # a prompt of medium length leaves the weights that the first eviction goes by
        ("weight_prompt_8k", dict(op="weight", B=1, T=8191, Lk=8191, H=HEADS, k=K, low=0, page=0)),
        # short chats trimmed to half
        ("evict_short", dict(op="evict", B=3, T=1, Lk=1021, keep=512, first=4, recent=64, low=1, page=64)),
        # one user's long document cut to a tenth
        ("evict_one_200k", dict(op="evict", B=1, T=1, Lk=200000, keep=20000, first=4, recent=1024, low=0, page=0)),
        # a batch of long contexts cut to a quarter
        ("evict_batch_64k", dict(op="evict", B=32, T=1, Lk=65536, keep=16384, first=16, recent=512, low=30000, page=64)),
    ]
    return [dict(c, name=n) for n, c in rows]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng: random.Random):
    op = rng.choice(["rows", "rows", "attn", "attn", "prompt", "weight", "weight_prompt", "evict", "evict"])
    page = rng.choice([0, 0, 64, 128])
    if op == "rows":
        T = _log(rng, 1, 65536)
        B = _log(rng, 1, max(1, min(48, 100000 // T)))
        L = T + _log(rng, 1, max(2, min(60000, 1000000 // B)))
        return dict(op="rows", B=B, T=T, Lk=L, low=rng.choice([0, 1]), page=page)
    if op in ("attn", "weight"):
        B, T = _log(rng, 1, 40), rng.choice([1, 1, 1, 2, 3])
        L = _log(rng, 300, min(200000, 1600000 // B))
        return dict(op=op, B=B, T=T, Lk=L, H=rng.choice([32, 32, rng.randint(1, 31)]), k=_log(rng, 33, K), low=rng.choice([0, 1]), page=page)
    if op in ("prompt", "weight_prompt"):
        T = _log(rng, 64, 16384 if op == "prompt" else 6000)
        return dict(op="attn" if op == "prompt" else "weight", B=rng.randint(1, 2 if T < 5000 else 1), T=T, Lk=T + rng.choice([0, _log(rng, 1, 20000)]),
                    H=rng.choice([32, rng.randint(1, 31)]), k=_log(rng, 129, K), low=0, page=page)
    B = _log(rng, 1, 32)
    L = _log(rng, 200, min(200000, 2000000 // B))
    keep = _log(rng, max(2, L // 20), max(3, L * 3 // 4))
    return dict(op="evict", B=B, T=1, Lk=L, keep=keep, first=min(4, keep // 4), recent=keep // rng.choice([4, 16]), low=rng.choice([0, 1]), page=page)


# ---- the 4-bit row ------------------------------------------------------------------------------------------------

def _pack(rows):
    """[.., 576] bf16 -> [.., 400] uint8.  Everything here is exact in 32 bits: scales are powers of two."""
    x = rows[..., :LAT].float()
    blocks = x.reshape(*x.shape[:-1], LAT // BLOCK, BLOCK)
    amax = blocks.abs().amax(-1)
    finite = torch.isfinite(amax)
    m, e = torch.frexp(torch.where(finite, amax, torch.ones_like(amax)))      # amax = m 2^e, m in [0.5, 1): <= 6 2^(e-3) up to m = 0.75
    e = torch.where(amax > 0, e - 3 + (m > 0.75).int(), torch.full_like(e, MIN_E)).clamp(MIN_E, MAX_E)
    y = torch.where(finite[..., None], torch.ldexp(blocks, -e[..., None]), torch.zeros_like(blocks))
    a = y.abs()
    # to the nearest of the eight, ties to the one with an even code
    code = ((a > 0.25).int() + (a >= 0.75).int() + (a > 1.25).int() + (a >= 1.75).int() + (a > 2.5).int() + (a >= 3.5).int() + (a > 5.0).int())
    code = (code | (torch.signbit(y).int() << 3)).to(torch.uint8).reshape(*x.shape[:-1], LAT // 2, 2)
    scale = torch.where(finite, e + 127, torch.full_like(e, 255)).to(torch.uint8)
    pad = torch.zeros(*scale.shape[:-1], ROW - 388, dtype=torch.uint8, device=rows.device)
    return torch.cat([code[..., 0] | (code[..., 1] << 4), rows[..., LAT:].contiguous().view(torch.uint8), scale, pad], -1)


def _unpack(packed):
    """[.., 400] uint8 -> [.., 576] fp32"""
    levels = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device=packed.device)
    c = packed[..., :LAT // 2]
    v = levels[torch.stack([c & 15, c >> 4], -1).int()].reshape(*c.shape[:-1], LAT // BLOCK, BLOCK)
    b = packed[..., 384:388].int()
    s = torch.where(b == 255, torch.full_like(b, 0, dtype=torch.float32) * math.nan, torch.ldexp(torch.ones_like(b, dtype=torch.float32), b - 127))
    return torch.cat([(v * s[..., None]).flatten(-2), packed[..., 256:384].contiguous().view(torch.bfloat16).float()], -1)


def _unpack_exact(packed):
    """The same in 64 bits, by arithmetic on the fields of a code instead of a table."""
    c = packed[..., :LAT // 2]
    q = torch.stack([c % 16, c // 16], -1).flatten(-2).double()
    sign, mag = 1 - 2 * torch.floor(q / 8), q % 8
    ex, fr = torch.floor(mag / 2), mag % 2
    v = sign * torch.where(ex > 0, (1 + fr / 2) * torch.exp2(ex - 1), fr / 2)
    b = packed[..., 384:388].double()
    s = torch.where(b == 255, b * math.nan, torch.exp2(b - 127)).repeat_interleave(BLOCK, -1)
    return torch.cat([v * s, packed[..., 256:384].contiguous().view(torch.bfloat16).double()], -1)


# ---- inputs -------------------------------------------------------------------------------------------------------

def _gen(seed, name):
    return torch.Generator(device="cuda").manual_seed((seed * 1000003 + sum(ord(c) * 131 ** i for i, c in enumerate(name))) % (1 << 62))


def _randn(shape, g):
    return torch.randn(shape, generator=g, device="cuda")


def _latents(n, g):
    """Rows of a latent cache: channels of different widths, a few of them wide, as a trained projection leaves them."""
    width = torch.exp(0.4 * _randn((576,), g))
    width[torch.randperm(LAT, generator=g, device="cuda")[:8]] *= 4
    step = 1 << 18
    out = torch.empty((n, 576), dtype=torch.bfloat16, device="cuda")
    for i in range(0, n, step):
        out[i:i + step] = _randn((min(step, n - i), 576), g) * width
    return out


def _cache(n, g):
    step = 1 << 17
    out = torch.empty((n, ROW), dtype=torch.uint8, device="cuda")
    for i in range(0, n, step):
        out[i:i + step] = _pack(_latents(min(step, n - i), g))
    return out


def _lens(case, g):
    """Lengths of the sequences; the longest has Lk, the shortest `low` where the batch is ragged."""
    B, L = case["B"], case["Lk"]
    if not case["low"]:
        return None
    n = (case["low"] + torch.rand((B,), generator=g, device="cuda") ** 2 * (L - case["low"])).int().clamp(1, L)
    n[0] = L
    n[-1] = case["low"]
    return n


def _pages(case, lens, g):
    """(table [B, pages], rows of the pool): the pages of all sequences, in an order of their own."""
    B, L, ps = case["B"], case["Lk"], case["page"]
    per = -(-L // ps)
    used = (torch.full((B,), per, device="cuda") if lens is None else (lens.long() + ps - 1) // ps)
    have = torch.arange(per, device="cuda") < used[:, None]
    total = int(used.sum())
    table = torch.zeros((B, per), dtype=torch.int32, device="cuda")
    table[have] = torch.randperm(total, generator=g, device="cuda").int()
    return table, total * ps


def _selected(case, lens, g):
    """Index rows as a causal top-k leaves them: ascending positions, -1 behind them; half of what a row takes, its neighbours take too."""
    B, T, L, k = case["B"], case["T"], case["Lk"], case["k"]
    j = torch.arange(k, device="cuda")
    shared = torch.rand((1, 1, k), generator=g, device="cuda")
    idx = torch.empty((B, T, k), dtype=torch.int32, device="cuda")
    n_b = torch.full((B,), L, device="cuda") if lens is None else lens.long()
    step = max(1, (1 << 24) // (B * k))
    for t0 in range(0, T, step):
        t = torch.arange(t0, min(T, t0 + step), device="cuda")
        n = (n_b[:, None] - T + 1 + t)[..., None]                                          # what the row sees
        u = torch.where(j % 2 == 0, shared, torch.rand((B, t.numel(), k), generator=g, device="cuda"))
        lo, hi = j * n // k, (j + 1) * n // k
        pick = lo + (u * (hi - lo)).long().clamp(max=1 << 40).minimum(hi - lo - 1)
        idx[:, t0:t0 + step] = torch.where(n <= k, torch.where(j < n, j, -1), pick).int()
    return idx


def prepare(case, seed):
    g = _gen(seed, case["op"])
    B, T, L, op = case["B"], case["T"], case["Lk"], case["op"]
    lens = _lens(case, g)
    table, n_rows = _pages(case, lens, g) if case["page"] else (None, B * L)
    s = {"case": case, "lens": lens, "table": table, "n_rows": n_rows}
    if op == "rows":
        s["new"] = _latents(B * T, g).reshape(B, T, 576)
        s["kv4"] = torch.zeros((n_rows, ROW), dtype=torch.uint8, device="cuda")
        return s
    s["kv4"] = _cache(n_rows, g)
    if op == "evict":
        # what the counters hold after a while: a few heavy positions, many light ones, many that nothing ever selected
        w = torch.exp(2.5 * _randn((B, L), g)) * (torch.rand((B, L), generator=g, device="cuda") < 0.6)
        s["weight"] = w
        s["ik"] = _randn((n_rows, 128), g).to(torch.bfloat16)
        keep = case["keep"]
        if case["page"]:
            per = -(-keep // case["page"])
            s["dst_table"] = torch.randperm(B * per, generator=g, device="cuda").int().reshape(B, per)
            s["dst_rows"] = B * per * case["page"]
        else:
            s["dst_table"], s["dst_rows"] = None, B * keep
        s["dst_kv4"] = torch.zeros((s["dst_rows"], ROW), dtype=torch.uint8, device="cuda")
        s["dst_ik"] = torch.zeros((s["dst_rows"], 128), dtype=torch.bfloat16, device="cuda")
        return s
    s["Q"] = (1.5 * _randn((B, T, case["H"], 576), g)).to(torch.bfloat16)
    s["idx"] = _selected(case, lens, g)
    if op == "weight":
        s["lse"] = torch.cat([x[1] for x in _attn_parts(s, lse_only=True)], 1)
        s["weight"] = torch.rand((B, L), generator=g, device="cuda")
    return s


# ---- plain forms --------------------------------------------------------------------------------------------------

def _physical(s, pos, table=None, L=None):
    """Rows of the pool (or of the dense cache) of logical positions [B, ..]."""
    table, ps = (s["table"] if table is None else table), s["case"]["page"]
    b = torch.arange(pos.shape[0], device=pos.device).reshape(-1, *[1] * (pos.dim() - 1))
    if table is None:
        return b * (s["case"]["Lk"] if L is None else L) + pos
    return table.long()[b, pos // ps] * ps + pos % ps


def _positions(s):
    """Positions [B, T] that the new rows go to (negative: none), the last T of each sequence."""
    c = s["case"]
    n = torch.full((c["B"],), c["Lk"], device="cuda") if s["lens"] is None else s["lens"].long()
    return n[:, None] - c["T"] + torch.arange(c["T"], device="cuda")


def _attn_parts(s, lse_only=False):
    """Per run of query rows: (weights of the selected rows, the heads' mean [B,t,k]; log-sum-exps [B,t,H]; outputs [B,t,H,512]; the positions' weights [B,Lk])."""
    c, Q, idx = s["case"], s["Q"], s["idx"]
    B, T, H, k = c["B"], c["T"], c["H"], c["k"]
    whole = _unpack(s["kv4"]) if s["n_rows"] <= B * T * k else None
    step = max(1, (1 << 18) // (B * k))
    out = []
    for t0 in range(0, T, step):
        i = idx[:, t0:t0 + step]
        t = i.shape[1]
        rows = _physical(s, i.clamp(min=0).long()).reshape(-1)
        kv = (_unpack(s["kv4"][rows]) if whole is None else whole[rows]).reshape(B * t, k, 576)
        z = torch.bmm(Q[:, t0:t0 + step].reshape(B * t, H, 576).float(), kv.transpose(1, 2).contiguous()) * SCALE
        z = torch.where((i >= 0).reshape(B * t, 1, k), z, torch.full_like(z, -math.inf))
        m = z.amax(-1, keepdim=True)
        m = torch.where(torch.isfinite(m), m, torch.zeros_like(m))
        p = torch.exp(z - m)
        l = p.sum(-1, keepdim=True)
        lse = (m + torch.log(l)).reshape(B, t, H)
        p = torch.where(l > 0, p / l, torch.zeros_like(p))
        O = None if lse_only else torch.bmm(p, kv[..., :LAT].contiguous()).to(torch.bfloat16).reshape(B, t, H, LAT)
        got = add = None
        if c["op"] == "weight" and not lse_only:
            got = p.reshape(B, t, H, k).mean(2)
            at = torch.zeros((B, t, c["Lk"]), device="cuda").scatter_add_(2, i.clamp(min=0).long(), torch.where(i >= 0, got, torch.zeros_like(got)))
            add = at.sum(1, dtype=torch.float64)
        out.append((got, lse, O, add))
    return out


def _plain(s):
    c, op = s["case"], s["case"]["op"]
    if op == "rows":
        pos = _positions(s)
        there = pos >= 0
        rows = _physical(s, pos.clamp(min=0))
        s["kv4"][rows[there]] = _pack(s["new"][there])
        back = _unpack(s["kv4"][rows]).to(torch.bfloat16)
        return torch.where(there[..., None], back, torch.zeros_like(back))
    if op == "attn":
        parts = _attn_parts(s)
        return {"O": torch.cat([x[2] for x in parts], 1), "lse": torch.cat([x[1] for x in parts], 1)}
    if op == "weight":
        parts = _attn_parts(s)
        p = torch.cat([x[0] for x in parts], 1)
        w = s["weight"].double() + sum(x[3] for x in parts)
        return {"probs": p, "weight": w.float()}
    return _evict(s, s["weight"])


def _evict(s, weight):
    c, B, L, n_keep = s["case"], s["case"]["B"], s["case"]["Lk"], s["case"]["keep"]
    n = (torch.full((B,), L, device="cuda") if s["lens"] is None else s["lens"].long())[:, None]
    pos = torch.arange(L, device="cuda")
    w = torch.where((pos < c["first"]) | (pos >= n - c["recent"]), torch.full_like(weight, math.inf), weight)
    w = torch.where(pos < n, w, torch.full_like(weight, -math.inf))
    best = torch.sort(w, dim=1, descending=True, stable=True)[1][:, :n_keep]
    best = torch.where(torch.arange(n_keep, device="cuda") < n, best, L)
    keep = torch.sort(best, dim=1)[0]
    there = keep < L
    keep = torch.where(there, keep, -1)
    src = _physical(s, keep.clamp(min=0))[there]
    dst = _physical(s, torch.arange(n_keep, device="cuda").expand(B, n_keep), s["dst_table"], n_keep)[there]
    s["dst_kv4"][dst] = s["kv4"][src]
    s["dst_ik"][dst] = s["ik"][src]
    kept = torch.where(there, weight.gather(1, keep.clamp(min=0)), torch.zeros((), device="cuda", dtype=weight.dtype))
    return {"keep": keep.int(), "lens": n[:, 0].clamp(max=n_keep).int(), "weight": kept, "kv4": s["dst_kv4"], "ik": s["dst_ik"]}


# ---- the framework's calls ----------------------------------------------------------------------------------------

def _own(s):
    import paper_2603_12201_amd as ic
    c, op = s["case"], s["case"]["op"]
    B, T, L, ps = c["B"], c["T"], c["Lk"], c["page"]
    pc = ic.paged_cache(s["lens"], s["table"], ps) if s["lens"] is not None or ps else None
    kv4 = s["kv4"] if ps else s["kv4"].view(B, L, ROW)
    if op == "rows":
        ic.kv4_write(s["new"], kv4, pos0=L - T, Lk=L, pc=pc)
        return ic.kv4_read(kv4, B, T, pos0=L - T, Lk=L, pc=pc)
    if op == "attn":
        O, lse = ic.sparse_attn_kv4(s["Q"], kv4, s["idx"], SCALE, Lk=L, pc=pc, want_lse=True)
        return {"O": O, "lse": lse}
    if op == "weight":
        p = ic.attn_probs_kv4(s["Q"], kv4, s["idx"], SCALE, s["lse"], Lk=L, pc=pc)
        return {"probs": p, "weight": ic.attn_weight_add(p, s["idx"], s["weight"], out=torch.empty_like(s["weight"]))}
    keep, lens, kept = ic.evict_keep(s["weight"], c["keep"], n_first=c["first"], n_recent=c["recent"], seq_lens=s["lens"])
    dst_pc = ic.paged_cache(None, s["dst_table"], ps) if ps else None
    d_kv4, ik, d_ik = s["dst_kv4"], s["ik"], s["dst_ik"]
    if not ps:
        d_kv4, ik, d_ik = d_kv4.view(B, c["keep"], ROW), ik.view(B, L, 128), d_ik.view(B, c["keep"], 128)
    ic.cache_compact([(kv4, d_kv4), (ik, d_ik)], keep, L, src_pc=ic.paged_cache(None, s["table"], ps) if ps else None, dst_pc=dst_pc)
    return {"keep": keep, "lens": lens, "weight": kept, "kv4": s["dst_kv4"], "ik": s["dst_ik"]}


def run(state):
    return _own(state) if own else _plain(state)


# ---- what a pass cannot do without --------------------------------------------------------------------------------

def work(case):
    B, T, L, op = case["B"], case["T"], case["Lk"], case["op"]
    if op == "rows":
        return {"bytes": B * T * (1152 + ROW + ROW + 1152), "flops": 0}
    if op == "evict":
        keep = min(L, case["keep"])
        return {"bytes": B * L * 4 + B * keep * (4 + 4 + 2 * (ROW + 256)), "flops": 0}
    H, k = case["H"], case["k"]
    per = min(k, L) if T == 1 else k
    held = sum(min(per, L - T + 1 + t) for t in range(T))           # rows selected by the queries of a sequence
    once = min(L, held) * ROW                                       # a row that several queries select is read once
    if op == "attn":
        return {"bytes": B * (once + T * (H * 576 * 2 + k * 4 + H * LAT * 2 + H * 4)), "flops": 2 * B * held * H * (576 + LAT)}
    return {"bytes": B * (once + T * (H * 576 * 2 + 2 * k * 4 + H * 4) + L * 8), "flops": 2 * B * held * H * 576}


# ---- from the definitions, in 64 bits -----------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    op, B, T = case["op"], case["B"], case["T"]
    if op == "rows":
        pos = _positions(s)
        x = s["new"].double()
        out = x.clone()
        levels = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device="cuda", dtype=torch.float64)
        for j in range(0, LAT, BLOCK):
            part = x[..., j:j + BLOCK]
            top = part.abs().amax(-1, keepdim=True).clamp(min=2.0 ** -200)
            e = torch.floor(torch.log2(top / 6))
            e = torch.where(top > 6 * torch.exp2(e), e + 1, e).clamp(MIN_E, MAX_E)
            y = part.abs() / torch.exp2(e)
            hi = torch.searchsorted(levels, y.clamp(max=6.0)).clamp(max=7)
            lo = (hi - 1).clamp(min=0)
            dl, dh = y - levels[lo], levels[hi] - y
            pick = torch.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
            out[..., j:j + BLOCK] = torch.sign(part) * levels[pick] * torch.exp2(e)
        return torch.where((pos >= 0)[..., None], out, torch.zeros_like(out))
    if op == "evict":
        return None
    H, k = case["H"], case["k"]
    O = torch.zeros((B, T, H, LAT), dtype=torch.float64, device="cuda") if op == "attn" else None
    lse = torch.full((B, T, H), -math.inf, dtype=torch.float64, device="cuda")
    probs = torch.zeros((B, T, k), dtype=torch.float64, device="cuda") if op == "weight" else None
    w = s["weight"].double() if op == "weight" else None
    step = max(1, (1 << 17) // k)
    for b in range(B):
        for t0 in range(0, T, step):
            i = s["idx"][b, t0:t0 + step].long()
            t = i.shape[0]
            if case["page"]:
                at = s["table"][b].long()[i.clamp(min=0) // case["page"]] * case["page"] + i.clamp(min=0) % case["page"]
            else:
                at = b * case["Lk"] + i.clamp(min=0)
            kv = _unpack_exact(s["kv4"][at.reshape(-1)]).reshape(t, k, 576)
            z = torch.bmm(s["Q"][b, t0:t0 + step].double(), kv.transpose(1, 2).contiguous()) * SCALE
            z = z.masked_fill((i < 0)[:, None, :], -math.inf)
            lse[b, t0:t0 + step] = torch.logsumexp(z, -1)
            # a row's own distribution; the weights go by the log-sum-exps they are given
            norm = lse[b, t0:t0 + step] if op == "attn" else s["lse"][b, t0:t0 + step].double()
            p = torch.nan_to_num(torch.exp(z - norm[..., None]), nan=0.0)
            if op == "attn":
                O[b, t0:t0 + step] = torch.bmm(p, kv[..., :LAT].contiguous())
            else:
                probs[b, t0:t0 + step] = p.mean(1)
                w[b].scatter_add_(0, i.clamp(min=0).flatten(), torch.where(i >= 0, p.mean(1), torch.zeros_like(p[:, 0])).flatten())
    return {"O": O, "lse": lse} if op == "attn" else {"probs": probs, "weight": w}
