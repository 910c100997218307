"""The operators around a paged cache of keys and values, as a list of measurable cases.

``rope`` turns heads by their positions, ``kv_append`` writes the new tokens' keys and values to the pages of a cache (keys and
queries turned on the way), ``attn_paged`` is the attention of the new tokens over it, ``kv_free`` / ``kv_fork`` / ``kv_compact`` keep
the pages.  A cache is [pages][key heads][page size][d] (or another order of the middle two: a strided view); a packed batch of
sequences is described by ``q_start`` [S+1] (first new token of each), ``kv_len`` [S] (tokens in the cache, the new ones among them) and
``table`` [S][entries] (the pages of each sequence).  ``run`` has each in its plain form, elementary torch operations in 32 bits (angles
in 64), and as the library's call; ``exact`` has the definitions in 64 bits.

Ranges:  attention 1 ... 256 sequences of 1 ... 65536 tokens, 1 ... 4096 new ones, 2 ... 64 heads on 1 ... 16 key heads, d 64 and 128, pages
of 16 ... 256 tokens, caches in 16 and 8 bits; rope and append 1 ... 32768 tokens; caches of 64 ... 4096 pages.
"""
from __future__ import annotations

import math

import torch

own = False

TYPE = {"fp16": torch.float16, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
BYTES = {"fp16": 2, "bf16": 2, "e4m3": 1}


def _attn(name, S, q_lo, q_hi, kv_lo, kv_hi, H, Hkv, d, dtype, cache, page, causal=True, order="head", pad=0):
    return {"name": name, "op": "attn", "S": S, "q_lo": q_lo, "q_hi": q_hi, "kv_lo": kv_lo, "kv_hi": kv_hi, "H": H, "Hkv": Hkv, "d": d, "dtype": dtype,
            "cache": cache, "page": page, "causal": causal, "order": order, "pad": pad}


def _append(name, S, q_lo, q_hi, kv_hi, H, Hkv, d, rot, layout, dtype, cache, page, pad=0):
    return {"name": name, "op": "append", "S": S, "q_lo": q_lo, "q_hi": q_hi, "kv_hi": kv_hi, "H": H, "Hkv": Hkv, "d": d, "rot": rot, "layout": layout,
            "dtype": dtype, "cache": cache, "page": page, "pad": pad}


def _rope(name, B, H, N, d, rot, layout, dtype, first, inverse, packed):
    return {"name": name, "op": "rope", "B": B, "H": H, "N": N, "d": d, "rot": rot, "layout": layout, "dtype": dtype, "first": first,
            "inverse": inverse, "packed": packed}


def _pages(name, op, layers, pages, page, Hkv, d, dtype, rows, fan):
    return {"name": name, "op": op, "layers": layers, "pages": pages, "page": page, "Hkv": Hkv, "d": d, "dtype": dtype, "rows": rows, "fan": fan}


def listed():
    return [
        # One sequence at the start of its answer, two heads: launches and latency.
        _attn("attn_step_smallest", 1, 1, 1, 128, 128, 2, 2, 64, "fp16", "fp16", 16),
        # A server's step: a token for each of 64 sequences of all lengths, four query heads on a key head.
        _attn("attn_step_batch", 64, 1, 1, 300, 16384, 32, 8, 128, "bf16", "bf16", 16),
        # Few very long sequences over a cache in 8 bits, large pages, eight query heads on a key head.
        _attn("attn_step_long_e4m3", 3, 1, 1, 40000, 65536, 64, 8, 128, "bf16", "e4m3", 64),
        # Drafted tokens being checked: several new tokens a sequence, as many key heads as query heads, d = 64, tokens before heads.
        _attn("attn_draft", 33, 3, 7, 200, 2309, 16, 16, 64, "fp16", "fp16", 32, order="token"),
        # A long prompt being read in chunks: 4096 new tokens at the end of 16384.
        _attn("attn_chunk", 1, 4096, 4096, 16384, 16384, 32, 8, 128, "bf16", "bf16", 64),
        # Short chunks of odd lengths beside each other, none with anything cached before it or with much.
        _attn("attn_chunks_ragged", 12, 1, 777, 900, 4001, 16, 4, 128, "fp16", "fp16", 16),
        # A step's tokens go to the cache: a latency.
        _append("append_step", 16, 1, 1, 16384, 32, 8, 128, 128, "half", "bf16", "bf16", 16),
        # Prompts of odd lengths go to a cache in 8 bits; half of the head is turned, pairs side by side.
        _append("append_chunk_e4m3", 5, 900, 4001, 16384, 32, 8, 128, 64, "interleaved", "fp16", "e4m3", 64),
        # Q of a training or prefill step in the attention call's own layout.
        _rope("rope_forward", 4, 16, 4096, 128, 128, "half", "bf16", 0, False, False),
        # The gradient of a packed slice, at far positions of a stretched context, part of the head.
        _rope("rope_gradient_far", 1, 32, 2309, 128, 96, "interleaved", "fp16", 1000003, True, True),
        # Several continuations of each of a few sequences: the old ones go, new ones share the full pages and copy the last.
        _pages("pages_fork", "fork", 8, 1024, 32, 8, 128, "bf16", 16, 7),
        # A cache with holes all over moves together.
        _pages("pages_compact", "compact", 8, 1024, 32, 8, 128, "bf16", 48, 0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges above; sizes spread over their logarithm."""
    kind = rng.choice(("step", "step", "chunk", "chunk", "append", "rope", "fork", "compact"))
    d, dtype = rng.choice((64, 128)), rng.choice(("fp16", "bf16"))
    cache = rng.choice((dtype, dtype, "e4m3"))
    page = rng.choice((16, 32, 64, 128, 256))
    Hkv = rng.choice((1, 2, 4, 8, 16))
    H = Hkv * rng.choice([g for g in (1, 2, 3, 4, 5, 7, 8, 16) if g * Hkv <= 64])
    order, pad = rng.choice(("head", "token")), rng.choice((0, 0, 1, 13))
    if kind == "step":
        S = _log_int(rng, 1, 256)
        hi = _log_int(rng, 1, max(1, min(65536, 24000000 // (S * Hkv * d // 16))))
        q = rng.choice((1, 1, 1, rng.randint(2, 9)))
        return _attn("", S, 1, q, max(q, hi // rng.choice((1, 3, 40))), max(q, hi), H, Hkv, d, dtype, cache, page, rng.random() < 0.9, order, pad)
    if kind == "chunk":
        q = _log_int(rng, 10, 4096)
        hi = max(q, _log_int(rng, q, 16384))
        S = _log_int(rng, 1, 24)
        S = max(1, min(S, int(1.5e9 // (q * hi * H))))
        if q * hi * H > 1.5e9:
            hi = max(q, int(1.5e9 // (q * H)))
        return _attn("", S, max(1, q // rng.choice((1, 4, 50))), q, max(1, hi // rng.choice((1, 2, 10))), hi, H, Hkv, d, dtype, cache, page, rng.random() < 0.8, order, pad)
    rot = rng.choice((d, d, d // 2, d - 16))
    layout = rng.choice(("half", "interleaved"))
    if kind == "append":
        S = _log_int(rng, 1, 64)
        q = _log_int(rng, 1, 8192 // S)
        return _append("", S, max(1, q // rng.choice((1, 3))), q, _log_int(rng, q, 16384), H, Hkv, d, rot, layout, dtype, cache, page, pad)
    if kind == "rope":
        N = _log_int(rng, 1, 16384)
        B = _log_int(rng, 1, max(1, 32768 // N))
        return _rope("", 1 if N > 8192 else B, min(H, 32), N, d, rot, layout, dtype, rng.choice((0, 17, 4000000)), rng.random() < 0.5, rng.random() < 0.5)
    layers, pages = _log_int(rng, 1, 16), _log_int(rng, 64, 4096)
    page = min(page, 64)
    while layers * pages * page * Hkv * d > 6e8:
        pages = max(64, pages // 2)
        layers = max(1, layers // 2)
    return _pages("", kind, layers, pages, page, Hkv, d, rng.choice(("fp16", "bf16", "e4m3")), _log_int(rng, 2, 64), rng.randint(1, 9))


# ---------------------------------------------------------------- inputs

def _normal(shape, dtype, gen, factor=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * factor).to(TYPE[dtype])


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _lengths(c):
    """New tokens and all tokens of each sequence, spread over their logarithm; one of each is the longest.  They belong to the case: every seed has
    the same ones."""
    gen = torch.Generator().manual_seed(c["S"])

    def spread(lo, hi):
        u = torch.rand(c["S"], generator=gen, dtype=torch.float64)
        u[c["S"] // 3] = 1.0
        return torch.exp(math.log(lo) + u * (math.log(hi) - math.log(lo))).round().long().clamp(lo, hi)

    q_len = spread(c["q_lo"], c["q_hi"])
    return q_len, torch.maximum(spread(c.get("kv_lo", 1), c["kv_hi"]), q_len)


def _held(c):
    """Tokens of each row that holds pages; together they fill about 6 of 10 pages, the continuations of a fork among them."""
    gen = torch.Generator().manual_seed(c["rows"])
    held = max(c["rows"], c["pages"] * 6 // 10 - (c["rows"] * c["fan"] if c["op"] == "fork" else 0))
    lens = torch.rand(c["rows"], generator=gen, dtype=torch.float64) + 0.05
    return (lens / lens.sum() * (held - c["rows"]) * c["page"]).long().clamp(min=1)


def _cache(pages, Hkv, page, d, dtype, order, gen, layers=None):
    """A cache of such values as a model's keys have, [pages][heads][tokens][d] whichever of heads and tokens lies further out."""
    lead = () if layers is None else (layers,)
    if order == "token":
        return _normal(lead + (pages, page, Hkv, d), dtype, gen).transpose(-3, -2)
    return _normal(lead + (pages, Hkv, page, d), dtype, gen)


def _frequencies(rot, stretched):
    """Radians per position of each pair; `stretched`: the slow ones by a factor of 8 (a context longer than the trained 4096), and an amplitude."""
    f = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    if not stretched:
        return f.cuda(), 1.0
    keep = ((4096 * f / (2 * math.pi) - 1) / 31).clamp(0, 1)
    return (f * keep + f / 8 * (1 - keep)).cuda(), 0.1 * math.log(8.0) + 1


def prepare(case, seed):
    gen, host = torch.Generator(device="cuda"), torch.Generator()
    gen.manual_seed(int(seed))
    host.manual_seed(int(seed))
    c = case
    if c["op"] in ("attn", "append"):
        S, page, Hkv, H, d = c["S"], c["page"], c["Hkv"], c["H"], c["d"]
        q_len, kv_len = _lengths(c)
        q_start = torch.cat((torch.zeros(1, dtype=torch.long), q_len.cumsum(0)))
        used = -(-kv_len // page)
        entries, total = int(used.max()), int(used.sum())
        pages = total + 3
        ids = torch.randperm(pages, generator=host)[:total]          # pages in no order, as after hours of serving
        table = torch.full((S, entries), -1, dtype=torch.int32)
        table[torch.arange(entries)[None] < used[:, None]] = ids.int()
        T = int(q_start[-1]) + c["pad"]
        s = {"case": c, "q_start": q_start.int().cuda(), "kv_len": kv_len.int().cuda(), "table": table.cuda(), "max_q": int(q_len.max()), "max_kv": int(kv_len.max()),
             "k_scale": None, "v_scale": None}
        order = c.get("order", "head")
        s["k_cache"], s["v_cache"] = (_cache(pages, Hkv, page, d, c["cache"], order, gen) for _ in "kv")
        if c["cache"] == "e4m3":
            s["k_scale"], s["v_scale"] = (torch.rand(Hkv, generator=gen, device="cuda") * 0.5 + 0.5 for _ in "kv")
        if c["op"] == "attn":
            s["q"] = _normal((T, H, d), c["dtype"], gen)
            s["o"] = torch.zeros((T, H, d), dtype=TYPE[c["dtype"]], device="cuda")
            s["lse"] = torch.zeros((T, H), device="cuda")
            s["scale"] = 1.0 / math.sqrt(d)
        else:
            qkv = _normal((T, H + 2 * Hkv, d), c["dtype"], gen)      # one projection's result
            s["q"], s["k"], s["v"] = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
            s["q_out"] = torch.zeros((T, H, d), dtype=TYPE[c["dtype"]], device="cuda")
            s["freq"], s["amplitude"] = _frequencies(c["rot"], False)
        return s
    if c["op"] == "rope":
        B, H, N, d = c["B"], c["H"], c["N"], c["d"]
        if c["packed"]:
            x = _normal((B, N, H, d), c["dtype"], gen).transpose(1, 2)
            y = torch.empty((B, N, H, d), dtype=TYPE[c["dtype"]], device="cuda").transpose(1, 2)
        else:
            x = _normal((B, H, N, d), c["dtype"], gen)
            y = torch.empty_like(x)
        pos = (torch.randint(0, 1 + c["first"] // 2, (B, 1), generator=host) + c["first"] + torch.arange(N)).int().cuda()
        f, a = _frequencies(c["rot"], c["first"] > 4096)
        return {"case": c, "x": x, "y": y, "pos": pos, "freq": f, "amplitude": a}
    # fork, compact: a cache of `layers` layers
    rows, pages, page, fan = c["rows"], c["pages"], c["page"], c["fan"]
    s = {"case": c}
    s["k_cache"], s["v_cache"] = (_cache(pages, c["Hkv"], page, c["d"], c["dtype"], "head", gen, c["layers"]) for _ in "kv")
    children = rows * fan if c["op"] == "fork" else 0
    lens = _held(c)
    used = -(-lens // page)                                          # (together at most `pages`)
    width = int(used.max()) + 2
    table = torch.full((rows + children, width), -1, dtype=torch.int32)
    table[:rows][torch.arange(width)[None] < used[:, None]] = torch.randperm(pages, generator=host)[:int(used.sum())].int()
    ref = torch.zeros(pages, dtype=torch.int32)
    ref[table[table >= 0].long()] = 1
    kv_len = torch.zeros(rows + children, dtype=torch.int32)
    kv_len[:rows] = lens.int()
    s |= {"table0": table.cuda(), "ref0": ref.cuda(), "len0": kv_len.cuda(), "missing": _ints([0])}
    s |= {"table": s["table0"].clone(), "ref": s["ref0"].clone(), "kv_len": s["len0"].clone()}
    if c["op"] == "fork":
        s["src"] = _ints(torch.arange(rows).repeat_interleave(fan).tolist())
        s["dst"] = _ints((rows + torch.randperm(children, generator=host)).tolist())
    return s


# ---------------------------------------------------------------- plain forms

def _tokens(s):
    """Sequence and position of every token of the batch."""
    q_start, kv_len = s["q_start"].long(), s["kv_len"].long()
    tok = torch.arange(s["q"].shape[0] - s["case"]["pad"], device="cuda")
    seq = (q_start[1:-1][None] <= tok[:, None]).sum(1)
    return tok, seq, kv_len[seq] - (q_start[seq + 1] - tok)


def _turn(x, pos, freq, amplitude, rot, layout, inverse):
    """x [..., d] in 32 bits, turned by pos (broadcast over x without its last dimension)."""
    angle = pos.double()[..., None] * freq
    cos, sin = (angle.cos() * amplitude).float(), (angle.sin() * (-amplitude if inverse else amplitude)).float()
    if layout == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    else:
        a, b = x[..., :rot:2], x[..., 1:rot:2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    return torch.cat((turned, x[..., rot:]), -1)


def _plain_attn(s):
    c = s["case"]
    S, H, Hkv, d, page, max_q, n = c["S"], c["H"], c["Hkv"], c["d"], c["page"], s["max_q"], s["max_kv"]
    G = H // Hkv
    q_start, kv_len = s["q_start"].long(), s["kv_len"].long()
    q_len = q_start[1:] - q_start[:-1]
    i, j = torch.arange(max_q, device="cuda"), torch.arange(n, device="cuda")
    here = i[None] < q_len[:, None]
    tok = (q_start[:-1, None] + i[None])[here]
    q = torch.zeros((S, max_q, H, d), device="cuda")
    q[here] = s["q"][tok].float()
    q = q.view(S, max_q, Hkv, G, d).transpose(1, 2).reshape(S, Hkv, max_q * G, d)
    at = s["table"].long()[:, j // page]
    valid = (j[None] < kv_len[:, None]) & (at >= 0)
    at = at.clamp(min=0)

    def rows(cache, scale):
        x = cache.view(torch.uint8)[at, :, j % page].view(cache.dtype).float() if cache.dtype == TYPE["e4m3"] else cache[at, :, j % page].float()
        x = torch.where(valid[..., None, None], x, 0.0)
        return x if scale is None else x * scale[:, None]

    k = rows(s["k_cache"], s["k_scale"]).permute(0, 2, 3, 1).contiguous()
    scores = torch.matmul(q, k).mul_(s["scale"])
    del k
    seen = valid[:, None, :].expand(S, max_q, n)
    if c["causal"]:
        seen = seen & (j <= (kv_len - q_len)[:, None, None] + i[:, None])
    scores.masked_fill_(~seen.repeat_interleave(G, 1)[:, None], -math.inf)
    top = scores.amax(-1, keepdim=True).clamp(min=-3e38)
    scores.sub_(top).exp_()
    total = scores.sum(-1, keepdim=True)
    v = rows(s["v_cache"], s["v_scale"]).transpose(1, 2).contiguous()
    o = torch.matmul(scores, v) / total
    lse = (top + total.log())[..., 0]
    s["o"][tok] = o.view(S, Hkv, max_q, G, d).transpose(1, 2).reshape(S, max_q, H, d)[here].to(s["o"].dtype)
    s["lse"][tok] = lse.view(S, Hkv, max_q, G).transpose(1, 2).reshape(S, max_q, H)[here]
    return s["o"], s["lse"]


def _plain_append(s):
    c = s["case"]
    tok, seq, pos = _tokens(s)
    where = s["table"].long()[seq, pos // c["page"]]
    turned = [_turn(s[x][tok].float(), pos[:, None], s["freq"], s["amplitude"], c["rot"], c["layout"], False) for x in "qk"]
    s["q_out"][tok] = turned[0].to(s["q_out"].dtype)
    k, v = turned[1], s["v"][tok].float()
    if c["cache"] == "e4m3":
        k, v = ((x / y[:, None]).clamp(-448, 448).to(TYPE["e4m3"]).view(torch.uint8) for x, y in ((k, s["k_scale"]), (v, s["v_scale"])))
        s["k_cache"].view(torch.uint8)[where, :, pos % c["page"]] = k
        s["v_cache"].view(torch.uint8)[where, :, pos % c["page"]] = v
    else:
        s["k_cache"][where, :, pos % c["page"]] = k.to(s["k_cache"].dtype)
        s["v_cache"][where, :, pos % c["page"]] = v.to(s["v_cache"].dtype)
    return s["q_out"], s["k_cache"], s["v_cache"]


def _plain_rope(s):
    c = s["case"]
    x = s["x"]
    s["y"].copy_(_turn(x.float(), s["pos"][:, None], s["freq"], s["amplitude"], c["rot"], c["layout"], c["inverse"]).to(x.dtype))
    return s["y"]


def _bytes_of(cache):
    return cache.view(torch.uint8) if cache.dtype == TYPE["e4m3"] else cache


def _plain_fork(s):
    page, table, ref, kv_len = s["case"]["page"], s["table"], s["ref"], s["kv_len"]
    src, dst = s["src"].long(), s["dst"].long()
    at = torch.arange(table.shape[1], device="cuda")
    # the rows that go
    old = table[dst]
    held = (at < ((kv_len[dst] + page - 1) // page)[:, None]) & (old >= 0)
    ref.index_add_(0, old[held].long(), torch.full((1,), -1, dtype=torch.int32, device="cuda").expand(int(held.sum())))
    table[dst] = -1
    kv_len[dst] = 0
    # the rows that come
    length = kv_len[src]
    full, part = length // page, length % page > 0
    shared = torch.where(at < full[:, None], table[src], -1)
    taken = shared[shared >= 0].long()
    ref.index_add_(0, taken, torch.ones_like(taken, dtype=torch.int32))
    free = (ref == 0).nonzero()[:, 0]
    rank = part.long().cumsum(0) - 1
    got = part & (rank < len(free))
    new, from_ = free[rank[got]], table[src[got], full[got].long()].long()
    shared[got, full[got].long()] = new.int()
    table[dst] = shared
    ref[new] = 1
    kv_len[dst] = length
    s["missing"].copy_((part & ~got).sum())
    for cache in (_bytes_of(s["k_cache"]), _bytes_of(s["v_cache"])):
        cache[:, new] = cache[:, from_]


def _plain_compact(s):
    page, table, ref, kv_len = s["case"]["page"], s["table"], s["ref"], s["kv_len"]
    live = ref > 0
    n = int(live.sum())
    to, from_ = (~live[:n]).nonzero()[:, 0], live[n:].nonzero()[:, 0] + n
    at = torch.arange(len(ref), device="cuda")
    at[from_] = to
    held = (torch.arange(table.shape[1], device="cuda") < ((kv_len + page - 1) // page)[:, None]) & (table >= 0)
    table.copy_(torch.where(held, at[table.long().clamp(min=0)].int(), table))
    ref[to] = ref[from_]
    ref[from_] = 0
    for cache in (_bytes_of(s["k_cache"]), _bytes_of(s["v_cache"])):
        cache[:, to] = cache[:, from_]


# ---------------------------------------------------------------- the pass

def run(s):
    c = s["case"]
    if own:
        return _own(s)
    if c["op"] == "attn":
        return _plain_attn(s)
    if c["op"] == "append":
        return _plain_append(s)
    if c["op"] == "rope":
        return _plain_rope(s)
    if c["op"] == "fork":
        _plain_fork(s)
    else:
        s["table"].copy_(s["table0"])            # the same holes in every pass
        s["ref"].copy_(s["ref0"])
        _plain_compact(s)
    return s["k_cache"], s["v_cache"], s["table"], s["ref"], s["kv_len"], s["missing"]


def _own(s):
    from paper_2510_14719_amd import kv_cache as kv
    c = s["case"]
    layout = kv.HALF if c.get("layout") == "half" else kv.INTERLEAVED
    if c["op"] == "attn":
        if "workspace" not in s:                 # kept by the program, like the output buffers
            n = kv.attn_paged_workspace(s["q"], s["k_cache"], c["S"], s["max_q"], s["max_kv"])
            s["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda")
        kv.attn_paged(s["q"], s["k_cache"], s["v_cache"], s["q_start"], s["kv_len"], s["table"], s["o"], s["lse"], s["max_q"], s["max_kv"], s["scale"], c["causal"],
                      k_scale=s["k_scale"], v_scale=s["v_scale"], workspace=s["workspace"])
        return s["o"], s["lse"]
    if c["op"] == "append":
        kv.kv_append(s["k"], s["v"], s["k_cache"], s["v_cache"], s["q_start"], s["kv_len"], s["table"], s["max_q"], s["max_kv"], q=s["q"], q_out=s["q_out"],
                     freq=s["freq"], layout=layout, amplitude=s["amplitude"], k_scale=s["k_scale"], v_scale=s["v_scale"])
        return s["q_out"], s["k_cache"], s["v_cache"]
    if c["op"] == "rope":
        kv.rope(s["x"], s["y"], s["freq"], s["pos"], layout=layout, amplitude=s["amplitude"], inverse=c["inverse"])
        return s["y"]
    if c["op"] == "fork":
        kv.kv_free(s["ref"], s["table"], s["kv_len"], s["dst"], c["page"])
        kv.kv_fork(s["k_cache"], s["v_cache"], s["ref"], s["table"], s["kv_len"], s["src"], s["dst"], s["missing"])
    else:
        if "workspace" not in s:
            s["workspace"] = torch.empty(kv.kv_compact_workspace(c["pages"]), dtype=torch.uint8, device="cuda")
        s["table"].copy_(s["table0"])
        s["ref"].copy_(s["ref0"])
        kv.kv_compact(s["k_cache"], s["v_cache"], s["ref"], s["table"], s["kv_len"], s["workspace"])
    return s["k_cache"], s["v_cache"], s["table"], s["ref"], s["kv_len"], s["missing"]


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    c = case
    if c["op"] == "attn":
        q, n = (x.double() for x in _lengths(c))
        pairs = c["H"] * float((q * (n - (q - 1) / 2 if c["causal"] else n)).sum())
        return {"bytes": float(n.sum()) * 2 * c["Hkv"] * c["d"] * BYTES[c["cache"]] + float(q.sum()) * c["H"] * (4 * c["d"] + 4), "flops": 4.0 * pairs * c["d"]}
    if c["op"] == "append":
        tokens = float(_lengths(c)[0].sum())
        return {"bytes": tokens * c["d"] * (4 * c["H"] + 2 * c["Hkv"] * (2 + BYTES[c["cache"]])), "flops": tokens * 3.0 * c["rot"] * (c["H"] + c["Hkv"])}
    if c["op"] == "rope":
        rows = c["B"] * c["H"] * c["N"]
        return {"bytes": rows * 4.0 * c["d"], "flops": rows * 3.0 * c["rot"]}
    one = 2 * c["layers"] * c["Hkv"] * c["page"] * c["d"] * BYTES[c["dtype"]]
    lens = _held(c)
    held = int((-(-lens // c["page"])).sum())
    moved = int((lens % c["page"] > 0).sum()) * c["fan"] if c["op"] == "fork" else held * (1 - held / c["pages"])     # (the latter as is expected)
    return {"bytes": 2.0 * moved * one + 8 * c["pages"], "flops": 0}


# ---------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    c = case
    if c["op"] == "attn":
        H, Hkv, d, page = c["H"], c["Hkv"], c["d"], c["page"]
        G = H // Hkv
        o, lse = s["o"].double(), s["lse"].double()
        first, lens, table = s["q_start"].tolist(), s["kv_len"].tolist(), s["table"].long()
        for b in range(c["S"]):
            n, m = lens[b], first[b + 1] - first[b]
            ids = table[b, :-(-n // page)]
            for h in range(Hkv):
                k, v = ((s[x + "_cache"][:, h].view(torch.uint8)[ids].view(s[x + "_cache"].dtype) if c["cache"] == "e4m3" else s[x + "_cache"][:, h][ids])
                        .reshape(-1, d)[:n].double() * (1.0 if s[x + "_scale"] is None else s[x + "_scale"][h].double()) for x in "kv")
                step = max(1, int(2e9 // (8 * G * n)))
                for i in range(0, m, step):
                    e = min(m, i + step)
                    q = s["q"][first[b] + i:first[b] + e, h * G:(h + 1) * G].double().reshape(-1, d)
                    w = (q @ k.T) / math.sqrt(d)
                    if c["causal"]:
                        last = torch.arange(i, e, device="cuda").repeat_interleave(G) + n - m
                        w[torch.arange(n, device="cuda")[None] > last[:, None]] = -math.inf
                    z = torch.logsumexp(w, 1)
                    o[first[b] + i:first[b] + e, h * G:(h + 1) * G] = (torch.exp(w - z[:, None]) @ v).view(-1, G, d)
                    lse[first[b] + i:first[b] + e, h * G:(h + 1) * G] = z.view(-1, G)
        return o, lse
    if c["op"] in ("append", "rope"):
        def turned(x, pos, sign):
            x = x.double()
            z = torch.polar(torch.full_like(s["freq"], s["amplitude"]), torch.zeros_like(s["freq"])) * torch.exp(1j * sign * pos.double()[..., None] * s["freq"])
            r, y = c["rot"], x.clone()
            pairs = (slice(0, r // 2), slice(r // 2, r)) if c["layout"] == "half" else (slice(0, r, 2), slice(1, r, 2))
            w = torch.complex(x[..., pairs[0]], x[..., pairs[1]]) * z
            y[..., pairs[0]], y[..., pairs[1]] = w.real, w.imag
            return y

        if c["op"] == "rope":
            return turned(s["x"], s["pos"][:, None], -1 if c["inverse"] else 1)
        q, kc, vc = s["q_out"].double(), s["k_cache"].double(), s["v_cache"].double()
        first, lens = s["q_start"].tolist(), s["kv_len"].tolist()
        for b in range(c["S"]):
            at = torch.arange(first[b], first[b + 1], device="cuda")
            pos = at - first[b + 1] + lens[b]
            q[at] = turned(s["q"][at], pos[:, None], 1)
            k, v = turned(s["k"][at], pos[:, None], 1), s["v"][at].double()
            if c["cache"] == "e4m3":
                k, v = ((x / y.double()[:, None]).clamp(-448, 448) for x, y in ((k, s["k_scale"]), (v, s["v_scale"])))
            ids = s["table"][b].long()[pos // c["page"]]
            kc[ids, :, pos % c["page"]], vc[ids, :, pos % c["page"]] = k, v
        return q, kc, vc
    # fork, compact: a page's new place, page by page
    k, v = s["k_cache"].double(), s["v_cache"].double()
    table, ref, lens, page = s["table"].tolist(), s["ref"].tolist(), s["kv_len"].tolist(), c["page"]
    old, new = [], []
    if c["op"] == "fork":
        pairs = list(zip(s["src"].tolist(), s["dst"].tolist()))
        free = [p for p in range(len(ref)) if ref[p] == 0]
        for a, b in pairs:
            if lens[a] % page and free:
                old.append(table[a][lens[a] // page])
                new.append(free.pop(0))
    else:
        n = sum(r > 0 for r in ref)
        new = [p for p in range(n) if ref[p] == 0]
        old = [p for p in range(n, len(ref)) if ref[p] > 0]
    k[:, new], v[:, new] = k[:, old], v[:, old]
    return k, v, None, None, None, None
