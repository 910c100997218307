"""Helpers of the tests around the paged cache: batches with everything that nobody wrote filled with NaN, and the attention in 64 bits
from its definition, with a bound for every output."""
import math

import numpy as np
import torch

TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
HALF_STEP = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
O_FILL, LSE_FILL = 77.0, 1234.5


def to_nan(t):
    """A tensor of a type filled with NaN."""
    if t.dtype == torch.float8_e4m3fn:
        t.view(torch.uint8).fill_(0x7f)
    else:
        t.fill_(float("nan"))
    return t


class Batch:
    """New tokens and a cache on the CPU, and copies on the device.  ``lens``: (new tokens, all tokens) of each sequence; where there are fewer tokens than new
    ones the sequence has none in the cache."""

    def __init__(self, lens, heads, key_heads, d, dtype="fp16", cache="fp16", page=16, order="head", pad=0, seed=1, spare=2, holes=(), peaky=False, width=None):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.heads, self.key_heads, self.d, self.page, self.pad = lens, heads, key_heads, d, page, pad
        self.dtype, self.cache_dtype = TYPES[dtype], TYPES[cache]
        n = sum(a for a, _ in lens)
        self.tokens = max(1, n + pad)
        self.q = torch.randn((self.tokens, heads, d), generator=g).to(self.dtype)
        used = [-(-b // page) for _, b in lens]
        pages = sum(used) + spare
        ids = (torch.randperm(pages - 1, generator=g) + 1).tolist()                 # page 0 is nobody's
        width = width or max(1, max(used))
        self.table = torch.full((len(lens), width), -7, dtype=torch.int32)
        shape = (pages, page, key_heads, d) if order == "token" else (pages, key_heads, page, d)
        self.k_cache, self.v_cache = (to_nan(torch.empty(shape, dtype=self.cache_dtype)) for _ in "kv")
        if order == "token":
            self.k_cache, self.v_cache = self.k_cache.transpose(1, 2), self.v_cache.transpose(1, 2)
        self.k_scale = self.v_scale = None
        if cache == "e4m3":
            self.k_scale, self.v_scale = (torch.rand(key_heads, generator=g) + 0.5 for _ in "kv")
        self.k, self.v = [], []
        for s, (_, b) in enumerate(lens):
            mine = [ids.pop() for _ in range(used[s])]
            self.table[s, :used[s]] = torch.tensor(mine, dtype=torch.int32)
            k, v = (torch.randn((b, key_heads, d), generator=g) for _ in "kv")
            if peaky:
                k *= torch.where(torch.rand((b, 1, 1), generator=g) < 0.05, 8.0, 1.0)
            self.k.append(k.to(self.cache_dtype))
            self.v.append(v.to(self.cache_dtype))
            for j in range(b):
                self.put(s, j)
        self.holes = set(holes)                                                     # (sequence, entry): no page there
        for s, e in holes:
            self.table[s, e] = (-1, pages, 2 ** 31 - 1, -2 ** 31)[(s + e) % 4]
        self.q_start = torch.tensor([0] + np.cumsum([a for a, _ in lens]).tolist(), dtype=torch.int32)
        self.kv_len = torch.tensor([b for _, b in lens], dtype=torch.int32)
        self.max_q, self.max_kv = max(1, max(a for a, _ in lens)), max(1, max(b for _, b in lens))

    def put(self, s, j):
        """Token j of sequence s to its place."""
        p = int(self.table[s, j // self.page])
        for cache, x in ((self.k_cache, self.k), (self.v_cache, self.v)):
            if self.cache_dtype == torch.float8_e4m3fn:
                cache.view(torch.uint8)[p, :, j % self.page] = x[s][j].view(torch.uint8)
            else:
                cache[p, :, j % self.page] = x[s][j]

    def seen(self, s, causal):
        """[new tokens][keys]: which keys a new token sees."""
        a, b = self.lens[s]
        j = np.arange(b)
        ok = np.ones((a, b), bool) if not causal else j[None] <= (b - a + np.arange(a))[:, None]
        for e in range(-(-b // self.page)):
            if (s, e) in self.holes:
                ok[:, e * self.page:(e + 1) * self.page] = False
        return ok

    def reference(self, scale, causal):
        """O, LSE and their bounds, float64 [tokens][heads][d] and [tokens][heads]; rows of nobody keep the fill values.

        Weights are rounded to the type of the tokens (half a step u relative; in fp16 also 2^-25 of the largest, below its normal numbers), the
        result once more.  Scores are sums of d exact products in fp32, (d + 2) 2^-24 of the sum of their absolute values; the exponent s c - m c
        adds three roundings of values up to |s|max, and exp2 and the scales 2^-22.  That changes weights by a factor exp(delta).  Sums over n
        keys in fp32 add n 2^-23 of the sum of absolute values."""
        o = np.full((self.tokens, self.heads, self.d), O_FILL)
        lse = np.full((self.tokens, self.heads), LSE_FILL)
        bo, bl = np.zeros_like(o), np.zeros_like(lse)
        u, G = HALF_STEP[self.dtype], self.heads // self.key_heads
        for s, (a, b) in enumerate(self.lens):
            t0, ok = int(self.q_start[s]), self.seen(s, causal)
            for h in range(self.heads):
                hk = h // G
                q = self.q[t0:t0 + a, h].double().numpy()
                k, v = self.k[s][:, hk].double().numpy(), self.v[s][:, hk].double().numpy()
                if self.k_scale is not None:
                    k, v = k * float(self.k_scale[hk]), v * float(self.v_scale[hk])
                for i in range(a):
                    at = np.flatnonzero(ok[i])
                    if len(at) == 0:
                        o[t0 + i, h], lse[t0 + i, h] = 0.0, -np.inf
                        continue
                    x = scale * (k[at] @ q[i])
                    m = x.max() if not np.isnan(x).any() else np.nan
                    w = np.exp(x - m)
                    p = w / w.sum()
                    o[t0 + i, h], lse[t0 + i, h] = p @ v[at], m + math.log(w.sum()) if not np.isnan(m) else np.nan
                    size = scale * (np.abs(k[at]) @ np.abs(q[i])).max()
                    delta = (self.d + 2) * 2.0 ** -24 * size + 3 * 2.0 ** -24 * 2 * np.abs(x).max() + 2.0 ** -21
                    e = np.maximum(u * p, np.minimum(p, 2.0 ** -25 * p.max()) if self.dtype == torch.float16 else 0) + (2 * delta + len(at) * 2.0 ** -23) * p
                    bo[t0 + i, h] = (e @ np.abs(v[at])) * (1 + 2 * u) + (u + 2.0 ** -22) * np.abs(o[t0 + i, h]) + 2.0 ** -25
                    bl[t0 + i, h] = delta + len(at) * 2.0 ** -24 + 2.0 ** -22 * (abs(lse[t0 + i, h]) + abs(m)) + 1e-6
        return o, lse, bo, bl

    def cuda(self):
        """Name -> device tensor of everything that a call takes; strides are kept."""
        def up(x):
            y = torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device="cuda")
            if x.dtype == torch.float8_e4m3fn:
                y.view(torch.uint8).copy_(x.view(torch.uint8))
            else:
                y.copy_(x)
            return y
        d = {n: up(getattr(self, n)) for n in ("q", "k_cache", "v_cache", "q_start", "kv_len", "table")}
        d["scales"] = {} if self.k_scale is None else {"k_scale": self.k_scale.cuda(), "v_scale": self.v_scale.cuda()}
        d["o"] = torch.full_like(d["q"], O_FILL)
        d["lse"] = torch.full((self.tokens, self.heads), LSE_FILL, device="cuda")
        return d


def workspace_for(kv, q, k_cache, sequences, max_q, max_kv):
    """A workspace full of NaN, or None where none is needed."""
    n = kv.attn_paged_workspace(q, k_cache, sequences, max_q, max_kv)
    return None if n == 0 else torch.full((n,), 0xff, dtype=torch.uint8, device="cuda")


def check(o, lse, ref, what=""):
    """Device outputs inside the bounds; NaN and infinities where the reference has them."""
    o, lse = o.double().cpu().numpy(), lse.double().cpu().numpy()
    o_ref, l_ref, bo, bl = ref
    for x, y, b, name in ((o, o_ref, bo, "O"), (lse, l_ref, bl, "LSE")):
        fine = np.isfinite(y)
        assert np.array_equal(np.isnan(x), np.isnan(y)), "%s %s: NaN at other places" % (what, name)
        assert np.array_equal(x[~fine & ~np.isnan(y)], y[~fine & ~np.isnan(y)]), "%s %s: infinities" % (what, name)
        err = np.abs(x[fine] - y[fine])
        worst = (err / np.maximum(b[fine], 1e-300)).max() if err.size and (err > 0).any() else 0.0
        print("%s %s: max error %.2e, of its bound %.2f" % (what, name, err.max() if err.size else 0.0, worst), flush=True)
        assert (err <= b[fine]).all(), "%s %s: %.2e, %.2f of the bound" % (what, name, err.max(), worst)
