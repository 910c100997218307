"""What the header promises of the operators around a paged cache where pages, lengths or values are not as they should be."""
import copy
import math
import random

import numpy as np
import pytest
import torch

from tests.paged_util import HALF_STEP, Batch, check, workspace_for
from tests.test_gpu_kv_pages import Model, ints

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    from paper_2510_14719_amd import kv_cache
    return kv_cache


class Pages(Model):
    """A continuation of a row whose last page is missing has none there either, and takes none."""

    def fork(self, src, dst):
        free, missing, bare = self.free_pages(), 0, 0
        for s, d in zip(src, dst):
            if not (0 <= s < self.rows and 0 <= d < self.rows) or s == d:
                continue
            n = self.len[s]
            full = n // self.page
            self.table[d] = self.table[s][:full] + [-1] * (self.width - full)
            for p in self.table[s][:full]:
                if 0 <= p < self.pages:
                    self.ref[p] += 1
            if n % self.page:
                old = self.table[s][full]
                if not 0 <= old < self.pages:
                    bare += 1
                elif free:
                    p = free.pop(0)
                    self.table[d][full] = p
                    self.ref[p] = 1
                    for x in self.want:
                        x[:, p] = x[:, old]
                else:
                    missing += 1
            self.len[d] = n
        self.bare = getattr(self, "bare", 0) + bare
        return missing


@pytest.mark.parametrize("layers,pages,heads,page,d,dtype,rows,width,order", [
    (3, 60, 2, 16, 128, torch.bfloat16, 9, 12, "token"), (2, 400, 3, 32, 64, torch.float8_e4m3fn, 40, 30, "head"),
    (1, 9001, 1, 16, 64, torch.float8_e4m3fn, 300, 80, "token"), (1, 50, 1, 16, 64, torch.float16, 30, 6, "head")])
def test_forks_of_rows_with_missing_pages(kv, layers, pages, heads, page, d, dtype, rows, width, order):
    m = Pages(layers, pages, heads, page, d, dtype, rows, width, order)
    rng = random.Random(pages + 1)
    for turn in range(8):
        grow = rng.sample(range(rows), rows // 2 + 1)
        lens = [rng.randint(1, width * page) for _ in grow]
        missing = m.reserve(grow, lens)
        kv.kv_reserve(*m.dev, ints(grow), ints(lens), m.missing, page)
        m.check("turn %d reserve" % turn, missing)
        order_ = rng.sample(range(rows), rows)
        src, dst = order_[:rows // 3], order_[rows // 3:rows // 2]
        src = [rng.choice(src) for _ in dst]
        m.release(dst)
        kv.kv_free(*m.dev, ints(dst), page)
        missing = m.fork(src, dst)
        kv.kv_fork(*m.kv, *m.dev, ints(src), ints(dst), m.missing)
        m.check("turn %d fork" % turn, missing)
    assert m.bare > 0                           # (the case has been there)


@pytest.mark.parametrize("cache", ["fp16", "e4m3"])
def test_a_continuation_sees_what_its_source_sees(kv, cache):
    """The source's last page is missing; all free pages are full of NaN, as a last owner may have left them."""
    b = Batch([(2, 40), (2, 40)], 4, 2, 64, "fp16", cache, 16, holes=[(0, 2), (1, 2)], spare=6)
    dev = b.cuda()
    pages = b.k_cache.shape[0]
    table = dev["table"]
    table[1] = -1
    ref = torch.zeros(pages, dtype=torch.int32, device="cuda")
    ref[table[0, :2].long()] = 1
    kv_len, missing = ints([40, 0]), ints([9])
    kv.kv_fork(dev["k_cache"][None], dev["v_cache"][None], ref, table, kv_len, ints([0]), ints([1]), missing)
    dev["q"][2:] = dev["q"][:2]
    kv.attn_paged(dev["q"], dev["k_cache"], dev["v_cache"], dev["q_start"], kv_len, table, dev["o"], dev["lse"], 2, 40, 1 / 8,
                  workspace=workspace_for(kv, dev["q"], dev["k_cache"], 2, 2, 40), **dev["scales"])
    torch.cuda.synchronize()
    assert table.tolist()[1] == table.tolist()[0][:2] + [-1] and missing.tolist() == [0] and kv_len.tolist() == [40, 40] and int(ref.sum()) == 4
    assert math.isfinite(float(dev["o"].float().abs().sum())) and torch.equal(dev["o"][2:], dev["o"][:2]) and torch.equal(dev["lse"][2:], dev["lse"][:2])


@pytest.mark.parametrize("d,dtype,cache", [(128, "bf16", "bf16"), (64, "fp16", "e4m3")])
def test_an_odd_number_of_partial_results_beside_chunks(kv, d, dtype, cache):
    """65 sequences, an odd number of tokens and one head: small tiles, cut chunks and the lists of both in one workspace."""
    lens = [(1, 2500)] + [(1, 1 + 7 * i % 60) for i in range(62)] + [(100, 2400), (40, 1300)]
    b = Batch(lens, 1, 1, d, dtype, cache, 16)
    b.max_kv = 2503                             # (five pieces of 512, and 203 tokens)
    dev = b.cuda()
    dev["table"] = torch.nn.functional.pad(dev["table"], (0, 1), value=-1)
    kv.attn_paged(dev["q"], dev["k_cache"], dev["v_cache"], dev["q_start"], dev["kv_len"], dev["table"], dev["o"], dev["lse"], b.max_q, b.max_kv, 1 / math.sqrt(d),
                  workspace=workspace_for(kv, dev["q"], dev["k_cache"], len(lens), b.max_q, b.max_kv), **dev["scales"])
    torch.cuda.synchronize()
    check(dev["o"], dev["lse"], b.reference(1 / math.sqrt(d), True))


@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "e4m3")])
@pytest.mark.parametrize("lens,H,Hk,d", [
    ([(64, 64)], 4, 2, 64), ([(1, 700), (3, 90), (1, 5000)], 16, 2, 128),         # small tiles, whole and in pieces
    ([(2100, 2100)], 16, 16, 128), ([(64, 4000)] * 8, 16, 4, 128),                # chunks, whole and in pieces
])
def test_a_row_is_a_mean_of_its_values(kv, lens, H, Hk, d, dtype, cache):
    """Values are in 1 ... 1 + w.  A weight p rounded to the type is off by u p at most (u half a step; in fp16 by 2^-25 of the largest, too), so the mean with
    rounded weights, divided by THEIR sum, is off by (u + n 2^-25) w; scores that are off by delta change weights by 2 delta p; the result is rounded, half a step u of values in 1 ... 2.
    (Divided by the sum of the weights as they are it would be off by another u, 16 or 8 times as much.)  Scores have a standard deviation of 2, so few keys have a say."""
    b = Batch(lens, H, Hk, d, dtype, cache, 16)
    g = torch.Generator().manual_seed(3)
    width = 1 / 8 if cache == "e4m3" else 1 / 16
    dev = b.cuda()
    for s, (_, n) in enumerate(lens):           # (values of the type itself, so that they are what the reference has)
        b.v[s] = (1 + width * torch.randint(0, 2 if cache == "e4m3" else 9, (n, Hk, d), generator=g) / (1 if cache == "e4m3" else 8)).to(b.cache_dtype)
        at = torch.arange(n)
        page, slot = b.table[s].long()[at // 16].cuda(), (at % 16).cuda()
        dev["v_cache"].view(torch.uint8).unflatten(-1, (d, -1))[page, :, slot] = b.v[s].cuda().view(torch.uint8).unflatten(-1, (d, -1))
    scales = {"k_scale": b.k_scale.cuda(), "v_scale": torch.ones(Hk, device="cuda")} if cache == "e4m3" else {}
    scale = 2 / math.sqrt(d)
    kv.attn_paged(dev["q"], dev["k_cache"], dev["v_cache"], dev["q_start"], dev["kv_len"], dev["table"], dev["o"], None, b.max_q, b.max_kv, scale,
                  workspace=workspace_for(kv, dev["q"], dev["k_cache"], len(lens), b.max_q, b.max_kv), **scales)
    u = HALF_STEP[b.dtype]
    for s, (m, n) in enumerate(lens):
        t0 = int(b.q_start[s])
        for h in range(H):
            q, k, v = b.q[t0:t0 + m, h].cuda().double(), b.k[s][:, h // (H // Hk)].cuda().double(), b.v[s][:, h // (H // Hk)].cuda().double()
            if cache == "e4m3":
                k = k * float(b.k_scale[h // (H // Hk)])
            x = scale * (q @ k.t().contiguous())
            x.masked_fill_(torch.arange(n, device="cuda")[None] > (n - m + torch.arange(m, device="cuda"))[:, None], -math.inf)
            want = x.softmax(-1) @ v
            # (scores: d products in fp32, and three roundings of the exponent)
            delta = (d + 2) * 2.0 ** -24 * scale * float(q.norm(dim=1).max() * k.norm(dim=1).max()) + 6 * 2.0 ** -24 * float(x[x > -math.inf].abs().max()) + 2.0 ** -21
            bound = u + (1 + u) * ((u + n * 2.0 ** -25 + 2 * delta) * width + n * 2.0 ** -23)
            err = float((dev["o"][t0:t0 + m, h].double() - want).abs().max())
            assert err <= bound, "sequence %d, head %d: %.3e, %.3f of the bound" % (s, h, err, err / bound)


SHORT = [(5, 40), (2, 9), (7, 30), (10, 5), (1, 36)]
MIXED = [(1 + i % 4, 8 + 7 * i % 90) for i in range(150)]
for at, long in ((3, (40, 1500)), (64, (20, 900)), (70, (70, 70)), (127, (9, 1100)), (149, (36, 1499))):
    MIXED[at] = long
CUT = [(SHORT, 3, 40), (SHORT, 10, 36), (SHORT, 4, 28), (SHORT, 1, 1), ([(6, 3000), (3, 1200), (1, 5)], 4, 2996), (MIXED, 33, 1496)]


def cut_lens(lens, max_q, max_kv):
    """What is left of (new tokens, all tokens) of each sequence: the first max_q new ones, at positions below max_kv."""
    out = []
    for n, kv in lens:
        first = kv - n
        m = max(0, min(n, max_q, max_kv - first))
        out.append((m, max(0, min(first + m, max_kv))))
    return out


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens,max_q,max_kv", CUT)
def test_attention_of_sequences_beyond_the_bounds(kv, lens, max_q, max_kv, causal):
    b = Batch(lens, 4, 1, 64, "fp16", "fp16", 16, pad=2)
    dev = b.cuda()
    kv.attn_paged(dev["q"], dev["k_cache"], dev["v_cache"], dev["q_start"], dev["kv_len"], dev["table"], dev["o"], dev["lse"], max_q, max_kv, 1 / 8, causal,
                  workspace=workspace_for(kv, dev["q"], dev["k_cache"], len(lens), max_q, max_kv))
    torch.cuda.synchronize()
    want = copy.copy(b)
    want.lens = cut_lens(lens, max_q, max_kv)
    # (the token of a sequence whose new tokens outnumber it has a negative position: it sees nothing with the mask, and what there is without)
    seen = want.seen

    def at_its_position(s, causal):
        ok = seen(s, causal)
        if causal:
            first = lens[s][1] - lens[s][0]
            ok &= np.arange(ok.shape[1])[None] <= (first + np.arange(ok.shape[0]))[:, None]
        return ok
    want.seen = at_its_position
    check(dev["o"], dev["lse"], want.reference(1 / 8, causal))


@pytest.mark.parametrize("cache", ["fp16", "e4m3"])
@pytest.mark.parametrize("lens,max_q,max_kv", CUT)
def test_append_of_sequences_beyond_the_bounds(kv, lens, max_q, max_kv, cache):
    """The tokens that are left get the places and angles that they have in the whole call; nothing else is written."""
    b = Batch(lens, 4, 2, 64, "fp16", cache, 16, pad=2)
    g = torch.Generator().manual_seed(4)
    k, v = (torch.randn((b.tokens, 2, 64), generator=g).half().cuda() for _ in "kv")
    freq = kv.rope_frequencies(64).cuda()
    results = []
    for bounds in ((b.max_q, b.max_kv), (max_q, max_kv)):
        dev = b.cuda()
        q_out = torch.full_like(dev["q"], 55.0)
        kv.kv_append(k, v, dev["k_cache"], dev["v_cache"], dev["q_start"], dev["kv_len"], dev["table"], *bounds, q=dev["q"], q_out=q_out, freq=freq, **dev["scales"])
        results.append((dev["k_cache"].view(torch.uint8).cpu(), dev["v_cache"].view(torch.uint8).cpu(), q_out.cpu()))
    before = [b.k_cache.view(torch.uint8), b.v_cache.view(torch.uint8)]
    for i in range(2):                          # a place of a token that is left as in the whole call, others as before
        want = before[i].clone()
        for s, (m, _) in enumerate(cut_lens(lens, max_q, max_kv)):
            for pos in range(max(0, lens[s][1] - lens[s][0]), lens[s][1] - lens[s][0] + m):
                page = int(b.table[s, pos // 16])
                want[page, :, pos % 16] = results[0][i][page, :, pos % 16]
        assert torch.equal(results[1][i], want)
    q_want = torch.full_like(results[0][2], 55.0)
    for s, (m, _) in enumerate(cut_lens(lens, max_q, max_kv)):
        t0 = int(b.q_start[s])
        q_want[t0:t0 + m] = results[0][2][t0:t0 + m]
    assert torch.equal(results[1][2], q_want)


@pytest.mark.parametrize("loose", [1, 12])
def test_pieces_beside_many_prompts(kv, loose):
    """Sequences of up to 32 rows are cut in a batch that has far more tokens than they have rows, with bounds that are tight and that are not."""
    lens = [(40, 45)] * 130
    for at, some in ((0, (3, 4500)), (33, (20, 4200)), (65, (1, 9)), (129, (32, 4497))):
        lens[at] = some
    b = Batch(lens, 4, 4, 128, "bf16", "bf16", 16, pad=1)
    dev = b.cuda()
    dev["table"] = torch.nn.functional.pad(dev["table"], (0, (loose - 1) * dev["table"].shape[1]), value=-1)
    workspace = workspace_for(kv, dev["q"], dev["k_cache"], 130, 40, 4500 * loose)
    kv.attn_paged(dev["q"], dev["k_cache"], dev["v_cache"], dev["q_start"], dev["kv_len"], dev["table"], dev["o"], dev["lse"], 40, 4500 * loose, 1 / math.sqrt(128),
                  workspace=workspace)
    torch.cuda.synchronize()
    check(dev["o"], dev["lse"], b.reference(1 / math.sqrt(128), True))


@pytest.mark.parametrize("down", [2.5, 20.0])
@pytest.mark.parametrize("lens,H,Hk,d,cache,value", [(*case, value) for case in (
    ([(6, 200), (1, 40), (3, 3)], 4, 2, 64, "fp16"), ([(6, 2000), (2, 40)], 4, 2, 128, "e4m3"), ([(64, 4000)] * 8, 16, 4, 128, "fp16"), ([(2100, 2100)], 16, 16, 128, "e4m3"))
    for value in ((math.nan,) if case[-1] == "e4m3" else (math.nan, math.inf, -math.inf))])       # (E4M3 has no infinities)
def test_values_that_are_not_finite_show_whatever_their_weight(kv, lens, H, Hk, d, cache, down, value):
    """Keys are 0 but for three, which score -scale d down = -20 and -160: weights of 2e-9, nothing in fp16, and of nothing in float32.  One of them all rows see in a whole
    tile, one only some, one is the newest.  Values are 1, so O is 1 where no row sees what is not finite."""
    b = Batch(lens, H, Hk, d, "fp16", cache, 16)
    b.k_scale = b.v_scale = None
    dev = b.cuda()
    dev["q"].fill_(1.0)
    features = {}                               # (sequence, key) -> feature
    for s, (n, m) in enumerate(lens):
        for i, key in enumerate({3, max(0, m - 1 - n // 2), m - 1}):
            features[s, key] = i
    for s, (n, m) in enumerate(lens):
        k, v = torch.zeros((m, Hk, d)), torch.ones((m, Hk, d))
        for (seq, key), f in features.items():
            if seq == s and key < m:
                k[key] = -down
                v[key, :, f] = value
        at = torch.arange(m)
        page, slot = b.table[s].long()[at // 16].cuda(), (at % 16).cuda()
        for name, x in (("k_cache", k), ("v_cache", v)):
            dev[name].view(torch.uint8).unflatten(-1, (d, -1))[page, :, slot] = x.to(b.cache_dtype).cuda().view(torch.uint8).unflatten(-1, (d, -1))
    scale = 8 / d
    kv.attn_paged(dev["q"], dev["k_cache"], dev["v_cache"], dev["q_start"], dev["kv_len"], dev["table"], dev["o"], None, b.max_q, b.max_kv, scale,
                  workspace=workspace_for(kv, dev["q"], dev["k_cache"], len(lens), b.max_q, b.max_kv))
    o = dev["o"].float().cpu()
    for s, (n, m) in enumerate(lens):
        t0 = int(b.q_start[s])
        shows = torch.zeros((n, d), dtype=torch.bool)
        for (seq, key), f in features.items():
            if seq == s and key < m:
                shows[:, f] |= m - n + torch.arange(n) >= key
        x, shows = o[t0:t0 + n], shows[:, None].expand(n, H, d)
        assert not x[shows].isfinite().any() and (not math.isnan(value) or x[shows].isnan().all())
        # (the weights are alike: a mean of ones is off by the sums' rounding, m 2^-24, and the result's)
        assert ((x[~shows] - 1).abs() <= m * 2.0 ** -23 + 2.0 ** -11).all()


def test_a_row_with_missing_pages_is_taken_up_again(kv):
    """As the header says: another call alone fills nothing; with kv_len set back to what the row has, it does, and no page is lost."""
    m = Pages(1, 6, 1, 16, 64, torch.float16, 3, 5, "head")
    for rows, lens, missing in (([0], [40], 0), ([1, 2], [30, 70], 4)):
        assert m.reserve(rows, lens) == missing
        kv.kv_reserve(*m.dev, ints(rows), ints(lens), m.missing, 16)
        m.check("reserve", missing)
    m.release([0])
    kv.kv_free(*m.dev, ints([0]), 16)
    assert m.reserve([2], [70]) == 0
    kv.kv_reserve(*m.dev, ints([2]), ints([70]), m.missing, 16)
    m.check("the same again", 0)
    assert m.table[2][:5] == [5, -1, -1, -1, -1]
    m.len[2] = 16
    m.dev[2][2] = 16
    assert m.reserve([2], [70]) == 1
    kv.kv_reserve(*m.dev, ints([2]), ints([70]), m.missing, 16)
    m.check("taken up", 1)
    assert m.table[2][:5] == [5, 0, 1, 2, -1] and m.ref == [1] * 6


def test_numbers_beyond_an_int(kv):
    b = Batch([(2, 40), (1, 9)], 4, 2, 64, "fp16", "fp16", 16)
    dev = b.cuda()
    big = 2 ** 32
    args = (dev["q_start"], dev["kv_len"], dev["table"])
    x = dev["q"].transpose(0, 1)[None]
    freq = kv.rope_frequencies(64).cuda()
    for call in (lambda: kv.attn_paged(dev["q"], dev["k_cache"], dev["v_cache"], *args, dev["o"], None, big + 2, 40, 1 / 8),
                 lambda: kv.attn_paged(dev["q"], dev["k_cache"], dev["v_cache"], *args, dev["o"], None, 2, big + 40, 1 / 8),
                 lambda: kv.kv_append(dev["q"][:, :2], dev["q"][:, :2], dev["k_cache"], dev["v_cache"], *args, big + 2, 40), lambda: kv.rope(x, torch.empty_like(x), freq, layout=big + 1),
                 lambda: kv.kv_free(torch.zeros(5, dtype=torch.int32, device="cuda"), dev["table"], dev["kv_len"], ints([0]), big + 16)):
        with pytest.raises(kv.KvCacheError) as e:
            call()
        assert e.value.code == -5


def test_many_chunks_of_many_heads(kv):
    """512 prompts of 1024 tokens, 64 heads: 131072 workgroups.  All read the same pages with the same Q, so all results are those of one prompt."""
    S, N, H, d = 512, 1024, 64, 64
    b = Batch([(N, N)], H, H, d, "bf16", "bf16", 64)
    dev = b.cuda()
    one, lse1 = torch.empty_like(dev["q"]), torch.empty((N, H), device="cuda")
    kv.attn_paged(dev["q"], dev["k_cache"], dev["v_cache"], dev["q_start"], dev["kv_len"], dev["table"], one, lse1, N, N, 1 / 8,
                  workspace=workspace_for(kv, dev["q"], dev["k_cache"], 1, N, N))
    q, o, lse = dev["q"].repeat(S, 1, 1), torch.empty((S * N, H, d), dtype=torch.bfloat16, device="cuda"), torch.empty((S * N, H), device="cuda")
    kv.attn_paged(q, dev["k_cache"], dev["v_cache"], torch.arange(S + 1, dtype=torch.int32, device="cuda") * N, dev["kv_len"].repeat(S), dev["table"].repeat(S, 1), o, lse, N, N, 1 / 8,
                  workspace=workspace_for(kv, q, dev["k_cache"], S, N, N))
    del q
    o, lse = o.view(S, N * H * d), lse.view(S, N * H)
    for s in range(1, S):
        assert torch.equal(o[s], o[0]) and torch.equal(lse[s], lse[0]), s
    # (another cut along the keys: both round the weights, 2 u of values up to 6 each, and the result)
    assert float((o[0].float() - one.flatten().float()).abs().max()) <= 2 * 2 * 2.0 ** -8 * 6 and float((lse[0] - lse1.flatten()).abs().max()) <= 1e-4
    assert bool(o[0].isfinite().all())


def test_scales_below_the_normal_numbers(kv):
    """Of an E4M3 cache: what is stored is the quotient all the same, zeros are zeros."""
    b = Batch([(3, 40), (2, 9)], 4, 2, 64, "bf16", "e4m3", 16)
    g = torch.Generator().manual_seed(6)
    scale = torch.tensor([1e-39, 2.0 ** -130])
    x = (torch.randn((b.tokens, 2, 64), generator=g) * 200 * scale[None, :, None]).bfloat16()                # (quotients in the range of E4M3)
    x[0] = 0.0
    x[1, :, ::2] = 1.0                          # (far beyond it)
    dev = b.cuda()
    kv.kv_append(x.cuda(), x.cuda(), dev["k_cache"], dev["v_cache"], dev["q_start"], dev["kv_len"], dev["table"], b.max_q, b.max_kv, k_scale=scale.cuda(), v_scale=scale.cuda())
    want = (x.double() / scale.double()[None, :, None]).clamp(-448, 448).float().to(torch.float8_e4m3fn).view(torch.uint8)
    for name in ("k_cache", "v_cache"):
        got = dev[name].view(torch.uint8).cpu()
        for s, (n, m) in enumerate(b.lens):
            for i in range(n):
                pos = m - n + i
                assert torch.equal(got[int(b.table[s, pos // 16]), :, pos % 16], want[int(b.q_start[s]) + i]), (name, s, i)


@pytest.mark.parametrize("lens,H,Hk,d", [([(6, 200), (2, 5)], 4, 2, 64), ([(2100, 2100)], 16, 16, 128)])
def test_scales_whose_product_is_zero(kv, lens, H, Hk, d):
    """In float32; all keys that a row sees weigh the same, and the others nothing."""
    b = Batch(lens, H, Hk, d, "bf16", "e4m3", 16)
    dev = b.cuda()
    dev["scales"] = {"k_scale": torch.full((Hk,), 1e-30, device="cuda"), "v_scale": torch.ones(Hk, device="cuda")}
    kv.attn_paged(dev["q"], dev["k_cache"], dev["v_cache"], dev["q_start"], dev["kv_len"], dev["table"], dev["o"], dev["lse"], b.max_q, b.max_kv, 1e-30,
                  workspace=workspace_for(kv, dev["q"], dev["k_cache"], len(lens), b.max_q, b.max_kv), **dev["scales"])
    for s, (n, m) in enumerate(lens):
        t0 = int(b.q_start[s])
        v = b.v[s].double()
        count = torch.arange(m - n + 1, m + 1).double()
        want = (v.cumsum(0)[m - n:] / count[:, None, None]).repeat_interleave(H // Hk, 1)
        size = (v.abs().cumsum(0)[m - n:] / count[:, None, None]).repeat_interleave(H // Hk, 1)
        got = dev["o"][t0:t0 + n].double().cpu()
        assert ((got - want).abs() <= 2.0 ** -8 * want.abs() + m * 2.0 ** -23 * size).all()
        assert torch.allclose(dev["lse"][t0:t0 + n].double().cpu(), count.log()[:, None].expand(n, H), rtol=2.0 ** -21, atol=m * 2.0 ** -24)


def guarded(like, fill):
    """A tensor of the same kind, 64 rows of `fill` before and behind it, and all of them."""
    whole = torch.full((like.shape[0] + 128, *like.shape[1:]), fill, dtype=like.dtype, device="cuda")
    return whole[64:64 + like.shape[0]], whole


# sequences, tokens, max_q, max_kv, heads, key heads, d: small tiles in pieces; pieces beside chunks; chunks in pieces; prompts
GARBAGE = [(6, 20, 4, 3000, 4, 1, 64), (150, 700, 33, 1500, 4, 1, 64), (8, 512, 64, 4000, 16, 4, 128), (3, 4200, 1500, 1500, 8, 2, 128), (130, 5200, 40, 4600, 4, 4, 128)]


@pytest.mark.parametrize("cache", ["fp16", "e4m3"])
@pytest.mark.parametrize("S,T,max_q,max_kv,H,Hk,d", GARBAGE)
def test_starts_and_lengths_that_make_no_sense_write_nothing_else(kv, S, T, max_q, max_kv, H, Hk, d, cache):
    """Falling, overlapping and endless starts, lengths and pages of all kinds: what lies beside O, LSE, the workspace, Q and the cache is left, and so are the rows that
    no sequence can have."""
    pages, rng = 40, random.Random(S)
    b = Batch([(1, 1)], H, Hk, d, "fp16", cache, 64)
    shape = (pages, Hk, 64, d)
    q = torch.randn((T, H, d), device="cuda").half()
    width = -(-max_kv // 64)
    strange = [0, 1, -1, T - 1, T, T + 5, 2 ** 31 - 1, -2 ** 31]
    for turn in range(4):
        caches = [guarded(torch.zeros(shape, device="cuda").to(b.cache_dtype) if cache == "fp16" else torch.zeros(shape, dtype=torch.uint8, device="cuda"), 57) for _ in "kv"]
        for c, _ in caches:
            c.fill_(1)
        k_cache, v_cache = (c if cache == "fp16" else c.view(b.cache_dtype) for c, _ in caches)
        o, o_all = guarded(q, 77.0)
        lse, lse_all = guarded(torch.empty((T, H), device="cuda"), 1234.5)
        starts = [rng.choice(strange) if rng.random() < 0.2 else rng.randint(0, T) for _ in range(S + 1)]
        if turn == 3:
            starts = sorted(s for s in starts)
        lens = [rng.choice([0, 1, -5, max_kv, max_kv + 1, 2 ** 31 - 1, -2 ** 31]) if rng.random() < 0.3 else rng.randint(0, max_kv) for _ in range(S)]
        table = torch.randint(-3, pages + 3, (S, width), dtype=torch.int32)
        args = (ints(starts), ints(lens), table.cuda())
        n = kv.attn_paged_workspace(q, k_cache, S, max_q, max_kv)
        work, work_all = guarded(torch.empty(max(n, 16), dtype=torch.uint8, device="cuda"), 0xa5)
        kv.attn_paged(q, k_cache, v_cache, *args, o, lse, max_q, max_kv, 1 / 8, turn != 1, workspace=work[:n] if n else None)
        q_out, q_all = guarded(q, 55.0)
        kv.kv_append(q[:, :Hk], q[:, :Hk], k_cache, v_cache, *args, max_q, max_kv, q=q, q_out=q_out, freq=kv.rope_frequencies(d).cuda())
        torch.cuda.synchronize()
        for whole, fill in ((o_all, 77.0), (lse_all, 1234.5), (work_all, 0xa5), (q_all, 55.0), (caches[0][1], 57), (caches[1][1], 57)):
            assert bool((whole[:64] == fill).all()) and bool((whole[-64:] == fill).all())
        owned = torch.zeros(T, dtype=torch.bool)
        for s in range(S):
            q0 = min(max(starts[s], 0), T)
            q1 = min(max(starts[s + 1], q0), T)
            owned[q0:min(q1, q0 + max_q)] = True
        for x, fill in ((o, 77.0), (lse, 1234.5), (q_out, 55.0)):
            assert bool((x[~owned.cuda()] == fill).all())


@pytest.mark.parametrize("lens", [[(1, 40), (2, 9), (1, 1300)], [(9, 700), (1, 30), (40, 90)]])
@pytest.mark.parametrize("cache", ["fp16", "e4m3"])
def test_more_heads_on_a_key_head_than_rows_of_a_chunk(kv, lens, cache):
    b = Batch(lens, 300, 1, 64, "fp16", cache, 16, pad=1)
    dev = b.cuda()
    kv.attn_paged(dev["q"], dev["k_cache"], dev["v_cache"], dev["q_start"], dev["kv_len"], dev["table"], dev["o"], dev["lse"], b.max_q, b.max_kv, 1 / 8,
                  workspace=workspace_for(kv, dev["q"], dev["k_cache"], len(lens), b.max_q, b.max_kv), **dev["scales"])
    torch.cuda.synchronize()
    check(dev["o"], dev["lse"], b.reference(1 / 8, True))


def test_more_sequences_than_two_steps_of_a_search(kv):
    """5000 sequences, some without new tokens: each token finds its own, and attention sees what was appended."""
    g = torch.Generator().manual_seed(8)
    n = torch.randint(0, 3, (5000,), generator=g)
    lens = [(int(a), int(a) + i % 40) for i, a in enumerate(n)]
    b = Batch(lens, 1, 1, 64, "fp16", "fp16", 16, pad=2)
    dev = b.cuda()
    k, v = (torch.zeros((b.tokens, 1, 64), dtype=torch.float16) for _ in "kv")
    for s, (a, m) in enumerate(lens):
        t0 = int(b.q_start[s])
        k[t0:t0 + a], v[t0:t0 + a] = b.k[s][m - a:], b.v[s][m - a:]
        for pos in range(m - a, m):             # (what append has to bring is not there yet)
            for name in ("k_cache", "v_cache"):
                getattr(b, name)[int(b.table[s, pos // 16]), :, pos % 16] = float("nan")
    before = [dev["k_cache"].clone(), dev["v_cache"].clone()]
    dev["k_cache"].copy_(b.k_cache)
    dev["v_cache"].copy_(b.v_cache)
    kv.kv_append(k.cuda(), v.cuda(), dev["k_cache"], dev["v_cache"], dev["q_start"], dev["kv_len"], dev["table"], 2, b.max_kv)
    for name, x in zip(("k_cache", "v_cache"), before):
        assert torch.equal(dev[name].view(torch.int16), x.view(torch.int16))
    kv.attn_paged(dev["q"], dev["k_cache"], dev["v_cache"], dev["q_start"], dev["kv_len"], dev["table"], dev["o"], dev["lse"], 2, b.max_kv, 1 / 8,
                  workspace=workspace_for(kv, dev["q"], dev["k_cache"], 5000, 2, b.max_kv))
    torch.cuda.synchronize()
    check(dev["o"], dev["lse"], b.reference(1 / 8, True))
