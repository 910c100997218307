"""Rotary positions and the writing of new tokens to a paged cache against their definitions in 64 bits."""
import math

import numpy as np
import pytest
import torch

from tests.paged_util import HALF_STEP, TYPES, Batch, check, workspace_for

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    from paper_2510_14719_amd import kv_cache
    return kv_cache


def turned(x, pos, freq, layout, amplitude=1.0, sign=1):
    """x [..., d] float64 turned by pos [...], and a bound of the error of doing it in 32 bits: cosine and sine are off by 2^-21 at most (their argument by 2 pi 2^-25,
    the function by 2^-23, the factor by 2^-24), products and sum by 2^-23 of their size."""
    rot = 2 * len(freq)
    a, b = (x[..., :rot // 2], x[..., rot // 2:rot]) if layout == 0 else (x[..., :rot:2], x[..., 1:rot:2])
    angle = pos[..., None].double() * freq
    c, s = amplitude * angle.cos(), sign * amplitude * angle.sin()
    ya, yb = a * c - b * s, b * c + a * s
    bound = abs(amplitude) * (a.abs() + b.abs()) * 2.0 ** -20
    y, e = x.clone(), torch.zeros_like(x)
    if layout == 0:
        y[..., :rot], e[..., :rot] = torch.cat((ya, yb), -1), torch.cat((bound, bound), -1)
    else:
        y[..., :rot], e[..., :rot] = torch.stack((ya, yb), -1).flatten(-2), torch.stack((bound, bound), -1).flatten(-2)
    return y, e


def near(got, want, bound, dtype, what=""):
    got = got.double().cpu()
    tol = want.abs() * HALF_STEP[dtype] + bound * (1 + HALF_STEP[dtype]) + (2.0 ** -25 if dtype == torch.float16 else 0)
    worst = ((got - want).abs() / tol.clamp(min=1e-300)).max().item()
    print("%s: %.2f of the bound" % (what, worst), flush=True)
    assert ((got - want).abs() <= tol).all(), "%s: %.2f of the bound" % (what, worst)


CASES = [(1, 1, 1, 16, 16), (1, 2, 1, 64, 64), (2, 3, 5, 128, 128), (1, 32, 33, 128, 96), (3, 4, 17, 64, 32), (1, 5, 300, 80, 48), (2, 1, 1000, 256, 16), (1, 7, 3, 1024, 1024)]


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("B,H,N,d,rot", CASES)
def test_rope_and_its_gradient(kv, B, H, N, d, rot, layout):
    for dtype, first, inverse in ((torch.bfloat16, 0, False), (torch.float16, 4000000, False), (torch.float16, 99991, True), (torch.bfloat16, 2 ** 31 - 1 - N, True)):
        g = torch.Generator().manual_seed(N + rot)
        x = torch.randn((B, H, N, d), generator=g).to(dtype)
        pos = first + torch.arange(B * N).reshape(B, N) % max(1, N)
        freq = kv.rope_frequencies(rot, 10000.0, kv.PARTS, 8.0, trained=4096.0)
        amplitude = 1.0 + 0.1 * math.log(8.0)
        want, bound = turned(x.double(), pos[:, None].expand(B, H, N), freq, layout, np.float32(amplitude).item(), -1 if inverse else 1)
        dx, dpos, dfreq = x.cuda(), pos.int().cuda(), freq.cuda()
        y = torch.full_like(dx, float("nan"))
        kv.rope(dx, y, dfreq, dpos, layout, amplitude, inverse)
        near(y, want, bound, dtype, "contiguous")
        packed = torch.full((B, N, H + 2, d), 9.0, dtype=dtype, device="cuda")       # a slice of a projection, turned in place
        view = packed[:, :, 1:H + 1].transpose(1, 2)
        view.copy_(dx)
        kv.rope(view, view, dfreq, dpos, layout, amplitude, inverse)
        assert torch.equal(view.contiguous(), y) and bool((packed[:, :, 0] == 9).all()) and bool((packed[:, :, -1] == 9).all())


def test_many_tokens_with_long_heads(kv):
    """The most sines and cosines that a workgroup keeps."""
    x = torch.randn((1, 1, 16389, 1024), generator=torch.Generator().manual_seed(2)).half()
    f = kv.rope_frequencies(1024)
    y = torch.full_like(x, float("nan"), device="cuda")
    kv.rope(x.cuda(), y, f.cuda(), layout=kv.INTERLEAVED)
    want, bound = turned(x.double(), torch.arange(16389).expand(1, 1, 16389), f, 1)
    near(y, want, bound, torch.float16)


def test_positions_by_default_and_shared(kv):
    x = torch.randn((3, 2, 50, 64), generator=torch.Generator().manual_seed(3)).half().cuda()
    f = kv.rope_frequencies(64).cuda()
    ys = [torch.empty_like(x) for _ in range(3)]
    kv.rope(x, ys[0], f)
    kv.rope(x, ys[1], f, torch.arange(50, dtype=torch.int32, device="cuda"))
    kv.rope(x, ys[2], f, torch.arange(50, dtype=torch.int32, device="cuda").repeat(3, 1))
    assert torch.equal(ys[0], ys[1]) and torch.equal(ys[0], ys[2])
    want, bound = turned(x.double().cpu(), torch.arange(50).expand(3, 2, 50), f.cpu(), 0)
    near(ys[0], want, bound, torch.float16)


@pytest.mark.parametrize("layout", [0, 1])
def test_the_inverse_is_the_gradient(kv, layout):
    """The map is linear, so its gradient is its transpose: <g, R x> = <R^T g, x> up to the roundings of both sides (half a step of every
    term), and the difference quotient of one element is a column of R."""
    N, d, rot = 40, 64, 48
    gen = torch.Generator().manual_seed(7)
    x, g = (torch.randn((1, 2, N, d), generator=gen).half().cuda() for _ in "xg")
    f, pos = kv.rope_frequencies(rot).cuda(), torch.arange(1000, 1000 + N, dtype=torch.int32, device="cuda")
    y, gx = torch.empty_like(x), torch.empty_like(x)
    kv.rope(x, y, f, pos, layout, 1.25)
    kv.rope(g, gx, f, pos, layout, 1.25, inverse=True)
    left, right = (g.double() * y.double()), (gx.double() * x.double())
    slack = (left.abs().sum() + right.abs().sum()).item() * (2.0 ** -11 + 2.0 ** -19) + 4 * N * d * 2.0 ** -20
    assert abs(left.sum().item() - right.sum().item()) <= slack
    step = x.clone()
    step[..., 5] += 1.0
    y2 = torch.empty_like(y)
    kv.rope(step, y2, f, pos, layout, 1.25)
    delta = (step.double() - x.double())[..., 5]
    unit = torch.zeros((1, 2, N, d), dtype=torch.float64)
    unit[..., 5] = 1.0
    column, _ = turned(unit, pos.cpu().expand(1, 2, N), f.cpu(), layout, 1.25)
    off = ((y2.double() - y.double()).cpu() - column * delta.cpu()[..., None]).abs()
    assert (off <= (y2.double().abs() + y.double().abs()).cpu() * (2.0 ** -11 + 2.0 ** -18) + 2.0 ** -17).all()


def test_rope_streams_and_graphs(kv):
    x = torch.randn((2, 4, 33, 64), generator=torch.Generator().manual_seed(8)).bfloat16().cuda()
    f, pos = kv.rope_frequencies(64).cuda(), torch.arange(33, dtype=torch.int32, device="cuda")
    y, z = torch.zeros_like(x), torch.zeros_like(x)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        kv.rope(x, y, f, pos)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kv.rope(x, z, f, pos)
    for first in (0, 500, 70000):
        pos.copy_(torch.arange(first, first + 33, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        want, bound = turned(x.double().cpu(), (first + torch.arange(33)).expand(2, 4, 33), f.cpu(), 0)
        near(z, want, bound, torch.bfloat16)
        if first == 0:
            assert torch.equal(y, z)


def stored_bound(x, scale):
    """E4M3 of x / scale: half a step (2^-4 of normal values, 2^-10 below 2^-6), a quotient in 32 bits; beyond 448 it is 448."""
    return x.abs() / scale * (2.0 ** -4 + 2.0 ** -22) + 2.0 ** -10


@pytest.mark.parametrize("lens,H,Hk,d,rot,layout,dtype,cache,page,order", [
    ([(1, 1)], 2, 2, 64, 64, 0, "fp16", "fp16", 16, "head"), ([(1, 17), (1, 300), (1, 16)], 32, 8, 128, 128, 0, "bf16", "bf16", 16, "head"),
    ([(3, 3), (0, 9), (40, 77), (1, 1), (5, 2), (0, 0), (17, 33)], 6, 2, 128, 64, 1, "fp16", "e4m3", 32, "token"),
    ([(130, 130), (2, 40)], 3, 1, 64, 48, 1, "bf16", "bf16", 64, "token"), ([(700, 900), (9, 5), (333, 333)], 8, 8, 64, 64, 0, "bf16", "e4m3", 16, "head"),
    ([(2000, 2100)] + [(1, i + 1) for i in range(200)], 4, 2, 128, 16, 0, "fp16", "fp16", 128, "head")])
def test_append(kv, lens, H, Hk, d, rot, layout, dtype, cache, page, order):
    b = Batch(lens, H, Hk, d, dtype, cache, page, order, pad=2, seed=4)
    dev, T = b.cuda(), b.tokens
    g = torch.Generator().manual_seed(6)
    k, v = (torch.randn((T, Hk, d), generator=g).to(TYPES[dtype]) for _ in "kv")
    v[T // 2] *= 2000                                                             # (saturates in 8 bits)
    qkv = torch.cat((b.q, k, v), 1).cuda()
    freq = kv.rope_frequencies(rot)
    before = {n: (dev[n].view(torch.uint8) if cache == "e4m3" else dev[n]).clone() for n in ("k_cache", "v_cache")}
    q_out = torch.full_like(dev["q"], 7.0)
    args = (qkv[:, H:H + Hk], qkv[:, H + Hk:], dev["k_cache"], dev["v_cache"], dev["q_start"], dev["kv_len"], dev["table"], b.max_q, b.max_kv)
    kv.kv_append(*args, q=qkv[:, :H], q_out=q_out, freq=freq.cuda(), layout=layout, amplitude=1.5, **dev["scales"])
    torch.cuda.synchronize()
    n = int(b.q_start[-1])
    seq = torch.cat([torch.full((a,), s) for s, (a, _) in enumerate(lens)]).long() if n else torch.zeros(0).long()
    pos = b.kv_len.long()[seq] - (b.q_start.long()[seq + 1] - torch.arange(n))
    want, bound = turned(b.q[:n].double(), pos[:, None].expand(n, H), freq, layout, 1.5)
    near(q_out[:n], want, bound, b.dtype, "q")
    assert bool((q_out[n:] == 7).all())
    stored = torch.nonzero(pos >= 0)[:, 0]
    where, at = b.table.long()[seq[stored], pos[stored] // page], pos[stored] % page
    kw, kb = turned(k[stored].double(), pos[stored][:, None].expand(len(stored), Hk), freq, layout, 1.5)
    for name, x, e in (("k", kw, kb), ("v", v[stored].double(), torch.zeros_like(kw))):
        now, old = dev[name + "_cache"], before[name + "_cache"]
        raw = now.view(torch.uint8) if cache == "e4m3" else now
        same = (raw == old) | ((raw != raw) & (old != old))
        same[where.cuda(), :, at.cuda()] = True
        assert bool(same.all()), name + ": another place was written"
        got = raw[where.cuda(), :, at.cuda()].cpu()
        if cache == "e4m3":
            scale = getattr(b, name + "_scale").double()[:, None]
            y, z = got.view(torch.float8_e4m3fn).double(), (x / scale).clamp(-448, 448)
            assert ((y - z).abs() <= stored_bound(z * scale, scale) + e / scale * 1.1).all(), name
            if name == "v":                                                       # (nothing is computed but the quotient: the nearest value itself)
                exact = (x.float() / scale.float()).clamp(-448, 448).to(torch.float8_e4m3fn)
                assert torch.equal(got, exact.view(torch.uint8))
        elif name == "v":
            assert torch.equal(got, v[stored])
        else:
            near(got, x, e, b.dtype, name)
    # in place, and without turning
    one = qkv.clone()
    kv.kv_append(one[:, H:H + Hk], one[:, H + Hk:], *args[2:], q=one[:, :H], q_out=one[:, :H], freq=freq.cuda(), layout=layout, amplitude=1.5, **dev["scales"])
    assert torch.equal(one[:n, :H], q_out[:n]) and torch.equal(one[n:], qkv[n:]) and torch.equal(one[:, H:], qkv[:, H:])
    kv.kv_append(*args, **dev["scales"])
    torch.cuda.synchronize()
    got = (dev["k_cache"].view(torch.uint8) if cache == "e4m3" else dev["k_cache"])[where.cuda(), :, at.cuda()].cpu()
    plain = k[stored]
    assert torch.equal(got, (plain.float() / b.k_scale[:, None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8) if cache == "e4m3" else plain)


def test_append_where_there_is_no_page_and_nan(kv):
    b = Batch([(20, 40), (3, 3)], 2, 1, 64, "fp16", "e4m3", 16, holes=[(0, 2), (1, 0)])
    dev = b.cuda()
    k, v = torch.ones((23, 1, 64)).half(), torch.full((23, 1, 64), -3.0).half()
    k[0, 0, 5], v[0, 0, 6], v[0, 0, 7] = math.nan, math.inf, -math.inf
    before = dev["k_cache"].view(torch.uint8).clone()
    kv.kv_append(k.cuda(), v.cuda(), dev["k_cache"], dev["v_cache"], dev["q_start"], dev["kv_len"], dev["table"], 20, 40)
    torch.cuda.synchronize()
    page, at = int(b.table[0, 1]), 4                                              # token 20 of the first sequence; 32 ... 39 have no page
    changed = (dev["k_cache"].view(torch.uint8) != before).nonzero()
    assert set(changed[:, 0].tolist()) <= {page}
    row = dev["k_cache"][page, 0].float().cpu(), dev["v_cache"][page, 0].float().cpu()
    assert bool((row[0][at + 1:] == 1).all()) and bool((row[1][at + 1:] == -3).all())
    assert math.isnan(row[0][at, 5]) and row[1][at, 6] == 448 and row[1][at, 7] == -448


@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("fp16", "e4m3")])
def test_a_sequence_from_prompt_to_answer(kv, dtype, cache):
    """Pages reserved, tokens appended (turned on the way) and attended to: a prompt, a second chunk, single tokens; one sequence forks on the way.  Every
    result is that of the definition on what the cache then stands for."""
    H, Hk, d, page, rows = 4, 2, 64, 16, 4
    gen = torch.Generator().manual_seed(11)
    kc, vc = (torch.full((1, 40, Hk, page, d), 0x7f, dtype=torch.uint8, device="cuda").view(TYPES[cache]) if cache == "e4m3" else
              torch.full((1, 40, Hk, page, d), math.nan, dtype=TYPES[cache], device="cuda") for _ in "kv")
    ref, table = torch.zeros(40, dtype=torch.int32, device="cuda"), torch.full((rows, 12), -1, dtype=torch.int32, device="cuda")
    kv_len, missing = torch.zeros(rows, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    freq = kv.rope_frequencies(d).cuda()
    scales = {"k_scale": torch.full((Hk,), 0.02, device="cuda"), "v_scale": torch.full((Hk,), 0.03, device="cuda")} if cache == "e4m3" else {}
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    want = [0, 0, 0, 0]

    def step(news):
        for r, n in enumerate(news):
            want[r] += n
        kv.kv_reserve(ref, table, kv_len, ints(0, 1, 2, 3), ints(*want), missing, page)
        T = sum(news)
        q, k, v = (torch.randn((T, h, d), generator=gen).to(TYPES[dtype]).cuda() for h in (H, Hk, Hk))
        q_start = ints(0, *np.cumsum(news).tolist())
        qr, o, lse = torch.empty_like(q), torch.empty_like(q), torch.empty((T, H), device="cuda")
        most = max(news), max(want)
        kv.kv_append(k, v, kc[0], vc[0], q_start, kv_len, table, *most, q=q, q_out=qr, freq=freq, **scales)
        kv.attn_paged(qr, kc[0], vc[0], q_start, kv_len, table, o, lse, *most, 0.125, workspace=workspace_for(kv, qr, kc[0], rows, *most), **scales)
        torch.cuda.synchronize()
        assert int(missing) == 0 and kv_len.tolist() == want
        b = Batch([(n, w) for n, w in zip(news, want)], H, Hk, d, dtype, cache, page)
        b.q = qr.cpu()
        if scales:
            b.k_scale, b.v_scale = scales["k_scale"].cpu(), scales["v_scale"].cpu()
        for r, w in enumerate(want):
            ids = table[r, :-(-w // page)].long()
            b.k[r], b.v[r] = (c[0].view(torch.uint8)[ids].view(c.dtype).cpu().transpose(1, 2).reshape(-1, Hk, d)[:w] if scales else
                              c[0][ids].cpu().transpose(1, 2).reshape(-1, Hk, d)[:w] for c in (kc, vc))
        check(o, lse, b.reference(0.125, True), "news %s" % (news,))

    step([50, 3, 0, 0])
    step([33, 1, 16, 0])
    kv.kv_fork(kc, vc, ref, table, kv_len, ints(0), ints(3), missing)
    want[3] = want[0]
    for _ in range(3):
        step([1, 1, 1, 1])
    kv.kv_free(ref, table, kv_len, ints(0), page)
    want[0] = 0
    kv.kv_compact(kc, vc, ref, table, kv_len, torch.empty(kv.kv_compact_workspace(40), dtype=torch.uint8, device="cuda"))
    step([0, 1, 2, 1])
    step([5, 1, 0, 1])
