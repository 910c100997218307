"""The operators around the paged cache on a machine without a GPU: every symbol is there, bad arguments are refused before any HIP call,
frequencies are those of their formulas."""
import ctypes
import math
import os
import re

import pytest
import torch

from paper_2510_14719_amd import kv_cache as kv

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NULL, SHAPE, SCALE, ALIGN, OVERFLOW, ALIAS, STRIDE, WORKSPACE = -1, -2, -3, -4, -5, -7, -8, -9
K, V, Q, O, L, W, I = (i << 36 for i in range(1, 8))                              # validation never dereferences them


@pytest.fixture(scope="module")
def lib():
    return kv._load()


def pages(**kw):
    a = dict(k=K, v=V, layers=1, pages=100, heads=2, page_size=16, d=64, dtype=0)
    a.update(kw)
    d, t, h = a["d"], a["page_size"], a["heads"]
    for name, value in (("token_stride", d), ("head_stride", d * t), ("page_stride", d * t * h), ("layer_stride", d * t * h * a["pages"])):
        a.setdefault(name, value)
    return kv._Pages(**a)


def batch(**kw):
    a = dict(q_start=I, kv_len=I + 4096, table=I + 8192, sequences=3, tokens=12, table_width=40, table_stride=40, max_q=4, max_kv=640)
    a.update(kw)
    return kv._Batch(**a)


def rows(p, heads, d=64, **kw):
    return kv._Rows(**{"p": p, "token_stride": heads * d, "head_stride": d, **kw})


def test_symbols_are_exported(lib):
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "kv_cache.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b((?:kv|rope|attn_paged)\w*)\s*\(", src)))
    assert {"attn_paged", "attn_paged_workspace", "rope", "rope_frequencies", "kv_append", "kv_reserve", "kv_free", "kv_fork", "kv_compact", "kv_copy_pages",
            "kv_strerror"} <= set(names)
    for n in names:
        assert hasattr(lib, n), n
    texts = [lib.kv_strerror(code) for code in range(-10, 1)]
    assert len(set(texts)) == 11 and texts[-1] == b"success"


def test_attention_refuses(lib):
    def f(c=None, b=None, q=None, o=None, lse=L, heads=4, scale=0.125, dtype=0, ws=W, n=1 << 40):
        return lib.attn_paged_check_args(c or pages(), b or batch(), q or rows(Q, heads), o or rows(O, heads), lse, heads, scale, dtype, ws, n)

    assert f() == 0 and f(lse=None) == 0 and f(c=pages(dtype=1), dtype=1) == 0
    assert f(c=pages(dtype=2, k_scale=I, v_scale=I + 64), dtype=1) == 0 and f(c=pages(dtype=2)) == 0
    for c in (pages(k=None), pages(v=None), pages(dtype=2, k_scale=I)):
        assert f(c=c) == NULL
    for b in (batch(q_start=None), batch(kv_len=None), batch(table=None)):
        assert f(b=b) == NULL
    assert f(q=rows(None, 4)) == NULL and f(o=rows(None, 4)) == NULL
    for c in (pages(d=96), pages(page_size=8), pages(page_size=24), pages(page_size=8192), pages(dtype=3), pages(dtype=1), pages(pages=0), pages(heads=0), pages(layers=0),
              pages(k_scale=I, v_scale=I)):
        assert f(c=c) == SHAPE
    for b in (batch(sequences=0), batch(tokens=0), batch(max_q=0), batch(max_kv=0), batch(max_kv=641), batch(table_width=0)):
        assert f(b=b) == SHAPE
    assert f(heads=3, q=rows(Q, 3), o=rows(O, 3)) == SHAPE and f(heads=0) == SHAPE and f(dtype=2) == SHAPE
    for bad in (0.0, -1.0, math.nan, math.inf):
        assert f(scale=bad) == SCALE
    assert f(c=pages(k=K + 8)) == ALIGN and f(c=pages(token_stride=68)) == ALIGN and f(q=rows(Q + 2, 4)) == ALIGN and f(q=rows(Q, 4, token_stride=260)) == ALIGN
    assert f(lse=L + 2) == ALIGN and f(b=batch(table=I + 2)) == ALIGN and f(c=pages(dtype=2, k_scale=I + 1, v_scale=I)) == ALIGN
    assert f(c=pages(token_stride=0)) == STRIDE and f(c=pages(page_stride=-2048)) == STRIDE and f(b=batch(table_stride=39)) == STRIDE
    assert f(o=rows(O, 4, token_stride=64)) == STRIDE and f(o=rows(O, 4, head_stride=0)) == STRIDE      # (rows of O would meet)
    assert f(q=rows(Q, 4, token_stride=0)) == 0 and f(o=rows(O, 4, head_stride=64 * 12, token_stride=64)) == 0
    assert f(c=pages(page_size=4096, token_stride=1 << 20), b=batch(table_width=1, table_stride=1)) == OVERFLOW
    assert f(b=batch(sequences=1 << 23)) == OVERFLOW and f(b=batch(max_kv=(1 << 30) + 1, table_width=1 << 27, table_stride=1 << 27)) == OVERFLOW
    assert f(c=pages(page_stride=1 << 45)) == OVERFLOW
    assert f(o=rows(Q, 4)) == ALIAS and f(o=rows(K + 64, 4)) == ALIAS and f(lse=Q) == ALIAS and f(lse=O + 16) == ALIAS
    b = batch(max_kv=60000, table_width=4000, table_stride=4000)
    need = lib.attn_paged_workspace(pages(), b, 4)
    assert need > 0 and f(b=b, n=need) == 0 and f(b=b, n=need - 1) == WORKSPACE and f(b=b, ws=None) == NULL and f(b=b, ws=W + 4) == ALIGN
    assert f(b=b, ws=O) == ALIAS and f(b=b, ws=L) == ALIAS
    # Q and O as two slices of the heads of one array
    assert f(q=rows(Q, 8), o=rows(Q + 512, 8)) == 0 and f(q=rows(Q, 8), o=rows(Q + 384, 8)) == ALIAS
    assert lib.attn_paged_workspace(pages(), batch(), 3) == -1 and lib.attn_paged_workspace(pages(d=32), batch(), 4) == -1
    assert lib.attn_paged(None, None, None, None, None, 1, 0.1, 1, 0, None, 0, None) == NULL


def test_rope_refuses(lib):
    def t(p, h=4, n=10, d=64, **kw):
        return kv._Tensor(**{"p": p, "batch_stride": h * n * d, "head_stride": n * d, "token_stride": d, **kw})

    def f(x=None, y=None, b=2, h=4, n=10, d=64, pos=I, stride=10, freq=I + 4096, rot=64, layout=0, amp=1.0, dtype=0):
        return lib.rope_check_args(x or t(Q), y or t(O), b, h, n, d, pos, stride, freq, rot, layout, amp, dtype)

    assert f() == 0 and f(pos=None) == 0 and f(stride=0) == 0 and f(y=t(Q)) == 0 and f(x=t(Q, batch_stride=0)) == 0
    assert f(x=t(None)) == NULL and f(y=t(None)) == NULL and f(freq=None) == NULL
    for kw in ({"b": 0}, {"h": 0}, {"n": 0}, {"d": 8}, {"d": 1040}, {"d": 72}, {"rot": 8}, {"rot": 80}, {"rot": 24}, {"rot": 0}, {"layout": 2}, {"dtype": 2}):
        assert f(**kw) == SHAPE, kw
    assert f(amp=math.nan) == SCALE and f(amp=math.inf) == SCALE and f(amp=-1.0) == 0
    assert f(x=t(Q + 8)) == ALIGN and f(y=t(O, token_stride=68)) == ALIGN and f(freq=I + 4) == ALIGN and f(pos=I + 2) == ALIGN
    assert f(stride=9) == STRIDE and f(x=t(Q, token_stride=32)) == STRIDE and f(y=t(O, batch_stride=0)) == STRIDE and f(y=t(O, batch_stride=64 * 39)) == STRIDE
    assert f(h=70000, x=t(Q, h=70000), y=t(O, h=70000)) == OVERFLOW and f(b=2 ** 30, pos=None) == OVERFLOW
    assert f(y=t(Q + 128)) == ALIAS and f(y=t(Q, token_stride=256, head_stride=64)) == ALIAS and f(freq=O) == ALIAS and f(pos=O) == ALIAS
    assert lib.rope(None, None, 1, 1, 1, 64, None, 0, None, 64, 0, 1.0, 0, 0, None) == NULL


def test_append_refuses(lib):
    def f(c=None, b=None, k=None, v=None, q=None, o=None, heads=4, freq=I + (1 << 20), rot=64, layout=1, amp=1.0, dtype=0):
        return lib.kv_append_check_args(c or pages(), b or batch(), k or rows(L, 2), v or rows(W, 2), q or rows(Q, 4), o or rows(O, 4), heads, freq, rot, layout, amp, dtype)

    none = kv._Rows()
    assert f() == 0 and f(q=none, o=none) == 0 and f(q=none, o=none, freq=None, rot=0) == 0 and f(o=rows(Q, 4)) == 0
    assert f(c=pages(dtype=2, k_scale=I, v_scale=I), dtype=1) == 0
    assert f(q=none) == NULL and f(o=none) == NULL and f(freq=None, rot=0) == NULL and f(k=rows(None, 2)) == NULL and f(v=rows(None, 2)) == NULL
    for kw in ({"rot": 0}, {"rot": 80}, {"rot": 24}, {"layout": 2}, {"heads": 0}, {"dtype": 1}, {"dtype": 2}, {"c": pages(page_size=17)}, {"b": batch(max_kv=700)}):
        assert f(**kw) == SHAPE, kw
    assert f(q=none, o=none, freq=None, rot=64) == SHAPE
    assert f(amp=math.inf) == SCALE and f(freq=I + 4) == ALIGN and f(k=rows(L + 8, 2)) == ALIGN and f(v=rows(W, 2, head_stride=8)) == STRIDE
    assert f(k=rows(K, 2)) == ALIAS and f(v=rows(V + 128, 2)) == ALIAS and f(o=rows(L, 4)) == ALIAS and f(o=rows(K, 4)) == ALIAS and f(o=rows(Q + 64, 4)) == ALIAS
    one = dict(token_stride=8 * 64)                                               # Q, K and V of one projection, Q in place
    assert f(q=rows(Q, 4, **one), o=rows(Q, 4, **one), k=rows(Q + 512, 2, **one), v=rows(Q + 768, 2, **one)) == 0
    assert f(q=rows(Q, 4, **one), o=rows(Q, 4, **one), k=rows(Q + 384, 2, **one), v=rows(Q + 768, 2, **one)) == ALIAS
    assert lib.kv_append(None, None, None, None, None, None, 0, None, 0, 0, 1.0, 0, None) == NULL


def test_pages_refuse(lib):
    def book(**kw):
        return kv._Book(**{"ref": I, "table": I + (1 << 20), "kv_len": I + (1 << 24), "pages": 100, "rows": 9, "table_width": 20, "table_stride": 20, "page_size": 16, **kw})

    def each(b, code):
        assert lib.kv_reserve(b, L, L, 1, W, None) == code and lib.kv_free(b, L, 1, None) == code
        assert lib.kv_fork(pages(), b, L, L, 1, W, None) == code and lib.kv_compact(pages(), b, W, 1 << 20, None) == code

    for name in ("ref", "table", "kv_len"):
        each(book(**{name: None}), NULL)
        each(book(**{name: I + (1 << 26) + 2}), ALIGN)
    for kw in ({"pages": 0}, {"rows": 0}, {"table_width": 0}, {"page_size": 15}, {"page_size": 8}, {"page_size": 8192}):
        each(book(**kw), SHAPE)
    each(book(table_stride=19), STRIDE)
    each(book(table_width=1 << 28, table_stride=1 << 28), OVERFLOW)
    each(book(kv_len=I), ALIAS)
    each(book(table=I + 16), ALIAS)
    b = book()
    for n in (-1, 8193):
        assert lib.kv_reserve(b, L, L, n, W, None) == lib.kv_free(b, L, n, None) == lib.kv_fork(pages(), b, L, L, n, W, None) == lib.kv_copy_pages(pages(), L, L, n, None) == SHAPE
    assert lib.kv_free(b, None, 0, None) == 0 and lib.kv_copy_pages(pages(), None, None, 0, None) == 0     # (nothing to do, nothing launched)
    assert lib.kv_reserve(b, None, L, 1, W, None) == lib.kv_reserve(b, L, None, 1, W, None) == lib.kv_reserve(b, L, L, 1, None, None) == NULL
    assert lib.kv_free(b, None, 1, None) == lib.kv_fork(pages(), b, L, None, 1, W, None) == lib.kv_fork(pages(), b, L, L, 1, None, None) == NULL
    assert lib.kv_free(b, L + 1, 1, None) == lib.kv_reserve(b, L, L, 1, W + 2, None) == lib.kv_copy_pages(pages(), L, L + 2, 1, None) == ALIGN
    for c in (pages(pages=99), pages(page_size=32)):
        assert lib.kv_fork(c, b, L, L, 1, W, None) == lib.kv_compact(c, b, W, 1 << 20, None) == SHAPE
    for c, code in ((pages(k=None), NULL), (pages(k=K + 4), ALIGN), (pages(layers=2, layer_stride=0), STRIDE), (pages(v=K), ALIAS)):
        assert lib.kv_fork(c, b, L, L, 1, W, None) == lib.kv_compact(c, b, W, 1 << 20, None) == lib.kv_copy_pages(c, L, L, 1, None) == code
    need = lib.kv_compact_workspace(100)
    assert lib.kv_compact(pages(), b, W, need - 1, None) == WORKSPACE and lib.kv_compact(pages(), b, None, need, None) == NULL
    assert lib.kv_compact(pages(), b, W + 8, need, None) == ALIGN and lib.kv_compact_workspace(0) == -1


def test_the_python_side_refuses():
    x = torch.zeros((3, 2, 64), dtype=torch.float16)
    c = torch.zeros((5, 2, 16, 64), dtype=torch.float16)
    n = torch.zeros(4, dtype=torch.int32)
    t = torch.zeros((3, 2), dtype=torch.int32)
    with pytest.raises(ValueError, match="device tensors"):
        kv.attn_paged(x, c, c, n, n[:3], t, x, None, 1, 1, 0.1)
    with pytest.raises(ValueError, match="contiguous"):
        kv.attn_paged(x[..., ::2], c, c, n, n[:3], t, x, None, 1, 1, 0.1)
    with pytest.raises(ValueError, match=r"\[tokens\]\[heads\]\[d\]"):
        kv.kv_append(x[:, :1], x, c, c, n, n[:3], t, 1, 1)
    y = torch.zeros((1, 2, 3, 64), dtype=torch.float16)
    with pytest.raises(ValueError, match="two tensors"):
        kv.rope(y, y[:, :1], torch.zeros(32, dtype=torch.float64))
    with pytest.raises(ValueError, match="pos"):
        kv.rope(y, y, torch.zeros(32, dtype=torch.float64), torch.zeros(4, dtype=torch.int32))
    with pytest.raises(ValueError, match="two tensors"):
        kv.kv_copy_pages(c, c, n, n)
    with pytest.raises(kv.KvCacheError) as e:
        kv.attn_paged_workspace(x, torch.zeros((5, 3, 16, 64), dtype=torch.float16), 1, 1, 1)
    assert e.value.code == -2
    with pytest.raises(ValueError, match="not supported"):
        kv.attn_paged_workspace(x, c.float(), 1, 1, 1)


def test_frequencies():
    plain = kv.rope_frequencies(64, 500.0)
    assert plain.dtype == torch.float64 and torch.allclose(plain, 500.0 ** (-torch.arange(32).double() / 32), rtol=1e-14)
    assert torch.allclose(kv.rope_frequencies(64, 500.0, kv.LINEAR, 4.0), plain / 4, rtol=1e-14)
    base = kv.rope_frequencies(64, 500.0, kv.BASE, 4.0)
    assert base[0] == 1 and math.isclose(base[-1], plain[-1] / 4, rel_tol=1e-12)                      # the slowest is stretched by the factor, the fastest stays
    parts = kv.rope_frequencies(64, 500.0, kv.PARTS, 4.0, 2048.0, 2.0, 20.0)
    turns = 2048 * plain / (2 * math.pi)
    assert torch.equal(parts[turns >= 20], plain[turns >= 20]) and torch.equal(parts[turns <= 2], plain[turns <= 2] / 4)
    mid = (turns > 2) & (turns < 20)
    keep = (turns - 2) / 18
    assert mid.any() and torch.allclose(parts[mid], (plain * keep + plain / 4 * (1 - keep))[mid], rtol=1e-13)
    lib, buf = kv._load(), (ctypes.c_double * 512)()
    ok = [buf, 64, 1e4, 3, 4.0, 100.0, 1.0, 32.0]
    assert lib.rope_frequencies(*ok) == 0 and lib.rope_frequencies(None, *ok[1:]) == NULL
    for i, bad in ((1, 0), (1, 3), (1, 1026), (2, 1.0), (2, math.inf), (2, math.nan), (3, 4), (3, -1), (4, 0.5), (4, math.nan), (5, 0.0), (5, math.inf), (6, -1.0), (7, 1.0), (7, math.inf)):
        assert lib.rope_frequencies(*ok[:i], bad, *ok[i + 1:]) == SHAPE, (i, bad)
    assert lib.rope_frequencies(buf, 2, 1e4, 2, 4.0, 0.0, 0.0, 0.0) == SHAPE


def test_what_the_extension_does_not_take():
    """CPU tensors, other counts of arguments and other types are left, untouched, to the general code."""
    from paper_2510_14719_amd import binding
    fast = binding._load_fast()
    x = torch.zeros((3, 2, 64), dtype=torch.float16)
    for f, n in ((fast.attn_paged, 16), (fast.kv_append, 17), (fast.rope, 8), (fast.kv_reserve, 8), (fast.kv_free, 6), (fast.kv_fork, 9), (fast.kv_compact, 7),
                 (fast.kv_copy_pages, 5)):
        for args in ([x] * n, [None] * n, [1] * n, [], [x] * (n + 1)):
            assert f(*args) is NotImplemented
    with pytest.raises(TypeError):
        fast.bind_kv(1)
    with pytest.raises(ValueError):
        fast.bind_kv(0, 0, 0, 0, 0, 0, 0, 0)
