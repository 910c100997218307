"""Calls around the paged cache that are refused before any HIP call, beyond those of test_kv_cache_abi.py."""
import pytest
import torch

from paper_2510_14719_amd import kv_cache as kv
from tests.test_kv_cache_abi import ALIAS, I, K, L, O, OVERFLOW, Q, V, W, batch, pages, rows  # noqa: F401


@pytest.fixture(scope="module")
def lib():
    return kv._load()


def book(**kw):
    return kv._Book(**{"ref": I, "table": I + (1 << 20), "kv_len": I + (1 << 24), "pages": 100, "rows": 9, "table_width": 20, "table_stride": 20, "page_size": 16, **kw})


def test_a_reserve_whose_pages_cannot_be_counted(lib):
    """8192 rows of 2^18 entries: with lengths that the device does not check, 2^31 pages would be wanted, and their sum is an int."""
    wide = book(rows=8192, table_width=1 << 18, table_stride=1 << 18, kv_len=I + (1 << 34))
    assert lib.kv_reserve(wide, L, L + (1 << 16), 8192, W, None) == OVERFLOW


def test_attention_whose_outputs_overlap_what_it_reads(lib):
    c = pages(dtype=2, k_scale=I + (1 << 20), v_scale=I + (1 << 20) + 256)
    b = batch(max_kv=60000, table_width=4000, table_stride=4000)                  # (a table of 48000 bytes)
    need = lib.attn_paged_workspace(c, b, 4)

    def f(o=O, lse=L, ws=W):
        return lib.attn_paged_check_args(c, b, rows(Q, 4), rows(o, 4), lse, 4, 0.125, 0, ws, need)

    assert need > 0 and f() == 0
    for inside in (I, I + 4096, I + 8192 + 47984, I + (1 << 20), I + (1 << 20) + 256):
        assert f(o=inside) == ALIAS and f(lse=inside) == ALIAS and f(ws=inside) == ALIAS, hex(inside)
    assert f(lse=I + 8192 + 48000) == 0 and f(lse=I + 4096 + 16) == 0              # (behind the table, behind the lengths)


def test_append_whose_outputs_overlap_what_it_reads(lib):
    freq = I + (1 << 21)
    scales = dict(dtype=2, k_scale=I + (1 << 20), v_scale=I + (1 << 20) + 256)

    def f(o=O, **kw):
        return lib.kv_append_check_args(pages(**scales, **kw), batch(), rows(L, 2), rows(W, 2), rows(Q, 4), rows(o, 4), 4, freq, 64, 0, 1.0, 0)

    assert f() == 0
    for inside in (I, I + 4096, I + 8192, I + (1 << 20), I + (1 << 20) + 256, freq + 240):
        assert f(o=inside) == ALIAS and f(k=inside) == ALIAS and f(v=inside) == ALIAS, hex(inside)
    assert f(o=freq + 256) == 0


def test_queries_without_a_place_and_a_place_without_queries():
    k, cache = torch.zeros((3, 2, 64), dtype=torch.float16), torch.zeros((5, 2, 16, 64), dtype=torch.float16)
    ints, table = torch.zeros(4, dtype=torch.int32), torch.zeros((3, 2), dtype=torch.int32)
    for half in ({"q": k}, {"q_out": k}):
        with pytest.raises(ValueError, match="both or neither"):
            kv.kv_append(k, k, cache, cache, ints, ints[:3], table, 1, 1, **half)


def test_numbers_beyond_an_int():
    """Not cut to their lower 32 bits, which would be another call's."""
    q, cache = torch.zeros((3, 2, 64), dtype=torch.float16), torch.zeros((5, 2, 16, 64), dtype=torch.float16)
    ints, table = torch.zeros(4, dtype=torch.int32), torch.zeros((3, 2), dtype=torch.int32)
    big = 2 ** 32
    for call in (lambda: kv.attn_paged_workspace(q, cache, big + 1, 1, 32), lambda: kv.attn_paged_workspace(q, cache, 1, big + 1, 32), lambda: kv.attn_paged_workspace(q, cache, 1, 1, big + 32),
                 lambda: kv.kv_compact_workspace(big + 5), lambda: kv.rope_frequencies(big + 64), lambda: kv._batch(ints, ints[:3], table, 3, big + 1, 32),
                 lambda: kv._batch(ints, ints[:3], table, 3, 1, big + 32)):
        with pytest.raises(kv.KvCacheError) as e:
            call()
        assert e.value.code == OVERFLOW


def meets(c, lib):
    """kv_copy_pages of nothing: only the cache is looked at."""
    return lib.kv_copy_pages(c, None, None, 0, None)


def test_keys_and_values_that_meet(lib):
    """Of a cache that is written.  Side by side in every order of the dimensions they do not meet; 16 bytes nearer they do."""
    P, H, T, d, layers = 6, 3, 16, 64, 2
    for dtype, es in ((0, 2), (2, 1)):
        for order in ("LPHT2", "LPH2T", "LP2HT", "L2PHT", "2LPHT", "LPTH2", "LPT2H", "PL2TH", "P2LHT"):
            size, stride = {"L": layers, "P": P, "H": H, "T": T, "2": 2}, {}
            at = d
            for x in reversed(order):
                stride[x] = at
                at *= size[x]
            c = dict(layers=layers, pages=P, heads=H, page_size=T, d=d, dtype=dtype, layer_stride=stride["L"], page_stride=stride["P"], head_stride=stride["H"],
                     token_stride=stride["T"], k=K)
            assert meets(pages(**c, v=K + stride["2"] * es), lib) == 0, order
            c["k"] = K + stride["2"] * es
            assert meets(pages(**c, v=K), lib) == 0, order
            for nearer in (16, -16):
                assert meets(pages(**c, v=c["k"] + nearer), lib) == ALIAS, (order, nearer)
    for v in range(K + 16, K + 100 * 2048, 2048 + 16):                            # one behind the other, but not far enough
        assert meets(pages(v=v), lib) == ALIAS
    assert meets(pages(v=K + 100 * 2 * 16 * 64 * 2), lib) == 0
    c = pages(v=K + 2048)
    assert lib.kv_append_check_args(c, batch(), rows(L, 2), rows(W, 2), kv._Rows(), kv._Rows(), 0, None, 0, 0, 1.0, 0) == ALIAS


def test_books_that_overlap_what_is_read_or_written(lib):
    b, small = book(), pages(pages=100)
    table, kv_len = I + (1 << 20), I + (1 << 24)
    for inside in (I, I + 396, table, table + 716, kv_len, kv_len + 32):
        assert lib.kv_reserve(b, inside, L, 2, W, None) == lib.kv_reserve(b, L, inside, 2, W, None) == lib.kv_reserve(b, L, L, 2, inside, None) == ALIAS
        assert lib.kv_free(b, inside, 2, None) == ALIAS
        assert lib.kv_fork(small, b, inside, L, 2, W, None) == lib.kv_fork(small, b, L, inside, 2, W, None) == lib.kv_fork(small, b, L, L, 2, inside, None) == ALIAS
    for at in (I, table, kv_len):
        assert lib.kv_compact(small, b, at, 1 << 20, None) == ALIAS
        for kw in ({"k": at}, {"v": at}):
            assert lib.kv_fork(pages(**kw), b, L, L, 2, W, None) == lib.kv_compact(pages(**kw), b, W, 1 << 20, None) == ALIAS
    for inside in (K, K + 16, V + 100 * 2 * 16 * 64 * 2 - 16):                     # in the cache
        assert lib.kv_fork(small, b, inside, L, 2, W, None) == lib.kv_fork(small, b, L, inside, 2, W, None) == lib.kv_fork(small, b, L, L, 2, inside, None) == ALIAS
        assert lib.kv_copy_pages(small, inside, L, 2, None) == lib.kv_copy_pages(small, L, inside, 2, None) == ALIAS
    assert lib.kv_compact(small, b, V, 1 << 20, None) == ALIAS
    assert lib.kv_reserve(b, L, L + 8, 2, L + 4, None) == lib.kv_fork(small, b, L, L + 8, 2, L + 12, None) == ALIAS       # `missing` in a list


def test_many_chunks_fit_a_grid(lib):
    """4194304 tokens of 64 heads on 16: 65536 chunks of each of 16 key heads, 2^20 workgroups of the 2^23 that there may be."""
    b = batch(sequences=64, tokens=1 << 22, max_q=1 << 16, max_kv=1 << 16, table_width=4096, table_stride=4096)
    wide = dict(token_stride=64 * 64)
    assert lib.attn_paged_check_args(pages(heads=16, pages=1 << 18), b, rows(1 << 42, 64, **wide), rows(1 << 43, 64, **wide), None, 64, 0.125, 0, 1 << 44, 1 << 40) == 0
    far = dict(heads=16, pages=1 << 18)
    b = batch(sequences=64, tokens=1 << 25, max_q=1 << 20, max_kv=1 << 16, table_width=4096, table_stride=4096)
    assert lib.attn_paged_check_args(pages(**far), b, rows(1 << 42, 64, **wide), rows(1 << 43, 64, **wide), None, 64, 0.125, 0, 1 << 44, 1 << 40) == OVERFLOW
