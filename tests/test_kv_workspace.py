"""Workspaces of the attention over a paged cache, on the CPU: their sizes, and where they may begin."""
import random

import pytest

from paper_2510_14719_amd import kv_cache as kv


def need(sequences, tokens, max_q, max_kv, heads, key_heads, d=128, dtype=0):
    return kv._load().attn_paged_workspace(kv._Pages(heads=key_heads, d=d, dtype=dtype),
                                           kv._Batch(sequences=sequences, tokens=tokens, max_q=max_q, max_kv=max_kv), heads)


def test_all_parts_are_aligned():
    """The lists at the end of a workspace are read 16 bytes at a time: what stands before them is a multiple of that, and so are they."""
    rng = random.Random(1)
    assert need(65, 101, 100, 2500, 1, 1) % 16 == 0
    for _ in range(3000):
        key_heads = rng.choice((1, 1, 3, 5))
        n = need(rng.randint(1, 200), rng.randint(1, 999) | 1, rng.randint(1, 300), rng.randint(1, 9000), key_heads * rng.choice((1, 3, 5)), key_heads, rng.choice((64, 128)),
                 rng.choice((0, 2)))
        assert n >= 0 and n % 16 == 0


def test_no_more_than_the_pieces_take():
    """Partial results are those of the pieces that there can be: sequences that go by chunks have their own, of one round of the chip, and small tiles at most 32 rows of 272 or
    528 bytes for a piece of 1.25 MiB of keys and values."""
    G = 1 << 30
    assert need(5, 5 * 2048, 2048, 4096, 64, 16) < G // 8                         # prompts: none of them has small tiles
    assert need(24, 24 * 4096, 4096, 16384, 64, 16) < G // 8
    assert need(256, 256 * 4096, 4096, 65536, 64, 16) < 2 * G
    assert need(1, 1, 1, 1 << 20, 64, 8) < G // 16 and need(100, 100, 1, 1 << 20, 32, 4) < G // 16
    assert need(256, 256, 1, 65536, 64, 16) < G // 4
    rng = random.Random(2)
    for _ in range(5000):
        sequences, max_q, max_kv = (int(2 ** rng.uniform(0, e)) for e in (8, 12, 20))
        max_q = min(max_q, max_kv)
        key_heads, d, dtype = rng.choice((1, 2, 4, 8, 16)), rng.choice((64, 128)), rng.choice((0, 2))
        heads = key_heads * rng.choice([g for g in (1, 2, 3, 4, 5, 7, 8, 16) if g * key_heads <= 64])
        tokens = rng.choice((sequences, sequences * max_q, sequences + max_q))
        cache = sequences * max_kv * key_heads * 2 * d * (1 if dtype == 2 else 2)
        assert 0 <= need(sequences, tokens, max_q, max_kv, heads, key_heads, d, dtype) <= G // 16 + cache // 50
