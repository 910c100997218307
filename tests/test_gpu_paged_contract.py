"""What the header promises of the operators around a paged cache where pages, lengths or values are not as they should be."""
import math
import random

import pytest
import torch

from tests.paged_util import Batch, check, workspace_for
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
