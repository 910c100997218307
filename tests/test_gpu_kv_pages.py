"""The upkeep of pages against a model in Python: tables, counts and lengths are equal after every call, and contents follow their pages."""
import random

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    from paper_2510_14719_amd import kv_cache
    return kv_cache


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Model:
    def __init__(self, layers, pages, heads, page, d, dtype, rows, width, order):
        self.page, self.rows, self.width, self.pages = page, rows, width, pages
        shape = (layers, pages, page, heads, d) if order == "token" else (layers, pages, heads, page, d)
        g = torch.Generator().manual_seed(1)
        self.kv = [torch.randint(0, 100, shape, generator=g).to(dtype).cuda() for _ in "kv"]
        if order == "token":
            self.kv = [x.transpose(2, 3) for x in self.kv]
        self.dev = [torch.zeros(pages, dtype=torch.int32, device="cuda"), torch.full((rows, width + 3), -5, dtype=torch.int32, device="cuda")[:, :width],
                    torch.zeros(rows, dtype=torch.int32, device="cuda")]
        self.missing = ints([99])
        self.ref, self.table, self.len = [0] * pages, [[-5] * width for _ in range(rows)], [0] * rows
        self.want = [x.cpu().clone() for x in self.kv]

    def held(self, n):
        return min(-(-min(max(n, 0), self.width * self.page) // self.page), self.width)

    def free_pages(self):
        return [p for p in range(self.pages) if self.ref[p] == 0]

    def check(self, what, missing=None):
        torch.cuda.synchronize()
        ref, table, length = (x.tolist() for x in self.dev)
        assert ref == self.ref, what + ": ref"
        assert table == self.table, what + ": table"
        assert length == self.len, what + ": kv_len"
        if missing is not None:
            assert self.missing.tolist() == [missing], what
        for x, y in zip(self.kv, self.want):
            assert torch.equal(x.cpu().view(torch.uint8), y.view(torch.uint8)), what + ": contents"

    def reserve(self, rows, lens):
        free, missing = self.free_pages(), 0
        for r, n in zip(rows, lens):
            if not 0 <= r < self.rows:
                continue
            n = min(n, self.width * self.page)
            for j in range(self.held(self.len[r]), self.held(n)):
                if free:
                    self.table[r][j] = free.pop(0)
                    self.ref[self.table[r][j]] = 1
                else:
                    self.table[r][j] = -1
                    missing += 1
            self.len[r] = max(self.len[r], n)
        return missing

    def release(self, rows):
        for r in rows:
            if 0 <= r < self.rows:
                for j in range(self.held(self.len[r])):
                    if 0 <= self.table[r][j] < self.pages:
                        self.ref[self.table[r][j]] -= 1
                    self.table[r][j] = -1
                self.len[r] = 0

    def fork(self, src, dst):
        free, missing = self.free_pages(), 0
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
                if free:
                    p, old = free.pop(0), self.table[s][full]
                    self.table[d][full] = p
                    self.ref[p] = 1
                    if 0 <= old < self.pages:
                        for x in self.want:
                            x[:, p] = x[:, old]
                else:
                    missing += 1
            self.len[d] = n
        return missing

    def compact(self):
        n = sum(r > 0 for r in self.ref)
        to = [p for p in range(n) if self.ref[p] <= 0]
        new = dict(zip([p for p in range(n, self.pages) if self.ref[p] > 0], to))
        for a, b in new.items():
            self.ref[b], self.ref[a] = self.ref[a], 0
            for x in self.want:
                x[:, b] = x[:, a]
        for r in range(self.rows):
            for j in range(self.held(self.len[r])):
                self.table[r][j] = new.get(self.table[r][j], self.table[r][j])


@pytest.mark.parametrize("layers,pages,heads,page,d,dtype,rows,width,order", [
    (1, 5, 1, 16, 64, torch.float16, 3, 3, "head"), (3, 60, 2, 16, 128, torch.bfloat16, 9, 12, "token"),
    (2, 400, 3, 32, 64, torch.float8_e4m3fn, 40, 30, "head"), (1, 9001, 1, 16, 64, torch.float8_e4m3fn, 300, 80, "token"),
    (1, 4096, 1, 16, 64, torch.float16, 1200, 4, "head"), (2, 30, 2, 1024, 128, torch.float16, 5, 7, "head")])
def test_against_the_model(kv, layers, pages, heads, page, d, dtype, rows, width, order):
    m = Model(layers, pages, heads, page, d, dtype, rows, width, order)
    rng = random.Random(pages)
    ws = torch.full((kv.kv_compact_workspace(pages),), 0xff, dtype=torch.uint8, device="cuda")
    some = lambda most: rng.sample(range(rows), rng.randint(1, max(1, min(rows, most))))  # noqa: E731
    for turn in range(14):
        what = rng.choice(("reserve", "reserve", "free", "fork", "compact")) if turn else "reserve"
        print("turn %d: %s" % (turn, what), flush=True)
        missing = None
        if what == "reserve":
            list_ = some(rows)
            lens = [rng.randint(0, min(width * page + 40, max(1, 3 * pages * page // rows))) for _ in list_]
            list_, lens = list_ + [-1, rows], lens + [50, 50]
            missing = m.reserve(list_, lens)
            kv.kv_reserve(*m.dev, ints(list_), ints(lens), m.missing, page)
        elif what == "free":
            list_ = some(max(1, rows // 2))
            list_ += [list_[0], -3, rows + 5]                                     # (a row twice counts once)
            m.release(list_)
            kv.kv_free(*m.dev, ints(list_), page)
        elif what == "fork":
            order_ = some(rows)
            cut = rng.randint(0, len(order_))
            src = [rng.choice(order_[:cut]) for _ in order_[cut:]] if cut else []
            dst = order_[cut:] if cut else []
            m.release(dst)
            kv.kv_free(*m.dev, ints(dst), page)
            src, dst = src + [rows, 0, 0], dst + [0, -1, 0]                       # (the last: onto itself, nothing happens)
            missing = m.fork(src, dst)
            kv.kv_fork(*m.kv, *m.dev, ints(src), ints(dst), m.missing)
        else:
            m.compact()
            kv.kv_compact(*m.kv, *m.dev, ws)
        m.check("turn %d %s" % (turn, what), missing)


def test_lists_of_many_and_of_none(kv):
    m = Model(1, 20000, 1, 16, 64, torch.float8_e4m3fn, 8192, 3, "head")
    kv.kv_reserve(*m.dev, ints([]), ints([]), m.missing, 16)
    m.check("empty reserve", 0)
    rows = list(range(8192))
    random.Random(3).shuffle(rows)
    lens = [(7 * r) % 49 for r in rows]
    missing = m.reserve(rows, lens)
    kv.kv_reserve(*m.dev, ints(rows), ints(lens), m.missing, 16)
    m.check("8192 rows", missing)
    m.release(rows[::3])
    kv.kv_free(*m.dev, ints(rows[::3]), 16)
    kv.kv_free(*m.dev, ints([]), 16)
    kv.kv_fork(*m.kv, *m.dev, ints([]), ints([]), m.missing)
    m.check("a third freed", 0)
    kv.kv_compact(*m.kv, *m.dev, torch.empty(kv.kv_compact_workspace(20000), dtype=torch.uint8, device="cuda"))
    m.compact()
    m.check("compacted")


def test_lengths_that_make_no_sense(kv):
    """Lengths beyond the table or below zero: nothing out of range is touched."""
    m = Model(1, 8, 1, 16, 64, torch.float16, 3, 2, "head")
    whole = m.dev[1]
    m.dev[2].copy_(ints([2 ** 31 - 1, -2 ** 31, 5]))
    kv.kv_reserve(*m.dev, ints([0, 1, 2]), ints([2 ** 31 - 1, -4, 2 ** 31 - 1]), m.missing, 16)
    kv.kv_fork(*m.kv, *m.dev, ints([0]), ints([1]), m.missing)
    kv.kv_compact(*m.kv, *m.dev, torch.empty(kv.kv_compact_workspace(8), dtype=torch.uint8, device="cuda"))
    kv.kv_free(*m.dev, ints([0, 1, 2]), 16)
    torch.cuda.synchronize()
    assert m.dev[2].tolist() == [0, 0, 0] and bool((whole._base[:, 2:] == -5).all() if whole._base is not None else True)


@pytest.mark.parametrize("dtype,order", [(torch.float16, "head"), (torch.float8_e4m3fn, "token")])
def test_copy_pages(kv, dtype, order):
    m = Model(3, 30, 2, 16, 64, dtype, 1, 1, order)
    src, dst = [3, 5, 3, -1, 7, 30, 2 ** 31 - 1], [10, 11, 12, 13, 30, 14, 15]
    kv.kv_copy_pages(*m.kv, ints(src), ints(dst))
    kv.kv_copy_pages(*m.kv, ints([]), ints([]))
    for x in m.want:
        x[:, [10, 11, 12]] = x[:, [3, 5, 3]]
    m.check("copy")


def test_a_captured_step(kv):
    """Fork, reserve and free in a graph: every replay equals the eager calls, with other work in between."""
    a, b = (Model(2, 64, 1, 16, 64, torch.float16, 6, 8, "head") for _ in "ab")
    src, dst, grow, lens = ints([0, 0, 1]), ints([3, 4, 5]), ints([3, 4]), ints([70, 100])

    def step(m):
        kv.kv_free(*m.dev, dst, 16)
        kv.kv_fork(*m.kv, *m.dev, src, dst, m.missing)
        kv.kv_reserve(*m.dev, grow, lens, m.missing, 16)

    for m in (a, b):
        kv.kv_reserve(*m.dev, ints([0, 1, 2]), ints([50, 33, 16]), m.missing, 16)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a)
    for turn in range(4):
        graph.replay()
        step(b)
        for m in (a, b):
            kv.kv_reserve(*m.dev, ints([turn % 3]), ints([50 + 9 * turn]), m.missing, 16)
        torch.cuda.synchronize()
        for x, y in zip(a.dev + a.kv, b.dev + b.kv):
            assert torch.equal(x, y)
