"""The page operations of the cache against a model in plain Python lists: which page goes where, reference counts, and the bytes that move (exactly)."""
import random

import pytest
import torch

from cache_cases import starts

pytestmark = pytest.mark.gpu


class Model:
    """What include/fbq.h says the operations do, one page and one token after another."""

    def __init__(self, layers, pages, page, heads, D, rows, width, dtype):
        self.page, self.width = page, width
        self.pool = torch.zeros(layers, pages, 2, heads, page, D, dtype=dtype)
        self.table = [[-1] * width for _ in range(rows)]
        self.lengths, self.refs = [0] * rows, [0] * pages

    def need(self, n):
        return -(-n // self.page)

    def free_pages(self):
        return [p for p, r in enumerate(self.refs) if r == 0]

    def reserve(self, count):
        free, start, asked, lacking = self.free_pages(), [], 0, 0
        had = len(free)
        for b, c in enumerate(count):
            c, n = max(c, 0), self.lengths[b]
            k = self.need(n + c) - self.need(n)
            if n + c > self.width * self.page:
                start.append(-1)
                continue
            asked += k
            if k and asked > had:
                start.append(-1)
                continue
            for i in range(k):
                p = free.pop(0)
                self.refs[p] = 1
                self.table[b][self.need(n) + i] = p
            start.append(n)
            self.lengths[b] = n + c
        return start, max(0, asked - had)

    def append(self, layer, k, v, start, counts):
        t = 0
        for b, c in enumerate(counts):
            for i in range(c):
                pos = start[b] + i
                if start[b] >= 0 and pos < self.width * self.page and self.table[b][pos // self.page] >= 0:
                    at = self.pool[layer, self.table[b][pos // self.page]]
                    at[0, :, pos % self.page], at[1, :, pos % self.page] = k[t], v[t]
                t += 1

    def free(self, rows):
        for b in rows:
            if 0 <= b < len(self.table):
                for p in self.table[b]:
                    if p >= 0:
                        self.refs[p] -= 1
                self.table[b], self.lengths[b] = [-1] * self.width, 0

    def fork(self, pairs):
        free, asked, skipped = self.free_pages(), 0, 0
        had, lengths = len(free), list(self.lengths)
        for a, b in pairs:
            if not (0 <= a < len(lengths) and 0 <= b < len(lengths)) or a == b or lengths[b]:
                skipped += 1
                continue
            n = lengths[a]
            part = n % self.page > 0
            asked += part
            if part and asked > had:
                skipped += 1
                continue
            for i in range(n // self.page):
                self.table[b][i] = self.table[a][i]
                self.refs[self.table[a][i]] += 1
            if part:
                p = free.pop(0)
                self.refs[p] = 1
                self.table[b][n // self.page] = p
                self.pool[:, p] = self.pool[:, self.table[a][n // self.page]]
            self.lengths[b] = n
        return max(0, asked - had), skipped

    def compact(self):
        live = [p for p, r in enumerate(self.refs) if r > 0]
        holes = [p for p in range(len(live)) if self.refs[p] == 0]
        moved = dict(zip([p for p in live if p >= len(live)], holes))
        for a, b in moved.items():
            self.pool[:, b] = self.pool[:, a]
            self.refs[a], self.refs[b] = 0, self.refs[a]
        self.table = [[moved.get(p, p) for p in row] for row in self.table]
        return len(live), len(moved)


class Pair:
    """The model and the library's cache, the same operations on both."""

    def __init__(self, layers, pages, page, heads, D, rows, width, dtype=torch.float16):
        import paper_2501_16385_amd as fbq
        self.fbq, self.m = fbq, Model(layers, pages, page, heads, D, rows, width, dtype)
        self.c = fbq.cache_create(layers, pages, page, heads, D, rows, width, dtype)
        self.c.pool.zero_()
        self.ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")

    def reserve(self, count):
        info = self.ints([99])
        start = self.fbq.cache_reserve(self.c, self.ints(count), info=info)
        want, lacking = self.m.reserve(count)
        assert start.tolist() == want and info.tolist() == [lacking]
        self.same()
        return start, want

    def append(self, counts, start, want, single=False, fused=0, seed=0):
        T, (layers, _, _, heads, _, D) = sum(counts), self.c.pool.shape
        g = torch.Generator().manual_seed(seed)
        for layer in range(layers):
            wide = torch.randn(T, 2 * heads + fused, D, generator=g).to(self.c.pool.dtype)
            k, v = wide[:, fused:fused + heads], wide[:, fused + heads:]
            dev = wide.cuda()
            self.fbq.cache_append(self.c, layer, dev[:, fused:fused + heads], dev[:, fused + heads:], start, q_start=None if single else starts(counts).cuda())
            self.m.append(layer, k, v, want, counts)
        self.same()

    def add(self, counts, **how):
        start, want = self.reserve(counts)
        self.append(counts, start, want, **how)

    def free(self, rows):
        self.fbq.cache_free(self.c, self.ints(rows))
        self.m.free(rows)
        self.same()

    def fork(self, pairs):
        info = self.ints([99, 99])
        self.fbq.cache_fork(self.c, self.ints([a for a, _ in pairs]), self.ints([b for _, b in pairs]), info=info)
        assert info.tolist() == list(self.m.fork(pairs))
        self.same()

    def compact(self, in_place):
        info = self.ints([99, 99])
        if in_place:
            self.fbq.cache_compact(self.c, info=info)
        else:
            before = self.c.table.clone(), self.c.refs.clone()
            out = self.fbq.Cache(self.c.pool, torch.full_like(self.c.table, 77), self.c.lengths, torch.full_like(self.c.refs, 77))
            assert self.fbq.cache_compact(self.c, out=out, info=info) is out
            assert torch.equal(self.c.table, before[0]) and torch.equal(self.c.refs, before[1])
            self.c = out
        assert info.tolist() == list(self.m.compact())
        self.same()

    def same(self):
        torch.cuda.synchronize()
        assert self.c.table.tolist() == self.m.table
        assert self.c.lengths.tolist() == self.m.lengths
        assert self.c.refs.tolist() == self.m.refs
        assert torch.equal(self.c.pool.cpu().view(torch.int16), self.m.pool.view(torch.int16))


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("heads,D,dtype", [(1, 16, torch.float16), (3, 72, torch.bfloat16), (2, 256, torch.float16)])
def test_append_across_pages(page, heads, D, dtype):
    p = Pair(2, 24, page, heads, D, 3, 7, dtype)
    p.add([page + 1, 0, 3], seed=1)
    p.add([1, 1, 1], single=True, seed=2)
    p.add([2 * page - 2, 5, page], fused=2, seed=3)
    p.add([0, 0, 1], seed=4)


def test_reserve_gives_nothing_to_those_for_whom_pages_do_not_suffice():
    p = Pair(1, 6, 16, 1, 16, 5, 4)
    p.add([20, 16, 1, 0, 0])                                   # four pages
    p.reserve([12, 0, 15, 33, 0])                              # none, none, none, three of two: refused
    p.reserve([1, 1, 1, 0, 0])                                 # one, one, one of two: the third refused
    p.reserve([0, 0, 0, 1, 0])
    p.free([1])
    p.reserve([5, -3, 0, 1, 0])
    p.reserve([1 << 30, 70, 64, 1, 2])                         # longer than a row of the table: refused, and no page counted


def test_reserve_of_more_rows_and_pages_than_a_block_has_threads():
    rnd = random.Random(5)
    p = Pair(1, 9000, 16, 1, 16, 2500, 6)
    p.reserve([rnd.randint(0, 60) for _ in range(2500)])
    p.free(rnd.sample(range(2500), 1300))
    p.reserve([rnd.choice([0, 0, 1, 20, 50]) for _ in range(2500)])
    p.free(rnd.sample(range(2500), 400))
    p.compact(True)
    p.reserve([rnd.randint(0, 96) for _ in range(2500)])       # more than there is
    p.compact(False)


def test_free_takes_rows_out_of_range_as_none():
    p = Pair(1, 10, 16, 1, 16, 3, 3)
    p.add([17, 4, 40])
    p.free([2, -1, 3, 0])
    p.add([1, 2, 3])


@pytest.mark.parametrize("layers,page,heads,D", [(1, 16, 1, 16), (3, 32, 2, 72), (2, 64, 5, 128)])
def test_fork_shares_full_pages_and_copies_the_last(layers, page, heads, D):
    p = Pair(layers, 40, page, heads, D, 12, 5)
    p.add([2 * page + 3, 2 * page, 0, 5] + [0] * 8, seed=1)
    p.fork([(0, 4), (1, 5), (2, 6), (3, 7), (0, 8)])
    p.add([1, 1, 1, 1, 1, 1, 1, 1, 1, 0, 0, 0], seed=2)         # nobody writes into a page of another's
    p.free([0, 4])
    p.fork([(8, 0), (5, 4), (5, 9)])
    p.fork([(8, 8), (8, 5), (-1, 10), (12, 10), (8, 12), (8, -2), (8, 11)])   # itself, not empty, out of range; the last is served
    p.free([8, 0, 11, 1, 5, 4, 9, 3, 7, 2, 6])
    assert all(r >= 0 for r in p.m.refs)


def test_fork_without_pages_for_all_and_chains():
    p = Pair(1, 4, 16, 1, 16, 8, 3)
    p.add([20, 0, 0, 0, 0, 0, 0, 0])
    p.fork([(0, 1), (1, 2), (0, 3), (0, 4), (0, 5)])           # a parent that is a child of the same call is still empty; two pages for three
    p.fork([(0, 6)])


def test_fork_of_many_pairs():
    rnd = random.Random(8)
    p = Pair(1, 5000, 16, 1, 16, 3000, 4)
    p.add([rnd.randint(0, 60) if b < 400 else 0 for b in range(3000)])
    p.fork([(rnd.randrange(400), b) for b in range(400, 3000)])
    p.free(list(range(0, 3000, 3)))
    p.compact(True)


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("layers,pages,page,heads,D", [(1, 2, 16, 1, 16), (2, 30, 16, 2, 64), (3, 50, 128, 2, 80), (1, 4097, 16, 1, 16), (1, 13000, 16, 1, 16)])
def test_compact(layers, pages, page, heads, D, in_place):
    rnd = random.Random(pages)
    rows = 9 if pages < 1000 else 900
    width = max(1, 3 * pages // rows // 2)
    p = Pair(layers, pages, page, heads, D, rows, width)
    p.compact(in_place)                                        # nothing in use
    p.add([rnd.randint(0, width * page) for _ in range(rows)] if pages > 2 else [16] + [0] * 8, seed=1)
    p.compact(in_place)                                        # already compact
    gone = rnd.sample(range(rows), rows // 2)
    p.free(gone)
    p.compact(in_place)
    p.fork([(a, b) for a, b in zip([r for r in range(rows) if r not in gone], gone)])
    p.free([r for r in range(rows) if r not in gone])
    p.compact(in_place)


@pytest.mark.parametrize("pages", [4096, 8192])
def test_compact_of_a_pool_in_use_to_the_last_page(pages):
    p = Pair(1, pages, 16, 1, 16, 4, pages)
    p.reserve([16 * pages // 2, 16 * pages // 2, 0, 0])
    p.compact(True)
    p.free([0])
    p.compact(False)


def test_copy_pages():
    import paper_2501_16385_amd as fbq
    cache = fbq.cache_create(3, 20, 64, 3, 80, 1, 1)
    cache.pool.normal_()
    want = cache.pool.clone()
    src, dst = [3, 5, 25, 7, 0], [9, 1, 2, -1, 19]             # two pairs name no page: skipped
    for a, b in zip(src, dst):
        if 0 <= a < 20 and 0 <= b < 20:
            want[:, b] = want[:, a]
    fbq.cache_copy(cache, torch.tensor(src, dtype=torch.int32).cuda(), torch.tensor(dst, dtype=torch.int32).cuda())
    assert torch.equal(cache.pool, want)


def test_append_skips_what_has_no_place():
    import paper_2501_16385_amd as fbq
    cache = fbq.cache_create(1, 4, 16, 1, 16, 4, 2)
    cache.pool.zero_()
    cache.table.copy_(torch.tensor([[0, 1 << 20], [1, -1], [2, 3], [-7, 3]]))
    k = torch.randn(4, 1, 16).half().cuda()
    fbq.cache_append(cache, 0, k, k, torch.tensor([16, 16, -1, 5], dtype=torch.int32).cuda())
    fbq.cache_append(cache, 0, k, k, torch.tensor([40, 1 << 30, 32, 0], dtype=torch.int32).cuda())
    assert (cache.pool == 0).all()
    # tokens outside every row's range of q_start go nowhere
    fbq.cache_append(cache, 0, k, k, torch.tensor([0, 0, 0, 0], dtype=torch.int32).cuda(), q_start=torch.tensor([1, 2, 2, 3, 3], dtype=torch.int32).cuda())
    want = torch.zeros_like(cache.pool)
    want[0, 0, :, :, 0], want[0, 2, :, :, 0] = k[1], k[2]
    assert torch.equal(cache.pool, want)


def test_random_life_of_a_cache():
    rnd = random.Random(11)
    p = Pair(2, 60, 16, 2, 24, 10, 8)
    for step in range(40):
        do = rnd.choice(["add", "add", "add", "free", "fork", "compact"])
        empty = [b for b in range(10) if p.m.lengths[b] == 0]
        if do == "add":
            p.add([rnd.choice([0, 1, 1, 2, 30]) for _ in range(10)], seed=step)
        elif do == "free":
            p.free(rnd.sample(range(10), rnd.randint(1, 4)))
        elif do == "fork" and empty:
            p.fork([(rnd.randrange(10), b) for b in rnd.sample(empty, rnd.randint(1, len(empty)))])
        else:
            p.compact(rnd.random() < 0.5)


def test_a_step_of_every_operation_in_a_replayed_graph():
    """reserve, append, attention, free, fork and compaction captured once: replays do on the device what eager calls do."""
    import paper_2501_16385_amd as fbq

    def build():
        p = Pair(1, 80, 16, 1, 64, 6, 12)
        p.add([20, 33, 0, 7, 0, 0], seed=3)
        return p.c

    def buffers():
        i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
        return {"k": torch.zeros(6, 1, 64, dtype=torch.float16, device="cuda"), "q": torch.zeros(6, 2, 64, dtype=torch.float16, device="cuda"), "count": i32(1, 1, 0, 1, 0, 0),
                "start": i32(*[0] * 6), "rows": i32(4, 5), "parent": i32(0, 1), "info": i32(0, 0), "out": torch.zeros(6, 2, 64, dtype=torch.float16, device="cuda")}

    def step(c, x, ws, stream=None):
        fbq.cache_reserve(c, x["count"], start=x["start"], stream=stream)
        fbq.cache_append(c, 0, x["k"], x["k"], x["start"], stream=stream)
        fbq.cache_free(c, x["rows"], stream=stream)
        fbq.cache_fork(c, x["parent"], x["rows"], workspace=ws[0], stream=stream)
        fbq.cache_compact(c, info=x["info"], workspace=ws[1], stream=stream)
        fbq.attention(c, 0, x["q"], out=x["out"], workspace=ws[2], stream=stream)

    eager, graphed = build(), build()
    x, y = buffers(), buffers()
    ws = [torch.empty(1 << 16, dtype=torch.uint8, device="cuda") for _ in range(2)] + [fbq.attention_workspace(eager, x["q"])]
    side = torch.cuda.Stream()
    warm = build()
    with torch.cuda.stream(side):
        step(warm, buffers(), ws, side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(graphed, y, ws, side)
    for it in range(5):
        for z in (x, y):
            z["k"].copy_(torch.randn(6, 1, 64, generator=torch.Generator().manual_seed(it)).half())
            z["q"].copy_(torch.randn(6, 2, 64, generator=torch.Generator().manual_seed(50 + it)).half())
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        step(eager, x, ws)
        torch.cuda.synchronize()
        assert torch.equal(x["out"], y["out"]) and torch.equal(eager.table, graphed.table) and torch.equal(eager.refs, graphed.refs), it
        assert torch.equal(eager.lengths, graphed.lengths) and torch.equal(eager.pool, graphed.pool) and torch.isfinite(x["out"]).all(), it


def test_the_workspace_that_a_cache_keeps_serves_larger_calls_and_graphs():
    """A captured fork goes on with the workspace it was captured with after a larger call has needed another."""
    rows = 700
    p = Pair(1, 900, 16, 1, 16, rows, 2)
    p.add([20, 5] + [0] * (rows - 2))
    parent, child = p.ints([0, 1]), p.ints([2, 3])
    p.fork([(0, 2), (1, 3)])
    p.free([2, 3])
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        p.fbq.cache_fork(p.c, parent, child, stream=side)
    p.fork([(0, b) for b in range(10, 600)])                   # more pairs than the first workspace holds
    filler = [torch.full((1 << 14,), 0x7F, dtype=torch.uint8, device="cuda") for _ in range(50)]
    torch.cuda.synchronize()
    graph.replay()
    p.m.fork([(0, 2), (1, 3)])
    p.same()
    assert all((f == 0x7F).all() for f in filler)
    p.compact(True)
