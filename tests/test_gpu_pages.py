"""The page calls through the C ABI against a plain model in Python lists: table, references and lengths equal, every slot of every layer equal.
Single calls at their edges, then random sequences of calls."""
import numpy as np
import pytest
import torch

from paper_2609_04774_b200 import binding
from tests.serving_util import D, generator

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


class Model:
    """What the header says, on lists."""

    def __init__(self, pages, rows, width, page):
        self.N, self.page, self.width = pages, page, width
        self.ref = [0] * pages
        self.table = [[-1] * width for _ in range(rows)]
        self.len = [0] * rows
        self.slots = None          # [layers * 2][pages][page] stamps
        self.bad = False

    def free_ids(self):
        return [i for i, r in enumerate(self.ref) if r == 0]

    def need(self, n, more):
        return -(-(n + more) // self.page) - -(-n // self.page)

    def extend(self, new):
        ids, failed = self.free_ids(), False
        for r, more in enumerate(new):
            if more < 0 or self.len[r] + more > self.width * self.page:
                self.bad = True
                continue
            n = self.need(self.len[r], more)
            if n and (failed or n > len(ids)):
                failed = self.bad = True
                continue
            first = -(-self.len[r] // self.page)
            for i in range(n):
                self.table[r][first + i] = ids.pop(0)
                self.ref[self.table[r][first + i]] = 1
            self.len[r] += more

    def drop(self, r, e):
        p, self.table[r][e] = self.table[r][e], -1
        if p == -1:
            return
        if not 0 <= p < self.N or self.ref[p] <= 0:
            self.bad = True
            return
        self.ref[p] -= 1

    def evict(self, window, sinks):
        for r, n in enumerate(self.len):
            for e in range(self.width):
                if e * self.page >= sinks and (e + 1) * self.page - 1 < n + 1 - window:
                    self.drop(r, e)

    def free(self, rows):
        for r in rows:
            if not 0 <= r < len(self.len):
                self.bad = True
                continue
            for e in range(self.width):
                self.drop(r, e)
            self.len[r] = 0

    def fork(self, parent, child):
        ids = self.free_ids()
        for p, c in zip(parent, child):
            if not (0 <= p < len(self.len) and 0 <= c < len(self.len) and p != c):
                self.bad = True
                continue
            n = self.len[p]
            full, part = n // self.page, n % self.page
            row = self.table[p][:full] + [-1] * (self.width - full)
            for e in range(full):
                if row[e] != -1:
                    self.ref[row[e]] += 1
            self.len[c] = n
            if part:
                src = self.table[p][full]
                if 0 <= src < self.N and ids:
                    row[full] = ids.pop(0)
                    self.ref[row[full]] = 1
                    self.slots[:, row[full], :part] = self.slots[:, src, :part]
                else:
                    self.bad = True
                    self.len[c] = full * self.page
            self.table[c] = row

    def compact(self):
        live = [i for i in range(self.N) if self.ref[i] > 0]
        n = len(live)
        holes = [i for i in range(n) if self.ref[i] == 0]
        new = [i if self.ref[i] > 0 else -1 for i in range(self.N)]
        for src, dst in zip([i for i in live if i >= n], holes):
            new[src] = dst
            self.ref[dst], self.ref[src] = self.ref[src], 0
            self.slots[:, dst] = self.slots[:, src]
        self.table = [[new[p] if 0 <= p < self.N and new[p] >= 0 else p for p in row] for row in self.table]
        return new, n


class State:
    """The same state on the device; a slot's row (all heads and elements) carries its stamp."""

    def __init__(self, pages=40, rows=7, width=9, page=16, layers=3, Hkv=2, fp8=False, strided=False, seed=0):
        self.m = Model(pages, rows, width, page)
        self.layers, self.Hkv = layers, Hkv
        g = generator(seed)
        stamps = torch.randint(0, 120, (2 * layers, pages, page), generator=g, device="cuda", dtype=torch.int32)
        self.m.slots = stamps.cpu().numpy().copy()
        dtype = torch.uint8 if fp8 else torch.bfloat16
        self.k, self.v = [], []
        for i in range(2 * layers):
            shape = (pages, page, Hkv, D)
            if strided:
                t = torch.zeros(pages, Hkv + 1, page + 1, D, dtype=dtype, device="cuda")[:, :Hkv, :page].permute(0, 2, 1, 3)
            else:
                t = torch.empty(shape, dtype=dtype, device="cuda")
            t.copy_(self.pattern(stamps[i]).to(dtype))
            (self.v if i & 1 else self.k).append(t)
        self.pool = binding.make_page_pool(self.k, self.v)
        self.ref = torch.zeros(pages, dtype=torch.int32, device="cuda")
        self.table = torch.full((rows, width), -1, dtype=torch.int32, device="cuda")
        self.len = torch.zeros(rows, dtype=torch.int32, device="cuda")
        self.ws = torch.full((binding.cp_workspace_bytes_pages(pages, 64),), 0xA5, dtype=torch.uint8, device="cuda")
        self.map, self.n_live = torch.zeros(pages, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")

    def pattern(self, stamps):
        """[..., Hkv, D] whole numbers below 256 (exact in both types) that differ between the rows and vectors of a slot."""
        h = torch.arange(self.Hkv, device="cuda")[:, None] * 16 + torch.arange(D, device="cuda")[None, :] // 8
        return (stamps[..., None, None] + h) % 256

    def ints(self, values):
        return torch.tensor(values, dtype=torch.int32, device="cuda")

    def extend(self, ctx, new):
        self.m.extend(new)
        binding.cp_pages_extend(ctx, self.pool, self.ref, self.table, self.len, self.ints(new), self.ws)

    def evict(self, ctx, window, sinks):
        self.m.evict(window, sinks)
        binding.cp_pages_evict(ctx, self.pool, self.ref, self.table, self.len, window, sinks)

    def free(self, ctx, rows):
        self.m.free(rows)
        binding.cp_pages_free(ctx, self.pool, self.ref, self.table, self.len, self.ints(rows))

    def fork(self, ctx, parent, child):
        self.m.fork(parent, child)
        binding.cp_pages_fork(ctx, self.pool, self.ref, self.table, self.len, self.ints(parent), self.ints(child), self.ws)

    def compact(self, ctx):
        new, n = self.m.compact()
        binding.cp_pages_compact(ctx, self.pool, self.ref, self.table, self.map, self.n_live, self.ws)
        assert self.map.tolist() == new and int(self.n_live) == n

    def copy(self, ctx, src, dst):
        for s, d in zip(src, dst):
            if 0 <= s < self.m.N and 0 <= d < self.m.N:
                self.m.slots[:, d] = self.m.slots[:, s]
            else:
                self.m.bad = True
        binding.cp_pages_copy(ctx, self.pool, self.ints(src), self.ints(dst), self.ws)

    def check(self, ctx, what=""):
        torch.cuda.synchronize()
        if self.m.bad:
            with pytest.raises(binding.CpError) as e:
                ctx.poll_status()
            assert e.value.code == binding.CP_ERR_BOUNDS, what
            self.m.bad = False
        ctx.poll_status()
        assert self.ref.tolist() == self.m.ref, what
        assert self.table.tolist() == self.m.table, what
        assert self.len.tolist() == self.m.len, what
        want = torch.from_numpy(self.m.slots).cuda()
        for i in range(2 * self.layers):
            got = (self.v if i & 1 else self.k)[i >> 1]
            assert torch.equal(got.to(torch.int32), self.pattern(want[i]).to(torch.int32)), (what, i)


@pytest.mark.parametrize("page,Hkv,fp8,strided", [(16, 2, False, False), (32, 1, True, False), (64, 3, False, True), (128, 8, True, True), (16, 16, False, False)])
def test_every_call_on_every_layout(ctx, page, Hkv, fp8, strided):
    s = State(page=page, Hkv=Hkv, fp8=fp8, strided=strided)
    s.extend(ctx, [1, 0, page, page + 1, 3 * page - 1, 5 * page, 0])
    s.check(ctx, "extend")
    s.fork(ctx, [4, 3], [1, 6])
    s.check(ctx, "fork")
    s.evict(ctx, page, 1)
    s.check(ctx, "evict")
    s.free(ctx, [3, 0])
    s.check(ctx, "free")
    s.compact(ctx)
    s.check(ctx, "compact")
    s.copy(ctx, [0, 1, 2], [30, 31, 39])
    s.check(ctx, "copy")


@pytest.mark.parametrize("seed", range(12))
def test_random_sequences_of_calls(ctx, seed):
    rng = np.random.default_rng(seed)
    page = [16, 32, 64, 128][seed % 4]
    rows, width = int(rng.integers(2, 40)), int(rng.integers(2, 12))
    s = State(pages=int(rng.integers(3, 120)), rows=rows, width=width, page=page, layers=1 + seed % 3, Hkv=1 + seed % 2, seed=seed)
    for step in range(40):
        op = rng.integers(0, 6)
        if op <= 1:
            s.extend(ctx, [int(x) if rng.random() < 0.5 else 0 for x in rng.integers(0, 2 * page, rows)])
        elif op == 2:
            s.evict(ctx, int(rng.integers(1, 3 * page)), int(rng.integers(0, 2 * page)))
        elif op == 3:
            s.free(ctx, [int(x) for x in rng.integers(0, rows, int(rng.integers(0, 4)))])
        elif op == 4:
            order = rng.permutation(rows)
            n = int(rng.integers(0, rows // 2 + 1))
            child = [int(x) for x in order[:n]]
            parent = [int(x) for x in rng.choice(order[n:], n)]
            if child:
                s.free(ctx, child)
            s.fork(ctx, parent, child)
        else:
            s.compact(ctx)
        s.check(ctx, (seed, step, int(op)))


def test_extend_when_the_pool_or_a_row_is_full(ctx):
    s = State(pages=5, rows=4, width=3)
    s.extend(ctx, [16, 33, 16, 5])                          # rows 0 and 1 take 4, row 2 takes the last, row 3 gets none
    s.check(ctx)
    assert s.len.tolist() == [16, 33, 16, 0]
    s.extend(ctx, [0, 14, 0, 0])                            # no new page needed
    s.check(ctx)
    s.extend(ctx, [0, 2, 0, 0])                             # the row's table is full
    s.check(ctx)
    s.extend(ctx, [-1, 0, 0, 0])
    s.check(ctx)
    s.free(ctx, [0])
    s.extend(ctx, [0, 0, 17, 3])                            # one page free, row 2 wants two: neither row gets any
    s.check(ctx)
    assert s.len.tolist() == [0, 47, 16, 0]


def test_fork_without_pages_and_with_bad_rows(ctx):
    s = State(pages=4, rows=6, width=4)
    s.extend(ctx, [40, 0, 0, 0, 0, 0])
    s.fork(ctx, [0, 0, 0], [1, 2, 3])                       # one free page for three partly filled tails
    s.check(ctx)
    assert s.len.tolist() == [40, 40, 32, 32, 0, 0]
    s.fork(ctx, [0, 9, -1, 4], [4, 5, 5, 4])
    s.check(ctx)


def test_fork_of_empty_full_and_evicted_rows(ctx):
    s = State(pages=30, rows=6, width=6)
    s.extend(ctx, [0, 32, 90, 0, 0, 0])
    s.evict(ctx, 20, 10)
    s.fork(ctx, [0, 1, 2], [3, 4, 5])
    s.check(ctx)
    assert s.table[5].tolist()[1:4] == [-1, -1, -1]
    s.free(ctx, [2, 5, 2])
    s.check(ctx)


def test_windows_of_evict(ctx):
    for window, sinks in ((1, 0), (16, 0), (17, 0), (5, 16), (5, 17), (binding.CP_NO_WINDOW, 0), (1, 10 ** 12), (2 ** 40, 3), (100, 40)):
        s = State(pages=40, rows=4, width=9)
        s.extend(ctx, [0, 16, 100, 144])
        s.evict(ctx, window, sinks)
        s.check(ctx, (window, sinks))


def test_entries_that_name_no_page_are_reported(ctx):
    s = State(pages=10, rows=3, width=4)
    s.extend(ctx, [40, 20, 0])
    s.table[0, 1] = 10
    s.m.table[0][1] = 10
    s.free(ctx, [0])
    s.check(ctx)
    s.table[2, 0] = int(s.ref.argmin())                     # a free page
    s.m.table[2][0] = int(s.ref.argmin())
    s.free(ctx, [2, 7])
    s.check(ctx)
    s.copy(ctx, [0, 10, 3, 4], [9, 1, -1, 8])
    s.check(ctx)


def test_compact_at_its_edges(ctx):
    s = State(pages=33, rows=3, width=12)
    s.compact(ctx)                                          # nothing in use
    s.check(ctx)
    s.extend(ctx, [33, 160, 160])
    s.compact(ctx)                                          # already dense
    s.check(ctx)
    s.free(ctx, [0])
    s.compact(ctx)
    s.check(ctx)
    full = State(pages=12, rows=1, width=12)
    full.extend(ctx, [192])
    full.compact(ctx)                                       # no page free
    full.check(ctx)


def test_large_pool(ctx):
    """More pages than one step of the scan, rows beyond one pass."""
    pages, rows, width = 30000, 2500, 12
    s = State(pages=pages, rows=rows, width=width, layers=1, Hkv=1)
    rng = np.random.default_rng(1)
    s.extend(ctx, [int(x) for x in rng.integers(0, 190, rows)])
    s.check(ctx, "extend")
    s.free(ctx, [int(x) for x in rng.permutation(rows)[:1200]])
    s.check(ctx, "free")
    child = [i for i in range(rows) if s.m.len[i] == 0][:1100]
    parent = [i for i in range(rows) if s.m.len[i] > 0]
    s.ws = torch.empty(binding.cp_workspace_bytes_pages(pages, 1100), dtype=torch.uint8, device="cuda")
    s.fork(ctx, [parent[i % len(parent)] for i in range(len(child))], child)
    s.check(ctx, "fork")
    s.free(ctx, parent[:600])
    s.compact(ctx)
    s.check(ctx, "compact")
    s.extend(ctx, [int(x) for x in rng.integers(0, 60, rows)])
    s.check(ctx, "extend again")


def test_captured_step_replays_on_changing_lengths(ctx):
    s = State(pages=40, rows=5, width=9)
    s.extend(ctx, [5, 30, 60, 0, 16])
    new = s.ints([1, 1, 1, 0, 1])
    torch.cuda.synchronize()
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        binding.cp_pages_evict(ctx, s.pool, s.ref, s.table, s.len, 20, 16, stream=stream)
        binding.cp_pages_extend(ctx, s.pool, s.ref, s.table, s.len, new, s.ws, stream=stream)
    for _ in range(40):
        graph.replay()
        s.m.evict(20, 16)
        s.m.extend([1, 1, 1, 0, 1])
    s.check(ctx)


def test_captured_forks_and_compaction(ctx):
    s = State(pages=60, rows=8, width=9, layers=2)
    s.extend(ctx, [5, 30, 60, 0, 0, 0, 0, 16])
    parent, child, drop = s.ints([1, 2, 1]), s.ints([3, 4, 5]), s.ints([1, 5])
    torch.cuda.synchronize()
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        binding.cp_pages_fork(ctx, s.pool, s.ref, s.table, s.len, parent, child, s.ws, stream=stream)
        binding.cp_pages_free(ctx, s.pool, s.ref, s.table, s.len, drop, stream=stream)
        binding.cp_pages_compact(ctx, s.pool, s.ref, s.table, s.map, s.n_live, s.ws, stream=stream)
    for more in ([0, 0, 3, 0, 0, 0, 0, 0], [0, 21, 0, 0, 0, 0, 0, 40]):
        graph.replay()
        s.m.fork([1, 2, 1], [3, 4, 5])
        s.m.free([1, 5])
        s.m.compact()
        s.check(ctx, "replay")
        s.free(ctx, [3, 4, 5])
        s.extend(ctx, more)
        s.check(ctx, "between")


def test_binding_refuses_what_the_call_would_misread(ctx):
    s = State()
    with pytest.raises(ValueError):
        binding.cp_pages_evict(ctx, s.pool, s.ref.long(), s.table, s.len, 5, 0)
    with pytest.raises(ValueError):
        binding.cp_pages_evict(ctx, s.pool, s.ref, s.table.T, s.len, 5, 0)
    with pytest.raises(ValueError):
        binding.cp_pages_evict(ctx, s.pool, s.ref[:3], s.table, s.len, 5, 0)
    with pytest.raises(ValueError):
        binding.make_page_pool(s.k, s.v[:1])
    with pytest.raises(binding.CpError) as e:
        binding.cp_pages_extend(ctx, s.pool, s.ref, s.table, s.len, s.len, s.ws[:256])
    assert e.value.code == binding.CP_ERR_WORKSPACE
