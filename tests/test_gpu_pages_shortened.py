"""Rows whose length the caller lowered (rejected draft tokens): the pages behind the new end stay theirs and the next extend uses them, so the
references always equal the table's entries."""
import numpy as np
import pytest
import torch

from paper_2609_04774_b200 import binding
from tests.test_gpu_pages import Model, State

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


class HeldModel(Model):
    """extend as the header says it: entries behind the end that name a page of the row's own are used again, shared ones are given up."""

    def extend(self, new):
        def span(r):
            return range(-(-self.len[r] // self.page), -(-(self.len[r] + new[r]) // self.page))
        fits = [more >= 0 and self.len[r] + more <= self.width * self.page for r, more in enumerate(new)]
        ref = list(self.ref)
        for r in range(len(new)):
            for e in span(r) if fits[r] else ():
                p = self.table[r][e]
                if 0 <= p < self.N and ref[p] == 1:
                    continue
                if 0 <= p < self.N and ref[p] > 1:
                    self.ref[p] -= 1
                self.table[r][e] = -1
        ids, failed = self.free_ids(), False
        for r, more in enumerate(new):
            if not fits[r]:
                self.bad = True
                continue
            missing = [e for e in span(r) if self.table[r][e] == -1]
            if missing and (failed or len(missing) > len(ids)):
                failed = self.bad = True
                continue
            for e in missing:
                self.table[r][e] = ids.pop(0)
                self.ref[self.table[r][e]] = 1
            self.len[r] += more


class Held(State):
    def __init__(self, **kw):
        super().__init__(**kw)
        m, self.m = self.m, HeldModel(self.m.N, len(self.m.table), self.m.width, self.m.page)
        self.m.slots = m.slots

    def shorten(self, rows, lens):
        for r, n in zip(rows, lens):
            assert n <= self.m.len[r]
            self.m.len[r] = n
            self.len[r] = n

    def balanced(self):
        """Every reference is an entry of the table."""
        t = self.table[self.table >= 0].long()
        assert torch.equal(torch.bincount(t, minlength=self.m.N).to(torch.int32), self.ref)


def test_rejected_drafts_over_a_page_boundary(ctx):
    s = Held(pages=6, rows=2, width=5)
    s.extend(ctx, [15, 3])
    for _ in range(20):                                    # four drafts, the first accepted: 19 -> 16, then 16 -> 17 and back by three
        s.extend(ctx, [4, 0])
        s.check(ctx)
        s.balanced()
        s.shorten([0], [min(s.m.len[0] - 3, 17)])
    assert int((s.ref > 0).sum()) == 3


def test_a_row_shortened_by_several_pages(ctx):
    s = Held(pages=12, rows=3, width=9)
    s.extend(ctx, [100, 20, 0])
    s.shorten([0], [5])
    s.extend(ctx, [40, 0, 0])                              # 5 -> 45: pages 1 and 2 are still there
    s.check(ctx)
    s.balanced()
    s.extend(ctx, [90, 0, 0])                              # to 135: four more held ones and two fresh
    s.check(ctx)
    s.balanced()
    s.shorten([0], [0])
    s.free(ctx, [0])
    s.check(ctx)
    s.balanced()


def test_a_full_pool_serves_the_rows_that_hold_their_pages(ctx):
    s = Held(pages=8, rows=3, width=9)
    s.extend(ctx, [80, 48, 0])
    s.shorten([0, 1], [33, 17])
    s.extend(ctx, [40, 31, 0])                             # no page is free, none is needed
    s.check(ctx)
    s.balanced()
    s.shorten([0], [10])
    s.extend(ctx, [100, 0, 1])                             # row 0 misses two pages: it and the row behind it get none
    s.check(ctx)
    s.balanced()


def test_entries_behind_the_end_that_are_shared_or_name_no_used_page(ctx):
    s = Held(pages=20, rows=4, width=6)
    s.extend(ctx, [64, 0, 0, 0])
    s.fork(ctx, [0, 0], [1, 2])                            # four full pages with three references each
    s.shorten([0, 1], [16, 32])
    s.extend(ctx, [48, 32, 0, 5])                          # pages 1 to 3 and 2 to 3 stay row 2's, the others take fresh ones
    s.check(ctx)
    s.balanced()
    s.shorten([0, 1, 2], [0, 0, 0])
    s.extend(ctx, [64, 64, 64, 0])                         # page 0 is given up by all three and handed out again
    s.check(ctx)
    s.balanced()
    s.table[3, 1], s.table[3, 2], s.table[3, 3] = 20, -9, int(s.ref.argmin())      # no page, no page, a free one
    s.m.table[3][1:4] = s.table[3, 1:4].tolist()
    s.extend(ctx, [0, 0, 0, 60])
    s.check(ctx)
    s.balanced()


@pytest.mark.parametrize("rows", [3, 1100])
def test_long_spans_and_many_rows(ctx, rows):
    """Spans far beyond the entries that one thread looks at by itself, rows beyond one pass."""
    s = Held(pages=rows * 24 + 200, rows=rows, width=60, layers=1, Hkv=1)
    rng = np.random.default_rng(rows)
    big = [int(x) for x in rng.permutation(rows)[:3]]
    s.extend(ctx, [16 * 50 if r in big else int(rng.integers(0, 200)) for r in range(rows)])
    s.shorten(range(rows), [int(rng.integers(0, n + 1)) if rng.random() < 0.7 else n for n in s.m.len])
    s.extend(ctx, [960 - s.m.len[r] if r in big else int(rng.integers(0, 150)) for r in range(rows)])
    s.check(ctx)
    s.balanced()


@pytest.mark.parametrize("seed", range(6))
def test_random_calls_with_rejected_tokens(ctx, seed):
    rng = np.random.default_rng(100 + seed)
    page = [16, 32, 64][seed % 3]
    rows, width = int(rng.integers(2, 20)), int(rng.integers(2, 10))
    s = Held(pages=int(rng.integers(10, 120)), rows=rows, width=width, page=page, layers=1, Hkv=1, seed=seed)
    for step in range(40):
        op = rng.integers(0, 5)
        if op <= 1:
            s.extend(ctx, [int(x) if rng.random() < 0.6 else 0 for x in rng.integers(0, 3 * page, rows)])
        elif op == 2:
            few = [int(x) for x in rng.permutation(rows)[:3]]
            s.shorten(few, [int(rng.integers(0, s.m.len[r] + 1)) for r in few])
        elif op == 3:
            s.free(ctx, [int(rng.integers(0, rows))])
        else:
            s.compact(ctx)
        s.check(ctx, (seed, step, int(op)))
        s.balanced()


def test_captured_step_with_rejected_tokens(ctx):
    s = Held(pages=40, rows=4, width=9)
    s.extend(ctx, [5, 30, 60, 0])
    new, back = s.ints([5, 5, 5, 0]), s.ints([3, 5, 1, 0])
    torch.cuda.synchronize()
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        binding.cp_pages_extend(ctx, s.pool, s.ref, s.table, s.len, new, s.ws, stream=stream)
        s.len.sub_(back)                                   # the lengths are lowered on the device
    for _ in range(15):
        graph.replay()
        s.m.extend([5, 5, 5, 0])
        s.m.len = [n - b for n, b in zip(s.m.len, [3, 5, 1, 0])]
        s.check(ctx)
        s.balanced()
