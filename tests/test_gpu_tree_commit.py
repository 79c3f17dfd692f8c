"""cp_tree_plan and cp_tree_commit through the C ABI against plain Python: every tree shape, padding, reports, paths whose slots overlap, page ends, every
kind of pool, strided pools, replayed graphs."""
import random

import pytest
import torch

from paper_2609_04774_b200 import binding
from tests.tree_util import as_i64, masks_of, random_tree

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def plan(ctx, parent, tree_len, kv_len, axes=1):
    B, n_q = parent.shape
    mask = torch.full((B, n_q), 77, dtype=torch.int64, device="cuda")
    positions = torch.full((axes, B * n_q), 77, dtype=torch.int32, device="cuda")
    seq, slot = torch.full((B * n_q,), 77, dtype=torch.int32, device="cuda"), torch.full((B * n_q,), 77, dtype=torch.int32, device="cuda")
    binding.cp_tree_plan(ctx, parent, tree_len, kv_len, mask, positions, seq, slot)
    torch.cuda.synchronize()
    return mask, positions, seq, slot


def bounds(ctx):
    with pytest.raises(binding.CpError) as e:
        ctx.poll_status()
    assert e.value.code == binding.CP_ERR_BOUNDS


@pytest.mark.parametrize("n_q", [1, 2, 5, 31, 32, 33, 63, 64])
@pytest.mark.parametrize("axes", [1, 3])
def test_plan(ctx, n_q, axes):
    rng = random.Random(n_q)
    parents, lens, kv = [], [], []
    for b in range(70):
        m = rng.choice([0, 1, n_q, rng.randrange(n_q + 1)])
        parents.append([random_tree(rng, m), list(range(-1, m - 1)), [-1] * m][b % 3])      # any, a chain, a bush
        lens.append(m)
        kv.append(m + rng.choice([0, 1, rng.randrange(100000)]))
    table = i32([p + [rng.randrange(-5, 99) for _ in range(n_q - len(p))] for p in parents])        # behind a tree: anything
    mask, positions, seq, slot = plan(ctx, table, i32(lens), i32(kv), axes)
    ctx.poll_status()
    for b, p in enumerate(parents):
        masks, m, base = masks_of(p), lens[b], kv[b] - lens[b]
        pad = n_q - m
        assert mask[b].tolist() == as_i64(masks) + [0] * pad
        at = slice(b * n_q, (b + 1) * n_q)
        for a in range(axes):
            assert positions[a, at].tolist() == [base + bin(x).count("1") - 1 for x in masks] + [0] * pad
        assert seq[at].tolist() == [b] * m + [-1] * pad
        assert slot[at].tolist() == [base + t for t in range(m)] + [0] * pad


def test_plan_without_lengths_and_reports(ctx):
    parent = i32([[-1, 0, 1], [-1, -1, 0]])
    mask, _, _, slot = plan(ctx, parent, None, i32([3, 10]))
    ctx.poll_status()
    assert mask.tolist() == [[1, 3, 7], [1, 2, 5]] and slot.tolist() == [0, 1, 2, 7, 8, 9]
    for bad in ([[-1, 1, 0]], [[-1, 2, 0]], [[-2, 0, 1]], [[0, -1, 1]], [[-1, 10 ** 9, 0]]):
        mask, _, _, _ = plan(ctx, i32(bad), None, i32([9]))
        bounds(ctx)
        fixed = [p if -1 <= p < t else -1 for t, p in enumerate(bad[0])]
        assert mask[0].tolist() == masks_of(fixed)
    for m, kv, counts in ((4, 9, 3), (-1, 9, 0), (3, 2, 2), (3, -5, 0)):
        mask, _, seq, _ = plan(ctx, i32([[-1, 0, 1]]), i32([m]), i32([kv]))
        bounds(ctx)
        assert mask[0].tolist() == [1, 3, 7][:counts] + [0] * (3 - counts) and seq.tolist() == [0] * counts + [-1] * (3 - counts)


class Pool:
    """Layers of random bytes in a shuffled pool; rows[b] tokens in sequence b."""

    def __init__(self, seed, rows, layers, Hkv, page, kind, pad=0, width=None):
        g = torch.Generator("cuda")
        g.manual_seed(seed)
        self.page = page
        counts = [-(-n // page) for n in rows]
        n = sum(counts) + 2
        ids = torch.randperm(n, generator=g, device="cuda").to(torch.int32)
        self.table = torch.full((len(rows), width or max(1, max(counts))), -1, dtype=torch.int32, device="cuda")
        at = 0
        for b, c in enumerate(counts):
            self.table[b, :c] = ids[at:at + c]
            at += c
        if kind == "mx4":
            shape, cut = (layers, n, page, binding.mx4_token_bytes(Hkv) + pad), binding.mx4_token_bytes(Hkv)
        else:
            shape, cut = (layers, n, page, Hkv, 128 + pad), 128
        make = lambda: torch.randint(0, 256, shape, generator=g, device="cuda", dtype=torch.uint8)[..., :cut]  # noqa: E731
        if kind == "bf16":
            make = lambda: torch.randint(-2 ** 15, 2 ** 15, shape, generator=g, device="cuda", dtype=torch.int16)[..., :cut].view(torch.bfloat16)  # noqa: E731
        self.k, self.v = make(), make()
        self.pool = (binding.make_page_pool_mx4 if kind == "mx4" else binding.make_page_pool)(self.k, self.v)

    def bits(self, x):
        return x.view(torch.int16) if x.dtype == torch.bfloat16 else x


def commit_reference(pool, parents, kv, lens, accepted):
    """What the call leaves behind: (k, v as integers, kv_len, paths)."""
    out = [pool.bits(pool.k).clone(), pool.bits(pool.v).clone()]
    before = [x.clone() for x in out]
    new_len, paths = [], []
    for b, p in enumerate(parents):
        path, a = [], accepted[b]
        while a >= 0:
            path.append(a)
            a = p[a]
        path.reverse()
        base = kv[b] - lens[b]
        for i, node in enumerate(path):
            src, dst = base + node, base + i
            ps, pd = int(pool.table[b, src // pool.page]), int(pool.table[b, dst // pool.page])
            for x, y in zip(before, out):
                y[:, pd, dst % pool.page] = x[:, ps, src % pool.page]
        new_len.append(base + len(path))
        paths.append(path)
    return out[0], out[1], new_len, paths


def run_commit(ctx, pool, parents, kv, lens, accepted, n_q, tree_len=True):
    table = i32([p + [5] * (n_q - len(p)) for p in parents])
    kv_len = i32(kv)
    path = torch.full(table.shape, 77, dtype=torch.int32, device="cuda")
    want = commit_reference(pool, parents, kv, lens, accepted)
    binding.cp_tree_commit(ctx, pool.pool, pool.table, kv_len, i32(lens) if tree_len else None, table, i32(accepted), path)
    torch.cuda.synchronize()
    assert torch.equal(pool.bits(pool.k), want[0]) and torch.equal(pool.bits(pool.v), want[1])
    assert kv_len.tolist() == want[2]
    for b, p in enumerate(want[3]):
        assert path[b].tolist() == p + [-1] * (n_q - len(p))


@pytest.mark.parametrize("kind,Hkv,pad", [("bf16", 2, 0), ("bf16", 3, 8), ("fp8", 2, 0), ("fp8", 5, 16), ("mx4", 8, 0), ("mx4", 3, 16), ("mx4", 1, 0)])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("n_q", [1, 9, 64])
def test_commit(ctx, kind, Hkv, pad, page, n_q):
    rng = random.Random(page + n_q)
    parents, lens, kv, accepted = [], [], [], []
    for b in range(13):
        m = rng.choice([1, n_q, rng.randrange(1, n_q + 1)]) if b else 0
        parents.append([random_tree(rng, m), list(range(-1, m - 1)), [-1] * m][b % 3])
        lens.append(m)
        kv.append(m + rng.choice([0, page - 1, page, rng.randrange(300)]))
        accepted.append(-1 if m == 0 else rng.choice([-1, m - 1, rng.randrange(m)]))
    pool = Pool(n_q, kv, 3, Hkv, page, kind, pad)
    run_commit(ctx, pool, parents, kv, lens, accepted, n_q)
    ctx.poll_status()


def test_paths_through_every_second_slot(ctx):
    """New slots are old slots of the same path: 1 -> 0, 3 -> 1, 5 -> 2, .. over more tokens than one batch of loads holds."""
    parent = [-1, -1] + [t - 2 for t in range(2, 64)]
    for base in (0, 7, 100):
        pool = Pool(base, [base + 64], 5, 4, 16, "bf16")
        run_commit(ctx, pool, [parent], [base + 64], [64], [63], 64, tree_len=False)
    ctx.poll_status()


def test_many_layers_and_sequences(ctx):
    rng = random.Random(1)
    B, n_q = 150, 16
    parents = [random_tree(rng, n_q) for _ in range(B)]
    kv = [n_q + rng.randrange(100) for _ in range(B)]
    pool = Pool(3, kv, 128, 1, 16, "fp8")
    run_commit(ctx, pool, parents, kv, [n_q] * B, [rng.randrange(-1, n_q) for _ in range(B)], n_q)
    ctx.poll_status()


def test_commit_reports(ctx):
    for accepted in (3, -2, 10 ** 9):
        pool = Pool(3, [20], 2, 2, 16, "bf16")
        k = pool.bits(pool.k).clone()
        kv_len, path = i32([20]), i32([[7, 7, 7, 7]])
        binding.cp_tree_commit(ctx, pool.pool, pool.table, kv_len, i32([3]), i32([[-1, 0, 1, 2]]), i32([accepted]), path)
        torch.cuda.synchronize()
        bounds(ctx)
        assert kv_len.tolist() == [17] and path.tolist() == [[-1] * 4] and torch.equal(pool.bits(pool.k), k)
    # a slot without a page: reported, the other tokens move
    for bad in (-1, 10 ** 8):
        pool = Pool(3, [40], 2, 2, 16, "bf16")
        k = pool.bits(pool.k).clone()
        page = int(pool.table[0, 1])
        pool.table[0, 2] = bad
        kv_len, path = i32([34]), i32([[7] * 6])
        binding.cp_tree_commit(ctx, pool.pool, pool.table, kv_len, None, i32([[-1, -1, 1, 2, 3, 4]]), i32([5]), path)      # slots 28..33, the last two on page 2
        torch.cuda.synchronize()
        bounds(ctx)
        want = k.clone()
        want[:, page, 12:15] = k[:, page, 13:16]
        assert torch.equal(pool.bits(pool.k), want) and kv_len.tolist() == [33] and path.tolist() == [[1, 2, 3, 4, 5, -1]]
    # a broken parent on the path ends it there
    pool = Pool(3, [20], 2, 2, 16, "bf16")
    kv_len, path = i32([20]), i32([[7] * 4])
    binding.cp_tree_commit(ctx, pool.pool, pool.table, kv_len, None, i32([[-1, 9, 1, 2]]), i32([3]), path)
    torch.cuda.synchronize()
    bounds(ctx)
    assert path.tolist() == [[1, 2, 3, -1]] and kv_len.tolist() == [19]


def test_empty_batches(ctx):
    pool = Pool(3, [20], 2, 2, 16, "bf16")
    e = lambda *s: torch.empty(s, dtype=torch.int32, device="cuda")  # noqa: E731
    binding.cp_tree_commit(ctx, pool.pool, e(0, 5), e(0), e(0), e(0, 4), e(0), e(0, 4))
    binding.cp_tree_plan(ctx, e(0, 4), None, e(0), torch.empty((0, 4), dtype=torch.int64, device="cuda"), e(1, 0), e(0), e(0))


def test_replayed_steps(ctx):
    """A captured commit follows the lengths, trees and accepted tokens of every replay."""
    rng = random.Random(4)
    n_q, kv = 12, [40, 90]
    pool = Pool(3, kv, 2, 2, 16, "bf16")
    parent, kv_len, tree_len, accepted, path = i32([[0] * n_q] * 2), i32(kv), i32([n_q] * 2), i32([-1, -1]), i32([[0] * n_q] * 2)
    mask, positions = torch.empty(2, n_q, dtype=torch.int64, device="cuda"), torch.empty(1, 2 * n_q, dtype=torch.int32, device="cuda")
    seq, slot = torch.empty(2 * n_q, dtype=torch.int32, device="cuda"), torch.empty(2 * n_q, dtype=torch.int32, device="cuda")
    parent.copy_(i32([random_tree(rng, n_q)] * 2))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        binding.cp_tree_plan(ctx, parent, tree_len, kv_len, mask, positions, seq, slot)
        binding.cp_tree_commit(ctx, pool.pool, pool.table, kv_len, tree_len, parent, accepted, path)
    for _ in range(4):
        lens = [rng.randrange(1, n_q + 1) for _ in range(2)]
        parents = [random_tree(rng, m) for m in lens]
        now = [rng.randrange(m, n + 1) for m, n in zip(lens, kv)]
        acc = [rng.randrange(-1, m) for m in lens]
        parent.copy_(i32([p + [-1] * (n_q - len(p)) for p in parents]))
        tree_len.copy_(i32(lens))
        kv_len.copy_(i32(now))
        accepted.copy_(i32(acc))
        want = commit_reference(pool, parents, now, lens, acc)
        graph.replay()
        torch.cuda.synchronize()
        ctx.poll_status()
        assert torch.equal(pool.bits(pool.k), want[0]) and torch.equal(pool.bits(pool.v), want[1]) and kv_len.tolist() == want[2]
        assert mask[0].tolist() == masks_of(parents[0]) + [0] * (n_q - lens[0])
