"""Tree attention through the C ABI against the definition in 64 bits: every kind of cache, narrow and wide forms, trees of different sizes, masks of any
bits, windows and sinks at every edge, unread slots that hold NaN, infinities in drafted values, strided pools, cut units, replayed graphs, refusals on
the device."""
import math
import random

import pytest
import torch

from paper_2609_04774_b200 import binding
from tests.tree_util import FULL, D, TreeStep, trees

pytestmark = pytest.mark.gpu
KINDS = ["bf16", "fp8", "mx4"]


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


BASES = [0, 1, 15, 16, 63, 100, 127, 128, 129, 500, 1999]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(8, 4), (16, 2), (12, 1)])
def test_bases_and_sizes(ctx, kind, page, Hq, Hkv):
    sizes = [1, 7, 3, 20, 5, 2, 11, 20, 1, 16, 9]
    TreeStep(page + Hq, BASES, trees(page, sizes), Hq, Hkv, page, kind).check(ctx)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("Hq,Hkv,n_q", [(1, 1, 1), (1, 1, 64), (5, 5, 9), (8, 1, 4), (33, 1, 1), (11, 1, 3), (2, 1, 32), (4, 1, 32), (43, 1, 3), (4, 2, 64), (8, 2, 64), (257, 1, 1),
                                        (9, 1, 29), (10, 2, 64), (24, 2, 64), (32, 4, 64), (16, 1, 64), (12, 6, 20), (8, 8, 40)])
def test_heads_and_rows(ctx, kind, Hq, Hkv, n_q):
    sizes = [n_q, max(1, n_q // 2), n_q]
    TreeStep(Hq + n_q, [5, 700, 131], trees(n_q, sizes), Hq, Hkv, 32, kind, n_q=n_q).check(ctx)


@pytest.mark.parametrize("Hq,Hkv,n_q", [(8, 8, 1), (8, 8, 8), (8, 8, 16), (8, 4, 8), (12, 6, 5), (16, 2, 2), (16, 8, 5)])
@pytest.mark.parametrize("width", [None, 100])
def test_4_bit_units_of_heads(ctx, Hq, Hkv, n_q, width):
    sizes = [n_q, max(1, n_q // 2), n_q, 1, n_q]
    TreeStep(Hq + n_q, [5, 700, 131, 0, 1100], trees(n_q, sizes), Hq, Hkv, 16, "mx4", n_q=n_q, width=width).check(ctx, 300, 3)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("Hq", [4, 16])
@pytest.mark.parametrize("window", [1, 2, 5, 16, 63, 64, 100, 128, 129, 500])
@pytest.mark.parametrize("sinks", [0, 1, 4, 130, 5000])
def test_windows_and_sinks(ctx, kind, Hq, window, sinks):
    TreeStep(window + sinks, [0, 3, 100, 128, 257, 700, 1300], trees(window, [24, 9, 24, 17, 24, 1, 24]), Hq, 2, 16, kind).check(ctx, window, sinks)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("Hq", [2, 8, 32])
@pytest.mark.parametrize("window,sinks", [(FULL, 0), (40, 2)])
def test_masks_of_any_bits(ctx, kind, Hq, window, sinks):
    """Rows that see no draft, not themselves, later tokens; bits behind the tree."""
    rng = random.Random(Hq)
    masks = [[rng.getrandbits(64) & rng.getrandbits(64) for _ in range(n)] for n in (33, 64, 1, 20)]
    masks[0][:3] = [0, 1 << 32, (1 << 64) - 1]
    masks[2][0] = 0
    s = TreeStep(Hq, [0, 300, 77, 128], masks, Hq, 2, 32, kind)
    s.check(ctx, window, sinks)
    assert bool(torch.isneginf(s.lse[:, 0]).all())                     # base 0 and no bits: nothing


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("bases,sizes,Hq,Hkv,window", [([40000], [20], 4, 1, FULL), ([100000, 3], [5, 64], 32, 2, FULL), ([33000, 60000, 1, 0], [40, 3, 40, 1], 16, 2, FULL),
                                                       ([50000], [9], 8, 8, 30000), ([19000, 900], [64, 64], 16, 1, FULL), ([70000], [64], 12, 2, FULL)])
def test_units_cut_over_many_ctas(ctx, kind, bases, sizes, Hq, Hkv, window):
    TreeStep(3, bases, trees(1, sizes), Hq, Hkv, 64, kind).check(ctx, window, 0 if window == FULL else 300)


@pytest.mark.parametrize("seed", range(12))
def test_random_batches(ctx, seed):
    rng = random.Random(seed)
    B = rng.randrange(1, 60)
    bases = [int(math.exp(rng.uniform(0, math.log(5000)))) if rng.random() < 0.9 else 0 for _ in range(B)]
    n_q = rng.choice([2, 7, 16, 33, 64])
    Hq, Hkv = rng.choice([(8, 2), (4, 4), (9, 3), (16, 4), (32, 4), (6, 6)])
    window = FULL if seed % 3 == 0 else int(math.exp(rng.uniform(0, math.log(3000))))
    s = TreeStep(100 + seed, bases, trees(seed, [rng.randrange(1, n_q + 1) for _ in range(B)]), Hq, Hkv, [16, 32, 64, 128][seed % 4], KINDS[seed // 4], n_q=n_q)
    s.check(ctx, window, rng.randrange(300), rows=set(rng.sample(range(B), min(B, 8))))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("Hq", [4, 40])
def test_many_short_requests(ctx, kind, Hq):
    rng = random.Random(Hq)
    B = 700
    s = TreeStep(9, [rng.randrange(40) for _ in range(B)], trees(3, [rng.randrange(1, 6) for _ in range(B)]), Hq, 4, 16, kind)
    s.check(ctx, rows=range(0, B, 23))


@pytest.mark.parametrize("kind,pad", [("bf16", 8), ("bf16", 24), ("fp8", 16), ("fp8", 48), ("mx4", 16), ("mx4", 48)])
@pytest.mark.parametrize("Hq", [4, 24])
def test_strided_pools(ctx, kind, pad, Hq):
    TreeStep(pad, [300, 17, 130], trees(2, [15, 9, 15]), Hq, 2, 32, kind, pad=pad).check(ctx)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("Hq", [2, 32])
def test_infinite_and_nan_values_stay_with_their_rows(ctx, kind, Hq):
    """V of drafted tokens, and of keys at the edge of some rows' windows, that is no finite number."""
    for window, sinks in ((FULL, 0), (70, 3)):
        s = TreeStep(5, [200, 0, 128], trees(8, [30, 30, 12]), Hq, 2, 16, kind)
        for b, (base, tree) in enumerate(zip(s.bases, s.trees)):
            odd = [base + 3, base + 9] + ([base - 60, base - 64] if base > 100 else [])
            for i, slot in enumerate(odd):
                page, at = s.kv.where(b, torch.tensor(slot, device="cuda"))
                if kind == "bf16":
                    s.kv.v[page, at, 0, 5 + i] = [math.inf, math.nan, -math.inf][i % 3]
                elif kind == "fp8":
                    s.kv.v[page, at, 0, 5 + i] = 0x7F
                else:
                    s.kv.v[page, at, 2 * 64 + i % 4] = 255
        s.check(ctx, window, sinks)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("Hq", [2, 32])
def test_keys_that_are_no_numbers(ctx, kind, Hq):
    """A NaN in K of a drafted token: rows that see it become NaN, the others do not."""
    s = TreeStep(6, [130], trees(8, [30]), Hq, 2, 16, kind)
    page, at = s.kv.where(0, torch.tensor(130 + 4, device="cuda"))
    if kind == "bf16":
        s.kv.k[page, at, 1, 7] = math.nan
    elif kind == "fp8":
        s.kv.k[page, at, 1, 7] = 0x7F
    else:
        s.kv.k[page, at, 2 * 64 + 4] = 255
    s.check(ctx)
    assert bool(torch.isnan(s.lse).any()) and bool(torch.isfinite(s.lse).any())


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("Hq", [4, 24])
def test_pages_given_back_and_ids_outside_the_pool(ctx, kind, Hq):
    """Pages behind the window are -1 or name no page; a hole among the seen keys reads as zeros."""
    s = TreeStep(7, [600, 90], trees(4, [14, 14]), Hq, 2, 16, kind)
    s.kv.table[0, 1:20] = torch.tensor([-1, 10 ** 9, -7] * 7, dtype=torch.int32, device="cuda")[:19]
    s.check(ctx, 200, 16)
    s = TreeStep(7, [600, 90], trees(4, [14, 14]), Hq, 2, 16, kind)
    s.kv.table[0, 30] = -1
    s.check(ctx)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("Hq", [4, 24])
def test_whole_trees_without_lengths_and_output_over_the_queries(ctx, kind, Hq):
    s = TreeStep(8, [77, 300], trees(4, [13, 13]), Hq, 2, 64, kind)
    q, tree_len = s.q.clone(), s.tree_len
    s.tree_len, s.out = None, s.q
    s.call(ctx)
    torch.cuda.synchronize()
    s.tree_len, s.q = tree_len, q
    s.compare()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("Hq", [4, 24])
def test_lengths_out_of_range_are_reported(ctx, kind, Hq):
    """A tree longer than n_q or than the sequence, a negative one, a length beyond the table: counted as the nearest, and reported."""
    good = TreeStep(8, [77, 300], trees(4, [13, 13]), Hq, 2, 64, kind)
    good.check(ctx)
    for b, value in ((0, 14), (1, 10 ** 6), (0, -1)):
        s = TreeStep(8, [77, 300], trees(4, [13, 13]), Hq, 2, 64, kind)
        s.tree_len[b] = value
        s.call(ctx)
        torch.cuda.synchronize()
        with pytest.raises(binding.CpError) as e:
            ctx.poll_status()
        assert e.value.code == binding.CP_ERR_BOUNDS
        ctx.poll_status()
        if value > 0:
            assert torch.equal(s.out, good.out) and torch.equal(s.lse, good.lse)
        else:
            assert bool((s.out[0] == 0).all()) and torch.equal(s.out[1], good.out[1])
    s = TreeStep(8, [77, 300], trees(4, [13, 13]), Hq, 2, 64, kind)
    s.kv_len[0] = 5                                                     # the tree has 13 tokens: 5 of them count
    s.call(ctx)
    torch.cuda.synchronize()
    with pytest.raises(binding.CpError):
        ctx.poll_status()
    assert bool((s.out[0, 5:] == 0).all()) and bool(torch.isneginf(s.lse[:, 5:13]).all())
    s = TreeStep(8, [77, 300], trees(4, [13, 13]), Hq, 2, 64, kind)
    s.kv_len[1] = 10 ** 8
    s.call(ctx)
    torch.cuda.synchronize()
    with pytest.raises(binding.CpError):
        ctx.poll_status()
    assert torch.equal(s.out[0], good.out[0])


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("Hq", [4, 24])
def test_replayed_with_other_lengths_and_trees(ctx, kind, Hq):
    s = TreeStep(11, [900, 40, 2000], trees(4, [13, 13, 13]), Hq, 2, 64, kind)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    s.call(ctx, stream=stream)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        s.call(ctx, stream=stream)
    for seed in range(3):
        rng = random.Random(seed)
        sizes = [rng.randrange(1, 14) for _ in range(3)]
        s.trees = trees(seed, sizes)
        s.bases = [rng.randrange(0, n - 13) for n in s.kv.lens]
        s.kv_len.copy_(torch.tensor([b + m for b, m in zip(s.bases, sizes)], dtype=torch.int32))
        s.tree_len.copy_(torch.tensor(sizes, dtype=torch.int32))
        s.mask.copy_(torch.tensor([t + [0] * (13 - len(t)) for t in s.trees], dtype=torch.int64))
        s.out.fill_(math.nan)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        ctx.poll_status()
        s.compare()


@pytest.mark.parametrize("kind", KINDS)
def test_two_streams_and_repeated_bits(ctx, kind):
    """Calls on two streams with workspaces of their own; the same call gives the same bits."""
    a, b = TreeStep(1, [3000, 500], trees(4, [40, 40]), 8, 2, 64, kind), TreeStep(2, [100, 2500], trees(5, [40, 40]), 8, 2, 64, kind)
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        a.call(ctx, stream=s1)
        b.call(ctx, stream=s2)
    torch.cuda.synchronize()
    a.compare()
    b.compare()
    first = a.out.clone()
    a.out.fill_(0)
    torch.cuda.synchronize()
    a.call(ctx)
    torch.cuda.synchronize()
    assert torch.equal(a.out, first)


@pytest.mark.parametrize("Hq,scale", [(4, 1e-3), (24, 1e-3), (4, 3.0), (24, 3.0)])
def test_scales(ctx, Hq, scale):
    """Nearly equal weights, and scores so large that the running maximum jumps.  Large scale: the scores' own fp32 error grows with it, so a weight's does."""
    s = TreeStep(4, [1500], trees(4, [13]), Hq, 2, 64, "bf16", scale=scale)
    s.call(ctx)
    torch.cuda.synchronize()
    ctx.poll_status()
    k, v = s.kv.values(0, 1513)
    from tests.tree_util import attention64_seen, check_rows, tree_seen
    ref = attention64_seen(s.q[0].double(), k, v, tree_seen(1500, s.trees[0], FULL, 0), scale)
    # |q k| scale adds up to at most about 130 * scale for normal inputs (128 products of mean magnitude 0.64, with margin), so 128 * 2^-23 of that
    err = 128 * 2.0 ** -23 * 130 * scale
    check_rows(s.out[0], s.lse, ref, scale, 2.0 ** -8 + 2 * err, lse_tol=2e-4 + 2 * err)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("Hq", [2, 8, 32])
@pytest.mark.parametrize("power", [-70, -20, 40, 70])
def test_queries_of_any_magnitude(ctx, kind, Hq, power):
    """Queries times a power of two and a softmax scale divided by it; a zero row and one of a single element among them."""
    s = TreeStep(6, [300, 20], trees(6, [13, 9]), Hq, 2, 64, kind, scale=D ** -0.5 * 2.0 ** -power)
    s.q.mul_(2.0 ** power)
    s.q[0, 3] = 0
    s.q[0, 5, :, 1:] = 0
    s.check(ctx)
    s.check(ctx, 30, 2)


@pytest.mark.parametrize("Hq", [4, 16, 64])
def test_signs_and_zeros_of_head_scales(ctx, Hq):
    """E4M3: scales of K that are negative or zero (all scores equal), scales of V that are negative or zero."""
    s = TreeStep(11, [200, 0, 700], trees(3, [12, 12, 5]), Hq, 4, 16, "fp8")
    s.kv.k_scale.copy_(torch.tensor([0.01, -0.013, 0.0, -0.0001], device="cuda"))
    s.kv.v_scale.copy_(torch.tensor([-0.01, 0.02, 0.015, 0.0], device="cuda"))
    s.check(ctx)
    s.check(ctx, 50, 3)
