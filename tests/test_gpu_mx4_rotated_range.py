"""cp_rope_append_mx4 at the ends of the range: rotated keys beyond the fp32 numbers, keys among the smallest ones, keys that are mostly zeros."""
import math

import pytest
import torch

from paper_2609_04774_b200 import binding
from tests.serving_util import generator, normal
from tests.test_gpu_mx4 import Rows, turned
from tests.tree_util import D, mx4_quantise, mx4_values

pytestmark = pytest.mark.gpu
LARGEST = 3.38953138925153547590470800371487866880e38       # of bf16


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


def written(ctx, r):
    """(K codes as written, K rows rotated in 64 bits), in the tokens' order."""
    r.run(ctx)
    ctx.poll_status()
    at = (r.table[r.seq.long(), r.slot.long() // r.page].long(), r.slot.long() % r.page)
    return r.k[at][:, :r.Hkv * 68], turned(r.k_rows, r.rope, r.positions)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("Hkv", [1, 8])
def test_finite_keys_that_leave_the_range_saturate(ctx, interleaved, Hkv):
    """Pairs of the largest bf16 numbers, turned by any angle: up to 2^128.5.  What leaves the fp32 range counts as its end: exponent byte 252, codes of 6, whatever
    the other blocks of the head hold."""
    g = generator(Hkv)
    n = 500
    k = normal(g, n, Hkv, D)
    # whole chunks of eight pairs, so that every value of a lane may be large: nothing else of the head then decides how it is rotated
    huge = (torch.rand(n, Hkv, D // 16, generator=g, device="cuda") < 0.1).repeat_interleave(8, -1)
    huge = torch.stack([huge, huge], -1).flatten(-2) if interleaved else torch.cat([huge, huge], -1)
    k = torch.where(huge, torch.copysign(torch.tensor(LARGEST, device="cuda"), k.float()).bfloat16(), k)
    assert bool(torch.isfinite(k).all())
    r = Rows(2, n, 4, Hkv, 16, [64], interleaved, x=(k, normal(g, n, Hkv, D)))
    got, x = written(ctx, r)
    top = float(torch.finfo(torch.float32).max)
    assert bool((x.abs() > top).any())
    want = mx4_quantise(x.clamp(-top, top))
    assert torch.equal(got[:, Hkv * 64:], want[:, Hkv * 64:]) and int(got[:, Hkv * 64:].max()) == 252
    assert torch.equal(mx4_values(got, Hkv), mx4_values(want, Hkv))


@pytest.mark.parametrize("interleaved", [False, True])
def test_the_smallest_keys(ctx, interleaved):
    """Magnitudes of 2^-133 to 2^-120, where fp32 has fewer bits: the rotation's error is then a step of the smallest numbers, not a share of the value."""
    g = generator(9)
    n, Hkv = 2000, 8
    power = torch.randint(-133, -119, (n, Hkv, 1), generator=g, device="cuda").double()
    k = (normal(g, n, Hkv, D).double().clamp(-1.5, 1.5) * torch.exp2(power)).bfloat16()
    r = Rows(2, n, 4, Hkv, 16, [64], interleaved, x=(k, normal(g, n, Hkv, D)))
    got, x = written(ctx, r)
    want = mx4_quantise(x)
    assert torch.equal(got[:, Hkv * 64:], want[:, Hkv * 64:])
    assert torch.equal(mx4_values(got, Hkv), mx4_values(want, Hkv))


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("sections", [[64], [24]])
def test_keys_that_are_mostly_zeros(ctx, interleaved, sections):
    """Zeros of either sign, alone and in pairs, among other elements."""
    g = generator(4)
    n, Hkv = 300, 4
    zero = torch.copysign(torch.zeros(n, Hkv, D, device="cuda"), torch.randn(n, Hkv, D, generator=g, device="cuda")).bfloat16()
    r = None
    for share in (0.5, 0.97):
        k = torch.where(torch.rand(n, Hkv, D, generator=g, device="cuda") < share, zero, normal(g, n, Hkv, D))
        r = Rows(2, n, 4, Hkv, 16, sections, interleaved, x=(k, normal(g, n, Hkv, D)))
        r.check(ctx)
    r = Rows(2, n, 4, Hkv, 16, sections, interleaved, x=(zero, zero))
    got, _ = written(ctx, r)
    assert bool((got[:, :Hkv * 64] & 0x77 == 0).all()) and bool((got[:, Hkv * 64:] == 0).all())


@pytest.mark.parametrize("freq", [2e-7, 1e-6, 4e-6, 2e-5])
@pytest.mark.parametrize("interleaved", [False, True])
def test_blocks_of_what_a_small_turn_brings_over(ctx, interleaved, freq):
    """The first element of every pair is zero and the angle a few millionths: its rotated value is not much larger than the rotation's error in fp32."""
    g = generator(6)
    n, Hkv = 600, 4
    k = normal(g, n, Hkv, D)
    k[..., 0::2 if interleaved else 1][..., :D // 2] = 0
    r = Rows(2, n, 4, Hkv, 16, [64], interleaved, x=(k, normal(g, n, Hkv, D)))
    r.rope.freq[:] = [freq * (1 + i / 64) for i in range(64)]
    r.positions.copy_(torch.randint(-3, 4, r.positions.shape, generator=g, device="cuda"))
    r.check(ctx)


@pytest.mark.parametrize("interleaved", [False, True])
def test_zeros_cost_nothing(ctx, interleaved):
    """A cache of zeros in half of the pairs is written about as fast as one without (every head that goes through the rotation in 64 bits costs many times a
    head's time, and a chunk without an undecided value is the rule)."""
    g = generator(5)
    n, Hkv = 16384, 8
    dense, v = normal(g, n, Hkv, D), normal(g, n, Hkv, D)
    gone = torch.rand(n, Hkv, D // 2, generator=g, device="cuda") < 0.5
    gone = torch.stack([gone, gone], -1).flatten(-2) if interleaved else torch.cat([gone, gone], -1)

    def time(k):
        r = Rows(2, n, 4, Hkv, 64, [64], interleaved, x=(k, v))
        best = math.inf
        for _ in range(12):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            binding.cp_rope_append_mx4(ctx, r.rope, None, r.k_rows, r.v_rows, r.positions, r.seq, r.slot, r.cache, r.table, None)
            b.record()
            b.synchronize()
            best = min(best, a.elapsed_time(b))
        return best

    full, sparse = time(dense), time(dense.masked_fill(gone, 0))
    assert sparse <= 1.3 * full, (full, sparse)
