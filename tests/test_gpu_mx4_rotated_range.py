"""cp_rope_append_mx4 at the ends of the range: rotated keys beyond the fp32 numbers."""
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
