"""4-bit caches of huge keys under tiny queries: scores of ordinary size from factors near the ends of the fp32 range."""
import pytest
import torch

from paper_2609_04774_b200 import binding
from tests.test_gpu_mx4 import Decode
from tests.tree_util import D, TreeStep, trees

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


def lift(keys, Hkv, by):
    """Exponent bytes of all K rows that hold tokens, raised."""
    e = keys[..., Hkv * 64:Hkv * 68]
    e.copy_(torch.where(e == 255, 255, e.int() + by).to(torch.uint8))


@pytest.mark.parametrize("power", [60, 95, 106])
@pytest.mark.parametrize("n_q", [1, 4])
def test_decode(ctx, power, n_q):
    s = Decode(9, [300, 40], 8, 4, 16, n_q=n_q)
    lift(s.kv.k, 4, power)
    s.q.copy_((s.q.double() * 2.0 ** -power).bfloat16())
    s.check(ctx)


@pytest.mark.parametrize("power", [60, 95, 106])
@pytest.mark.parametrize("Hq", [2, 24])
def test_trees(ctx, power, Hq):
    s = TreeStep(9, [300, 40], trees(1, [6, 5]), Hq, 2, 16, "mx4")
    lift(s.kv.k, 2, power)
    s.q.copy_((s.q.double() * 2.0 ** -power).bfloat16())
    s.check(ctx)
