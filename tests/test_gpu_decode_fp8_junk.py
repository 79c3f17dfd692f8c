"""Decode over an E4M3 pool whose slots hold NaN codes wherever no visible token lies: behind the lengths, between sinks and window, in pages that
were given back and in pages of nobody."""
import pytest
import torch

from paper_2609_04774_b200 import binding
from tests.test_gpu_decode import FULL, Step

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


def bury(s, window, sinks):
    """Every slot that no row sees becomes 0x7F or 0xFF."""
    seen = torch.zeros(s.kv.k.shape[:2], dtype=torch.bool, device="cuda")
    for b, n in enumerate(s.lens):
        t = torch.arange(n, device="cuda")
        t = t[(t > n - s.n_q - window) | (t < sinks)]
        seen[s.kv.where(b, t)] = True
    s.kv.k[~seen] = 0x7F
    s.kv.v[~seen] = 0xFF


@pytest.mark.parametrize("n_q", [1, 4])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("Hq,Hkv", [(8, 2), (12, 1), (3, 3), (64, 2)])
@pytest.mark.parametrize("window,sinks", [(FULL, 0), (100, 0), (37, 5), (300, 70)])
def test_unseen_slots_hold_nan(ctx, window, sinks, Hq, Hkv, page, n_q):
    s = Step(60, [0, 1, 15, 17, 130, 1000, 9001], Hq, Hkv, page, n_q=n_q, fp8=True)
    bury(s, window, sinks)
    s.run(ctx, window, sinks)
    for pool, code in ((s.kv.k, 0x7F), (s.kv.v, 0xFF)):    # the formula multiplies hidden values by zero: it gets finite ones
        pool[pool == code] = 0
    s.compare(window, sinks)
