"""Batches of short requests with many rows per KV head: a CTA takes several units of one or two tiles each, so what a unit keeps in shared memory (the queries' exponents, the list
of keys whose V is no number) is soon used for the next but one."""
import random

import pytest
import torch

from paper_2609_04774_b200 import binding
from tests.tree_util import TreeStep, trees

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


def short_requests(seed, kind, Hq, n_q, B=420, most=200):
    """Requests of up to `most` keys, a seventh of them without drafts, two KV heads."""
    rng = random.Random(seed)
    sizes = [0 if b % 7 == 3 else rng.randrange(1, n_q + 1) for b in range(B)]
    bases = [rng.randrange(most - n_q) if b % 5 == 0 else rng.randrange(100 - n_q) for b in range(B)]
    return TreeStep(seed, bases, trees(seed, sizes), Hq, 2, 16, kind, n_q=n_q, width=-(-most // 16))


@pytest.mark.parametrize("Hq,n_q", [(2, 40), (8, 16), (16, 16), (32, 16), (64, 12)])
def test_queries_of_another_magnitude_in_every_request(ctx, Hq, n_q):
    """E4M3: every query row is scaled up by a power of two of its own; taken for another unit's, it would move the row's scores by that much."""
    s = short_requests(Hq + n_q, "fp8", Hq, n_q, most=120)
    rng = random.Random(n_q)
    power = torch.tensor([[[rng.choice([-3.0, 0.0, -1.0, -40.0]) for _ in range(Hq)] for _ in range(n_q)] for _ in s.bases], device="cuda")
    s.q.mul_(torch.exp2(power)[..., None].bfloat16())
    s.check(ctx, rows=range(0, len(s.bases), 7))
    first, lse = s.out.clone(), s.lse.clone()
    for _ in range(20):
        s.out.fill_(7.0)
        s.call(ctx)
        assert torch.equal(s.out, first) and torch.equal(s.lse, lse)
    ctx.poll_status()
