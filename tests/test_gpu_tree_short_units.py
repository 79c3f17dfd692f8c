"""Batches of short requests with many rows per KV head: a CTA takes several units of one or two tiles each, so what a unit keeps in shared memory (the queries' exponents, the list
of keys whose V is no number) is soon used for the next but one."""
import math
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


@pytest.mark.parametrize("kind", ["bf16", "fp8", "mx4"])
@pytest.mark.parametrize("Hq,n_q", [(2, 30), (2, 40), (8, 16), (16, 16), (32, 16), (64, 12)])
def test_upper_dims_of_drafts_that_are_no_numbers(ctx, kind, Hq, n_q):
    """The upper half of one draft's V row is infinite (bf16) or NaN in every second request and one of its heads: exactly the rows that see it become that.
    Up to 128 rows the warpgroups take the tiles in turn: the one without a tile has to wait for the warps that put such values into their rows."""
    s = short_requests(Hq + n_q, kind, Hq, n_q)
    G = Hq // 2
    want = torch.zeros(len(s.bases), n_q, Hq, 128, dtype=torch.bool, device="cuda")
    for b, (base, tree) in enumerate(zip(s.bases, s.trees)):
        if b % 2 or not tree:
            continue
        u, h = b // 2 % len(tree), b // 4 % 2
        page, at = s.kv.where(b, torch.tensor(base + u, device="cuda"))
        if kind == "bf16":
            s.kv.v[page, at, h, 64:] = math.inf
        elif kind == "fp8":
            s.kv.v[page, at, h, 64:] = 0x7F
        else:
            s.kv.v[page, at, 2 * 64 + 4 * h + 2:2 * 64 + 4 * h + 4] = 255
        sees = torch.tensor([bool(m >> u & 1) for m in tree], device="cuda")
        want[b, :len(tree), h * G:(h + 1) * G, 64:] = sees[:, None, None]
    for again in range(20):
        s.out.fill_(7.0)
        s.call(ctx)
        got = torch.isinf(s.out) if kind == "bf16" else torch.isnan(s.out)
        assert torch.equal(got, want), (again, torch.nonzero((got ^ want).flatten(1).any(1)).flatten().tolist())
        assert bool(torch.isfinite(s.out[~want]).all())
    ctx.poll_status()
    s.compare(rows=range(0, len(s.bases), 30))
