"""The log of the sum of rows that see a key, or hold a query, that is no number: their output is NaN, and so is their lse (-inf would say that they
see nothing).  Whole units and units cut over many CTAs, both caches."""
import pytest
import torch

from paper_2609_04774_b200 import binding
from tests.test_gpu_decode import Step

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


LENS = [[40, 300, 17], [20000]]                            # whole units, one cut into a piece per CTA


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("n_q", [1, 3])
@pytest.mark.parametrize("lens", LENS)
def test_keys_that_are_no_numbers(ctx, lens, n_q, fp8):
    s = Step(50, lens, 8, 2, 16, n_q=n_q, fp8=fp8)
    clean, clean_lse = (x.clone() for x in s.run(ctx))
    sees = torch.zeros(8, len(lens), n_q, dtype=torch.bool, device="cuda")
    for b, t in ((0, lens[0] - 1), (len(lens) - 1, lens[-1] // 2)):
        page, slot = s.kv.where(b, torch.tensor(t, device="cuda"))
        s.kv.k[page, slot, 1, 9] = 0xFF if fp8 else float("nan")
        sees[4:, b, t <= lens[b] - n_q + torch.arange(n_q, device="cuda")] = True
    out, lse = s.run(ctx)
    rows = sees.reshape(8, -1)
    assert bool((torch.isnan(lse) == rows).all())
    assert torch.equal(lse[~rows], clean_lse[~rows])
    at = sees.permute(1, 2, 0)
    assert bool((torch.isnan(out).all(-1) == at).all()) and torch.equal(out[~at], clean[~at])


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_queries_that_are_no_numbers(ctx, lens, bad, fp8):
    """An infinite element meets keys of both signs: some scores are +inf."""
    s = Step(51, lens, 8, 2, 16, fp8=fp8)
    clean_lse = s.run(ctx)[1].clone()
    s.q[0, 0, 6, 77] = bad
    out, lse = s.run(ctx)
    row = torch.zeros_like(lse, dtype=torch.bool)
    row[6, 0] = True
    assert bool(torch.isnan(out[0, 0, 6]).all()) and bool((torch.isnan(lse) == row).all())
    assert torch.equal(lse[~row], clean_lse[~row])
