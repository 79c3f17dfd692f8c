"""A padded batch of drafted trees without tree lengths: rows of the table that hold fewer than n_q tokens, none at all among them, are no error in any of the
calls of a step."""
import pytest
import torch

from paper_2609_04774_b200 import binding
from tests.test_gpu_tree_commit import Pool, i32, plan
from tests.tree_util import FULL, masks_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("Hq", [2, 16])
def test_idle_rows_of_a_step(ctx, Hq):
    n_q, kv = 6, [6, 0, 40, 3]
    chain = list(range(-1, n_q - 1))
    parent, kv_len = i32([chain] * 4), i32(kv)
    pool = Pool(3, kv, 1, 2, 16, "bf16")
    pool.k.zero_(), pool.v.fill_(1.0)
    mask, positions, seq, slot = plan(ctx, parent, None, kv_len)
    ctx.poll_status()
    for b, n in enumerate(kv):
        m = min(n, n_q)
        assert mask[b].tolist() == masks_of(chain[:m]) + [0] * (n_q - m)
        assert seq[b * n_q:(b + 1) * n_q].tolist() == [b] * m + [-1] * (n_q - m)
        assert slot[b * n_q:(b + 1) * n_q].tolist() == list(range(n - m, n)) + [0] * (n_q - m)
    q = torch.ones(4, n_q, Hq, 128, dtype=torch.bfloat16, device="cuda")
    out, lse = torch.empty_like(q), torch.empty(Hq, 4 * n_q, device="cuda")
    ws = torch.empty(binding.cp_workspace_bytes_tree(4, n_q, Hq, 2), dtype=torch.uint8, device="cuda")
    binding.cp_tree_attn(ctx, q, binding.make_cache(pool.k[0], pool.v[0]), pool.table, kv_len, None, mask, FULL, 0, 0.1, out, lse, ws)
    path = torch.empty_like(parent)
    binding.cp_tree_commit(ctx, pool.pool, pool.table, kv_len, None, parent, i32([1, -1, 2, 0]), path)
    torch.cuda.synchronize()
    ctx.poll_status()
    for b, n in enumerate(kv):
        m = min(n, n_q)
        assert bool((out[b, :m] == 1).all()) and bool((out[b, m:] == 0).all())
    assert kv_len.tolist() == [2, 0, 37, 1]
    # a length that is given and does not fit is still reported
    plan(ctx, parent, i32([6, 1, 6, 3]), i32(kv))
    with pytest.raises(binding.CpError):
        ctx.poll_status()
