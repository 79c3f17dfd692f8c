"""Windowed prefill where a unit is one head over a pair of query tiles (odd Hq / Hkv), without sinks: the second tile's rows see nothing of the
unit's first KV tile, and in the next one some rows of a warp find their first key while others still see none.  Window starts of every residue
modulo the 32 rows of a warp, whole units and units cut along the keys, both caches, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import fp8 as o8
from paper_2609_04774_b200 import binding
from tests.serving_util import D, attention64_blocks, check_attention
from tests.test_gpu_window import SCALE, Batch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


def check(ctx, reqs, Hq, Hkv, page, window, sinks, fp8, seed=41):
    b = Batch(seed, reqs, Hq, Hkv, page, fp8=fp8)
    if not fp8:
        b.check(ctx, window, sinks)
        return
    out, lse = b.run(ctx, window, sinks)
    codes, qs = o8.quantize_q(b.q.view(torch.int16).cpu().numpy().view(np.uint16))
    b.q = torch.from_numpy(o8.e4m3_decode(codes) * qs[..., None].astype(np.float64)).cuda()
    for i in range(len(reqs)):
        lo, hi = b.cu[i], b.cu[i + 1]
        # weights rounded to E4M3 are off by at most 2^-4 of themselves, as in the form with sinks
        check_attention(out[lo:hi], lse[:, lo:hi], b.reference(i, window, sinks), (i, window, sinks), weight_eps=2.0 ** -4)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("Hq,Hkv", [(4, 4), (6, 2), (5, 1), (7, 1)])
def test_every_residue_of_the_window_start(ctx, Hq, Hkv, fp8):
    check(ctx, [(300, 640 + i) for i in range(33)], Hq, Hkv, 64, 300, 0, fp8)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("window", [1, 127, 128, 256, 512, 1000])
def test_prompts_without_prefix(ctx, window, fp8):
    check(ctx, [(1300, 0), (257, 0)], 4, 4, 32, window, 0, fp8)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("sinks", [0, 5, 300])
@pytest.mark.parametrize("window", [15000, 15001, 15037, 15100])
def test_units_cut_along_the_keys(ctx, window, sinks, fp8):
    check(ctx, [(300, 20000)], 1, 1, 64, window, sinks, fp8)
    check(ctx, [(200, 17777), (256, 16000)], 3, 3, 128, window, sinks, fp8)


@pytest.mark.parametrize("window", [333, 1000])
def test_chunk_form(ctx, window):
    b = Batch(42, [(1500, 900)], 3, 1, 64)
    n, p = b.reqs[0]
    C = 2
    ws = torch.empty(binding.cp_workspace_bytes([n], [C], 3), dtype=torch.uint8, device="cuda")
    for chunk in range(2 * C):
        lo, hi = chunk * n // (2 * C), (chunk + 1) * n // (2 * C)
        oc, lc = torch.empty(hi - lo, 3, D, dtype=torch.bfloat16, device="cuda"), torch.empty(3, hi - lo, device="cuda")
        binding.cp_prefill_attn_window_chunk(ctx, b.q[lo:hi].contiguous(), b.cache, b.kv.table, p, n, C, chunk, window, 0, 3, SCALE, oc, lc, ws)
        ref = attention64_blocks(b.q[lo:hi].double(), *b.kv.keys_values(0, n + p), p + torch.arange(lo, hi, device="cuda"), window, 0, SCALE)
        check_attention(oc, lc, ref, chunk)
