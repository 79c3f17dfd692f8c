"""Key ranges that begin a few keys before a tile's end, with large scores: rows of one warp that see nothing of the range next to rows that see the
last keys of one tile and find a larger score in the next.  The former are zeros with lse = -inf."""
import numpy as np
import pytest
import torch

from oracle import fp8 as o8
from paper_2609_04774_b200 import binding
from tests.serving_util import D, Paged, attention64, generator, normal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("Hq,Hkv", [(8, 2), (5, 1), (4, 4)])
@pytest.mark.parametrize("kv_lo", [97, 120, 126, 127, 255, 383])
def test_rows_before_the_range(ctx, kv_lo, Hq, Hkv, fp8):
    P, R = 60, 500
    g = generator(kv_lo * 10 + Hq)
    kv = Paged(g, [P + R], Hkv, 64, fp8=fp8)
    q = normal(g, R, Hq, D)
    scale = 0.5
    out = torch.full((R, Hq, D), float("nan"), device="cuda")
    lse = torch.full((Hq, R), float("nan"), device="cuda")
    if fp8:
        ws = torch.empty(binding.cp_workspace_bytes_fp8([R], [1], Hq), dtype=torch.uint8, device="cuda")
        cache = binding.make_cache_fp8(kv.k, kv.v, kv.k_scale, kv.v_scale)
        binding.cp_prefill_attn_fp8_kvrange(ctx, q, cache, kv.table[0], P, R, kv_lo, P + R, Hq, scale, out, lse, ws)
        codes, qs = o8.quantize_q(q.view(torch.int16).cpu().numpy().view(np.uint16))
        q64 = torch.from_numpy(o8.e4m3_decode(codes) * qs[..., None].astype(np.float64)).cuda()
    else:
        ws = torch.empty(binding.cp_workspace_bytes([R], [1], Hq), dtype=torch.uint8, device="cuda")
        binding.cp_prefill_attn_kvrange(ctx, q, binding.make_cache(kv.k, kv.v), kv.table[0], P, R, kv_lo, P + R, Hq, scale, out, lse, ws)
        q64 = q.double()
    torch.cuda.synchronize()
    ctx.poll_status()
    none = P + torch.arange(R, device="cuda") < kv_lo
    assert bool((out[none] == 0).all()) and bool(torch.isneginf(lse[:, none]).all())
    k, v = kv.keys_values(0, P + R)
    # positions counted from the range's first key: rows before it are negative and see nothing
    ro, rl, ra = attention64(q64, k[kv_lo:], v[kv_lo:], P - kv_lo + torch.arange(R, device="cuda"), binding.CP_NO_WINDOW, 0, scale)
    assert bool(torch.isfinite(out).all())
    # a weight rounded to bf16 (E4M3) is off by at most 2^-8 (2^-4) of itself; scores reach about 60 * 0.5 = 30, sums of 128 products in fp32:
    # off by 128 * 2^-23 * 30 = 5e-4 (bound of the LSE twice over, and of a weight's relative error).  E4M3 weights below the format's
    # smallest normal number, 2^-6, are off by up to half a step of 2^-9 instead; they carry a factor of 2^4, and the row's sum is at least the 1
    # of the key that its reference comes from: 2^-14 of every visible |v| more
    bound = ((2.0 ** -4 if fp8 else 2.0 ** -8) + 2.0 ** -10) * ra
    if fp8:
        seen = v[kv_lo:].abs().cumsum(0)[(P - kv_lo + torch.arange(R, device="cuda")).clamp(min=0)]
        bound += 2.0 ** -14 * seen.repeat_interleave(Hq // Hkv, 1)
    assert ((out.double() - ro).abs() - bound).max().item() <= 0
    assert (lse.double() - rl).abs()[:, ~none].max().item() <= 1e-3
