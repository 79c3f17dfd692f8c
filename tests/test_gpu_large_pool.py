"""Pools whose byte and element offsets pass 32 bits: the pages in use lie at the far end (only they are filled)."""
import pytest
import torch

from paper_2609_04774_b200 import binding
from tests.serving_util import D, attention64, check_attention, e4m3_codes, generator, normal

pytestmark = pytest.mark.gpu
SCALE = D ** -0.5
PAGE, HKV, HQ = 64, 8, 16


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


class Far:
    def __init__(self, fp8):
        self.fp8 = fp8
        self.pages = 150000 if fp8 else 75000               # 9.8 GB each for K and V
        self.k = torch.empty(self.pages, PAGE, HKV, D, dtype=torch.uint8 if fp8 else torch.bfloat16, device="cuda")
        self.v = torch.empty_like(self.k)
        g = generator(31)
        self.ids = torch.arange(self.pages - 24, self.pages, dtype=torch.int32, device="cuda").flip(0)
        fill = e4m3_codes if fp8 else normal
        for t in (self.k, self.v):
            t[self.ids.long()] = fill(g, 24, PAGE, HKV, D)
        self.scale = torch.full((HKV,), 1 / 70.0, device="cuda")
        self.table = torch.full((2, 12), -1, dtype=torch.int32, device="cuda")
        self.table[0], self.table[1] = self.ids[:12], self.ids[12:]
        self.lens = [700, 333]
        self.kv_len = torch.tensor(self.lens, dtype=torch.int32, device="cuda")
        self.q = normal(g, 2, 1, HQ, D)
        self.g = g
        self.cache = binding.make_cache_fp8(self.k, self.v, self.scale, self.scale) if fp8 else binding.make_cache(self.k, self.v)

    def kv(self, b, n):
        t = torch.arange(n, device="cuda")
        ids = self.table[b, t // PAGE].long()
        if self.fp8:
            return tuple(x.view(torch.float8_e4m3fn)[ids, t % PAGE].double() / 70.0 for x in (self.k, self.v))
        return self.k[ids, t % PAGE].double(), self.v[ids, t % PAGE].double()

    def decode(self, ctx):
        out, lse = torch.empty(2, 1, HQ, D, dtype=torch.bfloat16, device="cuda"), torch.empty(HQ, 2, device="cuda")
        ws = torch.empty(binding.cp_workspace_bytes_decode(2, 1, HQ, HKV), dtype=torch.uint8, device="cuda")
        f = binding.cp_decode_attn_fp8 if self.fp8 else binding.cp_decode_attn
        f(ctx, self.q, self.cache, self.table, self.kv_len, binding.CP_NO_WINDOW, 0, SCALE, out, lse, ws)
        torch.cuda.synchronize()
        ctx.poll_status()
        for b, n in enumerate(self.lens):
            ref = attention64(self.q[b].double(), *self.kv(b, n), torch.tensor([n - 1], device="cuda"), binding.CP_NO_WINDOW, 0, SCALE)
            check_attention(out[b], lse[:, b:b + 1], ref, (b, n), weight_eps=2.0 ** -8)


@pytest.mark.parametrize("fp8", [False, True])
def test_far_pages(ctx, fp8):
    s = Far(fp8)
    s.decode(ctx)
    # a token appended behind each sequence, rotated by nothing
    row, slot = torch.arange(2, dtype=torch.int32, device="cuda"), s.kv_len.clone()
    kr, vr = normal(s.g, 2, HKV, D), normal(s.g, 2, HKV, D)
    f = binding.cp_rope_append_fp8 if fp8 else binding.cp_rope_append
    f(ctx, binding.make_rope([64]), None, kr, vr, torch.zeros(1, 2, dtype=torch.int32, device="cuda"), row, slot, s.cache, s.table, None)
    s.lens = [n + 1 for n in s.lens]
    s.kv_len += 1
    at = (s.table[row.long(), slot.long() // PAGE].long(), slot.long() % PAGE)
    if not fp8:
        assert torch.equal(s.k[at], kr) and torch.equal(s.v[at], vr)
    s.decode(ctx)
    if not fp8:                                             # windowed prefill of the last 40 tokens of the first sequence
        q = normal(s.g, 40, HQ, D)
        out, lse = torch.empty_like(q), torch.empty(HQ, 40, device="cuda")
        ws = torch.empty(binding.cp_workspace_bytes([40], [1], HQ), dtype=torch.uint8, device="cuda")
        binding.cp_prefill_attn_window(ctx, q, s.cache, s.table[0], 661, 40, 1, 200, 4, HQ, SCALE, out, lse, ws)
        ref = attention64(q.double(), *s.kv(0, 701), 661 + torch.arange(40, device="cuda"), 200, 4, SCALE)
        check_attention(out, lse, ref, "prefill")
    # copies across the pool, then everything moves to the front
    pool = binding.make_page_pool([s.k], [s.v])
    ws = torch.empty(binding.cp_workspace_bytes_pages(s.pages, 2), dtype=torch.uint8, device="cuda")
    src, dst = s.ids[:2].clone(), torch.tensor([0, s.pages - 30], dtype=torch.int32, device="cuda")
    binding.cp_pages_copy(ctx, pool, src, dst, ws)
    for a, b in zip(src.tolist(), dst.tolist()):
        assert torch.equal(s.k[a], s.k[b]) and torch.equal(s.v[a], s.v[b])
    ref = torch.zeros(s.pages, dtype=torch.int32, device="cuda")
    ref[s.ids.long()] = 1
    page_map, n_live = torch.empty_like(ref), torch.empty(1, dtype=torch.int32, device="cuda")
    binding.cp_pages_compact(ctx, pool, ref, s.table, page_map, n_live, ws)
    torch.cuda.synchronize()
    ctx.poll_status()
    assert int(n_live) == 24 and int(s.table.max()) == 23 and int((page_map >= 0).sum()) == 24
    s.decode(ctx)
