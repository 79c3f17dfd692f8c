"""Windowed prefill attention through the C ABI against the definition in 64 bits: windows and sinks around the tile size, head
groups of both unit kinds, ragged batches, page sizes, KV cuts, evicted pages, the chunk form, the FP8 form, refusals."""
import numpy as np
import pytest
import torch

from oracle import fp8 as o8
from paper_2609_04774_b200 import binding
from tests.gpu_util import Guarded
from tests.serving_util import D, Paged, attention64_blocks, check_attention, generator, normal

pytestmark = pytest.mark.gpu
SCALE = D ** -0.5


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


class Batch:
    def __init__(self, seed, reqs, Hq, Hkv, page, fp8=False):
        """reqs: (new, prefix) per request."""
        g = generator(seed)
        self.reqs, self.Hq, self.Hkv = reqs, Hq, Hkv
        self.kv = Paged(g, [n + p for n, p in reqs], Hkv, page, fp8=fp8)
        self.cu = [0]
        for n, _ in reqs:
            self.cu.append(self.cu[-1] + n)
        self.q = normal(g, self.cu[-1], Hq, D)
        self.C = [1 + i % 3 for i in range(len(reqs))]
        w = self.kv.table.shape[1]
        self.cu_pages = [i * w for i in range(len(reqs) + 1)]
        size = binding.cp_workspace_bytes_fp8 if fp8 else binding.cp_workspace_bytes
        self.g_ws = Guarded((size([n for n, _ in reqs], self.C, Hq),), torch.uint8, 0)
        self.g_out = Guarded((self.cu[-1], Hq, D), torch.bfloat16, float("nan"))
        self.g_lse = Guarded((Hq, self.cu[-1]), torch.float32, float("nan"))
        self.cache = (binding.make_cache_fp8(self.kv.k, self.kv.v, self.kv.k_scale, self.kv.v_scale) if fp8
                      else binding.make_cache(self.kv.k, self.kv.v))

    def run(self, ctx, window, sinks):
        call = binding.cp_prefill_attn_fp8_window_batch if self.kv.fp8 else binding.cp_prefill_attn_window_batch
        call(ctx, self.q, self.cache, self.kv.table, self.cu, [p for _, p in self.reqs], self.C, self.cu_pages, window, sinks,
             self.Hq, SCALE, self.g_out.tensor, self.g_lse.tensor, self.g_ws.tensor)
        torch.cuda.synchronize()
        ctx.poll_status()
        for g, what in ((self.g_out, "out"), (self.g_lse, "lse"), (self.g_ws, "workspace")):
            g.check(what)
        return self.g_out.tensor, self.g_lse.tensor

    def reference(self, b, window, sinks, table=None):
        n, p = self.reqs[b]
        k, v = self.kv.keys_values(b, n + p)
        pos = p + torch.arange(n, device="cuda")
        return attention64_blocks(self.q[self.cu[b]:self.cu[b + 1]].double(), k, v, pos, window, sinks, SCALE)

    def check(self, ctx, window, sinks):
        out, lse = self.run(ctx, window, sinks)
        for b in range(len(self.reqs)):
            lo, hi = self.cu[b], self.cu[b + 1]
            check_attention(out[lo:hi], lse[:, lo:hi], self.reference(b, window, sinks), (b, window, sinks))
        return out, lse


@pytest.mark.parametrize("window", [1, 2, 100, 127, 128, 129, 255, 256, 257, 700])
@pytest.mark.parametrize("sinks", [0, 4, 130])
def test_windows_and_sinks_around_the_tile(ctx, window, sinks):
    Batch(window * 7 + sinks, [(300, 700), (1, 0), (129, 1000)], 8, 2, 64).check(ctx, window, sinks)


@pytest.mark.parametrize("sinks", [1, 127, 128, 129, 256, 512, 900, 5000])
def test_sinks_up_to_and_beyond_the_window(ctx, sinks):
    Batch(sinks, [(200, 800), (333, 0)], 4, 2, 32).check(ctx, 200, sinks)


@pytest.mark.parametrize("Hq,Hkv", [(32, 8), (8, 8), (6, 2), (5, 1), (16, 16), (32, 4), (2, 1)])
@pytest.mark.parametrize("page", [16, 64, 128])
def test_head_groups_and_pages(ctx, Hq, Hkv, page):
    Batch(Hq * 100 + page, [(257, 511), (64, 4000), (700, 0), (1, 1), (1, 2500)], Hq, Hkv, page).check(ctx, 384, 3)


@pytest.mark.parametrize("seed", range(10))
def test_random_batches(ctx, seed):
    rng = np.random.default_rng(seed)
    reqs = [(int(rng.integers(1, 600)), int(rng.integers(0, 3000))) for _ in range(int(rng.integers(1, 9)))]
    Hq, Hkv = [(8, 2), (4, 4), (9, 3), (16, 2)][seed % 4]
    page = [16, 32, 64, 128][(seed // 2) % 4]
    Batch(1000 + seed, reqs, Hq, Hkv, page).check(ctx, int(np.exp(rng.uniform(0, np.log(2000)))), int(rng.integers(0, 200)))


@pytest.mark.parametrize("reqs,Hq,Hkv,window,sinks", [
    ([(1, 60000)], 2, 1, 50000, 4),          # one unit cut into many pieces
    ([(130, 30000)], 2, 2, 20000, 300),      # tile pairs, cut, sinks over several tiles
    ([(5, 40000), (128, 9000)], 4, 2, 30000, 64)])
def test_units_cut_along_the_window(ctx, reqs, Hq, Hkv, window, sinks):
    Batch(77, reqs, Hq, Hkv, 64).check(ctx, window, sinks)


def test_long_prompt(ctx):
    Batch(5, [(9000, 0)], 4, 1, 64).check(ctx, 1024, 4)


def test_a_window_beyond_every_length_is_the_plain_call(ctx):
    b = Batch(9, [(300, 500), (77, 0)], 8, 2, 64)
    out, lse = (x.clone() for x in b.run(ctx, 800, 0))
    for window, sinks in ((binding.CP_NO_WINDOW, 0), (1 << 40, 1 << 40), (801, 17)):
        o2, l2 = b.run(ctx, window, sinks)
        assert torch.equal(out, o2) and torch.equal(lse, l2)
    binding.cp_prefill_attn_batch(ctx, b.q, b.cache, b.kv.table, b.cu, [p for _, p in b.reqs], b.C, b.cu_pages, 8, SCALE,
                                  b.g_out.tensor, b.g_lse.tensor, b.g_ws.tensor)
    assert torch.equal(out, b.g_out.tensor) and torch.equal(lse, b.g_lse.tensor)


def test_sinks_that_reach_the_window_are_full_attention(ctx):
    b = Batch(10, [(300, 500)], 8, 2, 64)
    out, lse = (x.clone() for x in b.run(ctx, 100, 800))
    full = b.reference(0, binding.CP_NO_WINDOW, 0)
    check_attention(out, lse, full, "sinks cover everything")


def test_evicted_pages_are_not_needed(ctx):
    b = Batch(12, [(200, 3000), (64, 900)], 8, 2, 64)
    window, sinks = 500, 70
    out, lse = (x.clone() for x in b.run(ctx, window, sinks))
    for i, (n, p) in enumerate(b.reqs):
        first, last = -(-sinks // 64), max(0, p + 1 - window) // 64
        b.kv.table[i, first:last] = torch.tensor([-1, 10 ** 9, b.kv.k.shape[0]] * 100, dtype=torch.int32, device="cuda")[:max(0, last - first)]
    o2, l2 = b.run(ctx, window, sinks)
    assert torch.equal(out, o2) and torch.equal(lse, l2)


def test_chunk_form_and_schedule_reuse(ctx):
    b = Batch(13, [(700, 900)], 8, 2, 64)
    n, p = b.reqs[0]
    out, lse = (x.clone() for x in b.run(ctx, 300, 5))
    C = 3
    ws = torch.empty(binding.cp_workspace_bytes([n], [C], 8), dtype=torch.uint8, device="cuda")
    plan = binding.cp_plan(n, p, C)
    for k in range(C):
        for i, chunk in ((0, k), (1, 2 * C - 1 - k)):
            lo, hi = plan[k]["q_begin"][i], plan[k]["q_end"][i]
            oc = torch.empty(hi - lo, 8, D, dtype=torch.bfloat16, device="cuda")
            lc = torch.empty(8, hi - lo, dtype=torch.float32, device="cuda")
            binding.cp_prefill_attn_window_chunk(ctx, b.q[lo:hi].contiguous(), b.cache, b.kv.table, p, n, C, chunk, 300, 5, 8, SCALE, oc, lc, ws)
            ref = attention64_blocks(b.q[lo:hi].double(), *b.kv.keys_values(0, n + p), p + torch.arange(lo, hi, device="cuda"), 300, 5, SCALE)
            check_attention(oc, lc, ref, chunk)
    c2 = binding.Context(0)
    c2.cache_schedule(True)
    for window, sinks in ((300, 5), (300, 5), (40, 5), (40, 200), (300, 5)):      # a changed window is another schedule
        o2, l2 = b.run(c2, window, sinks)
        check_attention(o2, l2, b.reference(0, window, sinks), ("reuse", window, sinks))
    binding.cp_prefill_attn_window(c2, b.q, b.cache, b.kv.table, p, n, 1, 300, 5, 8, SCALE, b.g_out.tensor, b.g_lse.tensor, b.g_ws.tensor)
    torch.cuda.synchronize()
    c2.poll_status()
    c2.close()
    assert torch.equal(out, b.g_out.tensor) and torch.equal(lse, b.g_lse.tensor)


def test_empty_chunks(ctx):
    """Five tokens in 2 * 4 chunks: the trailing ones are empty and launch nothing."""
    b = Batch(16, [(5, 300)], 4, 2, 64)
    ws = torch.empty(binding.cp_workspace_bytes([5], [4], 4), dtype=torch.uint8, device="cuda")
    for chunk in range(8):
        lo, hi = min(5, chunk), min(5, chunk + 1)
        oc, lc = torch.empty(hi - lo, 4, D, dtype=torch.bfloat16, device="cuda"), torch.empty(4, hi - lo, device="cuda")
        binding.cp_prefill_attn_window_chunk(ctx, b.q[lo:hi].contiguous(), b.cache, b.kv.table, 300, 5, 4, chunk, 100, 2, 4, SCALE, oc, lc, ws)
        if hi > lo:
            ref = attention64_blocks(b.q[lo:hi].double(), *b.kv.keys_values(0, 305), 300 + torch.arange(lo, hi, device="cuda"), 100, 2, SCALE)
            check_attention(oc, lc, ref, chunk)
    torch.cuda.synchronize()
    ctx.poll_status()


def test_captured_call(ctx):
    b = Batch(14, [(200, 1500)], 8, 2, 64)
    out, lse = (x.clone() for x in b.run(ctx, 400, 4))
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        binding.cp_prefill_attn_window_batch(ctx, b.q, b.cache, b.kv.table, b.cu, [1500], b.C, b.cu_pages, 400, 4, 8, SCALE, b.g_out.tensor,
                                             b.g_lse.tensor, b.g_ws.tensor, stream=stream)
    b.g_out.tensor.zero_()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, b.g_out.tensor) and torch.equal(lse, b.g_lse.tensor)


@pytest.mark.parametrize("reqs,Hq,Hkv,page,window,sinks", [
    ([(300, 700), (1, 0), (129, 1000)], 8, 2, 64, 257, 4), ([(200, 800)], 3, 1, 16, 100, 130), ([(1, 20000)], 2, 1, 128, 15000, 0)])
def test_fp8_form(ctx, reqs, Hq, Hkv, page, window, sinks):
    """Weights rounded to E4M3: off by at most 2^-4 of themselves; the queries' codes are taken from the oracle's quantiser."""
    b = Batch(21, reqs, Hq, Hkv, page, fp8=True)
    out, lse = b.run(ctx, window, sinks)
    codes, qs = o8.quantize_q(b.q.view(torch.int16).cpu().numpy().view(np.uint16))
    b.q = torch.from_numpy(o8.e4m3_decode(codes) * qs[..., None].astype(np.float64)).cuda()
    for i in range(len(reqs)):
        lo, hi = b.cu[i], b.cu[i + 1]
        check_attention(out[lo:hi], lse[:, lo:hi], b.reference(i, window, sinks), i, weight_eps=2.0 ** -4)


def test_refusals(ctx):
    b = Batch(30, [(20, 50)], 4, 2, 64)

    def call(window=10, sinks=0, C=(1,), cu_pages=(0, 2), ws=None, Hq=4):
        binding.cp_prefill_attn_window_batch(ctx, b.q, b.cache, b.kv.table, b.cu, [50], C, cu_pages, window, sinks, Hq, SCALE,
                                             b.g_out.tensor, b.g_lse.tensor, b.g_ws.tensor if ws is None else ws)
    call()
    for kw, code in ((dict(window=0), binding.CP_ERR_INVALID_ARG), (dict(window=-5), binding.CP_ERR_INVALID_ARG),
                     (dict(sinks=-1), binding.CP_ERR_INVALID_ARG), (dict(C=(0,)), binding.CP_ERR_INVALID_ARG),
                     (dict(Hq=5), binding.CP_ERR_INVALID_ARG), (dict(cu_pages=(0, 1)), binding.CP_ERR_BOUNDS),
                     (dict(ws=torch.empty(256, dtype=torch.uint8, device="cuda")), binding.CP_ERR_WORKSPACE)):
        with pytest.raises(binding.CpError) as e:
            call(**kw)
        assert e.value.code == code, kw
    with pytest.raises(binding.CpError) as e:
        binding.cp_prefill_attn_window_chunk(ctx, b.q, b.cache, b.kv.table, 50, 20, 1, 2, 10, 0, 4, SCALE, b.g_out.tensor, b.g_lse.tensor,
                                             b.g_ws.tensor)
    assert e.value.code == binding.CP_ERR_INVALID_ARG
    torch.cuda.synchronize()
    ctx.poll_status()
