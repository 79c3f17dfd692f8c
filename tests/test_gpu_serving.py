"""The serving calls together, as a server uses them: two layers, prompts prefilled through the windowed call, decode steps with page work,
rotary append and decode attention, forks, evictions and a compaction in between; the whole of a step's decode part replayed from one graph.
Every attention output against the definition in 64 bits on keys and values kept in plain lists (the rotated, stored values)."""
import numpy as np
import pytest
import torch

from paper_2609_04774_b200 import binding
from tests.serving_util import D, attention64, check_attention, generator, normal

pytestmark = pytest.mark.gpu
SCALE = D ** -0.5
LAYERS = 2


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


class Server:
    def __init__(self, ctx, fp8, window, sinks, Hq=8, Hkv=2, page=16, pages=220, rows=6, width=40, seed=0):
        self.ctx, self.fp8, self.window, self.sinks, self.Hq, self.Hkv, self.page = ctx, fp8, window, sinks, Hq, Hkv, page
        self.g = generator(seed)
        dtype = torch.uint8 if fp8 else torch.bfloat16
        self.k = torch.zeros(LAYERS, pages, page, Hkv, D, dtype=dtype, device="cuda")
        self.v = torch.zeros_like(self.k)
        if fp8:
            self.ks, self.vs = (torch.rand(2, LAYERS, Hkv, generator=self.g, device="cuda") + 0.5) / 90.0
            self.caches = [binding.make_cache_fp8(self.k[i], self.v[i], self.ks[i], self.vs[i]) for i in range(LAYERS)]
        else:
            self.caches = [binding.make_cache(self.k[i], self.v[i]) for i in range(LAYERS)]
        self.pool = binding.make_page_pool(self.k, self.v)
        self.ref = torch.zeros(pages, dtype=torch.int32, device="cuda")
        self.table = torch.full((rows, width), -1, dtype=torch.int32, device="cuda")
        self.len = torch.zeros(rows, dtype=torch.int32, device="cuda")
        self.ws = torch.empty(max(binding.cp_workspace_bytes_pages(pages, rows), binding.cp_workspace_bytes_decode(rows, 1, Hq, Hkv)), dtype=torch.uint8, device="cuda")
        self.rope = binding.make_rope([16, 24, 24])
        self.rows = rows
        # the plain side: per layer and row, the stored keys and values of every token, in 64 bits
        self.K = [[torch.empty(0, Hkv, D, dtype=torch.float64, device="cuda") for _ in range(rows)] for _ in range(LAYERS)]
        self.V = [[torch.empty(0, Hkv, D, dtype=torch.float64, device="cuda") for _ in range(rows)] for _ in range(LAYERS)]

    def turned(self, x, pos):
        """Rotation in 64 bits."""
        freq = torch.tensor(list(self.rope.freq), dtype=torch.float64, device="cuda")
        ang = (pos[torch.tensor(list(self.rope.axis), device="cuda")].double().T * freq)[:, None]
        a, b = x.double()[..., :64], x.double()[..., 64:]
        return torch.cat([a * ang.cos() - b * ang.sin(), b * ang.cos() + a * ang.sin()], -1)

    def keep(self, layer, seq, slot, k_rows, v_rows, pos):
        """The plain side stores what the cache holds: read back after a check that it is the rotated row up to its rounding."""
        rk = self.turned(k_rows, pos)
        ids, at = self.table[seq.long(), slot.long() // self.page].long(), slot.long() % self.page
        if self.fp8:
            gk = self.k[layer].view(torch.float8_e4m3fn)[ids, at].double() * self.ks[layer].double()[:, None]
            gv = self.v[layer].view(torch.float8_e4m3fn)[ids, at].double() * self.vs[layer].double()[:, None]
            rk = rk.clamp(-448 * self.ks[layer].double()[:, None], 448 * self.ks[layer].double()[:, None])      # the format saturates
            step = 2.0 ** -4 + 2.0 ** -18
            low = 2.0 ** -10 * self.ks[layer].double()[:, None]
        else:
            gk, gv = self.k[layer][ids, at].double(), self.v[layer][ids, at].double()
            assert torch.equal(gv, v_rows.double())
            step, low = 2.0 ** -8, 2.0 ** -17
        assert bool(((gk - rk).abs() <= step * rk.abs() + low + 2.0 ** -17 * 6).all())
        for i in range(len(seq)):
            b = int(seq[i])
            assert self.K[layer][b].shape[0] == int(slot[i])
            self.K[layer][b] = torch.cat([self.K[layer][b], gk[i:i + 1]])
            self.V[layer][b] = torch.cat([self.V[layer][b], gv[i:i + 1]])

    def prefill(self, which):
        """{row: new tokens}: pages, rotary append and windowed attention of prompts (rows may hold tokens already)."""
        new = torch.zeros(self.rows, dtype=torch.int32)
        for r, n in which.items():
            new[r] = n
        before = self.len.clone()
        binding.cp_pages_extend(self.ctx, self.pool, self.ref, self.table, self.len, new.cuda(), self.ws)
        n = int(new.sum())
        seq = torch.cat([torch.full((c,), r, dtype=torch.int32) for r, c in which.items()]).cuda()
        slot = torch.cat([torch.arange(c, dtype=torch.int32) + int(before[r]) for r, c in which.items()]).cuda()
        pos = torch.stack([slot, slot // 7, slot % 7]).to(torch.int32).contiguous()
        cu, prefix = [0], []
        for r, c in which.items():
            cu.append(cu[-1] + c)
            prefix.append(int(before[r]))
        ws = torch.empty((binding.cp_workspace_bytes_fp8 if self.fp8 else binding.cp_workspace_bytes)(list(which.values()), [1] * len(which), self.Hq),
                         dtype=torch.uint8, device="cuda")
        table = self.table[list(which)].contiguous()
        for layer in range(LAYERS):
            q, k, v = normal(self.g, n, self.Hq, D), normal(self.g, n, self.Hkv, D), normal(self.g, n, self.Hkv, D)
            f = binding.cp_rope_append_fp8 if self.fp8 else binding.cp_rope_append
            f(self.ctx, self.rope, q, k, v, pos, seq, slot, self.caches[layer], self.table, q)
            self.keep(layer, seq, slot, k, v, pos)
            if self.fp8:
                continue                                    # the FP8 prefill rounds its queries: compared elsewhere
            out, lse = torch.empty_like(q), torch.empty(self.Hq, n, device="cuda")
            binding.cp_prefill_attn_window_batch(self.ctx, q, self.caches[layer], table, cu, prefix, [1] * len(which),
                                                 [i * table.shape[1] for i in range(len(which) + 1)], self.window, self.sinks, self.Hq, SCALE, out, lse, ws)
            for i, (r, c) in enumerate(which.items()):
                s = slice(cu[i], cu[i + 1])
                ref = attention64(q[s].double(), self.K[layer][r], self.V[layer][r], prefix[i] + torch.arange(c, device="cuda"), self.window, self.sinks, SCALE)
                check_attention(out[s], lse[:, s], ref, ("prefill", r, layer))

    def buffers(self):
        z = lambda *shape: torch.zeros(*shape, dtype=torch.bfloat16, device="cuda")
        i = lambda *shape: torch.zeros(*shape, dtype=torch.int32, device="cuda")
        self.new, self.seq, self.slot, self.pos = i(self.rows), i(self.rows), i(self.rows), i(3, self.rows)
        self.q = [z(self.rows, 1, self.Hq, D) for _ in range(LAYERS)]
        self.kr, self.vr = ([z(self.rows, self.Hkv, D) for _ in range(LAYERS)] for _ in range(2))
        self.out = [z(self.rows, 1, self.Hq, D) for _ in range(LAYERS)]
        self.lse = [torch.zeros(self.Hq, self.rows, device="cuda") for _ in range(LAYERS)]

    def device_step(self, stream=None):
        """One decode step on the device, as a graph holds it."""
        binding.cp_pages_evict(self.ctx, self.pool, self.ref, self.table, self.len, self.window, self.sinks, stream=stream)
        binding.cp_pages_extend(self.ctx, self.pool, self.ref, self.table, self.len, self.new, self.ws, stream=stream)
        rope = binding.cp_rope_append_fp8 if self.fp8 else binding.cp_rope_append
        attn = binding.cp_decode_attn_fp8 if self.fp8 else binding.cp_decode_attn
        for layer in range(LAYERS):
            q = self.q[layer].view(self.rows, self.Hq, D)
            rope(self.ctx, self.rope, q, self.kr[layer], self.vr[layer], self.pos, self.seq, self.slot, self.caches[layer], self.table, q, stream=stream)
            attn(self.ctx, self.q[layer], self.caches[layer], self.table, self.len, self.window, self.sinks, SCALE, self.out[layer], self.lse[layer], self.ws,
                 stream=stream)

    def fill(self, active):
        lens = self.len.cpu()
        on = torch.tensor([1 if r in active else 0 for r in range(self.rows)], dtype=torch.int32)
        self.new.copy_(on)
        self.seq.copy_(torch.where(on > 0, torch.arange(self.rows, dtype=torch.int32), torch.full((self.rows,), -1, dtype=torch.int32)))
        self.slot.copy_(lens)
        self.pos.copy_(torch.stack([lens, lens // 7, lens % 7]))
        for layer in range(LAYERS):
            self.q[layer].copy_(normal(self.g, self.rows, 1, self.Hq, D))
            self.kr[layer].copy_(normal(self.g, self.rows, self.Hkv, D))
            self.vr[layer].copy_(normal(self.g, self.rows, self.Hkv, D))

    def check_step(self, active):
        torch.cuda.synchronize()
        self.ctx.poll_status()
        rows = torch.tensor(sorted(active), device="cuda")
        for layer in range(LAYERS):
            self.keep(layer, self.seq[rows], self.slot[rows], self.kr[layer][rows], self.vr[layer][rows], self.pos[:, rows])
            for r in range(self.rows):
                n = int(self.len[r])
                assert n == self.K[layer][r].shape[0]
                if r not in active and n:
                    continue                                # an idle row's old token is attended again: its query was not rotated
                ref = attention64(self.q[layer][r].double(), self.K[layer][r], self.V[layer][r], torch.tensor([n - 1], device="cuda"), self.window, self.sinks, SCALE)
                check_attention(self.out[layer][r], self.lse[layer][:, r:r + 1], ref, ("decode", r, layer), weight_eps=2.0 ** -11 + 2.0 ** -16 if self.fp8 else 2.0 ** -8)

    def fork(self, parent, child):
        i = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
        binding.cp_pages_free(self.ctx, self.pool, self.ref, self.table, self.len, i(child))
        binding.cp_pages_fork(self.ctx, self.pool, self.ref, self.table, self.len, i(parent), i(child), self.ws)
        for layer in range(LAYERS):
            for p, c in zip(parent, child):
                self.K[layer][c], self.V[layer][c] = self.K[layer][p], self.V[layer][p]

    def free(self, rows):
        binding.cp_pages_free(self.ctx, self.pool, self.ref, self.table, self.len, torch.tensor(rows, dtype=torch.int32, device="cuda"))
        for layer in range(LAYERS):
            for r in rows:
                self.K[layer][r], self.V[layer][r] = self.K[layer][r][:0], self.V[layer][r][:0]

    def compact(self):
        page_map, n_live = torch.empty_like(self.ref), torch.empty(1, dtype=torch.int32, device="cuda")
        binding.cp_pages_compact(self.ctx, self.pool, self.ref, self.table, page_map, n_live, self.ws)
        n = int(n_live)
        assert bool((self.ref[:n] > 0).all()) and bool((self.ref[n:] == 0).all())

    def check_refs(self):
        held = self.table[self.table >= 0].long()
        assert torch.equal(torch.bincount(held, minlength=self.ref.numel()).to(torch.int32), self.ref)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("window,sinks", [(binding.CP_NO_WINDOW, 0), (50, 4), (16, 20)])
def test_a_server_from_prompt_to_answer(ctx, fp8, window, sinks):
    s = Server(ctx, fp8, window, sinks, seed=3 if fp8 else 4)
    s.buffers()
    s.prefill({0: 100, 2: 33, 3: 16})
    s.check_refs()
    stream, graph = torch.cuda.Stream(), None
    torch.cuda.synchronize()
    active = {0, 2, 3}
    for step in range(24):
        if step == 4:
            s.fork([0, 2], [1, 4])
            active |= {1, 4}
        if step == 9:
            s.free([2])
            active -= {2}
        if step == 12:
            s.compact()
        if step == 15:
            s.prefill({5: 70, 3: 21})
            active |= {5}
        s.fill(active)
        if step == 2:                                       # from here on the step is one graph
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                s.device_step(stream)
        torch.cuda.synchronize()
        if graph is None:
            s.device_step()
        else:
            graph.replay()
        s.check_step(active)
        s.check_refs()
    s.free(list(range(s.rows)))
    torch.cuda.synchronize()
    ctx.poll_status()
    assert int(s.ref.abs().sum()) == 0 and int((s.table != -1).sum()) == 0
