"""The tree and 4-bit calls together, as a server that drafts uses them: two layers, prompts (4-bit caches are gathered for the prefill), steps of pages, plan,
rotary append, tree attention and commit, replayed from graphs, forks and a compaction in between; large pools; streams and workspaces."""
import math
import random

import pytest
import torch

from paper_2609_04774_b200 import binding
from tests.serving_util import D, attention64, check_attention, e4m3_codes, generator, normal
from tests.tree_util import FULL, WEIGHT_EPS, TreeStep, as_i64, attention64_seen, check_rows, masks_of, mx4_quantise, mx4_values, random_tree, tree_seen, trees

pytestmark = pytest.mark.gpu
SCALE = D ** -0.5
LAYERS = 2
KINDS = ["bf16", "fp8", "mx4"]
ROPE = {"bf16": binding.cp_rope_append, "fp8": binding.cp_rope_append_fp8, "mx4": binding.cp_rope_append_mx4}
ATTN = {"bf16": binding.cp_tree_attn, "fp8": binding.cp_tree_attn_fp8, "mx4": binding.cp_tree_attn_mx4}
DECODE = {"bf16": binding.cp_decode_attn, "fp8": binding.cp_decode_attn_fp8, "mx4": binding.cp_decode_attn_mx4}


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Server:
    def __init__(self, ctx, kind, n_q, window, sinks, Hq=8, Hkv=2, page=16, pages=300, rows=5, width=48, seed=0):
        self.ctx, self.kind, self.n_q, self.window, self.sinks, self.Hq, self.Hkv, self.page, self.rows = ctx, kind, n_q, window, sinks, Hq, Hkv, page, rows
        self.g, self.rng = generator(seed), random.Random(seed)
        if kind == "mx4":
            self.k = torch.full((LAYERS, pages, page, binding.mx4_token_bytes(Hkv)), 0xFF, dtype=torch.uint8, device="cuda")
        else:
            self.k = torch.zeros(LAYERS, pages, page, Hkv, D, dtype=torch.uint8 if kind == "fp8" else torch.bfloat16, device="cuda")
        self.v = self.k.clone()
        if kind == "fp8":
            self.ks, self.vs = (torch.rand(2, LAYERS, Hkv, generator=self.g, device="cuda") + 0.5) / 90.0
            self.caches = [binding.make_cache_fp8(self.k[i], self.v[i], self.ks[i], self.vs[i]) for i in range(LAYERS)]
        else:
            make = (lambda k, v: binding.make_cache_mx4(k, v, Hkv)) if kind == "mx4" else binding.make_cache
            self.caches = [make(self.k[i], self.v[i]) for i in range(LAYERS)]
        self.pool = (binding.make_page_pool_mx4 if kind == "mx4" else binding.make_page_pool)(self.k, self.v)
        self.ref, self.table, self.len = torch.zeros(pages, dtype=torch.int32, device="cuda"), torch.full((rows, width), -1, dtype=torch.int32, device="cuda"), i32([0] * rows)
        self.ws = torch.empty(max(binding.cp_workspace_bytes_pages(pages, rows), binding.cp_workspace_bytes_tree(rows, n_q, Hq, Hkv)), dtype=torch.uint8, device="cuda")
        self.rope = binding.make_rope([16, 24, 24])
        self.kept = [0] * rows                               # tokens of a row, by the plain side
        # a step's buffers
        n = rows * n_q
        self.tree_len, self.parent, self.accepted, self.path = i32([0] * rows), i32([[-1] * n_q] * rows), i32([-1] * rows), i32([[7] * n_q] * rows)
        self.mask = torch.zeros(rows, n_q, dtype=torch.int64, device="cuda")
        self.pos, self.seq, self.slot = (torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((3, n), (n,), (n,)))
        self.q, self.q_in = ([torch.zeros(rows, n_q, Hq, D, dtype=torch.bfloat16, device="cuda") for _ in range(LAYERS)] for _ in range(2))
        self.kr, self.vr = ([torch.zeros(n, Hkv, D, dtype=torch.bfloat16, device="cuda") for _ in range(LAYERS)] for _ in range(2))
        self.out = [torch.zeros(rows, n_q, Hq, D, dtype=torch.bfloat16, device="cuda") for _ in range(LAYERS)]
        self.lse = [torch.zeros(Hq, n, device="cuda") for _ in range(LAYERS)]

    def turned(self, x, pos):
        freq = torch.tensor(list(self.rope.freq), dtype=torch.float64, device="cuda")
        ang = (pos[torch.tensor(list(self.rope.axis), device="cuda")].double().T * freq)[:, None]
        a, b = x.double()[..., :64], x.double()[..., 64:]
        return torch.cat([a * ang.cos() - b * ang.sin(), b * ang.cos() + a * ang.sin()], -1)

    def stored(self, layer, b, t):
        """K and V of the tokens in slots t of row b, in 64 bits."""
        ids, at = self.table[b, t // self.page].long(), t % self.page
        k, v = self.k[layer][ids, at], self.v[layer][ids, at]
        if self.kind == "fp8":
            return k.view(torch.float8_e4m3fn).double() * self.ks[layer].double()[:, None], v.view(torch.float8_e4m3fn).double() * self.vs[layer].double()[:, None]
        return (mx4_values(k, self.Hkv), mx4_values(v, self.Hkv)) if self.kind == "mx4" else (k.double(), v.double())

    def check_stored(self, layer, b, t, k_rows, v_rows, pos):
        """What the append stored is the rotated row up to its format's rounding."""
        k, v = self.stored(layer, b, t)
        for got, want, which in ((k, self.turned(k_rows, pos), "k"), (v, v_rows.double(), "v")):
            if self.kind == "mx4":                           # the quantisation of exactly those values; a rotation in doubles is off by far less than half a step
                top = want.abs().reshape(*want.shape[:-1], 4, 32).amax(-1, keepdim=True).expand(*want.shape[:-1], 4, 32).reshape(want.shape)
                assert bool(((got - want).abs() <= 0.5 * top).all())
                q = mx4_values(mx4_quantise(want), self.Hkv)
                assert (q != got).sum().item() <= 2 if which == "k" else torch.equal(q, got)
            elif self.kind == "fp8":
                s = (self.ks if which == "k" else self.vs)[layer].double()[:, None]
                want = want.clamp(-448 * s, 448 * s)
                assert bool(((got - want).abs() <= (2.0 ** -4 + 2.0 ** -18) * want.abs() + 2.0 ** -10 * s + 2.0 ** -17 * 6).all())
            else:
                assert bool(((got - want).abs() <= (2.0 ** -8 if which == "k" else 0.0) * want.abs() + (2.0 ** -14 if which == "k" else 0.0)).all())

    def prompt(self, b, n):
        """n tokens of row b appended and prefilled; the prefill of a 4-bit cache reads gathered rows."""
        before, new = self.kept[b], [0] * self.rows
        new[b] = n
        binding.cp_pages_extend(self.ctx, self.pool, self.ref, self.table, self.len, i32(new), self.ws)
        slot = torch.arange(before, before + n, dtype=torch.int32, device="cuda")
        seq, pos = torch.full_like(slot, b), slot.expand(3, n).contiguous()
        for layer in range(LAYERS):
            q, k, v = normal(self.g, n, self.Hq, D), normal(self.g, n, self.Hkv, D), normal(self.g, n, self.Hkv, D)
            ROPE[self.kind](self.ctx, self.rope, q, k, v, pos, seq, slot, self.caches[layer], self.table, q)
            self.check_stored(layer, b, slot.long(), k, v, pos)
            if self.kind == "fp8":
                continue                                     # the FP8 prefill rounds its queries: compared elsewhere
            cache, table = self.caches[layer], self.table[b]
            total = before + n
            if self.kind == "mx4":
                pages = -(-total // self.page)
                kv = torch.zeros(2, pages * self.page, self.Hkv, D, dtype=torch.bfloat16, device="cuda")
                binding.cp_kv_gather_mx4(self.ctx, cache, self.table[b], 0, total, kv[0, :total], kv[1, :total])
                cache, table = binding.make_cache(*kv.view(2, pages, self.page, self.Hkv, D)), torch.arange(pages, dtype=torch.int32, device="cuda")
            out, lse = torch.empty_like(q), torch.empty(self.Hq, n, device="cuda")
            ws = torch.empty(binding.cp_workspace_bytes([n], [1], self.Hq), dtype=torch.uint8, device="cuda")
            binding.cp_prefill_attn_window(self.ctx, q, cache, table, before, n, 1, self.window, self.sinks, self.Hq, SCALE, out, lse, ws)
            ref = attention64(q.double(), *self.stored(layer, b, torch.arange(total, device="cuda")), before + torch.arange(n, device="cuda"), self.window, self.sinks, SCALE)
            check_attention(out, lse, ref, ("prompt", b, layer))
        self.kept[b] += n

    def draft(self, stream=None):
        """Pages, plan, append and attention of all rows' trees, as a graph holds them."""
        binding.cp_pages_extend(self.ctx, self.pool, self.ref, self.table, self.len, self.tree_len, self.ws, stream=stream)
        binding.cp_tree_plan(self.ctx, self.parent, self.tree_len, self.len, self.mask, self.pos, self.seq, self.slot, stream=stream)
        for i in range(LAYERS):
            flat = (self.rows * self.n_q, self.Hq, D)
            ROPE[self.kind](self.ctx, self.rope, self.q_in[i].view(flat), self.kr[i], self.vr[i], self.pos, self.seq, self.slot, self.caches[i], self.table,
                            self.q[i].view(flat), stream=stream)
            ATTN[self.kind](self.ctx, self.q[i], self.caches[i], self.table, self.len, self.tree_len, self.mask, self.window, self.sinks, SCALE, self.out[i], self.lse[i],
                            self.ws, stream=stream)

    def commit(self, stream=None):
        binding.cp_tree_commit(self.ctx, self.pool, self.table, self.len, self.tree_len, self.parent, self.accepted, self.path, stream=stream)

    def fill(self, active):
        self.sizes = [self.rng.randrange(0, self.n_q + 1) if b in active else 0 for b in range(self.rows)]
        self.parents = [random_tree(self.rng, m) for m in self.sizes]
        self.picks = [self.rng.randrange(-1, m) if m else -1 for m in self.sizes]
        self.tree_len.copy_(i32(self.sizes))
        self.parent.copy_(i32([p + [-1] * (self.n_q - len(p)) for p in self.parents]))
        self.accepted.copy_(i32(self.picks))
        for layer in range(LAYERS):
            self.q_in[layer].copy_(normal(self.g, self.rows, self.n_q, self.Hq, D))
            self.kr[layer].copy_(normal(self.g, self.rows * self.n_q, self.Hkv, D))
            self.vr[layer].copy_(normal(self.g, self.rows * self.n_q, self.Hkv, D))

    def check_draft(self):
        torch.cuda.synchronize()
        self.ctx.poll_status()
        wide = self.n_q * self.Hq // self.Hkv > 32
        self.before = []
        for b, (m, parent) in enumerate(zip(self.sizes, self.parents)):
            base, masks, at = self.kept[b], masks_of(parent), slice(b * self.n_q, b * self.n_q + m)
            assert int(self.len[b]) == base + m
            depth = torch.tensor([base + bin(x).count("1") - 1 for x in masks], dtype=torch.int32, device="cuda")
            slots = torch.arange(base, base + m, device="cuda")
            assert torch.equal(self.slot[at], slots.int()) and torch.equal(self.pos[:, at], depth.expand(3, m)) and bool((self.seq[at] == b).all())
            assert self.mask[b, :m].tolist() == as_i64(masks) and bool((self.seq[b * self.n_q + m:(b + 1) * self.n_q] == -1).all())
            for layer in range(LAYERS):
                self.check_stored(layer, b, slots, self.kr[layer][at], self.vr[layer][at], self.pos[:, at])
                k, v = self.stored(layer, b, torch.arange(base + m, device="cuda"))
                self.before.append((k, v))
                ref = attention64_seen(self.q[layer][b, :m].double(), k, v, tree_seen(base, masks, self.window, self.sinks), SCALE)
                lse = self.lse[layer].view(self.Hq, self.rows, self.n_q)[:, b]
                check_rows(self.out[layer][b, :m], lse[:, :m], ref, (b, layer, base, m), 2.0 ** -8 if wide else WEIGHT_EPS[self.kind])
                assert bool((self.out[layer][b, m:] == 0).all()) and bool(torch.isneginf(lse[:, m:]).all())

    def check_commit(self):
        torch.cuda.synchronize()
        self.ctx.poll_status()
        for b, (parent, pick) in enumerate(zip(self.parents, self.picks)):
            path = []
            while pick >= 0:
                path.insert(0, pick)
                pick = parent[pick]
            base = self.kept[b]
            assert self.path[b].tolist() == path + [-1] * (self.n_q - len(path)) and int(self.len[b]) == base + len(path)
            take = torch.tensor(list(range(base)) + [base + x for x in path], dtype=torch.long, device="cuda")
            for layer in range(LAYERS):
                k, v = self.before[b * LAYERS + layer]
                got = self.stored(layer, b, torch.arange(base + len(path), device="cuda"))
                assert torch.equal(got[0], k[take]) and torch.equal(got[1], v[take])
            self.kept[b] += len(path)

    def fork(self, parent, child):
        binding.cp_pages_free(self.ctx, self.pool, self.ref, self.table, self.len, i32(child))
        binding.cp_pages_fork(self.ctx, self.pool, self.ref, self.table, self.len, i32(parent), i32(child), self.ws)
        for p, c in zip(parent, child):
            self.kept[c] = self.kept[p]
            for layer in range(LAYERS):
                t = torch.arange(self.kept[p], device="cuda")
                assert all(torch.equal(x, y) for x, y in zip(self.stored(layer, p, t), self.stored(layer, c, t)))

    def compact(self):
        old = [[self.stored(i, b, torch.arange(self.kept[b], device="cuda")) for b in range(self.rows)] for i in range(LAYERS)]
        page_map, n_live = torch.empty_like(self.ref), torch.empty(1, dtype=torch.int32, device="cuda")
        binding.cp_pages_compact(self.ctx, self.pool, self.ref, self.table, page_map, n_live, self.ws)
        for i in range(LAYERS):
            for b in range(self.rows):
                assert all(torch.equal(x, y) for x, y in zip(old[i][b], self.stored(i, b, torch.arange(self.kept[b], device="cuda"))))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n_q,window,sinks", [(4, FULL, 0), (4, 40, 3), (13, FULL, 0), (13, 30, 5)])
def test_a_server_that_drafts(ctx, kind, n_q, window, sinks):
    s = Server(ctx, kind, n_q, window, sinks, seed=n_q)
    for b, n in ((0, 100), (2, 33), (3, 16)):
        s.prompt(b, n)
    stream, graphs, active = torch.cuda.Stream(), None, {0, 2, 3}
    for step in range(14):
        if step == 4:
            s.fork([0, 2], [1, 4])
            active |= {1, 4}
        if step == 8:
            binding.cp_pages_free(ctx, s.pool, s.ref, s.table, s.len, i32([2]))
            s.kept[2] = 0
            s.compact()
        if step == 10:
            s.prompt(2, 45)
        s.fill(active)
        if step == 1:                                        # from here on the step is two graphs, which share a workspace
            torch.cuda.synchronize()
            graphs = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
            with torch.cuda.graph(graphs[0], stream=stream):
                s.draft(stream)
            with torch.cuda.graph(graphs[1], stream=stream):
                s.commit(stream)
        torch.cuda.synchronize()
        if graphs:
            graphs[0].replay()
        else:
            s.draft()
        s.check_draft()
        if graphs:
            graphs[1].replay()
        else:
            s.commit()
        s.check_commit()
        held = s.table[s.table >= 0].long()
        assert torch.equal(torch.bincount(held, minlength=s.ref.numel()).to(torch.int32), s.ref)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n_q,Hq", [(7, 32), (16, 32), (33, 8), (50, 32)])
def test_long_memory_bound_steps_replayed(ctx, kind, n_q, Hq):
    """Many long requests: the rings of K and V tiles run full and the tensor cores wait for memory; odd numbers of rows."""
    rng = random.Random(n_q)
    bases = [rng.choice([4096, 4100, 3999, 2000]) for _ in range(37)]
    s = TreeStep(n_q, bases, trees(n_q, [rng.randrange(1, n_q + 1) for _ in bases]), Hq, 8, 64, kind, n_q=n_q)
    stream = torch.cuda.Stream()
    s.call(ctx)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        for _ in range(10):
            s.call(ctx, stream=stream)
    s.out.fill_(math.nan)
    for _ in range(5):
        graph.replay()
    torch.cuda.synchronize()
    ctx.poll_status()
    s.compare(rows={0, 9, 36})
    first = s.out.clone()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(first, s.out)                         # sums in a fixed order


@pytest.mark.parametrize("kind", KINDS)
def test_two_streams_with_a_workspace_each(ctx, kind):
    steps = [TreeStep(i, [900 + 70 * i, 40, 1300], trees(i, [9, 5, 9]), 8 * (1 + 3 * i), 2, 32, kind) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in steps]
    torch.cuda.synchronize()
    for _ in range(20):
        for s, st in zip(steps, streams):
            s.call(ctx, 500, 4, stream=st)
    torch.cuda.synchronize()
    ctx.poll_status()
    for s in steps:
        s.compare(500, 4)


PAGE, HKV = 64, 8


@pytest.mark.parametrize("kind", KINDS)
def test_far_pages(ctx, kind):
    """Byte offsets, and for bf16 element offsets, beyond 32 bits: appends, attention of trees and tokens, gathers and commits at the far end of a pool."""
    g = generator(12)
    pages = {"bf16": 75000, "fp8": 150000, "mx4": 260000}[kind]                # 9 to 10 GB each for K and V
    row = binding.mx4_token_bytes(HKV)
    shape = (pages, PAGE, row) if kind == "mx4" else (pages, PAGE, HKV, D)
    k, v = (torch.empty(shape, dtype=torch.bfloat16 if kind == "bf16" else torch.uint8, device="cuda") for _ in range(2))
    ids = torch.arange(pages - 24, pages, dtype=torch.int32, device="cuda").flip(0)
    for t in (k, v):
        x = normal(g, 24, PAGE, HKV, D)
        t[ids.long()] = x if kind == "bf16" else (e4m3_codes(g, 24, PAGE, HKV, D) if kind == "fp8" else torch.nn.functional.pad(mx4_quantise(x), (0, row - 68 * HKV)))
    scale = torch.full((HKV,), 1 / 70.0, device="cuda")
    cache = binding.make_cache(k, v) if kind == "bf16" else (binding.make_cache_fp8(k, v, scale, scale) if kind == "fp8" else binding.make_cache_mx4(k, v, HKV))
    pool = binding.make_page_pool_mx4([k], [v]) if kind == "mx4" else binding.make_page_pool([k], [v])
    table, kv_len = ids.view(2, 12).contiguous(), i32([700, 333])

    def values(b, n):
        t = torch.arange(n, device="cuda")
        at = (table[b, t // PAGE].long(), t % PAGE)
        if kind == "mx4":
            return mx4_values(k[at], HKV), mx4_values(v[at], HKV)
        return (k[at].double(), v[at].double()) if kind == "bf16" else tuple(x[at].view(torch.float8_e4m3fn).double() / 70.0 for x in (k, v))

    for n_q, Hq in ((2, 16), (8, 64)):                       # few rows a head, and many
        parents = [random_tree(random.Random(n_q + b), n_q) for b in range(2)]
        masks = [masks_of(p) for p in parents]
        q, out = normal(g, 2, n_q, Hq, D), torch.empty(2, n_q, Hq, D, dtype=torch.bfloat16, device="cuda")
        lse, ws = torch.empty(Hq, 2 * n_q, device="cuda"), torch.empty(binding.cp_workspace_bytes_tree(2, n_q, Hq, HKV), dtype=torch.uint8, device="cuda")
        mask, pos, seq, slot = torch.empty(2, n_q, dtype=torch.int64, device="cuda"), i32([[0] * 2 * n_q]), i32([0] * 2 * n_q), i32([0] * 2 * n_q)
        kr, vr = normal(g, 2 * n_q, HKV, D), normal(g, 2 * n_q, HKV, D)
        base = kv_len.tolist()
        kv_len += n_q
        binding.cp_tree_plan(ctx, i32(parents), None, kv_len, mask, pos, seq, slot)
        ROPE[kind](ctx, binding.make_rope([64]), None, kr, vr, pos, seq, slot, cache, table, None)
        ATTN[kind](ctx, q, cache, table, kv_len, None, mask, FULL, 0, SCALE, out, lse, ws)
        torch.cuda.synchronize()
        ctx.poll_status()
        for b in range(2):
            K, V = values(b, base[b] + n_q)
            if kind != "fp8":
                want = vr.view(2, n_q, HKV, D)[b].double()
                assert torch.equal(V[base[b]:], mx4_values(mx4_quantise(want), HKV) if kind == "mx4" else want)
            ref = attention64_seen(q[b].double(), K, V, tree_seen(base[b], masks[b], FULL, 0), SCALE)
            check_rows(out[b], lse.view(Hq, 2, n_q)[:, b], ref, (b, n_q), 2.0 ** -8)
        if kind == "mx4":
            rows = torch.empty(2, base[1] + n_q, HKV, D, dtype=torch.bfloat16, device="cuda")
            binding.cp_kv_gather_mx4(ctx, cache, table[1], 0, base[1] + n_q, rows[0], rows[1])
            assert all(torch.equal(rows[i].double(), x) for i, x in enumerate(values(1, base[1] + n_q)))
        old = [values(b, base[b] + n_q) for b in range(2)]
        path = i32([[0] * n_q] * 2)
        binding.cp_tree_commit(ctx, pool, table, kv_len, None, i32(parents), i32([n_q - 1, 0]), path)
        torch.cuda.synchronize()
        ctx.poll_status()
        for b in range(2):
            keep = [x for x in path[b].tolist() if x >= 0]
            assert keep == [t for t in range(n_q) if masks[b][(n_q - 1, 0)[b]] >> t & 1] and int(kv_len[b]) == base[b] + len(keep)
            take = torch.tensor(list(range(base[b])) + [base[b] + x for x in keep], device="cuda")
            assert all(torch.equal(x[take], y) for x, y in zip(old[b], values(b, base[b] + len(keep))))
    q, out, lse = normal(g, 2, 1, 16, D), torch.empty(2, 1, 16, D, dtype=torch.bfloat16, device="cuda"), torch.empty(16, 2, device="cuda")
    ws = torch.empty(binding.cp_workspace_bytes_decode(2, 1, 16, HKV), dtype=torch.uint8, device="cuda")
    DECODE[kind](ctx, q, cache, table, kv_len, FULL, 0, SCALE, out, lse, ws)
    for b in range(2):
        n = int(kv_len[b])
        ref = attention64(q[b].double(), *values(b, n), torch.tensor([n - 1], device="cuda"), FULL, 0, SCALE)
        check_attention(out[b], lse[:, b:b + 1], ref, (b, n), weight_eps=2.0 ** -8)
