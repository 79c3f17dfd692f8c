"""Rotary append through the C ABI against the rotation in 64 bits: axes, both pair layouts, partial rotation, far positions, padding rows,
in-place queries, strided caches, FP8 caches, tokens and pages out of range, graph replay."""
import math

import numpy as np
import pytest
import torch

from paper_2609_04774_b200 import binding
from tests.gpu_util import Guarded
from tests.serving_util import D, e4m3_codes, generator, normal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


def rotate64(x, pos, rope):
    """x [n, H, 128] in 64 bits, pos [axes, n] -> rotated, and |a| + |b| of every element's pair (0 where nothing turns)."""
    n = rope.rot_dims // 2
    freq = torch.tensor(list(rope.freq)[:n], dtype=torch.float64, device=x.device)
    axis = torch.tensor(list(rope.axis)[:n], device=x.device)
    ang = (pos[axis].double().T * freq)[:, None]
    first = torch.arange(n, device=x.device) * (2 if rope.interleaved else 1)
    second = first + (1 if rope.interleaved else n)
    a, b = x[..., first], x[..., second]
    y, size = x.clone(), torch.zeros_like(x)
    y[..., first] = a * ang.cos() - b * ang.sin()
    y[..., second] = b * ang.cos() + a * ang.sin()
    size[..., first] = size[..., second] = a.abs() + b.abs()
    return y, size


def check_rotated(got, ref, size, what):
    """Half a bf16 step of the value, and the fp32 arithmetic: cosine and sine off by at most 2^-21 (an angle to 2^-23 of a turn's fraction, 2
    ulp of the function), three roundings of 2^-24 of the products; far positions lose 2^31 * 2^-53 * 2 pi < 2^-19 in the reference's angle."""
    excess = ((got.double() - ref).abs() - 2.0 ** -8 * ref.abs() - 2.0 ** -18 * size).max().item()
    assert excess <= 0, (what, excess)


class Case:
    def __init__(self, seed, n, Hq, Hkv, page, sections, interleaved=False, base=10000.0, fp8=False, strided=False, far=None, rows=4):
        g = generator(seed)
        rng = np.random.default_rng(seed)
        self.rope = binding.make_rope(sections, base=base, interleaved=interleaved)
        self.n, self.Hq, self.Hkv, self.page, self.fp8 = n, Hq, Hkv, page, fp8
        per = -(-n // rows)
        width = -(-(per + 5) // page)
        pool = rows * width + 2
        self.table = torch.randperm(pool, generator=g, device="cuda")[:rows * width].to(torch.int32).view(rows, width).contiguous()
        places = [(r, t) for r in range(rows) for t in range(per + 5)]
        order = rng.permutation(len(places))[:n]
        self.seq = torch.tensor([places[i][0] for i in order], dtype=torch.int32, device="cuda")
        self.slot = torch.tensor([places[i][1] for i in order], dtype=torch.int32, device="cuda")
        hi = far or 3000
        self.pos = torch.from_numpy(rng.integers(-hi if far else 0, hi, size=(len(sections), n))).to(torch.int32).cuda()
        self.q, self.kr, self.vr = normal(g, n, Hq, D), normal(g, n, Hkv, D), normal(g, n, Hkv, D)
        shape = (pool, page, Hkv, D)
        if strided:                                        # heads, then tokens, with a gap: a view of a larger pool
            big = (e4m3_codes(g, 2, pool, Hkv + 1, page + 1, D) if fp8 else normal(g, 2, pool, Hkv + 1, page + 1, D))
            self.k, self.v = (big[i, :, :Hkv, :page].permute(0, 2, 1, 3) for i in range(2))
        elif fp8:
            self.k, self.v = e4m3_codes(g, *shape), e4m3_codes(g, *shape)
        else:
            self.k, self.v = normal(g, *shape), normal(g, *shape)
        if fp8:
            self.ks = (torch.rand(Hkv, generator=g, device="cuda") + 0.5) / 100.0
            self.vs = (torch.rand(Hkv, generator=g, device="cuda") + 0.5) / 100.0
            self.cache = binding.make_cache_fp8(self.k, self.v, self.ks, self.vs)
        else:
            self.cache = binding.make_cache(self.k, self.v)
        self.g_out = Guarded((n, Hq, D), torch.bfloat16, float("nan"))

    def call(self, ctx, **kw):
        a = dict(q=self.q, k_rows=self.kr, v_rows=self.vr, positions=self.pos, token_seq=self.seq, token_slot=self.slot, page_table=self.table,
                 q_out=self.g_out.tensor, stream=None) | kw
        f = binding.cp_rope_append_fp8 if self.fp8 else binding.cp_rope_append
        f(ctx, self.rope, a["q"], a["k_rows"], a["v_rows"], a["positions"], a["token_seq"], a["token_slot"], self.cache, a["page_table"], a["q_out"],
          stream=a["stream"])

    def check(self, ctx, skipped=None):
        """skipped: bool [n], tokens whose k and v are not written."""
        k0, v0 = self.k.clone(), self.v.clone()
        self.call(ctx)
        torch.cuda.synchronize()
        ctx.poll_status()
        self.g_out.check("q_out")
        self.compare(k0, v0, torch.ones(self.n, dtype=torch.bool, device="cuda"))

    def compare(self, k0, v0, written):
        ref, size = rotate64(self.q.double(), self.pos, self.rope)
        check_rotated(self.g_out.tensor, ref, size, "q")
        tail = slice(self.rope.rot_dims, D)
        assert torch.equal(self.g_out.tensor[..., tail], self.q[..., tail])
        ids = self.table[self.seq.long().clamp(min=0), (self.slot.long() // self.page).clamp(0, self.table.shape[1] - 1)].long()
        where = (ids[written], (self.slot.long() % self.page)[written])
        kr, ksize = rotate64(self.kr.double(), self.pos, self.rope)
        if self.fp8:
            for got, ref, sc, sz, what in ((self.k, kr, self.ks, ksize, "k"), (self.v, self.vr.double(), self.vs, None, "v")):
                s = sc.double()[:, None]
                val = got[where].contiguous().view(torch.float8_e4m3fn).double() * s
                ref = ref[written]
                near = ref.clamp(-448 * s, 448 * s)
                # half an e4m3 step (2^-4 of the value, 2^-10 scale below 2^-6) on top of the fp32 arithmetic, which can also move a tie
                bound = 2.0 ** -4 * near.abs() + 2.0 ** -10 * s + (2.0 ** -18 * sz[written] if sz is not None else 0) + 2.0 ** -22 * near.abs()
                assert bool(((val - near).abs() <= bound).all()), what
        else:
            check_rotated(self.k[where], kr[written], ksize[written], "k")
            assert torch.equal(self.k[where][..., tail], self.kr[written][..., tail])
            assert torch.equal(self.v[where], self.vr[written])
        k0[where], v0[where] = self.k[where], self.v[where]
        assert torch.equal(k0, self.k) and torch.equal(v0, self.v), "slots that no token names were touched"


@pytest.mark.parametrize("sections", [[64], [16, 24, 24], [32, 32], [8, 8], [10, 20, 14, 4], [0, 40, 24], [24, 0, 0]])
@pytest.mark.parametrize("interleaved", [False, True])
def test_axes_layouts_and_partial_rotation(ctx, sections, interleaved):
    Case(len(sections) * 10 + sum(sections), 77, 8, 2, 16, sections, interleaved).check(ctx)


@pytest.mark.parametrize("n", [1, 2, 31, 500, 5000])
@pytest.mark.parametrize("Hq,Hkv", [(32, 8), (5, 1), (3, 3), (16, 16), (7, 7)])
def test_token_counts_and_heads(ctx, n, Hq, Hkv):
    Case(n + Hq, n, Hq, Hkv, 64, [16, 24, 24]).check(ctx)


@pytest.mark.parametrize("far", [1000000, 2 ** 31 - 1])
@pytest.mark.parametrize("base", [10000.0, 1e6, 3.0])
def test_far_and_negative_positions(ctx, far, base):
    Case(3, 300, 4, 1, 32, [32, 32], base=base, far=far).check(ctx)


def test_exact_quarter_turns(ctx):
    c = Case(4, 64, 4, 2, 16, [64])
    for i in range(64):
        c.rope.freq[i] = math.pi / 2
    c.pos.copy_(torch.arange(64, device="cuda", dtype=torch.int32)[None] * 1000003)
    c.call(ctx)
    x, y = c.q.float(), c.g_out.tensor.float()
    turn = (c.pos[0].long() * 1 % 4)[:, None, None]
    a, b = x[..., :64], x[..., 64:]
    ra = torch.where(turn == 0, a, torch.where(turn == 1, -b, torch.where(turn == 2, -a, b)))
    rb = torch.where(turn == 0, b, torch.where(turn == 1, a, torch.where(turn == 2, -b, -a)))
    assert (y[..., :64] - ra).abs().max() <= 2.0 ** -8 * 6 and (y[..., 64:] - rb).abs().max() <= 2.0 ** -8 * 6


def test_frequencies_beyond_a_turn_and_changed_axes(ctx):
    c = Case(5, 100, 4, 2, 16, [32, 32])
    for i in range(64):
        c.rope.freq[i], c.rope.axis[i] = -17.5 + 0.7 * i, i % 2
    c.check(ctx)


@pytest.mark.parametrize("page,Hkv", [(16, 3), (128, 8)])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("strided", [False, True])
def test_fp8_and_strided_caches(ctx, page, Hkv, fp8, strided):
    Case(6 + page, 200, 2 * Hkv, Hkv, page, [16, 24, 24], interleaved=page == 16, fp8=fp8, strided=strided).check(ctx)


def test_fp8_zero_rotation_equals_the_quantising_append(ctx):
    """At position 0 nothing turns: the stored bytes are those of cp_kv_append_fp8."""
    c = Case(7, 48, 8, 4, 16, [64], fp8=True, rows=1)
    c.slot.copy_(torch.arange(48, device="cuda"))
    c.pos.zero_()
    c.call(ctx)
    got = c.k.clone(), c.v.clone()
    c.k.zero_(), c.v.zero_()
    binding.cp_kv_append_fp8(ctx, c.cache, c.table[0], 0, 48, c.kr, c.vr)
    ids = c.table[0].long()
    for a, b in zip(got, (c.k, c.v)):
        assert torch.equal(a[ids].flatten(0, 1)[:48], b[ids].flatten(0, 1)[:48])


@pytest.mark.parametrize("scale", [1.0, 0.37, 2.0 ** -6, 1.7e-38, 1e30, 3e-39, 1e-41, 0.0, -0.02])
def test_fp8_codes_of_every_bf16_value(ctx, scale):
    """All 65536 bit patterns at position 0: the codes of the quantising append, ties and borders of the format among them."""
    c = Case(13, 64, 8, 8, 16, [64], fp8=True, rows=1)
    c.slot.copy_(torch.arange(64, device="cuda"))
    c.pos.zero_()
    bits = torch.arange(65536, device="cuda", dtype=torch.int32).to(torch.int16).view(torch.bfloat16).view(64, 8, D)
    # at angle 0 an element becomes x * 1 - y * 0: its pair's other half must be finite, so non-finite patterns go through v alone
    c.vr.copy_(bits)
    c.kr.copy_(torch.where(torch.isfinite(bits), bits, torch.zeros_like(bits)))
    c.ks.fill_(scale), c.vs.fill_(scale)
    c.call(ctx)
    ids = c.table[0].long()
    got = [x[ids].flatten(0, 1)[:64].clone() for x in (c.k, c.v)]
    binding.cp_kv_append_fp8(ctx, c.cache, c.table[0], 0, 64, c.kr, c.vr)
    want = [x[ids].flatten(0, 1)[:64] for x in (c.k, c.v)]
    # -0 keeps or loses its sign in x * 1 - y * 0: both codes stand for zero
    zero = lambda t: torch.where(t == 0x80, torch.zeros_like(t), t)
    assert torch.equal(zero(got[0]), zero(want[0])) and torch.equal(got[1], want[1])


def test_padding_rows_in_place_and_parts(ctx):
    c = Case(8, 90, 8, 2, 16, [64])
    pad = torch.arange(90, device="cuda") % 3 == 1
    c.seq[pad] = -1
    k0, v0, q0 = c.k.clone(), c.v.clone(), c.q.clone()
    c.call(ctx, q_out=c.q)                                  # q rotates in place
    torch.cuda.synchronize()
    ctx.poll_status()
    assert torch.equal(c.q[pad], q0[pad])
    out, c.q = c.q, q0
    c.g_out.tensor.copy_(out)
    ref, size = rotate64(q0.double(), c.pos, c.rope)
    c.g_out.tensor[pad] = ref[pad].to(torch.bfloat16)
    c.compare(k0, v0, ~pad)
    # queries alone, keys alone
    k1 = c.k.clone()
    c.g_out.tensor.fill_(float("nan"))
    c.call(ctx, k_rows=None, v_rows=None)
    assert torch.equal(c.g_out.tensor[~pad], out[~pad]) and bool(torch.isnan(c.g_out.tensor[pad]).all()) and torch.equal(c.k, k1)
    c.k.copy_(k0), c.v.copy_(v0)
    c.call(ctx, q=None, q_out=None)
    assert torch.equal(c.k, k1)


@pytest.mark.parametrize("kind", ["page below", "page above", "slot below", "slot behind", "row behind"])
def test_tokens_out_of_range_are_skipped_and_reported(ctx, kind):
    c = Case(9, 40, 4, 2, 16, [64])
    written = torch.ones(40, dtype=torch.bool, device="cuda")
    k0, v0 = c.k.clone(), c.v.clone()
    if kind.startswith("page"):
        entry = int(c.slot[11]) // 16
        hit = (c.seq == c.seq[11]) & (c.slot // 16 == entry)
        keep = int(c.table[int(c.seq[11]), entry])
        c.table[int(c.seq[11]), entry] = -3 if kind == "page below" else c.k.shape[0]
    else:
        hit = torch.arange(40, device="cuda") == 11
        if kind == "slot below":
            c.slot[11] = -1
        elif kind == "slot behind":
            c.slot[11] = c.table.shape[1] * 16
        else:
            c.seq[11] = 4
    c.call(ctx)
    torch.cuda.synchronize()
    with pytest.raises(binding.CpError) as e:
        ctx.poll_status()
    assert e.value.code == binding.CP_ERR_BOUNDS
    ctx.poll_status()
    if kind.startswith("page"):
        c.table[int(c.seq[11]), entry] = keep
    if kind == "row behind":
        c.seq[11] = 0
    written[hit] = False
    c.compare(k0, v0, written)


def test_captured_and_replayed_with_new_contents(ctx):
    c = Case(10, 64, 8, 2, 16, [16, 24, 24])
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        c.call(ctx, stream=stream)
    for seed in (1, 2):
        g = generator(100 + seed)
        c.q.copy_(normal(g, *c.q.shape)), c.kr.copy_(normal(g, *c.kr.shape))
        c.pos.add_(977)
        k0, v0 = c.k.clone(), c.v.clone()
        graph.replay()
        torch.cuda.synchronize()
        c.compare(k0, v0, torch.ones(64, dtype=torch.bool, device="cuda"))


def test_no_tokens(ctx):
    c = Case(12, 8, 4, 2, 16, [64])
    k0 = c.k.clone()
    c.call(ctx, q=c.q[:0], k_rows=c.kr[:0], v_rows=c.vr[:0], positions=c.pos[:, :0].contiguous(), token_seq=c.seq[:0], token_slot=c.slot[:0],
           q_out=c.g_out.tensor[:0])
    torch.cuda.synchronize()
    ctx.poll_status()
    assert torch.equal(c.k, k0)


def test_binding_refuses_what_the_call_would_misread(ctx):
    c = Case(11, 8, 4, 2, 16, [64])
    for kw in (dict(q=c.q.float()), dict(q=c.q.transpose(0, 1)), dict(positions=c.pos.long()), dict(positions=torch.cat([c.pos, c.pos])),
               dict(k_rows=c.kr[:4]), dict(token_slot=c.slot[:3]), dict(page_table=c.table.repeat(1, 2)[:, ::2]), dict(q_out=c.g_out.tensor.cpu())):
        with pytest.raises(ValueError):
            c.call(ctx, **kw)
    with pytest.raises(ValueError):
        c.call(ctx, k_rows=None)
    with pytest.raises(ValueError):
        c.call(ctx, q_out=None)
