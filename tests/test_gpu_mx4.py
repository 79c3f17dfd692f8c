"""4-bit caches through the C ABI: the codes that cp_rope_append_mx4 writes against the definition in 64 bits (all of them equal), what cp_kv_gather_mx4
reads back, cp_decode_attn_mx4 against attention over the stored values, page calls on such pools."""
import math
import random

import pytest
import torch

from paper_2609_04774_b200 import binding
from tests.serving_util import attention64, generator, normal
from tests.tree_util import FULL, Cache, D, attention64_seen, check_rows, mx4_quantise, mx4_values, tree_seen

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def turned(x, rope, positions):
    """[n, heads, 128] rotated in 64 bits; angles modulo one turn in whole arithmetic where they are large (Python integers would do: |angle| < 2^31 * 2 pi
    keeps 20 bits behind the point in a double, so the turns are taken from the fractions of freq / 2 pi in 2^-64)."""
    n = rope.rot_dims // 2
    y = x.double().clone()
    for i in range(n):
        step = int(math.floor((rope.freq[i] / (2 * math.pi)) % 1.0 * 2 ** 64)) & (2 ** 64 - 1)
        pos = positions[rope.axis[i]].tolist()
        half = torch.tensor([((p * step) & (2 ** 64 - 1)) / 2 ** 63 for p in pos], dtype=torch.float64, device="cuda")[:, None]
        c, s = torch.cos(half * math.pi), torch.sin(half * math.pi)
        a, b = (2 * i, 2 * i + 1) if rope.interleaved else (i, i + n)
        u, w = y[..., a].clone(), y[..., b].clone()
        y[..., a], y[..., b] = u * c - w * s, w * c + u * s
    return y


class Rows:
    def __init__(self, seed, n, Hq, Hkv, page, sections, interleaved=False, far=0, pad=0, x=None):
        g = generator(seed)
        self.Hkv = Hkv
        self.rope = binding.make_rope(sections, base=1e4, interleaved=interleaved)
        self.q = normal(g, n, Hq, D)
        self.k_rows, self.v_rows = (normal(g, n, Hkv, D), normal(g, n, Hkv, D)) if x is None else x
        self.positions = (far + torch.randint(0, 3000, (len(sections), n), generator=g, device="cuda")).to(torch.int32)
        rows = 3
        per = -(-n // rows)
        count = -(-(per + 5) // page)
        self.table = torch.randperm(rows * count + 2, generator=g, device="cuda")[:rows * count].to(torch.int32).view(rows, count)
        i = torch.arange(n, device="cuda")
        self.seq, self.slot = (i // per).to(torch.int32), (5 + i % per).to(torch.int32)
        shape = (rows * count + 2, page, binding.mx4_token_bytes(Hkv) + pad)
        self.page = page
        self.k, self.v = (torch.randint(0, 256, shape, generator=g, device="cuda", dtype=torch.uint8) for _ in range(2))
        self.k, self.v = self.k[..., :shape[2] - pad], self.v[..., :shape[2] - pad]
        self.cache = binding.make_cache_mx4(self.k, self.v, Hkv)

    def run(self, ctx):
        q_out = torch.empty_like(self.q)
        binding.cp_rope_append_mx4(ctx, self.rope, self.q, self.k_rows, self.v_rows, self.positions, self.seq, self.slot, self.cache, self.table, q_out)
        torch.cuda.synchronize()
        return q_out

    def check(self, ctx):
        want_k, want_v = self.k.clone(), self.v.clone()
        at = (self.table[self.seq.long(), self.slot.long() // self.page].long(), self.slot.long() % self.page)
        used = self.Hkv * 68
        keep = self.seq >= 0
        at = (at[0][keep], at[1][keep])
        turned_k = turned(self.k_rows, self.rope, self.positions)
        for want, x in ((want_k, turned_k), (want_v, self.v_rows)):
            rows = want[at]
            rows[:, :used] = mx4_quantise(x)[keep]
            want[at] = rows
        q_out = self.run(ctx)
        ctx.poll_status()
        # the sign of a value that the rotation makes zero (up to its error) is either; every other bit is the definition's
        zero = lambda rows: torch.stack([rows & 7, rows >> 4 & 7], -1) == 0  # noqa: E731
        for got, want in ((self.k, want_k), (self.v, want_v)):
            diff = got ^ want
            assert bool((diff[..., used:] == 0).all())
            codes = diff[..., :self.Hkv * 64]
            signs = torch.stack([codes & 8, codes >> 4 & 8], -1) != 0
            assert bool(((codes & 0x77) == 0).all()), "%d codes differ" % int((codes & 0x77 != 0).sum())
            assert bool((~signs | zero(want[..., :self.Hkv * 64])).all())
            assert bool((diff[..., self.Hkv * 64:used] == 0).all()), "exponents differ"
        want_q = turned(self.q, self.rope, self.positions)[keep]
        d = (q_out[keep].double() - want_q).abs()
        # one rounding to bf16, and the fp32 rotation's own error (angle 2^-25 of a turn, three roundings) of values up to about 6
        assert bool((d <= want_q.abs() * 2.0 ** -8 + 6 * 5e-7 * 2).all())


@pytest.mark.parametrize("Hkv", [1, 2, 3, 4, 8, 16])
@pytest.mark.parametrize("sections,interleaved", [([64], False), ([64], True), ([16, 24, 24], False), ([16], False), ([8], True), ([24], False), ([24], True), ([48], False)])
def test_append(ctx, Hkv, sections, interleaved):
    Rows(Hkv + len(sections), 37, 5, Hkv, 16, sections, interleaved).check(ctx)


@pytest.mark.parametrize("n", [1, 2, 3, 4000])
@pytest.mark.parametrize("interleaved", [False, True])
def test_append_sizes(ctx, n, interleaved):
    Rows(n, n, 32, 8, 64, [64], interleaved, far=10 ** 6).check(ctx)


@pytest.mark.parametrize("pad", [16, 64])
def test_append_strided(ctx, pad):
    Rows(pad, 50, 4, 3, 32, [64], pad=pad).check(ctx)


def test_append_at_the_borders(ctx):
    """Values on and next to the borders of the format, blocks whose largest element is a power of two or next to one, tiny, huge and empty blocks."""
    g = generator(3)
    borders = torch.tensor([0.0, -0.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 0.5, 1.0, 2.0, 4.0, 6.0, 7.0, 7.96875, 4.03125, 3.984375, 0.251953125, 0.2490234375, 5.03125,
                            4.96875, 1e-3, 3.0, 1.5], device="cuda")
    n, Hkv = 600, 4
    pick = lambda: borders[torch.randint(0, len(borders), (n, Hkv, D), generator=g, device="cuda")] * \
        torch.where(torch.rand(n, Hkv, D, generator=g, device="cuda") < 0.5, -1.0, 1.0)  # noqa: E731
    scale = torch.exp2(torch.randint(-120, 120, (n, Hkv, 4, 1), generator=g, device="cuda").float()).expand(n, Hkv, 4, 32).reshape(n, Hkv, D)
    v = (pick() * scale)
    v[::7] = 0.0
    v[1::7, :, :32] = 0.0
    k = pick()
    r = Rows(1, n, 4, Hkv, 32, [64], x=(k.bfloat16(), v.bfloat16()))
    r.positions.zero_()                                                  # no turn: the borders stay where they are
    r.positions[0, ::2] = torch.randint(0, 10 ** 6, (n // 2,), generator=g, device="cuda", dtype=torch.int32)
    r.check(ctx)


def test_append_of_infinities_and_nan(ctx):
    g = generator(4)
    k, v = normal(g, 40, 2, D), normal(g, 40, 2, D)
    v[3, 0, 40], v[5, 1, 127], v[9, 0, 0] = math.inf, math.nan, -math.inf
    k[4, 1, 100], k[6, 0, 3] = math.nan, math.inf
    r = Rows(2, 40, 4, 2, 16, [16], x=(k, v))                           # elements 32.. of k are not turned
    r.run(ctx)
    ctx.poll_status()
    at = (r.table[r.seq.long(), r.slot.long() // 16].long(), r.slot.long() % 16)
    vv, kk = mx4_values(r.v[at], 2), mx4_values(r.k[at], 2)
    for x, odd in ((vv, {(3, 0, 1), (5, 1, 3), (9, 0, 0)}), (kk, {(4, 1, 3), (6, 0, 0)})):
        blocks = x.view(40, 2, 4, 32)
        nan = torch.isnan(blocks)
        assert bool((nan.any(-1) == nan.all(-1)).all())
        assert {tuple(i) for i in torch.nonzero(nan.all(-1)).tolist()} == odd


def test_append_padding_reports_and_halves(ctx):
    r = Rows(5, 30, 4, 2, 16, [64])
    r.seq[::3] = -1
    q = r.q.clone()
    r.check(ctx)
    assert torch.equal(r.q, q)
    before = r.k.clone()
    for name, value in (("slot", 10 ** 6), ("slot", -1), ("seq", 3)):
        r = Rows(5, 30, 4, 2, 16, [64])
        getattr(r, name)[7] = value
        r.run(ctx)
        with pytest.raises(binding.CpError) as e:
            ctx.poll_status()
        assert e.value.code == binding.CP_ERR_BOUNDS
    r = Rows(5, 30, 4, 2, 16, [64])
    r.table[0, 0] = 10 ** 6
    r.run(ctx)
    with pytest.raises(binding.CpError):
        ctx.poll_status()
    # queries alone, keys alone
    r = Rows(5, 30, 4, 2, 16, [64])
    a = r.run(ctx)
    k = r.k.clone()
    b = torch.empty_like(r.q)
    binding.cp_rope_append_mx4(ctx, r.rope, r.q, None, None, r.positions, r.seq, None, r.cache, r.table, b)
    r.k.fill_(9)
    r.k[..., 136:] = k[..., 136:]
    binding.cp_rope_append_mx4(ctx, r.rope, None, r.k_rows, r.v_rows, r.positions, r.seq, r.slot, r.cache, r.table, None)
    torch.cuda.synchronize()
    at = (r.table[r.seq.long(), r.slot.long() // 16].long(), r.slot.long() % 16)
    assert torch.equal(a, b) and torch.equal(r.k[at], k[at])


# ---------------------------------------------------------------------------------------------------------------------- gather

@pytest.mark.parametrize("Hkv", [1, 3, 8])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("t_begin,n", [(0, 1), (0, 300), (17, 100), (128, 128), (299, 1), (5, 0)])
def test_gather(ctx, Hkv, page, t_begin, n):
    c = Cache(Hkv, [300], Hkv, page, "mx4", pad=16)
    k, v = (torch.full((n + 2, Hkv, D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    binding.cp_kv_gather_mx4(ctx, c.cache, c.table[0], t_begin, n, k[1:1 + n], v[1:1 + n])
    torch.cuda.synchronize()
    ctx.poll_status()
    for got, want in zip((k, v), c.values(0, 300)):
        assert torch.equal(got[1:1 + n].double(), want[t_begin:t_begin + n])
        assert bool((got[0] == 7).all()) and bool((got[n + 1:] == 7).all())


def test_gather_of_every_code_and_exponent(ctx):
    """All 16 codes with exponents 0..252 exactly (2^-128 .. 6 * 2^125), 255 as NaN; one of the pair alone; entries outside the pool."""
    rows = torch.zeros(16, 16, 80, dtype=torch.uint8, device="cuda")
    e = torch.arange(256, device="cuda", dtype=torch.uint8).view(16, 16)
    e = torch.where(e > 252, 255, e.int()).to(torch.uint8)
    rows[..., :64] = (torch.arange(64, device="cuda") * 37 + 16 * (torch.arange(64, device="cuda") % 16)).to(torch.uint8)
    rows[..., 64:68] = e[..., None]
    cache = binding.make_cache_mx4(rows, rows, 1)
    table = torch.arange(16, dtype=torch.int32, device="cuda")
    k = torch.empty(256, 1, D, dtype=torch.bfloat16, device="cuda")
    binding.cp_kv_gather_mx4(ctx, cache, table, 0, 256, k, None)
    torch.cuda.synchronize()
    want = mx4_values(rows.view(256, 80), 1)
    assert bool((torch.isnan(k) == torch.isnan(want)).all()) and torch.equal(k[:253].double(), want[:253])
    for bad in (-1, 16):
        table[3] = bad
        k.fill_(7)
        binding.cp_kv_gather_mx4(ctx, cache, table, 0, 256, None, k)
        torch.cuda.synchronize()
        with pytest.raises(binding.CpError) as err:
            ctx.poll_status()
        assert err.value.code == binding.CP_ERR_BOUNDS
        assert bool((k[48:64] == 7).all()) and torch.equal(k[64:253].double(), want[64:253]) and torch.equal(k[:48].double(), want[:48])


# ---------------------------------------------------------------------------------------------------------------------- decode

class Decode:
    def __init__(self, seed, lens, Hq, Hkv, page, n_q=1, pad=0, width=None, scale=D ** -0.5):
        self.kv = Cache(seed, lens, Hkv, page, "mx4", pad=pad, width=width)
        self.lens, self.Hq, self.n_q, self.scale = list(lens), Hq, n_q, scale
        B = len(lens)
        self.q = normal(generator(seed + 1), B, n_q, Hq, D)
        self.kv_len = i32(self.lens)
        self.out = torch.full((B, n_q, Hq, D), math.nan, dtype=torch.bfloat16, device="cuda")
        self.lse = torch.full((Hq, B * n_q), math.nan, dtype=torch.float32, device="cuda")
        self.ws = torch.full((binding.cp_workspace_bytes_decode(B, n_q, Hq, Hkv),), 0xFF, dtype=torch.uint8, device="cuda")

    def check(self, ctx, window=FULL, sinks=0, rows=None, lse_tol=2e-4, more=0.0):
        binding.cp_decode_attn_mx4(ctx, self.q, self.kv.cache, self.kv.table, self.kv_len, window, sinks, self.scale, self.out, self.lse, self.ws)
        torch.cuda.synchronize()
        ctx.poll_status()
        for b, n in enumerate(self.lens):
            if rows is not None and b not in rows:
                continue
            k, v = self.kv.values(b, n)
            p = n - self.n_q + torch.arange(self.n_q, device="cuda")
            j = torch.arange(n, device="cuda")
            seen = (j[None, :] <= p[:, None]) & ((p[:, None] - j[None, :] < window) | (j[None, :] < sinks))
            ref = attention64_seen(self.q[b].double(), k, v, seen, self.scale)
            check_rows(self.out[b], self.lse.view(self.Hq, -1, self.n_q)[:, b], ref, (b, n, window, sinks), 2.0 ** -8 + more, lse_tol)


LENS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 127, 128, 129, 300, 1000, 2049]


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("n_q", [1, 3])
@pytest.mark.parametrize("Hq,Hkv", [(8, 4), (8, 2)])
@pytest.mark.parametrize("width", [None, 160])
def test_decode_lengths(ctx, page, n_q, Hq, Hkv, width):
    """Wide tables: units of several heads; narrow ones: of one."""
    Decode(page + n_q, LENS, Hq, Hkv, page, n_q=n_q, width=width).check(ctx)


@pytest.mark.parametrize("Hq,Hkv,n_q", [(8, 8, 1), (16, 8, 3), (40, 8, 3), (64, 8, 8), (12, 6, 2), (24, 2, 1), (24, 2, 3), (28, 4, 4)])
@pytest.mark.parametrize("width", [None, 100])
def test_decode_units_of_heads(ctx, Hq, Hkv, n_q, width):
    Decode(Hq + n_q, [5, 700, 0, 1300, 64, 9], Hq, Hkv, 16, n_q=n_q, width=width).check(ctx)


@pytest.mark.parametrize("Hq,Hkv,n_q", [(1, 1, 1), (8, 8, 1), (7, 1, 1), (9, 1, 1), (16, 1, 1), (17, 1, 1), (33, 1, 1), (64, 8, 4), (128, 4, 1), (128, 4, 2), (5, 5, 7), (12, 4, 5),
                                        (4, 2, 64), (16, 16, 1), (12, 12, 3), (64, 4, 1)])
def test_decode_heads(ctx, Hq, Hkv, n_q):
    Decode(Hq + n_q, [5, 700, 0, 130], Hq, Hkv, 32, n_q=n_q).check(ctx)


@pytest.mark.parametrize("Hkv", [2, 4])
@pytest.mark.parametrize("window", [1, 2, 15, 16, 17, 100, 127, 128, 129, 500])
@pytest.mark.parametrize("sinks", [0, 1, 4, 130, 5000])
def test_decode_windows(ctx, Hkv, window, sinks):
    Decode(window + sinks, [0, 1, 100, 128, 129, 257, 700, 1300], 8, Hkv, 16, n_q=2).check(ctx, window, sinks)


@pytest.mark.parametrize("lens,Hq,Hkv,n_q,window,sinks", [([40000], 4, 1, 1, FULL, 0), ([100000, 3], 32, 4, 1, FULL, 0), ([33000, 60000, 1, 0], 16, 4, 4, FULL, 0),
                                                          ([50000], 8, 8, 1, 30000, 300), ([19000], 40, 1, 1, FULL, 0)])
def test_decode_cut_units(ctx, lens, Hq, Hkv, n_q, window, sinks):
    Decode(3, lens, Hq, Hkv, 64, n_q=n_q).check(ctx, window, sinks)


def test_decode_many(ctx):
    rng = random.Random(3)
    lens = [rng.randrange(0, 90) for _ in range(900)]
    Decode(5, lens, 8, 4, 16).check(ctx, rows=range(0, 900, 31))


@pytest.mark.parametrize("n_q", [1, 3])
@pytest.mark.parametrize("Hkv", [2, 4, 6])
def test_decode_of_all_magnitudes(ctx, n_q, Hkv):
    """V with exponents from 0 to 253 and K with a few large and tiny blocks: the weights' common factor has to follow, in single tiles and over several."""
    for seed, lo, hi in ((0, 0, 20), (1, 100, 140), (2, 120, 200), (3, 200, 250), (4, 60, 180)):
        s = Decode(seed, [500, 37, 3000], 2 * Hkv if Hkv > 4 else 8, Hkv, 32, n_q=n_q)
        g = generator(seed + 50)
        e = s.kv.v[..., Hkv * 64:Hkv * 68]
        e.copy_(torch.where(e == 255, 255, torch.randint(lo, hi + 1, e.shape, generator=g, device="cuda")).to(torch.uint8))
        k = s.kv.k[..., Hkv * 64:Hkv * 68]
        few = (torch.rand(k.shape, generator=g, device="cuda") < 0.02) & (k != 255)
        k.copy_(torch.where(few, torch.randint(0, 128, k.shape, generator=g, device="cuda"), k.int()).to(torch.uint8))
        if seed == 0:
            # results near 2^-110 are fp32 subnormals in the accumulators' scale (2^-16 of the values): half a step of 2^-149 + 16 per key, 3000 keys
            binding.cp_decode_attn_mx4(ctx, s.q, s.kv.cache, s.kv.table, s.kv_len, FULL, 0, s.scale, s.out, s.lse, s.ws)
            torch.cuda.synchronize()
            assert bool(torch.isfinite(s.out).all()) and bool((s.out.abs() <= 6 * 2.0 ** (20 - 127)).all())
        else:
            s.check(ctx)


@pytest.mark.parametrize("n_q", [1, 4])
@pytest.mark.parametrize("Hkv", [2, 4, 6, 8])
def test_decode_of_nan_blocks(ctx, n_q, Hkv):
    """A NaN block of V reaches its 32 elements of the rows that see the key, one of K whole rows; also beside large exponents."""
    s = Decode(7, [200, 500], 2 * Hkv if Hkv > 4 else 8, Hkv, 16, n_q=n_q)
    for b, t, which, byte in ((0, 199, "v", 2), (0, 198, "v", 7), (1, 40, "v", 1), (1, 499, "k", 5), (0, 150, "v", 4)):
        page, at = s.kv.where(b, torch.tensor(t, device="cuda"))
        getattr(s.kv, which)[page, at, Hkv * 64 + byte] = 255
    page, at = s.kv.where(1, torch.tensor(41, device="cuda"))
    s.kv.v[page, at, Hkv * 64] = 190
    s.check(ctx)
    s.check(ctx, 20, 0)


def test_decode_large_keys(ctx):
    """K with exponents beyond those of ordinary caches: scores in the thousands, so a weight's relative error is that of its score: 128 products of magnitude
    up to 2^9 * 6 * 4 * scale, 2^-23 each."""
    s = Decode(9, [300], 8, 4, 16, scale=2.0 ** -14)
    k = s.kv.k[..., 256:272]
    k.copy_(torch.where(k == 255, 255, 136).to(torch.uint8))
    err = 128 * 2.0 ** -23 * 2 ** 9 * 24 * 2.0 ** -14
    s.check(ctx, more=2 * err, lse_tol=2e-4 + 2 * err)


def test_decode_replayed(ctx):
    s = Decode(11, [900, 40, 2000], 8, 4, 64)
    s.check(ctx)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.cp_decode_attn_mx4(ctx, s.q, s.kv.cache, s.kv.table, s.kv_len, FULL, 0, s.scale, s.out, s.lse, s.ws)
    s.lens = [5, 0, 1999]
    s.kv_len.copy_(i32(s.lens))
    graph.replay()
    torch.cuda.synchronize()
    for b, n in enumerate(s.lens):
        k, v = s.kv.values(b, n)
        ref = attention64(s.q[b].double(), k, v, torch.tensor([n - 1], device="cuda"), FULL, 0, s.scale)
        check_rows(s.out[b], s.lse[:, b:b + 1], ref, b, 2.0 ** -8)


# ---------------------------------------------------------------------------------------------------------------------- pages

def test_page_calls_on_4_bit_pools(ctx):
    """fork copies the tokens of a partly filled page, compact and copy whole pages, byte by byte."""
    Hkv, page, layers, n = 3, 16, 2, 12
    g = generator(1)
    k, v = (torch.randint(0, 256, (layers, n, page, binding.mx4_token_bytes(Hkv) + 16), generator=g, device="cuda", dtype=torch.uint8)[..., :208] for _ in range(2))
    pool = binding.make_page_pool_mx4(k, v)
    ws = torch.empty(binding.cp_workspace_bytes_pages(n, 4), dtype=torch.uint8, device="cuda")
    table, refs, kv_len = i32([[7, 4, -1], [-1, -1, -1]]), torch.zeros(n, dtype=torch.int32, device="cuda"), i32([21, 0])
    refs[7] = refs[4] = 1
    k0, v0 = k.clone(), v.clone()
    binding.cp_pages_fork(ctx, pool, refs, table, kv_len, i32([0]), i32([1]), ws)
    torch.cuda.synchronize()
    assert table.tolist() == [[7, 4, -1], [7, 0, -1]] and kv_len.tolist() == [21, 21]
    for x, x0 in ((k, k0), (v, v0)):
        assert torch.equal(x[:, 0, :5], x0[:, 4, :5]) and torch.equal(x[:, 0, 5:], x0[:, 0, 5:]) and torch.equal(x[:, 1:], x0[:, 1:])
    binding.cp_pages_copy(ctx, pool, i32([7]), i32([9]), ws)
    torch.cuda.synchronize()
    assert torch.equal(k[:, 9], k0[:, 7]) and torch.equal(v[:, 9], v0[:, 7])
    page_map, n_live = torch.empty(n, dtype=torch.int32, device="cuda"), i32([0])
    binding.cp_pages_compact(ctx, pool, refs, table, page_map, n_live, ws)
    torch.cuda.synchronize()
    ctx.poll_status()
    assert n_live.item() == 3 and sorted(set(table.flatten().tolist())) == [-1, 0, 1, 2]
    assert torch.equal(k[:, int(table[0, 0])], k0[:, 7]) and torch.equal(v[:, int(table[0, 1])], v0[:, 4])
