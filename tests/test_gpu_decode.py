"""Decode attention through the C ABI against the definition in 64 bits: lengths from none to many pages, rows before position 0, head groups and
row groups, windows and sinks, both caches, strided pools, unread slots that hold NaN, pages given back, cut units, large batches, replayed graphs."""
import numpy as np
import pytest
import torch

from paper_2609_04774_b200 import binding
from tests.gpu_util import Guarded
from tests.serving_util import D, Paged, attention64, check_attention, generator, normal

pytestmark = pytest.mark.gpu
SCALE = D ** -0.5
FULL = binding.CP_NO_WINDOW


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


class Step:
    def __init__(self, seed, lens, Hq, Hkv, page, n_q=1, fp8=False, width=None, junk=float("nan"), scale=SCALE):
        g = generator(seed)
        self.kv = Paged(g, lens, Hkv, page, fp8=fp8, width=width, junk=junk)
        self.lens, self.Hq, self.Hkv, self.n_q, self.scale = list(lens), Hq, Hkv, n_q, scale
        B = len(lens)
        self.q = normal(g, B, n_q, Hq, D)
        self.kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.g_out = Guarded((B, n_q, Hq, D), torch.bfloat16, float("nan"))
        self.g_lse = Guarded((Hq, B * n_q), torch.float32, float("nan"))
        self.g_ws = Guarded((binding.cp_workspace_bytes_decode(B, n_q, Hq, Hkv),), torch.uint8, 0xFF)
        self.describe()

    def describe(self):
        kv = self.kv
        self.cache = binding.make_cache_fp8(kv.k, kv.v, kv.k_scale, kv.v_scale) if kv.fp8 else binding.make_cache(kv.k, kv.v)

    def call(self, ctx, window=FULL, sinks=0, stream=None, ws=None, kv_len=None):
        f = binding.cp_decode_attn_fp8 if self.kv.fp8 else binding.cp_decode_attn
        f(ctx, self.q, self.cache, self.kv.table, self.kv_len if kv_len is None else kv_len, window, sinks, self.scale, self.g_out.tensor,
          self.g_lse.tensor, self.g_ws.tensor if ws is None else ws, stream=stream)

    def run(self, ctx, window=FULL, sinks=0):
        self.g_out.tensor.fill_(float("nan"))
        self.g_lse.tensor.fill_(float("nan"))
        self.call(ctx, window, sinks)
        torch.cuda.synchronize()
        ctx.poll_status()
        for g, what in ((self.g_out, "out"), (self.g_lse, "lse"), (self.g_ws, "workspace")):
            g.check(what)
        return self.g_out.tensor, self.g_lse.tensor

    def compare(self, window=FULL, sinks=0, lens=None, rows=None):
        out, lse = self.g_out.tensor, self.g_lse.tensor
        for b, n in enumerate(lens or self.lens):
            if rows is not None and b not in rows:
                continue
            k, v = self.kv.keys_values(b, n)
            p = n - self.n_q + torch.arange(self.n_q, device="cuda")
            ref = attention64(self.q[b].double(), k, v, p, window, sinks, self.scale)
            check_attention(out[b], lse[:, b * self.n_q:(b + 1) * self.n_q], ref, (b, n, window, sinks),
                            weight_eps=2.0 ** -11 + 2.0 ** -16 if self.kv.fp8 else 2.0 ** -8)

    def check(self, ctx, window=FULL, sinks=0, rows=None):
        self.run(ctx, window, sinks)
        self.compare(window, sinks, rows=rows)


LENS = [0, 1, 2, 15, 16, 17, 63, 127, 128, 129, 300, 1000, 2049]


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("n_q", [1, 3])
def test_lengths(ctx, fp8, page, n_q):
    Step(page + n_q, LENS, 8, 2, page, n_q=n_q, fp8=fp8).check(ctx)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("Hq,Hkv,n_q", [(1, 1, 1), (8, 8, 1), (7, 1, 1), (8, 1, 1), (9, 1, 1), (16, 1, 1), (17, 1, 1), (32, 1, 1), (33, 1, 1), (64, 8, 4),
                                        (128, 1, 2), (5, 5, 7), (12, 4, 5), (4, 2, 64), (16, 16, 1)])
def test_heads_and_row_groups(ctx, fp8, Hq, Hkv, n_q):
    Step(Hq + n_q, [5, 700, 0, 130], Hq, Hkv, 32, n_q=n_q, fp8=fp8).check(ctx)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("window", [1, 2, 15, 16, 17, 100, 127, 128, 129, 500])
@pytest.mark.parametrize("sinks", [0, 1, 4, 130, 5000])
def test_windows_and_sinks(ctx, fp8, window, sinks):
    Step(window + sinks, [0, 1, 100, 128, 129, 257, 700, 1300], 8, 4, 16, n_q=2, fp8=fp8).check(ctx, window, sinks)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("lens,Hq,Hkv,n_q,window,sinks", [([40000], 4, 1, 1, FULL, 0), ([100000, 3], 32, 2, 1, FULL, 0), ([33000, 60000, 1, 0], 16, 2, 4, FULL, 0),
                                                          ([50000], 8, 8, 1, 30000, 300), ([19000], 40, 1, 1, FULL, 0)])
def test_units_cut_over_many_ctas(ctx, fp8, lens, Hq, Hkv, n_q, window, sinks):
    Step(3, lens, Hq, Hkv, 64, n_q=n_q, fp8=fp8).check(ctx, window, sinks)


@pytest.mark.parametrize("seed", range(10))
def test_random_batches(ctx, seed):
    rng = np.random.default_rng(seed)
    lens = [int(np.exp(rng.uniform(0, np.log(6000)))) if rng.random() < 0.9 else 0 for _ in range(int(rng.integers(1, 40)))]
    Hq, Hkv = [(8, 2), (4, 4), (9, 3), (16, 2)][seed % 4]
    window = FULL if seed % 3 == 0 else int(np.exp(rng.uniform(0, np.log(3000))))
    Step(100 + seed, lens, Hq, Hkv, [16, 32, 64, 128][seed % 4], n_q=1 + seed % 5, fp8=seed % 2 == 1).check(ctx, window, int(rng.integers(0, 300)))


@pytest.mark.parametrize("B", [255, 256, 257, 1500])
def test_large_batches(ctx, B):
    rng = np.random.default_rng(B)
    lens = [int(x) for x in rng.integers(0, 200, B)]
    s = Step(B, lens, 4, 2, 16)
    s.run(ctx)
    s.compare(rows=set(int(x) for x in rng.integers(0, B, 60)) | {0, 1, B - 1})
    assert not bool(torch.isnan(s.g_out.tensor).any()) and not bool(torch.isnan(s.g_lse.tensor).any())


@pytest.mark.parametrize("scale", [0.3, 2.0])
@pytest.mark.parametrize("fp8", [False, True])
def test_large_scores_raise_the_maximum_late(ctx, scale, fp8):
    """Scores up to about 60 sqrt(2 ln n) scale: the lse tolerance grows with the scores' fp32 error, 128 * 2^-23 * sum |q k| scale."""
    s = Step(6, [3000, 900], 8, 2, 64, fp8=fp8, scale=scale)
    out, lse = s.run(ctx)
    for b, n in enumerate(s.lens):
        k, v = s.kv.keys_values(b, n)
        ref = attention64(s.q[b].double(), k, v, torch.tensor([n - 1], device="cuda"), FULL, 0, scale)
        # sum |q k| is about 82 for unit normals; a weight is off by as much as the score, plus its rounding to bf16 or fp16
        score = 128 * 2.0 ** -23 * 130 * scale
        check_attention(out[b], lse[:, b:b + 1], ref, (b, scale), weight_eps=2.0 ** -8 + 2 * score, lse_tol=2e-4 + 2 * score)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("Hkv", [3, 4])
def test_strided_pool(ctx, fp8, Hkv):
    s = Step(8, [700, 33, 128], 2 * Hkv, Hkv, 32, fp8=fp8)
    for name in ("k", "v"):
        t = getattr(s.kv, name)
        big = torch.zeros(t.shape[0], Hkv + 1, 35, D, dtype=t.dtype, device="cuda")
        view = big[:, :Hkv, :32].permute(0, 2, 1, 3)
        view.copy_(t)
        setattr(s.kv, name, view)
    s.describe()
    s.check(ctx)
    s.check(ctx, 100, 4)


@pytest.mark.parametrize("fp8", [False, True])
def test_pages_given_back_and_bad_entries_behind_the_window(ctx, fp8):
    s = Step(9, [3000, 700, 64], 8, 2, 16, n_q=2, fp8=fp8)
    window, sinks = 333, 20
    out, lse = (x.clone() for x in s.run(ctx, window, sinks))
    for b, n in enumerate(s.lens):
        first, last = -(-sinks // 16), max(0, n - 2 + 1 - window) // 16
        gone = s.kv.table[b, first:last].long()
        if not fp8:
            s.kv.k[gone], s.kv.v[gone] = float("nan"), float("inf")
        s.kv.table[b, first:last] = torch.tensor([-1, 10 ** 9, s.kv.k.shape[0], -7] * 60, dtype=torch.int32, device="cuda")[:max(0, last - first)]
    o2, l2 = s.run(ctx, window, sinks)
    assert torch.equal(out, o2) and torch.equal(lse, l2)


def test_visible_entry_outside_the_pool_reads_as_zeros(ctx):
    s = Step(10, [200], 4, 2, 16)
    ids = s.kv.table[0].clone()
    for bad in (-1, s.kv.k.shape[0], 2 ** 31 - 1):
        s.kv.table[0, 5] = bad
        out, lse = s.run(ctx)
        s.kv.table[0, 5] = ids[5]
        keep = s.kv.k[ids[5].long()].clone(), s.kv.v[ids[5].long()].clone()
        s.kv.k[ids[5].long()], s.kv.v[ids[5].long()] = 0, 0
        s.compare()
        s.kv.k[ids[5].long()], s.kv.v[ids[5].long()] = keep


def test_lengths_out_of_range_are_clamped_and_reported(ctx):
    s = Step(11, [100, 64, 48], 4, 2, 16, width=8)
    s.kv.table[1, 4:] = s.kv.table[0, 4:5]
    s.call(ctx, kv_len=torch.tensor([100, 64, -5], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    with pytest.raises(binding.CpError) as e:
        ctx.poll_status()
    assert e.value.code == binding.CP_ERR_BOUNDS
    s.compare(lens=[100, 64, 0])
    full = Step(12, [128, 40], 4, 2, 16)
    full.call(ctx, kv_len=torch.tensor([5000, 40], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    with pytest.raises(binding.CpError) as e:
        ctx.poll_status()
    assert e.value.code == binding.CP_ERR_BOUNDS
    full.compare()


def test_replayed_with_growing_lengths_and_shared_workspace(ctx):
    """Two captured calls share one workspace and one stream; lengths grow between replays."""
    a, b = Step(13, [700, 2000, 0, 129], 8, 2, 16, junk=3e38), Step(14, [3000], 4, 1, 32, n_q=2, fp8=True)
    ws = torch.empty(max(x.g_ws.tensor.numel() for x in (a, b)), dtype=torch.uint8, device="cuda")
    for s in (a, b):
        s.call(ctx, ws=ws)                                  # kernels loaded before the capture
    torch.cuda.synchronize()
    stream, graphs = torch.cuda.Stream(), [torch.cuda.CUDAGraph() for _ in range(2)]
    for s, graph in zip((a, b), graphs):
        with torch.cuda.graph(graph, stream=stream):
            s.call(ctx, window=500, sinks=4, stream=stream, ws=ws)
    for lens_a, lens_b in (([700, 2000, 0, 129], [3000]), ([1, 5, 0, 100], [2]), ([650, 1999, 0, 3], [2999])):
        a.kv_len.copy_(torch.tensor(lens_a, dtype=torch.int32))
        b.kv_len.copy_(torch.tensor(lens_b, dtype=torch.int32))
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            for _ in range(3):
                graphs[0].replay()
                graphs[1].replay()
        torch.cuda.synchronize()
        a.compare(500, 4, lens=lens_a)
        b.compare(500, 4, lens=lens_b)


@pytest.mark.parametrize("fill", [0x00, 0x01, 0x5A, 0xFF])
def test_any_workspace_contents(ctx, fill):
    """The workspace needs no initial state, and calls of other shapes and contexts may have left theirs."""
    other = binding.Context(0)
    steps = [Step(28, [9000, 2000, 129], 8, 2, 16, junk=3e38), Step(29, [30000], 2, 1, 64, n_q=3), Step(30, [7000, 10], 16, 1, 32, fp8=True)]
    ws = torch.full((max(s.g_ws.tensor.numel() for s in steps),), fill, dtype=torch.uint8, device="cuda")
    for i in range(9):
        s = steps[(i * 2) % 3]
        s.g_out.tensor.fill_(float("nan"))
        s.call(ctx if i % 2 else other, ws=ws)
        torch.cuda.synchronize()
        s.compare()
    other.close()


def test_two_streams_with_their_own_workspaces(ctx):
    steps = [Step(15 + i, [5000, 300, 40 + i], 8, 2, 16) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in steps]
    torch.cuda.synchronize()
    for _ in range(20):
        for s, st in zip(steps, streams):
            s.call(ctx, stream=st)
    torch.cuda.synchronize()
    for s in steps:
        s.compare()


def test_fp8_scales_of_zero_and_below(ctx):
    """Bytes stand for scale * e4m3 whatever the scale: a head of zeros, and a negative one."""
    s = Step(24, [700, 5, 0, 129], 12, 3, 16, n_q=2, fp8=True)
    s.kv.k_scale[0], s.kv.v_scale[0] = 0.0, 0.0
    s.kv.k_scale[1], s.kv.v_scale[1] = -s.kv.k_scale[1], -s.kv.v_scale[1]
    s.check(ctx)
    s.check(ctx, 100, 3)


@pytest.mark.parametrize("size", [2.0 ** -60, 2.0 ** -20, 2.0 ** 30])
def test_fp8_queries_of_any_size(ctx, size):
    s = Step(25, [300, 17], 8, 2, 16, fp8=True, scale=SCALE / size)
    s.q.mul_(size)
    s.q[0, 0, 3] = 0
    s.check(ctx)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_query_that_is_no_number_stays_in_its_row(ctx, fp8, bad):
    s = Step(26, [300, 17], 8, 2, 16, n_q=2, fp8=fp8)
    s.q[0, 1, 3, 5] = bad
    out, lse = s.run(ctx)
    assert bool(torch.isnan(out[0, 1, 3]).all())
    s.q[0, 1, 3, 5] = 0
    keep = torch.ones(2, 2, 8, dtype=torch.bool, device="cuda")
    keep[0, 1, 3] = False
    first = out.clone()
    o2, _ = s.run(ctx)
    assert torch.equal(first[keep], o2[keep])


def test_fp8_queries_with_a_wide_range(ctx):
    """Elements from 2^-30 to 1 of a row: what fp16 drops below 2^-24 of the largest is far below the bound."""
    s = Step(27, [500], 8, 2, 16, fp8=True)
    s.q.mul_(torch.exp2(-torch.arange(D, device="cuda") / 4.3).to(torch.bfloat16))
    s.check(ctx)


def test_same_inputs_same_bits(ctx):
    s = Step(20, [9000, 300, 2222], 8, 2, 16)
    out, lse = (x.clone() for x in s.run(ctx))
    for _ in range(5):
        o2, l2 = s.run(ctx)
        assert torch.equal(out, o2) and torch.equal(lse, l2)


def test_partials_over_two_caches_merge(ctx):
    """Keys split over two caches (as two ranks would hold them): cp_merge joins the two calls' results."""
    s = Step(21, [900], 8, 2, 16)
    k, v = s.kv.keys_values(0, 900)
    outs, lses = [], []
    for lo, hi in ((0, 400), (400, 900)):
        half = Step(22, [hi - lo], 8, 2, 16)
        ids, slot = half.kv.where(0, torch.arange(hi - lo, device="cuda"))
        half.kv.k[ids, slot], half.kv.v[ids, slot] = k[lo:hi].to(torch.bfloat16), v[lo:hi].to(torch.bfloat16)
        half.q.copy_(s.q)
        o, l = half.run(ctx)
        outs.append(o.float().reshape(1, 8, D).clone())
        lses.append(l.clone())
    out, lse = torch.empty(1, 8, D, device="cuda"), torch.empty(8, 1, device="cuda")
    binding.cp_merge(ctx, torch.stack(outs), torch.stack(lses), out, lse)
    ref = attention64(s.q[0].double(), k, v, torch.tensor([899], device="cuda"), FULL, 0, SCALE)
    check_attention(out, lse, ref, "merged")


def test_empty_batch_and_binding_refusals(ctx):
    s = Step(23, [100, 40], 4, 2, 16)
    binding.cp_decode_attn(ctx, s.q[:0], s.cache, s.kv.table[:0], s.kv_len[:0], FULL, 0, SCALE, s.g_out.tensor[:0], s.g_lse.tensor[:, :0].contiguous(), s.g_ws.tensor)
    good = dict(q=s.q, page_table=s.kv.table, kv_len=s.kv_len, out=s.g_out.tensor, lse=s.g_lse.tensor)
    for kw in (dict(q=s.q.float()), dict(q=s.q.transpose(1, 2)), dict(page_table=s.kv.table[:1]), dict(kv_len=s.kv_len.long()), dict(kv_len=s.kv_len.cpu()),
               dict(out=s.g_out.tensor[:1]), dict(lse=s.g_lse.tensor.T)):
        a = good | kw
        with pytest.raises(ValueError):
            binding.cp_decode_attn(ctx, a["q"], s.cache, a["page_table"], a["kv_len"], FULL, 0, SCALE, a["out"], a["lse"], s.g_ws.tensor)
    with pytest.raises(ValueError):
        binding.cp_decode_attn_fp8(ctx, s.q, s.cache, s.kv.table, s.kv_len, FULL, 0, SCALE, s.g_out.tensor, s.g_lse.tensor, s.g_ws.tensor)
    with pytest.raises(binding.CpError) as e:
        s.call(ctx, ws=s.g_ws.tensor[:1024])
    assert e.value.code == binding.CP_ERR_WORKSPACE


@pytest.mark.parametrize("fp8,Hkv", [(False, 2), (True, 2), (True, 1)])
@pytest.mark.parametrize("G,n_q", [(1, 2), (4, 3), (8, 4), (8, 9)])
def test_values_that_are_no_numbers_stay_out_of_rows_that_do_not_see_them(ctx, fp8, Hkv, G, n_q):
    """Draft tokens whose V is infinite or NaN, and one at the edge of the windows: rows that do not see the key keep their bits, the others
    have the odd element and, in the others, what the formula gives."""
    window, lens = 200, [413, 40, 16, n_q]
    s = Step(28, lens, G * Hkv, Hkv, 16, n_q=n_q, fp8=fp8)
    bad = {}                                               # (request, key) -> dim
    for b, n in enumerate(lens):
        for i in range(1, n_q):
            bad[b, n - i] = (37 * i + 11 * b) % D
        if n > window + n_q:
            bad[b, n - n_q + 1 - window] = 126             # in the first row's window only
    def put(value):
        for i, ((b, t), dim) in enumerate(bad.items()):
            page, slot = s.kv.where(b, torch.tensor(t, device="cuda"))
            s.kv.v[page, slot, i % Hkv, dim] = value(i)
    put(lambda i: 0)
    clean, clean_lse = (x.clone() for x in s.run(ctx, window))
    s.compare(window)
    put(lambda i: (0x7F, 0xFF)[i % 2] if fp8 else (float("inf"), float("nan"), -float("inf"))[i % 3])
    out, lse = (x.clone() for x in s.run(ctx, window))
    assert torch.equal(lse, clean_lse)
    odd = torch.zeros(out.shape, dtype=torch.bool, device="cuda")
    sees = torch.zeros(out.shape, dtype=torch.bool, device="cuda")
    for i, ((b, t), dim) in enumerate(bad.items()):
        p = lens[b] - n_q + torch.arange(n_q, device="cuda")
        rows = (t <= p) & (p - t < window)
        heads = slice(i % Hkv * G, (i % Hkv + 1) * G)
        odd[b, rows, heads, dim] = True
        sees[b, rows, heads] = True
    assert bool((~torch.isfinite(out) == odd).all())
    assert torch.equal(out[~sees], clean[~sees])
    s.g_out.tensor.copy_(torch.where(odd, clean, out))     # the finite elements, against the formula
    put(lambda i: 0)
    s.compare(window)


@pytest.mark.parametrize("fp8", [False, True])
def test_keys_that_are_no_numbers_stay_out_of_rows_that_do_not_see_them(ctx, fp8):
    window, lens, n_q = 200, [413, 40, 3], 3
    s = Step(29, lens, 8, 2, 16, n_q=n_q, fp8=fp8)
    clean, clean_lse = (x.clone() for x in s.run(ctx, window))
    sees = torch.zeros(clean.shape, dtype=torch.bool, device="cuda")
    for b, n in enumerate(lens):
        for t in [n - 1] + ([n - n_q + 1 - window] if n > 300 else []):
            page, slot = s.kv.where(b, torch.tensor(t, device="cuda"))
            s.kv.k[page, slot, 1, 5] = 0x7F if fp8 else float("nan")
            p = n - n_q + torch.arange(n_q, device="cuda")
            sees[b, (t <= p) & (p - t < window), 4:] = True
    out, lse = s.run(ctx, window)
    assert bool((torch.isnan(out) == sees).all())
    rows = sees[..., 0].permute(2, 0, 1).reshape(8, -1)
    assert torch.equal(out[~sees], clean[~sees]) and torch.equal(lse[~rows], clean_lse[~rows])


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("n_q", [1, 5])
def test_output_over_the_queries(ctx, fp8, n_q):
    s = Step(30, [9000, 300, 2222, 0] + [200] * 60, 16, 2, 32, n_q=n_q, fp8=fp8)
    out, lse = (x.clone() for x in s.run(ctx))
    keep = s.q.clone()
    for _ in range(3):
        s.q.copy_(keep)
        f = binding.cp_decode_attn_fp8 if fp8 else binding.cp_decode_attn
        f(ctx, s.q, s.cache, s.kv.table, s.kv_len, FULL, 0, SCALE, s.q, s.g_lse.tensor, s.g_ws.tensor)
        torch.cuda.synchronize()
        assert torch.equal(s.q, out) and torch.equal(s.g_lse.tensor, lse)
    ctx.poll_status()
