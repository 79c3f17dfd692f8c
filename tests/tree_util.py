"""Helpers of the tests of drafted trees and 4-bit caches: paged sequences of every kind of cache with junk in the slots that hold no token, the 4-bit
format, trees, and the plain definitions in 64 bits."""
import math
import random

import torch

from paper_2609_04774_b200 import binding
from tests.serving_util import D, e4m3_codes, generator, normal

FULL = binding.CP_NO_WINDOW
MAGNITUDES = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
# a softmax weight's rounding: bf16 for bf16 and 4-bit caches, fp16 for E4M3 ones (2^-16 more: weights below 2^-14 of the largest are subnormals; with many
# rows, where a weight's reference may be 2^8 off, the bound of bf16 is used)
WEIGHT_EPS = {"bf16": 2.0 ** -8, "mx4": 2.0 ** -8, "fp8": 2.0 ** -11 + 2.0 ** -16}


def mx4_quantise(x):
    """[.., Hkv, 128] in 64 bits -> token rows [.., Hkv * 68] uint8 from the definition: every code by its distance to the value."""
    x = x.double()
    lead, Hkv = x.shape[:-2], x.shape[-2]
    y = x.reshape(*lead, Hkv, 4, 32)
    top = y.abs().amax(-1, keepdim=True)
    odd = ~torch.isfinite(y).all(-1, keepdim=True)
    e = torch.where(top > 0, torch.frexp(torch.where(odd, 1.0, top))[1].double() - 3, torch.tensor(-127.0, dtype=torch.float64, device=x.device)).clamp(min=-127)
    z = torch.where(odd, 0.0, y.abs()) * torch.exp2(-e)
    d = (z.clamp(max=6.0)[..., None] - MAGNITUDES.to(x.device)).abs()
    near = d <= d.amin(-1, keepdim=True)
    code = torch.where(near[..., 0::2].any(-1), 2 * near[..., 0::2].int().argmax(-1), 2 * near[..., 1::2].int().argmax(-1) + 1)      # a tie: the even code
    code = (code + 8 * torch.signbit(y)).reshape(*lead, Hkv * 64, 2)
    exps = torch.where(odd, 255, e.int() + 127).reshape(*lead, Hkv * 4)
    return torch.cat([(code[..., 0] + 16 * code[..., 1]).to(torch.uint8), exps.to(torch.uint8)], -1)


def mx4_values(rows, Hkv):
    """Token rows [.., bytes] -> [.., Hkv, 128] in 64 bits; blocks with an exponent byte of 255 are NaN."""
    m = MAGNITUDES.to(rows.device)
    value = torch.cat([m, -m])
    c = rows[..., :Hkv * 64].long()
    x = value[torch.stack([c & 15, c >> 4], -1)].reshape(*rows.shape[:-1], Hkv, 4, 32)
    e = rows[..., Hkv * 64:Hkv * 68].reshape(*rows.shape[:-1], Hkv, 4, 1).double()
    return torch.where(e == 255, math.nan, x * torch.exp2(e - 127)).reshape(*rows.shape[:-1], Hkv, D)


class Cache:
    """Sequences of the given lengths in a shuffled pool of one kind ("bf16", "fp8", "mx4"): table [B, width] (-1 behind a sequence's pages).  Slots
    that hold no token are NaN."""

    def __init__(self, seed, lens, Hkv, page, kind, width=None, spare=3, pad=0):
        g = generator(seed)
        self.lens, self.page, self.Hkv, self.kind = list(lens), page, Hkv, kind
        counts = [-(-n // page) for n in lens]
        # 4-bit kernels take several heads a unit unless the table is narrow: with an even number of heads it is wide here, by default
        width = width or max(1, max(counts), 65536 // page if kind == "mx4" and Hkv % 2 == 0 else 0)
        pool = sum(counts) + spare
        ids = torch.randperm(pool, generator=g, device="cuda").to(torch.int32)
        self.table = torch.full((len(lens), width), -1, dtype=torch.int32, device="cuda")
        at = 0
        for b, c in enumerate(counts):
            self.table[b, :c] = ids[at:at + c]
            at += c
        used = torch.zeros(pool, page, dtype=torch.bool, device="cuda")
        for b, n in enumerate(lens):
            t = torch.arange(n, device="cuda")
            used[self.table[b, t // page].long(), t % page] = True
        x = [normal(g, pool, page, Hkv, D) for _ in range(2)]
        if kind == "bf16":
            # pad: room between heads' rows, so that strides are not those of a dense pool
            self.pools = [torch.full((pool, page, Hkv, D + pad), math.nan, dtype=torch.bfloat16, device="cuda")[..., :D] for _ in x]
            for p, y in zip(self.pools, x):
                p[used] = y[used]
        elif kind == "fp8":
            self.pools = [torch.full((pool, page, Hkv, D + pad), 0x7F, dtype=torch.uint8, device="cuda")[..., :D] for _ in x]
            for p in self.pools:
                p[used] = e4m3_codes(g, pool, page, Hkv, D)[used]
            self.k_scale, self.v_scale = ((torch.rand(Hkv, generator=g, device="cuda") + 0.5) / 70.0 for _ in range(2))
        else:
            rows = binding.mx4_token_bytes(Hkv)
            self.pools = [torch.full((pool, page, rows + pad), 0xFF, dtype=torch.uint8, device="cuda")[..., :rows] for _ in x]
            for p, y in zip(self.pools, x):
                p[..., :Hkv * 68][used] = mx4_quantise(y)[used]
        self.k, self.v = self.pools
        self.describe()

    def describe(self):
        if self.kind == "bf16":
            self.cache = binding.make_cache(self.k, self.v)
        elif self.kind == "fp8":
            self.cache = binding.make_cache_fp8(self.k, self.v, self.k_scale, self.v_scale)
        else:
            self.cache = binding.make_cache_mx4(self.k, self.v, self.Hkv)

    def where(self, b, t):
        return self.table[b, t // self.page].long(), t % self.page

    def values(self, b, n):
        """K and V [n, Hkv, D] of sequence b in 64 bits."""
        ids, slot = self.where(b, torch.arange(n, device="cuda"))
        outside = (ids < 0) | (ids >= self.k.shape[0])                 # reads as zeros
        gone, ids = outside[:, None, None], ids.masked_fill(outside, 0)
        k, v = self.k[ids, slot], self.v[ids, slot]
        if self.kind == "fp8":
            k, v = k.view(torch.float8_e4m3fn).double() * self.k_scale.double()[:, None], v.view(torch.float8_e4m3fn).double() * self.v_scale.double()[:, None]
        elif self.kind == "mx4":
            k, v = mx4_values(k, self.Hkv), mx4_values(v, self.Hkv)
        return torch.where(gone, 0.0, k.double()), torch.where(gone, 0.0, v.double())


def random_tree(rng, n):
    """Parents of n drafted tokens: any earlier token, or the sequence."""
    return [rng.randrange(-1, t) if rng.random() < 0.9 else t - 1 for t in range(n)]


def masks_of(parent):
    m = []
    for t, p in enumerate(parent):
        m.append((m[p] if p >= 0 else 0) | 1 << t)
    return m


def as_i64(masks):
    return [m - (1 << 64) if m >= 1 << 63 else m for m in masks]


def tree_seen(base, masks, window, sinks):
    """[rows, base + rows] of a tree's masks (any bits): what each row sees, from the definition."""
    m = len(masks)
    inside = (1 << m) - 1
    pos = [base + bin(x & inside).count("1") - 1 for x in masks]
    seen = torch.zeros(m, base + m, dtype=torch.bool)
    j = torch.arange(base)
    for t in range(m):
        seen[t, :base] = (pos[t] - j < window) | (j < sinks)
        for u in range(m):
            seen[t, base + u] = bool(masks[t] >> u & 1) and (pos[t] - pos[u] < window or pos[u] < sinks)
    return seen.cuda()


def attention64_seen(q, k, v, seen, scale):
    """q [r, Hq, D], k / v [n, Hkv, D] in 64 bits, seen [r, n] -> O, LSE [Hq, r], A = sum p |v|; what a row does not see takes no part in it."""
    r, Hq, _ = q.shape
    G = Hq // k.shape[1]
    o, a = torch.zeros(r, Hq, D, dtype=torch.float64, device=q.device), torch.zeros(r, Hq, D, dtype=torch.float64, device=q.device)
    lse = torch.full((Hq, r), -math.inf, dtype=torch.float64, device=q.device)
    finite = bool(torch.isfinite(v).all())
    for h in range(Hq):
        s = ((q[:, h] @ k[:, h // G].T) * scale).masked_fill(~seen, -math.inf)
        top = s.amax(1, keepdim=True) if s.shape[1] else torch.full((r, 1), -math.inf, dtype=torch.float64, device=q.device)
        e = torch.exp(s - top.masked_fill(torch.isneginf(top), 0.0)).masked_fill(~seen, 0.0)
        l = e.sum(1, keepdim=True)
        w = e / l.masked_fill(l == 0, 1.0)
        lse[h] = (top + torch.log(l))[:, 0]
        vv = v[:, h // G]
        if finite:
            o[:, h], a[:, h] = w @ vv, w @ vv.abs()
        else:
            for t in range(r):
                o[t, h], a[t, h] = w[t, seen[t]] @ vv[seen[t]], w[t, seen[t]] @ vv[seen[t]].abs()
    return o, lse, a


def check_rows(out, lse, ref, what, weight_eps, lse_tol=2e-4):
    """check_attention's bound (serving_util), where the reference is finite; elsewhere infinities and NaN must be where it has them."""
    ro, rl, ra = ref
    fine = torch.isfinite(ro)
    assert bool((torch.isfinite(out) == fine).all()), (what, "infinities or NaN elsewhere")
    assert bool((torch.isnan(out) == torch.isnan(ro)).all()), (what, "NaN elsewhere")
    d = (out.double() - ro).abs()[fine]
    excess = (d - (weight_eps + 2.0 ** -8 + 2.0 ** -10) * ra[fine]).max().item() if d.numel() else 0.0
    assert excess <= 0, (what, "O beyond the bound by", excess, "largest error", d.max().item())
    plain = torch.isfinite(rl)
    assert bool((lse[~plain].double().nan_to_num(7e77) == rl[~plain].nan_to_num(7e77)).all()), (what, "lse of rows without keys or with NaN")
    dl = (lse.double() - rl).abs()[plain]
    assert dl.numel() == 0 or dl.max().item() <= lse_tol, (what, "lse", dl.max().item())


class TreeStep:
    """A call of cp_tree_attn*: trees[b] are the masks of sequence b's drafted tokens, behind bases[b] tokens."""

    def __init__(self, seed, bases, trees, Hq, Hkv, page, kind, n_q=None, scale=D ** -0.5, width=None, pad=0):
        self.bases, self.trees, self.Hq, self.Hkv, self.kind, self.scale = list(bases), [list(t) for t in trees], Hq, Hkv, kind, scale
        B = len(self.bases)
        self.n_q = n_q or max(len(t) for t in trees)
        self.kv = Cache(seed, [b + len(t) for b, t in zip(bases, trees)], Hkv, page, kind, width=width, pad=pad)
        self.q = normal(generator(seed + 1), B, self.n_q, Hq, D)
        self.kv_len = torch.tensor(self.kv.lens, dtype=torch.int32, device="cuda")
        self.tree_len = torch.tensor([len(t) for t in trees], dtype=torch.int32, device="cuda")
        self.mask = torch.tensor([as_i64(t) + [-1] * (self.n_q - len(t)) for t in trees], dtype=torch.int64, device="cuda")      # behind the tree: ignored
        self.out = torch.full((B, self.n_q, Hq, D), math.nan, dtype=torch.bfloat16, device="cuda")
        self.lse = torch.full((Hq, B * self.n_q), math.nan, dtype=torch.float32, device="cuda")
        self.ws = torch.full((binding.cp_workspace_bytes_tree(B, self.n_q, Hq, Hkv),), 0xFF, dtype=torch.uint8, device="cuda")

    def call(self, ctx, window=FULL, sinks=0, stream=None):
        f = {"bf16": binding.cp_tree_attn, "fp8": binding.cp_tree_attn_fp8, "mx4": binding.cp_tree_attn_mx4}[self.kind]
        f(ctx, self.q, self.kv.cache, self.kv.table, self.kv_len, self.tree_len, self.mask, window, sinks, self.scale, self.out, self.lse, self.ws, stream=stream)

    def compare(self, window=FULL, sinks=0, rows=None):
        for b, (base, tree) in enumerate(zip(self.bases, self.trees)):
            if rows is not None and b not in rows:
                continue
            m = len(tree)
            k, v = self.kv.values(b, base + m)
            ref = attention64_seen(self.q[b, :m].double(), k, v, tree_seen(base, tree, window, sinks), self.scale)
            lse = self.lse.view(self.Hq, -1, self.n_q)[:, b]
            wide = self.n_q * self.Hq // self.Hkv > 32
            check_rows(self.out[b, :m], lse[:, :m], ref, (b, base, m, window, sinks), 2.0 ** -8 if wide else WEIGHT_EPS[self.kind])
            assert bool((self.out[b, m:] == 0).all()) and bool(torch.isneginf(lse[:, m:]).all()), (b, "rows behind the tree")

    def check(self, ctx, window=FULL, sinks=0, rows=None):
        self.call(ctx, window, sinks)
        torch.cuda.synchronize()
        ctx.poll_status()
        self.compare(window, sinks, rows)


def trees(seed, sizes):
    rng = random.Random(seed)
    return [masks_of(random_tree(rng, n)) for n in sizes]
