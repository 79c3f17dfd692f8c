"""Helpers of the serving-operator tests: paged sequences on the device and the plain definition of windowed attention
in 64 bits (torch, every (query, key) pair looked at)."""
import torch

D = 128


def normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32).to(torch.bfloat16)


def generator(seed):
    g = torch.Generator("cuda")
    g.manual_seed(seed)
    return g


def e4m3_codes(g, *shape):
    """Finite E4M3 bytes of normal values spread over the format."""
    x = torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32) * 70.0
    return x.clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)


class Paged:
    """Sequences of the given lengths in a shuffled pool: table [B, width] (-1 behind a sequence's pages), k / v pages.
    bf16 pools hold huge finite values in the slots no token maps to (they must not reach a result)."""

    def __init__(self, g, lens, Hkv, page, fp8=False, width=None, spare=3, junk=3e38):
        self.lens, self.page, self.Hkv, self.fp8 = list(lens), page, Hkv, fp8
        counts = [-(-n // page) for n in lens]
        width = width or max(1, max(counts))
        pool = sum(counts) + spare
        ids = torch.randperm(pool, generator=g, device="cuda").to(torch.int32)
        self.table = torch.full((len(lens), width), -1, dtype=torch.int32, device="cuda")
        at = 0
        for b, c in enumerate(counts):
            self.table[b, :c] = ids[at:at + c]
            at += c
        shape = (pool, page, Hkv, D)
        if fp8:
            self.k, self.v = e4m3_codes(g, *shape), e4m3_codes(g, *shape)
            self.k_scale = (torch.rand(Hkv, generator=g, device="cuda") + 0.5) / 70.0
            self.v_scale = (torch.rand(Hkv, generator=g, device="cuda") + 0.5) / 70.0
        else:
            self.k, self.v = torch.full(shape, junk, dtype=torch.bfloat16, device="cuda"), torch.full(shape, -junk, dtype=torch.bfloat16, device="cuda")
            for b, n in enumerate(lens):
                ids_b, slot = self.where(b, torch.arange(n, device="cuda"))
                self.k[ids_b, slot] = normal(g, n, Hkv, D)
                self.v[ids_b, slot] = normal(g, n, Hkv, D)

    def where(self, b, t):
        return self.table[b, t // self.page].long(), t % self.page

    def keys_values(self, b, n):
        """K and V [n, Hkv, D] of sequence b in 64 bits."""
        ids, slot = self.where(b, torch.arange(n, device="cuda"))
        if self.fp8:
            return (self.k.view(torch.float8_e4m3fn)[ids, slot].double() * self.k_scale.double()[:, None],
                    self.v.view(torch.float8_e4m3fn)[ids, slot].double() * self.v_scale.double()[:, None])
        return self.k[ids, slot].double(), self.v[ids, slot].double()


def visible(p, j, window, sinks):
    return (j[None, :] <= p[:, None]) & ((p[:, None] - j[None, :] < window) | (j[None, :] < sinks))


def attention64(q, k, v, p, window, sinks, scale):
    """q [r, Hq, D], k / v [n, Hkv, D] in 64 bits, p [r] positions -> O [r, Hq, D], LSE [Hq, r], A = sum p |v| [r, Hq, D].
    A row that sees nothing gives zeros and -inf."""
    r, Hq, _ = q.shape
    G = Hq // k.shape[1]
    seen = visible(p, torch.arange(k.shape[0], device=q.device), window, sinks)
    o, a = torch.zeros(r, Hq, D, dtype=torch.float64, device=q.device), torch.zeros(r, Hq, D, dtype=torch.float64, device=q.device)
    lse = torch.full((Hq, r), -float("inf"), dtype=torch.float64, device=q.device)
    some = seen.any(1)
    if k.shape[0] == 0 or not bool(some.any()):
        return o, lse, a
    for h in range(Hq):
        s = (q[:, h] @ k[:, h // G].T) * scale
        s = s.masked_fill(~seen, -float("inf"))[some]
        m = s.amax(1, keepdim=True)
        e = torch.exp(s - m)
        l = e.sum(1, keepdim=True)
        o[some, h] = (e @ v[:, h // G]) / l
        a[some, h] = (e @ v[:, h // G].abs()) / l
        lse[h, some] = (m + torch.log(l))[:, 0]
    return o, lse, a


def attention64_blocks(q, k, v, p, window, sinks, scale, block=512):
    parts = [attention64(q[i:i + block], k, v, p[i:i + block], window, sinks, scale) for i in range(0, q.shape[0], block)]
    return torch.cat([x[0] for x in parts]), torch.cat([x[1] for x in parts], 1), torch.cat([x[2] for x in parts])


def check_attention(out, lse, ref, what, weight_eps=2.0 ** -8, lse_tol=2e-4):
    """Element by element: a softmax weight rounded to the format of the P*V product is off by at most weight_eps of itself, so O by
    at most weight_eps * A; the bf16 output by at most 2^-8 |O| <= 2^-8 A; 2^-10 A more covers the fp32 arithmetic (a score is a sum
    of 128 products, |q k| scale adds up to about 7 for normal inputs, so its fp32 error is at most 128 * 2^-23 * 7 = 1.1e-4, and
    a weight's relative error the same) and the products of these.  LSE: the score error twice over (the scores' and the sum's)."""
    ro, rl, ra = ref
    d = (out.double() - ro).abs()
    assert bool(torch.isfinite(out).all()), what
    excess = (d - (weight_eps + 2.0 ** -8 + 2.0 ** -10) * ra).max().item()
    assert excess <= 0, (what, "O beyond the bound by", excess, "largest error", d.max().item())
    none = torch.isneginf(rl)
    assert bool((torch.isneginf(lse) == none).all()), (what, "rows that see nothing")
    dl = (lse.double() - rl).abs()[~none]
    assert dl.numel() == 0 or dl.max().item() <= lse_tol, (what, "lse", dl.max().item())
