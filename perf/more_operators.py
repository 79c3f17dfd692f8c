"""Operators for drafted trees and for 4-bit caches, as cases with plain forms.

Four groups of calls that belong together in a serving loop:

  tree     attention of a tree of drafted tokens over a paged cache (bf16, E4M3 or 4-bit): every token sees the sequence and
           its own ancestors, with or without a window; lengths, trees and page tables live on the device
  commit   the step around it: masks, positions and slots from the parents of the drafted tokens, and, once a path has been accepted,
           its keys and values moved to consecutive slots in every layer
  prompt   a chunk of a prompt appended to a 4-bit cache (rotated and quantised on the way), and the rows of the whole
           context read back in bf16, as the prefill attention over such a cache takes them
  decode   attention of one or a few new tokens per request over a 4-bit cache

Logical token t of a sequence lives in page table[t // page], slot t % page.  Row t of a tree of m tokens behind `base` tokens sits in
slot base + t, at position base + depth(t); it sees key j if j is a token of the sequence, itself or one of its ancestors, and
(its position - position of j < window or position of j < sinks); window 0 in a case means no window.

4-bit cache: blocks of 32 elements with an exponent byte e and 32 codes of 1-2-1 bits (0, .5, 1, 1.5, 2, 3, 4, 6 and their negatives), which stand
for code * 2^(e - 127); e - 127 = floor(log2(largest magnitude)) - 2.  A token's row: Hkv * 64 bytes of codes, then Hkv * 4 exponents.
"""
import math
import random

import torch

own = False

D = 128
NO_WINDOW = 0x7FFFFFFF


# ----------------------------------------------------------------------------------------------------------------------
# Cases
# ----------------------------------------------------------------------------------------------------------------------

def listed():
    return [
        # one user with a small tree: latency counts
        dict(name="tree_single", op="tree", B=1, n_q=16, ragged=False, len_lo=4000, len_hi=4000, window=0, sinks=0, Hq=32, Hkv=8, page=64, kind="bf16", mix=1),
        # a serving batch of ragged lengths, every request with a tree of 32 tokens
        dict(name="tree_batch", op="tree", B=32, n_q=32, ragged=False, len_lo=257, len_hi=16384, window=0, sinks=0, Hq=32, Hkv=8, page=64, kind="bf16", mix=2),
        # few long contexts with large trees: as much arithmetic as memory traffic
        dict(name="tree_long", op="tree", B=4, n_q=64, ragged=False, len_lo=100000, len_hi=131072, window=0, sinks=0, Hq=32, Hkv=4, page=64, kind="bf16", mix=3),
        # long conversations of a model with a window, E4M3 cache, trees of different sizes
        dict(name="tree_window_fp8", op="tree", B=64, n_q=12, ragged=True, len_lo=1000, len_hi=65536, window=4096, sinks=4, Hq=64, Hkv=8, page=32, kind="fp8", mix=4),
        # small trees over a 4-bit cache
        dict(name="tree_mx4", op="tree", B=48, n_q=7, ragged=True, len_lo=333, len_hi=16384, window=0, sinks=0, Hq=32, Hkv=8, page=64, kind="mx4", mix=5),
        # the bookkeeping of one step of a small batch: latency counts
        dict(name="commit_step", op="commit", B=8, n_q=16, ragged=True, layers=4, len_lo=100, len_hi=2000, Hkv=8, page=64, kind="fp8", mix=6),
        # all layers of a model, a large batch
        dict(name="commit_layers", op="commit", B=64, n_q=64, ragged=True, layers=32, len_lo=100, len_hi=2000, Hkv=8, page=64, kind="bf16", mix=7),
        # a chat turn: a few new tokens behind a cached conversation
        dict(name="prompt_turn", op="prompt", n=37, prefix=700, axes=1, pairs=False, rot=128, Hq=32, Hkv=8, page=64, mix=8),
        # a chunk of a long document (text and images)
        dict(name="prompt_chunk", op="prompt", n=16384, prefix=32768, axes=3, pairs=False, rot=128, Hq=32, Hkv=8, page=64, mix=9),
        # one user, one token: latency counts
        dict(name="decode_single", op="decode", B=1, n_q=1, len_lo=4097, len_hi=4097, window=0, sinks=0, Hq=32, Hkv=8, page=64, mix=10),
        # a serving batch of ragged lengths
        dict(name="decode_batch", op="decode", B=128, n_q=1, len_lo=257, len_hi=16384, window=0, sinks=0, Hq=32, Hkv=8, page=64, mix=11),
        # long contexts of a model with a window, two drafted tokens each
        dict(name="decode_window", op="decode", B=96, n_q=2, len_lo=1000, len_hi=65536, window=8192, sinks=4, Hq=64, Hkv=8, page=32, mix=12),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["tree", "tree", "commit", "prompt", "decode"])
    page = rng.choice([16, 32, 64, 128])
    Hq, Hkv = rng.choice([(32, 8), (32, 4), (16, 16), (8, 8), (64, 8), (5, 1), (16, 2), (12, 6)])
    mix = rng.randrange(1 << 20)
    if op == "tree":
        B, n_q = _log(rng, 1, 64), _log(rng, 1, 64)
        hi = _log(rng, 16, max(32, min(131072, 1600000 // (B * Hkv), 700000000 // (B * n_q * Hq))))
        return dict(op=op, B=B, n_q=n_q, ragged=rng.random() < 0.5, len_lo=max(1, hi // rng.choice([1, 8, 64])), len_hi=hi,
                    window=rng.choice([0, 0, _log(rng, 1, 8192)]), sinks=rng.choice([0, 4, rng.randrange(300)]), Hq=Hq, Hkv=Hkv, page=page,
                    kind=rng.choice(["bf16", "bf16", "fp8", "mx4"]), mix=mix)
    if op == "commit":
        return dict(op=op, B=_log(rng, 1, 64), n_q=_log(rng, 1, 64), ragged=rng.random() < 0.5, layers=rng.randrange(1, 25), len_lo=1, len_hi=_log(rng, 20, 2000),
                    Hkv=min(Hkv, 8), page=page, kind=rng.choice(["bf16", "fp8"]), mix=mix)
    if op == "prompt":
        return dict(op=op, n=_log(rng, 1, 12000), prefix=rng.choice([0, _log(rng, 1, 32768)]), axes=rng.choice([1, 2, 3]), pairs=rng.random() < 0.5,
                    rot=rng.choice([128, 128, 64, 96]), Hq=min(Hq, 32), Hkv=min(Hkv, 8), page=page, mix=mix)
    B = _log(rng, 1, 128)
    hi = _log(rng, 16, min(131072, 500000 * 8 // (B * Hkv)))
    return dict(op=op, B=B, n_q=rng.choice([1, 1, 2, 3]), len_lo=max(1, hi // rng.choice([1, 8, 64])), len_hi=hi, window=rng.choice([0, _log(rng, 1, 8192)]),
                sinks=rng.choice([0, 4, rng.randrange(300)]), Hq=Hq, Hkv=Hkv, page=page, mix=mix)


def _tree(rng, n):
    """Parents of n drafted tokens, level by level as drafting makes them: -1 behind the sequence itself."""
    levels = min(n, rng.randint(2, 8))
    cuts = [0] + sorted(rng.sample(range(1, n), levels - 1)) + [n]
    return [rng.randrange(cuts[i - 1], cuts[i]) if i else -1 for i in range(levels) for _ in range(cuts[i + 1] - cuts[i])]


def _accepted(rng, parent):
    """The last token of an accepted path, -1: none.  Of the paths those whose new slots hold no token of the same path elsewhere, so
    that a pass can be repeated on the same buffers."""
    fine = [-1]
    for a in range(len(parent)):
        path = [a]
        while parent[path[-1]] >= 0:
            path.append(parent[path[-1]])
        path.reverse()
        if all(node == i or node >= len(path) for i, node in enumerate(path)):
            fine.append(a)
    return rng.choice(fine[-max(1, len(fine) // 2):])


def _requests(case):
    """(tokens before the new ones, new tokens, parents of the new ones, accepted) of every request: they belong to the case, not to the seed of the values."""
    rng = random.Random(case["mix"])
    found = []
    for _ in range(case["B"]):
        base = _log(rng, case["len_lo"], case["len_hi"])
        m = rng.randint(1, case["n_q"]) if case.get("ragged") else case["n_q"]
        parent = _tree(rng, m)
        found.append((base, m, parent, _accepted(rng, parent)))
    return found


# ----------------------------------------------------------------------------------------------------------------------
# Inputs
# ----------------------------------------------------------------------------------------------------------------------

def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32).to(torch.bfloat16)


def _codes(g, *shape):
    """E4M3 bytes of normal values spread over the format's range."""
    return (torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32) * 70.0).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _token_bytes(Hkv):
    return -(-Hkv * 68 // 16) * 16


def _blocks(g, pages, page, Hkv):
    """4-bit token rows [pages, page, bytes] of normal values."""
    pool = torch.zeros(pages, page, _token_bytes(Hkv), dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 25) // (page * Hkv * D))
    for p in range(0, pages, step):
        x = torch.randn(min(step, pages - p), page, Hkv, D, generator=g, device="cuda", dtype=torch.float32)
        pool[p:p + step, :, :Hkv * 68] = _quantise(x)
    return pool


def _scatter_pages(g, counts, width, spare):
    """A table [rows, width] whose row r has counts[r] pages, drawn without order from a pool."""
    total = sum(counts)
    ids = torch.randperm(total + spare, generator=g, device="cuda")[:total].to(torch.int32)
    c = torch.tensor(counts, device="cuda")
    at = torch.arange(width, device="cuda")[None, :]
    base = (torch.cumsum(c, 0) - c)[:, None]
    return torch.where(at < c[:, None], ids[(base + at).clamp(max=max(total - 1, 0))], -1).contiguous(), total + spare


def _cache(s, g, kind, pool, page, Hkv):
    if kind == "mx4":
        s["k"], s["v"] = _blocks(g, pool, page, Hkv), _blocks(g, pool, page, Hkv)
    elif kind == "fp8":
        s["k"], s["v"] = _codes(g, pool, page, Hkv, D), _codes(g, pool, page, Hkv, D)
        s["k_scale"] = (torch.rand(Hkv, generator=g, device="cuda") + 0.5) / 70.0
        s["v_scale"] = (torch.rand(Hkv, generator=g, device="cuda") + 0.5) / 70.0
    else:
        s["k"], s["v"] = _normal(g, pool, page, Hkv, D), _normal(g, pool, page, Hkv, D)


def prepare(case, seed):
    g = torch.Generator("cuda")
    g.manual_seed(int(seed) * 7919 + 29)
    s = {"case": case}
    op, page, Hkv = case["op"], case["page"], case["Hkv"]
    if op in ("tree", "decode"):
        reqs = _requests(case)
        B, n_q = case["B"], case["n_q"]
        lens = [base + m for base, m, _, _ in reqs]
        # with a window, the pages wholly behind it (and behind the sinks) have been given back: their entries are -1
        counts = [-(-n // page) for n in lens]
        width = max(counts)
        window = case["window"] or NO_WINDOW
        first = [-(-case["sinks"] // page) for _ in lens]
        last = [max(f, max(0, base + 1 - window) // page) for (base, _, _, _), f in zip(reqs, first)]
        held = [c - max(0, min(b, c) - a) for c, a, b in zip(counts, first, last)]
        dense, pool = _scatter_pages(g, held, width, 3)
        at = torch.arange(width, device="cuda")[None, :]
        a, b, c = (torch.tensor(x, device="cuda")[:, None] for x in (first, last, counts))
        gap = (b.minimum(c) - a).clamp(min=0)
        gone = (at >= a) & (at < a + gap)
        src = torch.where(at < a, at, at - gap).clamp(min=0)
        s["table"] = torch.where(gone | (at >= c), -1, dense.gather(1, src.clamp(max=width - 1))).to(torch.int32).contiguous()
        s["kv_len"] = _i32(lens)
        s["q"] = _normal(g, B, n_q, case["Hq"], D)
        _cache(s, g, case.get("kind", "mx4"), pool, page, Hkv)
        if op == "tree":
            s["tree_len"] = _i32([m for _, m, _, _ in reqs])
            s["mask"] = _ancestors(_i32([p + [-1] * (n_q - m) for _, m, p, _ in reqs]), s["tree_len"])[1]
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(case["Hq"], B * n_q, dtype=torch.float32, device="cuda")
    elif op == "commit":
        reqs = _requests(case)
        B, n_q = case["B"], case["n_q"]
        counts = [-(-(base + m) // page) for base, m, _, _ in reqs]
        s["table"], pool = _scatter_pages(g, counts, max(counts), 3)
        s["kv_len"], s["tree_len"] = _i32([base + m for base, m, _, _ in reqs]), _i32([m for _, m, _, _ in reqs])
        s["parent"] = _i32([p + [-1] * (n_q - m) for _, m, p, _ in reqs])
        s["accepted"] = _i32([a for _, _, _, a in reqs])
        shape = (case["layers"], pool, page, Hkv, D)
        s["k"], s["v"] = (_codes(g, *shape), _codes(g, *shape)) if case["kind"] == "fp8" else (_normal(g, *shape), _normal(g, *shape))
        s["new_mask"] = torch.empty(B, n_q, dtype=torch.int64, device="cuda")
        s["positions"] = torch.empty(1, B * n_q, dtype=torch.int32, device="cuda")
        s["seq"], s["slot"] = (torch.empty(B * n_q, dtype=torch.int32, device="cuda") for _ in range(2))
        s["path"] = torch.empty(B, n_q, dtype=torch.int32, device="cuda")
    else:
        n, prefix = case["n"], case["prefix"]
        rng = random.Random(case["mix"])
        count = -(-(prefix + n) // page)
        s["table"], pool = _scatter_pages(g, [count], count, 2)
        i = torch.arange(n, device="cuda")
        s["seq"], s["slot"] = torch.zeros_like(i, dtype=torch.int32), (prefix + i).to(torch.int32)
        # text positions go far; rows and columns of images stay small and start behind the text
        far = prefix + rng.choice([0, 5000, 100000])
        t = [far + i, far + i // 32 % 48, far + i % 32]
        s["positions"] = torch.stack(t[:case["axes"]]).to(torch.int32).contiguous()
        s["q"] = _normal(g, n, case["Hq"], D)
        s["k_rows"], s["v_rows"] = _normal(g, n, Hkv, D), _normal(g, n, Hkv, D)
        s["q_out"] = torch.empty_like(s["q"])
        _cache(s, g, "mx4", pool, page, Hkv)
        s["k_all"], s["v_all"] = (torch.empty(prefix + n, Hkv, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    return s


# ----------------------------------------------------------------------------------------------------------------------
# The framework's calls
# ----------------------------------------------------------------------------------------------------------------------

_handles = {}


def _binding():
    from paper_2609_04774_b200 import binding
    return binding


def _ctx():
    """One library context for the process, as a server keeps it."""
    if "ctx" not in _handles:
        _handles["ctx"] = _binding().Context(0)
    return _handles["ctx"]


def _kept(s, name, make):
    """What a program makes once for its buffers and keeps: workspaces, cache and pool descriptors."""
    if name not in s:
        s[name] = make()
    return s[name]


def _cache_of(s):
    b, kind = _binding(), s["case"].get("kind", "mx4")
    if kind == "mx4":
        return _kept(s, "cache", lambda: b.make_cache_mx4(s["k"], s["v"], s["case"]["Hkv"]))
    if kind == "fp8":
        return _kept(s, "cache", lambda: b.make_cache_fp8(s["k"], s["v"], s["k_scale"], s["v_scale"]))
    return _kept(s, "cache", lambda: b.make_cache(s["k"], s["v"]))


def _own_tree(s):
    b, c = _binding(), s["case"]
    call = {"bf16": b.cp_tree_attn, "fp8": b.cp_tree_attn_fp8, "mx4": b.cp_tree_attn_mx4}[c["kind"]]
    ws = _kept(s, "ws", lambda: torch.empty(b.cp_workspace_bytes_tree(c["B"], c["n_q"], c["Hq"], c["Hkv"]), dtype=torch.uint8, device="cuda"))
    call(_ctx(), s["q"], _cache_of(s), s["table"], s["kv_len"], s["tree_len"], s["mask"], c["window"] or NO_WINDOW, c["sinks"], D ** -0.5, s["out"], s["lse"], ws)
    return [s["out"], s["lse"]]


def _own_commit(s):
    b = _binding()
    kv_len = s["kv_len"].clone()
    pool = _kept(s, "pool", lambda: b.make_page_pool(s["k"], s["v"]))
    b.cp_tree_plan(_ctx(), s["parent"], s["tree_len"], kv_len, s["new_mask"], s["positions"], s["seq"], s["slot"])
    b.cp_tree_commit(_ctx(), pool, s["table"], kv_len, s["tree_len"], s["parent"], s["accepted"], s["path"])
    return [s["new_mask"], s["positions"], s["seq"], s["slot"], kv_len, s["path"], _values(s["k"]), _values(s["v"])]


def _own_prompt(s):
    b, c = _binding(), s["case"]
    rope = _kept(s, "rope", lambda: b.make_rope(_sections(c), base=_BASE, interleaved=c["pairs"]))
    b.cp_rope_append_mx4(_ctx(), rope, s["q"], s["k_rows"], s["v_rows"], s["positions"], s["seq"], s["slot"], _cache_of(s), s["table"], s["q_out"])
    b.cp_kv_gather_mx4(_ctx(), _cache_of(s), s["table"], 0, c["prefix"] + c["n"], s["k_all"], s["v_all"])
    return [s["q_out"], s["k_all"], s["v_all"]]


def _own_decode(s):
    b, c = _binding(), s["case"]
    ws = _kept(s, "ws", lambda: torch.empty(b.cp_workspace_bytes_decode(c["B"], c["n_q"], c["Hq"], c["Hkv"]), dtype=torch.uint8, device="cuda"))
    b.cp_decode_attn_mx4(_ctx(), s["q"], _cache_of(s), s["table"], s["kv_len"], c["window"] or NO_WINDOW, c["sinks"], D ** -0.5, s["out"], s["lse"], ws)
    return [s["out"], s["lse"]]


# ----------------------------------------------------------------------------------------------------------------------
# Plain forms
# ----------------------------------------------------------------------------------------------------------------------

_BASE = 1000000.0
_MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
_BORDERS = (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)       # between neighbours; a tie goes to the even code


def _sections(c):
    """Rotated pairs of each axis."""
    n = c["rot"] // 2
    if c["axes"] == 1:
        return [n]
    if c["axes"] == 2:
        return [n // 2, n - n // 2]
    return [n // 4, (n - n // 4) // 2, n - n // 4 - (n - n // 4) // 2]


def _values(pool):
    """The values that a pool's bytes stand for, up to the scale of their head."""
    return pool.view(torch.float8_e4m3fn) if pool.dtype == torch.uint8 else pool


def _quantise(x):
    """[.., Hkv, 128] -> 4-bit token rows [.., Hkv * 68]."""
    lead, Hkv = x.shape[:-2], x.shape[-2]
    y = x.reshape(*lead, Hkv, 4, 32)
    top = y.abs().amax(-1, keepdim=True)
    e = torch.frexp(top)[1] - 3                                                             # top = m 2^(e + 3), m in [1/2, 1)
    e = torch.where(top > 0, e, -127).clamp(min=-127)
    z = torch.ldexp(y.abs(), -e)
    index = torch.arange(7, device=x.device)
    border = torch.tensor(_BORDERS, dtype=x.dtype, device=x.device)
    above = torch.where(index % 2 == 0, z[..., None] > border, z[..., None] >= border)      # behind an odd code a tie goes up
    code = above.sum(-1) + 8 * torch.signbit(y)
    code = code.reshape(*lead, Hkv * 64, 2)
    return torch.cat([(code[..., 0] + 16 * code[..., 1]).to(torch.uint8), (e + 127).reshape(*lead, Hkv * 4).to(torch.uint8)], -1)


def _dequantise(rows, Hkv):
    """4-bit token rows [.., bytes] -> [.., Hkv, 128] in 32 bits."""
    m = torch.tensor(_MAGNITUDES, device=rows.device)
    value = torch.cat([m, -m])
    byte = torch.arange(256, device=rows.device)
    pairs = torch.stack([value[byte % 16], value[byte // 16]], -1)
    x = pairs[rows[..., :Hkv * 64].int()].reshape(*rows.shape[:-1], Hkv, 4, 32)
    e = rows[..., Hkv * 64:Hkv * 68].reshape(*rows.shape[:-1], Hkv, 4, 1).int() - 127
    return torch.ldexp(x, e).reshape(*rows.shape[:-1], Hkv, D)


def _ancestors(parent, tree_len):
    """parent [B, n] -> (ancestor or self [B, n, n], the same as bits of 64-bit masks [B, n]); rows behind the tree have none."""
    B, n = parent.shape
    index = torch.arange(n, device=parent.device)
    step = (parent[:, :, None] == index).double() + torch.eye(n, dtype=torch.float64, device=parent.device)
    reach = (torch.linalg.matrix_power(step, n) > 0) & (index < tree_len[:, None])[:, :, None]
    return reach, (reach.long() << index).sum(-1)


def _softmax_product(q, k, v, seen, scale):
    """q [.., r, d], k and v [.., n, d], seen [.., r, n] -> (output, log of the sum); a row that sees nothing gives 0 and -inf."""
    s = (q @ k.transpose(-1, -2)) * scale
    s = s.masked_fill(~seen, -math.inf)
    m = s.amax(-1, keepdim=True)
    e = torch.exp(s - m.masked_fill(m == -math.inf, 0.0))
    l = e.sum(-1, keepdim=True)
    o = (e @ v) / l.masked_fill(l == 0, 1.0)
    return o, (m + torch.log(l)).squeeze(-1)


def _plain_attention(s):
    """Trees, and chains of new tokens as trees in which every token is the parent of the next."""
    c = s["case"]
    B, n_q, Hkv, G, page = c["B"], c["n_q"], c["Hkv"], c["Hq"] // c["Hkv"], c["page"]
    W, S = c["window"] or NO_WINDOW, c["sinks"]
    bit = torch.arange(n_q, device="cuda")
    if c["op"] == "tree":
        m, reach = s["tree_len"].long()[:, None], (s["mask"][:, :, None] >> bit & 1).bool()
    else:
        m, reach = torch.full((B, 1), n_q, device="cuda"), (bit[:, None] >= bit).expand(B, n_q, n_q)
    n = s["kv_len"].long()[:, None]
    base = n - m
    pos = base + reach.sum(-1) - 1                                                          # of the new tokens
    # candidate keys of every request: the sinks, then the last ones
    cap = s["table"].shape[1] * page
    span = min(cap, W + n_q)
    tail = n - span + torch.arange(span, device="cuda")[None, :]
    head = torch.arange(min(S, cap), device="cuda")[None, :].expand(B, -1)
    at = torch.cat([head, tail], 1)
    use = torch.cat([(head < n) & (head < n - span), tail >= 0], 1)
    at = at.clamp(min=0)
    new = (at - base).clamp(0, n_q - 1)
    key_pos = torch.where(at >= base, pos.gather(1, new), at)
    linked = reach.gather(2, new[:, None, :].expand(B, n_q, -1)) | (at < base)[:, None, :]
    seen = use[:, None, :] & linked & ((pos[:, :, None] - key_pos[:, None, :] < W) | (key_pos[:, None, :] < S)) & (bit < m)[:, :, None]
    pages = s["table"].gather(1, (at // page).clamp(max=s["table"].shape[1] - 1)).clamp(min=0).long()
    k, v = (x[pages, at % page] for x in (s["k"], s["v"]))                                  # [B, keys, ..]
    kind = c.get("kind", "mx4")
    if kind == "mx4":
        k, v = _dequantise(k, Hkv), _dequantise(v, Hkv)
    elif kind == "fp8":
        k, v = _values(k).float() * s["k_scale"][:, None], _values(v).float() * s["v_scale"][:, None]
    q = s["q"].float().view(B, n_q, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, n_q * G, D)
    rows = seen[:, None, :, None, :].expand(B, 1, n_q, G, at.shape[1]).reshape(B, 1, n_q * G, at.shape[1])
    o, l = _softmax_product(q, k.permute(0, 2, 1, 3).float(), v.permute(0, 2, 1, 3).float(), rows, D ** -0.5)
    s["out"].copy_(o.view(B, Hkv, n_q, G, D).permute(0, 2, 1, 3, 4).reshape(B, n_q, c["Hq"], D))
    s["lse"].copy_(l.view(B, Hkv, n_q, G).permute(1, 3, 0, 2).reshape(c["Hq"], B * n_q))
    return [s["out"], s["lse"]]


def _plain_commit(s):
    page, parent, tree_len = s["case"]["page"], s["parent"], s["tree_len"]
    B, n_q = parent.shape
    reach, mask = _ancestors(parent, tree_len)
    inside = torch.arange(n_q, device="cuda") < tree_len[:, None]
    base = (s["kv_len"] - tree_len)[:, None]
    index = torch.arange(n_q, device="cuda", dtype=torch.int32)
    positions = torch.where(inside, base + reach.sum(-1) - 1, 0).to(torch.int32).view(1, -1)
    seq = torch.where(inside, torch.arange(B, device="cuda")[:, None], -1).to(torch.int32).view(-1)
    slot = torch.where(inside, base + index, 0).to(torch.int32).view(-1)
    # the accepted path: node number i of it moves to slot base + i
    a = s["accepted"].long()
    on = reach[torch.arange(B, device="cuda"), a.clamp(min=0)] & (a >= 0)[:, None]
    b, node = torch.nonzero(on, as_tuple=True)
    i = (torch.cumsum(on, 1) - 1)[b, node]
    path = torch.full((B, n_q), -1, dtype=torch.int32, device="cuda")
    path[b, i] = node.to(torch.int32)
    src, dst = base[b, 0] + node, base[b, 0] + i
    where = lambda t: (s["table"][b, t // page].long(), t % page)  # noqa: E731
    (p_src, t_src), (p_dst, t_dst) = where(src), where(dst)
    s["k"][:, p_dst, t_dst] = s["k"][:, p_src, t_src]
    s["v"][:, p_dst, t_dst] = s["v"][:, p_src, t_src]
    return [mask, positions, seq, slot, (base[:, 0] + on.sum(1)).to(torch.int32), path, _values(s["k"]), _values(s["v"])]


def _plain_prompt(s):
    c = s["case"]
    pairs = c["rot"] // 2
    axis = torch.repeat_interleave(torch.arange(c["axes"], device="cuda"), torch.tensor(_sections(c), device="cuda"), output_size=pairs)
    freq = torch.pow(torch.tensor(_BASE, dtype=torch.float64, device="cuda"), -torch.arange(pairs, dtype=torch.float64, device="cuda") / pairs)
    angle = s["positions"].double()[axis].T * freq
    cos, sin = torch.cos(angle)[:, None], torch.sin(angle)[:, None]

    def rotate(x):                                       # in 64 bits: the codes of values next to a border depend on the last bits
        x = x.double()
        a, b = (x[..., 0:2 * pairs:2], x[..., 1:2 * pairs:2]) if c["pairs"] else (x[..., :pairs], x[..., pairs:2 * pairs])
        u, w = a * cos - b * sin, b * cos + a * sin
        turned = torch.stack([u, w], -1).flatten(-2) if c["pairs"] else torch.cat([u, w], -1)
        return torch.cat([turned, x[..., 2 * pairs:]], -1)

    s["q_out"].copy_(rotate(s["q"]))
    used = c["Hkv"] * 68
    where = (s["table"][0, s["slot"].long() // c["page"]].long(), s["slot"].long() % c["page"])
    s["k"][..., :used][where] = _quantise(rotate(s["k_rows"]))
    s["v"][..., :used][where] = _quantise(s["v_rows"].float())
    t = torch.arange(c["prefix"] + c["n"], device="cuda")
    where = (s["table"][0, t // c["page"]].long(), t % c["page"])
    s["k_all"].copy_(_dequantise(s["k"][where], c["Hkv"]))
    s["v_all"].copy_(_dequantise(s["v"][where], c["Hkv"]))
    return [s["q_out"], s["k_all"], s["v_all"]]


_OWN = {"tree": _own_tree, "commit": _own_commit, "prompt": _own_prompt, "decode": _own_decode}
_PLAIN = {"tree": _plain_attention, "commit": _plain_commit, "prompt": _plain_prompt, "decode": _plain_attention}


def run(state):
    op = state["case"]["op"]
    if own:
        return _OWN[op](state)
    return _PLAIN[op](state)


# ----------------------------------------------------------------------------------------------------------------------
# What a pass cannot do without
# ----------------------------------------------------------------------------------------------------------------------

def _depths(parent):
    d = []
    for p in parent:
        d.append(0 if p < 0 else d[p] + 1)
    return d


def work(case):
    op, Hkv = case["op"], case["Hkv"]
    if op in ("tree", "decode"):
        W, S, n_q = case["window"] or NO_WINDOW, case["sinks"], case["n_q"]
        row = {"bf16": 2 * D, "fp8": D, "mx4": 68}[case.get("kind", "mx4")]
        pairs = keys = new = 0
        for base, m, parent, _ in _requests(case):
            depth = _depths(parent) if op == "tree" else range(m)
            for d in depth:
                low = max(0, base + d + 1 - W)
                pairs += base + d + 1 - low + min(S, low)
            low = max(0, base + 1 - W)
            keys += base + m - low + min(S, low)
            new += m
        return {"bytes": keys * Hkv * 2 * row + new * case["Hq"] * 2 * D + case["B"] * n_q * case["Hq"] * (2 * D + 4), "flops": 4 * D * case["Hq"] * pairs}
    if op == "commit":
        moved = nodes = 0
        for _, m, parent, a in _requests(case):
            path = []
            while a >= 0:
                path.append(a)
                a = parent[a]
            moved += sum(i != node for i, node in enumerate(reversed(path)))
            nodes += m
        elem = 1 if case["kind"] == "fp8" else 2
        return {"bytes": moved * case["layers"] * Hkv * D * elem * 4 + nodes * 4 + case["B"] * (case["n_q"] * 24 + 16), "flops": 0}
    n, prefix = case["n"], case["prefix"]
    return {"bytes": n * (case["Hq"] * 4 * D + Hkv * 2 * (2 * D + 68)) + (prefix + n) * Hkv * 2 * (68 + 2 * D), "flops": n * 3 * case["rot"] * (case["Hq"] + Hkv)}


# ----------------------------------------------------------------------------------------------------------------------
# The definition in 64 bits
# ----------------------------------------------------------------------------------------------------------------------

def _element(rows, Hkv):
    """4-bit token rows in 64 bits, from the bits of a code: sign, two of exponent, one of mantissa."""
    packed = rows[..., :Hkv * 64].long()
    code = torch.stack([packed & 15, packed >> 4], -1).flatten(-2)
    sign, exponent, half = 1 - 2.0 * (code >> 3), code >> 1 & 3, code & 1
    x = sign * torch.where(exponent == 0, 0.5 * half.double(), (1 + 0.5 * half) * torch.exp2(exponent.double() - 1))
    scale = torch.exp2(rows[..., Hkv * 64:Hkv * 68].double() - 127).repeat_interleave(32, -1)
    return (x * scale).reshape(*rows.shape[:-1], Hkv, D)


def exact(case, seed):
    op, page, Hkv = case["op"], case["page"], case["Hkv"]
    if op == "commit":
        return None                               # whole numbers and copies
    s = prepare(case, seed)
    if op in ("tree", "decode"):
        W, S, n_q, Hq = case["window"] or NO_WINDOW, case["sinks"], case["n_q"], case["Hq"]
        kind = case.get("kind", "mx4")
        out = torch.zeros(case["B"], n_q, Hq, D, dtype=torch.float64, device="cuda")
        lse = torch.full((Hq, case["B"], n_q), -math.inf, dtype=torch.float64, device="cuda")
        for b, (base, m, parent, _) in enumerate(_requests(case)):
            t = torch.arange(base + m, device="cuda")
            ids = s["table"][b, t // page].long().clamp(min=0)     # a page that was given back holds keys that nobody sees
            if kind == "mx4":
                k, v = (_element(x[ids, t % page], Hkv) for x in (s["k"], s["v"]))
            elif kind == "fp8":
                k, v = (x.view(torch.float8_e4m3fn)[ids, t % page].double() * f.double()[:, None] for x, f in ((s["k"], s["k_scale"]), (s["v"], s["v_scale"])))
            else:
                k, v = s["k"][ids, t % page].double(), s["v"][ids, t % page].double()
            depth = _depths(parent) if op == "tree" else list(range(m))
            up = parent if op == "tree" else list(range(-1, m - 1))
            seen = torch.zeros(m, base + m, dtype=torch.bool, device="cuda")
            before = torch.arange(base, device="cuda")
            for i in range(m):
                seen[i, :base] = (base + depth[i] - before < W) | (before < S)
                j = i
                while j >= 0:
                    seen[i, base + j] = depth[i] - depth[j] < W or base + depth[j] < S
                    j = up[j]
            for h in range(Hq):
                g = h // (Hq // Hkv)
                score = (s["q"][b, :m, h].double() @ k[:, g].T / math.sqrt(D)).masked_fill(~seen, -math.inf)
                z = torch.logsumexp(score, 1)
                lse[h, b, :m] = z
                out[b, :m, h] = torch.exp(score - z[:, None]) @ v[:, g]
        return [out, lse.reshape(Hq, -1)]
    # prompt: pair i of a head is a complex number, turned by exp(1j * angle); the blocks' exponents and codes by search over the 16 values
    n = case["rot"] // 2
    which = [a for a, m in enumerate(_sections(case)) for _ in range(m)]
    rate = torch.tensor([math.exp(-math.log(_BASE) * i / n) for i in range(n)], dtype=torch.float64, device="cuda")
    angle = s["positions"][torch.tensor(which, device="cuda")].double().T * rate
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]

    def turned(x):
        y = x.double().clone()
        first = slice(0, 2 * n, 2) if case["pairs"] else slice(0, n)
        second = slice(1, 2 * n, 2) if case["pairs"] else slice(n, 2 * n)
        z = torch.complex(y[..., first].contiguous(), y[..., second].contiguous()) * turn
        y[..., first], y[..., second] = z.real, z.imag
        return y

    def nearest(x):
        y = x.reshape(*x.shape[:-1], 4, 32)
        scale = torch.exp2(torch.floor(torch.log2(y.abs().amax(-1, keepdim=True))) - 2)
        even, odd = (torch.tensor(v, dtype=torch.float64, device="cuda") for v in ((0.0, 1.0, 2.0, 4.0), (0.5, 1.5, 3.0, 6.0)))
        z = (y.abs() / scale).clamp(max=6.0)
        a, b = (v[torch.argmin((z[..., None] - v).abs(), -1)] for v in (even, odd))
        return (torch.sign(y) * torch.where((z - a).abs() <= (z - b).abs(), a, b) * scale).reshape(x.shape)

    t = torch.arange(case["prefix"], device="cuda")
    ids = s["table"][0, t // page].long()
    k, v = (_element(x[ids, t % page], Hkv) for x in (s["k"], s["v"]))
    return [turned(s["q"]), torch.cat([k, nearest(turned(s["k_rows"]))]), torch.cat([v, nearest(s["v_rows"].double())])]
