"""Serving operators behind a paged K/V cache, as cases with plain forms.

Four operators that belong together in a serving loop:

  window   prefill attention of new tokens over a paged cache with a sliding window and a few first tokens (sinks)
           that stay visible
  decode   attention of one or a few new tokens per request over a paged cache (bf16 or E4M3), with or without a window;
           lengths and page tables live on the device
  rope     rotary positions with one to three axes (time, height, width) applied to q and k, and k, v appended to the paged
           cache in the same call
  pages    the care of the pages: fork (share full pages, copy a partly filled one), extend + evict (a decode step's page
           work), compact (live pages moved to the front of the pool)

Logical token t of a sequence lives in page table[t // page], slot t % page.  A token at position p sees key j if j <= p and
(p - j < window or j < sinks); window 0 in a case means no window.
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
        # a chat turn: a few hundred new tokens behind a cached conversation
        dict(name="window_turn", op="window", B=1, new_lo=333, new_hi=333, prefix=1500, window=1024, sinks=4, Hq=32, Hkv=8, page=64, mix=1),
        # a prefill batch of mixed requests with partial prefix hits
        dict(name="window_batch", op="window", B=16, new_lo=200, new_hi=6000, prefix=12288, window=4096, sinks=64, Hq=32, Hkv=8, page=64, mix=2),
        # one long document, no prefix
        dict(name="window_document", op="window", B=1, new_lo=32768, new_hi=32768, prefix=0, window=4096, sinks=4, Hq=32, Hkv=8, page=64, mix=3),
        # one user, one token: latency counts
        dict(name="decode_single", op="decode", B=1, n_q=1, len_lo=4097, len_hi=4097, window=0, sinks=0, Hq=32, Hkv=8, page=64, fp8=False, mix=4),
        # a serving batch of ragged lengths
        dict(name="decode_batch", op="decode", B=64, n_q=1, len_lo=257, len_hi=16384, window=0, sinks=0, Hq=32, Hkv=8, page=64, fp8=False, mix=5),
        # long conversations of a model with a window, E4M3 cache, pages behind the window given back
        dict(name="decode_window_fp8", op="decode", B=128, n_q=1, len_lo=1000, len_hi=65536, window=4096, sinks=4, Hq=64, Hkv=8, page=32, fp8=True, mix=6),
        # few long contexts, four draft tokens each checked in one step
        dict(name="decode_draft", op="decode", B=4, n_q=4, len_lo=100000, len_hi=131072, window=0, sinks=0, Hq=32, Hkv=4, page=64, fp8=False, mix=7),
        # the new tokens of a decode step
        dict(name="rope_step", op="rope", n=64, Hq=32, Hkv=8, page=64, axes=1, pairs=True, rot=128, fp8=False, mix=8),
        # a prompt of images and video
        dict(name="rope_video", op="rope", n=16384, Hq=32, Hkv=8, page=64, axes=3, pairs=False, rot=128, fp8=False, mix=9),
        # parallel samples of a few prompts: full pages shared, the partly filled page of every sample copied in every layer
        dict(name="pages_fork", op="fork", forks=32, parents=4, len_lo=1000, len_hi=6000, layers=32, pool=512, Hkv=8, page=64, mix=10),
        # the page work of one decode step of windowed sequences
        dict(name="pages_step", op="step", rows=64, len_lo=200, len_hi=65536, new_hi=4, window=4096, sinks=64, pool=16384, page=64, mix=11),
        # a pool with holes made dense again
        dict(name="pages_compact", op="compact", rows=48, layers=4, pool=2048, live=1200, Hkv=8, page=64, mix=12),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["window", "decode", "rope", "fork", "step", "compact"])
    page = rng.choice([16, 32, 64, 128])
    Hq, Hkv = rng.choice([(32, 8), (32, 4), (16, 16), (8, 8), (64, 8), (5, 1), (16, 2)])
    mix = rng.randrange(1 << 20)
    if op == "window":
        Hq, Hkv = rng.choice([(32, 8), (32, 4), (16, 16), (8, 2), (6, 2)])
        B = _log(rng, 1, 24)
        hi = _log(rng, 1, 32768 // B)
        return dict(op=op, B=B, new_lo=max(1, hi // 8), new_hi=hi, prefix=rng.choice([0, _log(rng, 1, 16384)]), window=_log(rng, 1, 4096),
                    sinks=rng.choice([0, 1, 4, rng.randrange(200)]), Hq=Hq, Hkv=Hkv, page=page, mix=mix)
    if op == "decode":
        B = _log(rng, 1, 128)
        hi = _log(rng, 16, min(131072, 500000 * 4 // (B * Hkv)))
        return dict(op=op, B=B, n_q=rng.choice([1, 1, 1, 2, 3, 4]), len_lo=max(1, hi // rng.choice([1, 8, 64])), len_hi=hi,
                    window=rng.choice([0, _log(rng, 1, 8192)]), sinks=rng.choice([0, 4, rng.randrange(300)]), Hq=Hq, Hkv=Hkv, page=page,
                    fp8=rng.random() < 0.5, mix=mix)
    if op == "rope":
        return dict(op=op, n=_log(rng, 1, 12000), Hq=min(Hq, 32), Hkv=min(Hkv, 8), page=page, axes=rng.choice([1, 2, 3]), pairs=rng.random() < 0.5,
                    rot=rng.choice([128, 128, 64, 96]), fp8=rng.random() < 0.5, mix=mix)
    if op == "fork":
        parents = rng.randrange(1, 7)
        return dict(op=op, forks=_log(rng, 1, 32), parents=parents, len_lo=1, len_hi=_log(rng, 20, 400 * page // parents), layers=rng.randrange(1, 25),
                    pool=rng.randrange(450, 1000), Hkv=min(Hkv, 8), page=min(page, 64), mix=mix)
    if op == "step":
        window = _log(rng, 16, 8192)
        return dict(op=op, rows=_log(rng, 1, 128), len_lo=1, len_hi=_log(rng, 64, 65536), new_hi=rng.choice([1, 4, 100]), window=window, sinks=rng.choice([0, 4, 130]),
                    pool=80000, page=page, mix=mix)
    pool = _log(rng, 20, 2048)
    return dict(op=op, rows=rng.randrange(1, 60), layers=rng.randrange(1, 5), pool=pool, live=rng.randrange(pool + 1), Hkv=min(Hkv, 8), page=min(page, 64), mix=mix)


def _lengths(case):
    """The lengths that a case stands for: they belong to the case, not to the seed of the values."""
    rng = random.Random(case["mix"])
    if case["op"] == "window":
        return [(_log(rng, case["new_lo"], case["new_hi"]), rng.randint(case["prefix"] // 2, case["prefix"])) for _ in range(case["B"])]
    if case["op"] == "decode":
        return [_log(rng, case["len_lo"], case["len_hi"]) for _ in range(case["B"])]
    if case["op"] == "fork":
        lens = [_log(rng, case["len_lo"], case["len_hi"]) for _ in range(case["parents"])]
        return lens, [rng.randrange(case["parents"]) for _ in range(case["forks"])]
    if case["op"] == "step":
        lens = [_log(rng, case["len_lo"], case["len_hi"]) for _ in range(case["rows"])]
        return lens, [rng.randint(0, case["new_hi"]) for _ in range(case["rows"])]
    raise ValueError(case["op"])


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


def _scatter_pages(g, counts, width, spare):
    """A table [rows, width] whose row r has counts[r] pages, drawn without order from a pool."""
    total = sum(counts)
    ids = torch.randperm(total + spare, generator=g, device="cuda")[:total].to(torch.int32)
    c = torch.tensor(counts, device="cuda")
    at = torch.arange(width, device="cuda")[None, :]
    base = (torch.cumsum(c, 0) - c)[:, None]
    return torch.where(at < c[:, None], ids[(base + at).clamp(max=max(total - 1, 0))], -1).contiguous(), total + spare


def prepare(case, seed):
    g = torch.Generator("cuda")
    g.manual_seed(int(seed) * 7919 + 17)
    s = {"case": case}
    op, page = case["op"], case["page"]
    if op == "window":
        lens = _lengths(case)
        counts = [-(-(n + p) // page) for n, p in lens]
        s["table"], pool = _scatter_pages(g, counts, max(counts), 3)
        total = sum(n for n, _ in lens)
        s["q"] = _normal(g, total, case["Hq"], D)
        s["k"], s["v"] = _normal(g, pool, page, case["Hkv"], D), _normal(g, pool, page, case["Hkv"], D)
        s["lens"] = lens
        s["out"], s["lse"] = torch.empty_like(s["q"]), torch.empty(case["Hq"], total, dtype=torch.float32, device="cuda")
    elif op == "decode":
        lens = _lengths(case)
        # with a window, the pages wholly behind it (and behind the sinks) have been given back: their entries are -1
        counts = [-(-n // page) for n in lens]
        width = max(counts)
        window, n_q = case["window"] or NO_WINDOW, case["n_q"]
        first = [-(-case["sinks"] // page) for _ in lens]
        last = [max(f, max(0, n - n_q + 1 - window) // page) for n, f in zip(lens, first)]
        held = [c - max(0, min(b, c) - a) for c, a, b in zip(counts, first, last)]
        dense, pool = _scatter_pages(g, held, width, 3)
        at = torch.arange(width, device="cuda")[None, :]
        a, b, c = (torch.tensor(x, device="cuda")[:, None] for x in (first, last, counts))
        gap = (b.minimum(c) - a).clamp(min=0)
        gone = (at >= a) & (at < a + gap)
        src = torch.where(at < a, at, at - gap).clamp(min=0)
        s["table"] = torch.where(gone | (at >= c), -1, dense.gather(1, src.clamp(max=width - 1))).to(torch.int32).contiguous()
        s["kv_len"] = _i32(lens)
        s["q"] = _normal(g, len(lens), n_q, case["Hq"], D)
        shape = (pool, page, case["Hkv"], D)
        if case["fp8"]:
            s["k"], s["v"] = _codes(g, *shape), _codes(g, *shape)
            s["k_scale"] = (torch.rand(case["Hkv"], generator=g, device="cuda") + 0.5) / 70.0
            s["v_scale"] = (torch.rand(case["Hkv"], generator=g, device="cuda") + 0.5) / 70.0
        else:
            s["k"], s["v"] = _normal(g, *shape), _normal(g, *shape)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(case["Hq"], len(lens) * n_q, dtype=torch.float32, device="cuda")
    elif op == "rope":
        n = case["n"]
        rng = random.Random(case["mix"])
        rows = max(1, min(n, rng.randint(1, 64)))
        per = -(-n // rows)
        offset = rng.randint(0, 500)
        counts = [-(-(offset + per) // page)] * rows
        s["table"], pool = _scatter_pages(g, counts, counts[0], 2)
        i = torch.arange(n, device="cuda")
        s["seq"], s["slot"] = (i // per).to(torch.int32), (offset + i % per).to(torch.int32)
        # text positions go far; frames, rows and columns of images and video stay small and start behind the text
        far = rng.choice([0, 5000, 1000000])
        t = [far + i % per, far + (i % per) // 32 % 48, far + i % 32]
        s["positions"] = torch.stack(t[:case["axes"]]).to(torch.int32).contiguous()
        s["q"] = _normal(g, n, case["Hq"], D)
        s["k_rows"], s["v_rows"] = _normal(g, n, case["Hkv"], D), _normal(g, n, case["Hkv"], D)
        s["q_out"] = torch.empty_like(s["q"])
        shape = (pool, page, case["Hkv"], D)
        if case["fp8"]:
            s["k"], s["v"] = _codes(g, *shape), _codes(g, *shape)
            s["k_scale"] = (torch.rand(case["Hkv"], generator=g, device="cuda") + 0.5) / 70.0
            s["v_scale"] = (torch.rand(case["Hkv"], generator=g, device="cuda") + 0.5) / 70.0
        else:
            s["k"], s["v"] = _normal(g, *shape), _normal(g, *shape)
    elif op == "fork":
        lens, parent = _lengths(case)
        counts = [-(-n // page) for n in lens]
        table, _ = _scatter_pages(g, counts, max(counts) + 1, case["pool"] - sum(counts))
        s["table"] = torch.cat([table, torch.full((case["forks"], table.shape[1]), -1, dtype=torch.int32, device="cuda")])
        s["kv_len"] = _i32(lens + [0] * case["forks"])
        s["refcount"] = torch.zeros(case["pool"], dtype=torch.int32, device="cuda")
        s["refcount"][table[table >= 0].long()] = 1
        s["parent"], s["child"] = _i32(parent), _i32([case["parents"] + i for i in range(case["forks"])])
        shape = (case["layers"], case["pool"], page, case["Hkv"], D)
        s["k"], s["v"] = _normal(g, *shape), _normal(g, *shape)
    elif op == "step":
        lens, new = _lengths(case)
        width = -(-(max(lens) + case["new_hi"]) // page)
        first = -(-case["sinks"] // page)
        # behind the last step's window everything is gone already, the step before this one's is not
        last = [max(first, max(0, n + 1 - case["window"] - page) // page) for n in lens]
        counts = [-(-n // page) for n in lens]
        held = [max(0, min(c, first)) + max(0, c - max(b, min(c, first))) for c, b in zip(counts, last)]
        dense, _ = _scatter_pages(g, held, width, case["pool"] - sum(held))
        at = torch.arange(width, device="cuda")[None, :]
        b, c = torch.tensor(last, device="cuda")[:, None], torch.tensor(counts, device="cuda")[:, None]
        gone = (at >= first) & (at < b)
        src = torch.where(at < first, at, at - (b - first))
        s["table"] = torch.where(gone | (at >= c), -1, dense.gather(1, src.clamp(0, width - 1))).to(torch.int32).contiguous()
        s["refcount"] = torch.zeros(case["pool"], dtype=torch.int32, device="cuda")
        s["refcount"][s["table"][s["table"] >= 0].long()] = 1
        s["kv_len"], s["new"] = _i32(lens), _i32(new)
        s["k"] = s["v"] = torch.zeros(1, case["pool"], page, 1, D, dtype=torch.bfloat16, device="cuda")
    else:
        pool, live, rows = case["pool"], case["live"], case["rows"]
        ids = torch.randperm(pool, generator=g, device="cuda")[:live]
        s["refcount"] = torch.zeros(pool, dtype=torch.int32, device="cuda")
        s["refcount"][ids] = torch.randint(1, 4, (live,), generator=g, device="cuda", dtype=torch.int32)
        width = max(1, -(-live // rows))
        table = torch.full((rows * width,), -1, dtype=torch.int32, device="cuda")
        table[:live] = ids.to(torch.int32)
        s["table"] = table.view(rows, width)
        shape = (case["layers"], pool, page, case["Hkv"], D)
        s["k"], s["v"] = _normal(g, *shape), _normal(g, *shape)
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
    b = _binding()
    if "k_scale" in s:
        return _kept(s, "cache", lambda: b.make_cache_fp8(s["k"], s["v"], s["k_scale"], s["v_scale"]))
    return _kept(s, "cache", lambda: b.make_cache(s["k"], s["v"]))


def _pool_of(s):
    return _kept(s, "pool", lambda: _binding().make_page_pool(s["k"], s["v"], s["refcount"].numel()))


def _own_window(s):
    b, c = _binding(), s["case"]
    lens, width = s["lens"], s["table"].shape[1]
    C = [1] * len(lens)
    ws = _kept(s, "ws", lambda: torch.empty(b.cp_workspace_bytes([n for n, _ in lens], C, c["Hq"]), dtype=torch.uint8, device="cuda"))
    cu = [0]
    for n, _ in lens:
        cu.append(cu[-1] + n)
    b.cp_prefill_attn_window_batch(_ctx(), s["q"], _cache_of(s), s["table"], cu, [p for _, p in lens], C, [i * width for i in range(len(lens) + 1)],
                                   c["window"], c["sinks"], c["Hq"], D ** -0.5, s["out"], s["lse"], ws)
    return [s["out"], s["lse"]]


def _own_decode(s):
    b, c = _binding(), s["case"]
    call = b.cp_decode_attn_fp8 if c["fp8"] else b.cp_decode_attn
    ws = _kept(s, "ws", lambda: torch.empty(b.cp_workspace_bytes_decode(c["B"], c["n_q"], c["Hq"], c["Hkv"]), dtype=torch.uint8, device="cuda"))
    call(_ctx(), s["q"], _cache_of(s), s["table"], s["kv_len"], c["window"] or NO_WINDOW, c["sinks"], D ** -0.5, s["out"], s["lse"], ws)
    return [s["out"], s["lse"]]


def _own_rope(s):
    b, c = _binding(), s["case"]
    rope = _kept(s, "rope", lambda: b.make_rope(_sections(c), base=_BASE, interleaved=c["pairs"]))
    call = b.cp_rope_append_fp8 if c["fp8"] else b.cp_rope_append
    call(_ctx(), rope, s["q"], s["k_rows"], s["v_rows"], s["positions"], s["seq"], s["slot"], _cache_of(s), s["table"], s["q_out"])
    return [s["q_out"], _values(s["k"]), _values(s["v"])]


def _own_fork(s):
    b = _binding()
    table, refcount, kv_len = s["table"].clone(), s["refcount"].clone(), s["kv_len"].clone()
    ws = _kept(s, "ws", lambda: torch.empty(b.cp_workspace_bytes_pages(s["refcount"].numel(), s["parent"].numel()), dtype=torch.uint8, device="cuda"))
    b.cp_pages_fork(_ctx(), _pool_of(s), refcount, table, kv_len, s["parent"], s["child"], ws)
    return [table, refcount, kv_len, s["k"], s["v"]]


def _own_step(s):
    b, c = _binding(), s["case"]
    table, refcount, kv_len = s["table"].clone(), s["refcount"].clone(), s["kv_len"].clone()
    ws = _kept(s, "ws", lambda: torch.empty(b.cp_workspace_bytes_pages(s["refcount"].numel(), kv_len.numel()), dtype=torch.uint8, device="cuda"))
    b.cp_pages_evict(_ctx(), _pool_of(s), refcount, table, kv_len, c["window"], c["sinks"])
    b.cp_pages_extend(_ctx(), _pool_of(s), refcount, table, kv_len, s["new"], ws)
    return [table, refcount, kv_len]


def _own_compact(s):
    b = _binding()
    table, refcount = s["table"].clone(), s["refcount"].clone()
    page_map = _kept(s, "map", lambda: torch.empty_like(s["refcount"]))
    n_live = _kept(s, "n_live", lambda: torch.empty(1, dtype=torch.int32, device="cuda"))
    ws = _kept(s, "ws", lambda: torch.empty(b.cp_workspace_bytes_pages(s["refcount"].numel(), table.shape[0]), dtype=torch.uint8, device="cuda"))
    b.cp_pages_compact(_ctx(), _pool_of(s), refcount, table, page_map, n_live, ws)
    return [table, refcount, page_map, n_live, s["k"], s["v"]]


# ----------------------------------------------------------------------------------------------------------------------
# Plain forms
# ----------------------------------------------------------------------------------------------------------------------

_BASE = 1000000.0
_ROWS = 512          # query rows of a plain window block: bounds its score matrix


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


def _fetch(pool, table_row, at, scale):
    """Keys or values at logical positions `at` of one sequence in 32 bits; entries without a page read as page 0 (they are masked)."""
    page = pool.shape[1]
    x = _values(pool)[table_row[at // page].clamp(min=0).long(), at % page].float()
    return x if scale is None else x * scale[:, None]


def _softmax_product(q, k, v, seen, scale):
    """q [.., r, d], k and v [.., n, d], seen [.., r, n] -> (output, log of the sum); a row that sees nothing gives 0 and -inf."""
    s = (q @ k.transpose(-1, -2)) * scale
    s = s.masked_fill(~seen, -math.inf)
    m = s.amax(-1, keepdim=True)
    e = torch.exp(s - m.masked_fill(m == -math.inf, 0.0))
    l = e.sum(-1, keepdim=True)
    o = (e @ v) / l.masked_fill(l == 0, 1.0)
    return o, (m + torch.log(l)).squeeze(-1)


def _plain_window(s):
    c = s["case"]
    out, lse = s["out"], s["lse"]
    Hkv, G, W, S = c["Hkv"], c["Hq"] // c["Hkv"], c["window"], c["sinks"]
    row = 0
    for b, (n, prefix) in enumerate(s["lens"]):
        for r0 in range(0, n, _ROWS):
            r1 = min(n, r0 + _ROWS)
            low = max(0, prefix + r0 - W + 1)
            head = torch.arange(min(S, low), device="cuda")
            at = torch.cat([head, torch.arange(low, prefix + r1, device="cuda")])
            k, v = (_fetch(x, s["table"][b], at, None).permute(1, 0, 2) for x in (s["k"], s["v"]))
            p = prefix + torch.arange(r0, r1, device="cuda")
            seen = (at[None, :] <= p[:, None]) & ((p[:, None] - at[None, :] < W) | (at[None, :] < S))
            q = s["q"][row + r0:row + r1].float().view(r1 - r0, Hkv, G, D).permute(1, 2, 0, 3)
            o, l = _softmax_product(q, k[:, None], v[:, None], seen, D ** -0.5)
            out[row + r0:row + r1] = o.permute(2, 0, 1, 3).reshape(r1 - r0, c["Hq"], D).to(torch.bfloat16)
            lse[:, row + r0:row + r1] = l.reshape(c["Hq"], r1 - r0)
        row += n
    return [out, lse]


def _plain_decode(s):
    c = s["case"]
    out, lse = s["out"], s["lse"]
    B, n_q, Hkv, G = c["B"], c["n_q"], c["Hkv"], c["Hq"] // c["Hkv"]
    W, S, page = c["window"] or NO_WINDOW, c["sinks"], c["page"]
    cap = s["table"].shape[1] * page
    n = s["kv_len"].long()[:, None]
    # candidate keys of every request: the sinks, then the last ones
    span = min(cap, W + n_q - 1)
    tail = n - span + torch.arange(span, device="cuda")[None, :]
    head = torch.arange(min(S, cap), device="cuda")[None, :].expand(B, -1)
    at = torch.cat([head, tail], 1)
    use = torch.cat([(head < n) & (head < n - span), tail >= 0], 1)
    at = at.clamp(min=0)
    p = n - n_q + torch.arange(n_q, device="cuda")[None, :]                                  # positions of the new tokens
    seen = use[:, None, :] & (at[:, None, :] <= p[:, :, None]) & ((p[:, :, None] - at[:, None, :] < W) | (at[:, None, :] < S))
    pages = s["table"].gather(1, (at // page).clamp(max=s["table"].shape[1] - 1)).clamp(min=0).long()
    k, v = (_values(x)[pages, at % page] for x in (s["k"], s["v"]))                         # [B, n, Hkv, D]
    k, v = k.float(), v.float()
    if c["fp8"]:
        k, v = k * s["k_scale"][:, None], v * s["v_scale"][:, None]
    q = s["q"].float().view(B, n_q, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, n_q * G, D)
    rows = seen[:, None, :, None, :].expand(B, 1, n_q, G, at.shape[1]).reshape(B, 1, n_q * G, at.shape[1])
    o, l = _softmax_product(q, k.permute(0, 2, 1, 3), v.permute(0, 2, 1, 3), rows, D ** -0.5)
    out.copy_(o.view(B, Hkv, n_q, G, D).permute(0, 2, 1, 3, 4).reshape(B, n_q, c["Hq"], D))
    lse.copy_(l.view(B, Hkv, n_q, G).permute(1, 3, 0, 2).reshape(c["Hq"], B * n_q))
    return [out, lse]


def _rotate(x, cos, sin, c):
    n = c["rot"] // 2
    x = x.float()
    a, b = (x[..., 0:2 * n:2], x[..., 1:2 * n:2]) if c["pairs"] else (x[..., :n], x[..., n:2 * n])
    u, w = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([u, w], -1).flatten(-2) if c["pairs"] else torch.cat([u, w], -1)
    return torch.cat([turned, x[..., 2 * n:]], -1)


def _plain_rope(s):
    c = s["case"]
    pairs = c["rot"] // 2
    axis = torch.repeat_interleave(torch.arange(c["axes"], device="cuda"), torch.tensor(_sections(c), device="cuda"), output_size=pairs)
    freq = torch.pow(torch.tensor(_BASE, dtype=torch.float64, device="cuda"), -torch.arange(pairs, dtype=torch.float64, device="cuda") / pairs)
    angle = s["positions"].double()[axis].T * freq                                          # in 64 bits: positions go far
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    s["q_out"].copy_(_rotate(s["q"], cos, sin, c))
    k, v = _rotate(s["k_rows"], cos, sin, c), s["v_rows"].float()
    where = (s["table"][s["seq"].long(), s["slot"].long() // c["page"]].long(), s["slot"].long() % c["page"])
    if c["fp8"]:
        k, v = (k / s["k_scale"][:, None]).clamp(-448, 448), (v / s["v_scale"][:, None]).clamp(-448, 448)
        s["k"][where] = k.to(torch.float8_e4m3fn).view(torch.uint8)
        s["v"][where] = v.to(torch.float8_e4m3fn).view(torch.uint8)
    else:
        s["k"][where] = k.to(torch.bfloat16)
        s["v"][where] = v.to(torch.bfloat16)
    return [s["q_out"], _values(s["k"]), _values(s["v"])]


def _free_ids(refcount):
    """Page ids, the free ones first, each kind in ascending order."""
    return torch.argsort((refcount != 0).to(torch.int8), stable=True)


def _plain_fork(s):
    page = s["case"]["page"]
    table, refcount, kv_len = s["table"].clone(), s["refcount"].clone(), s["kv_len"].clone()
    parent, child = s["parent"].long(), s["child"].long()
    n = kv_len[parent].long()
    full, part = n // page, n % page
    rows = table[parent]
    at = torch.arange(table.shape[1], device="cuda")[None, :]
    shared = torch.where(at < full[:, None], rows, -1)
    need = (part > 0).long()
    fresh = _free_ids(refcount)[torch.cumsum(need, 0) - need]
    kept = shared[shared >= 0].long()
    refcount.index_add_(0, kept, torch.ones_like(kept, dtype=torch.int32))
    i = torch.nonzero(part).squeeze(1)
    src, dst = rows[i, full[i]].long(), fresh[i]
    refcount[dst] = 1
    table[child] = shared
    table[child[i], full[i]] = dst.to(torch.int32)
    kv_len[child] = kv_len[parent]
    used = torch.arange(page, device="cuda")[None, :] < part[i][:, None]
    pair, slot = torch.nonzero(used, as_tuple=True)
    for pool in (s["k"], s["v"]):
        pool[:, dst[pair], slot] = pool[:, src[pair], slot]
    return [table, refcount, kv_len, s["k"], s["v"]]


def _plain_step(s):
    c = s["case"]
    page = c["page"]
    table, refcount, kv_len = s["table"].clone(), s["refcount"].clone(), s["kv_len"].clone()
    at = torch.arange(table.shape[1], device="cuda")[None, :]
    n = kv_len.long()[:, None]
    gone = (at >= -(-c["sinks"] // page)) & ((at + 1) * page <= n + 1 - c["window"]) & (table >= 0)
    ids = table[gone].long()
    refcount.index_add_(0, ids, torch.full_like(ids, -1, dtype=torch.int32))
    table[gone] = -1
    first, last = (n[:, 0] + page - 1) // page, (n[:, 0] + s["new"].long() + page - 1) // page
    need = last - first
    base = torch.cumsum(need, 0) - need
    take = (at >= first[:, None]) & (at < last[:, None])
    fresh = _free_ids(refcount)[(base[:, None] + at - first[:, None]).clamp(min=0, max=refcount.numel() - 1)]
    table = torch.where(take, fresh.to(torch.int32), table)
    refcount[fresh[take]] = 1
    return [table, refcount, kv_len + s["new"]]


def _plain_compact(s):
    refcount = s["refcount"]
    N = refcount.numel()
    at = torch.arange(N, device="cuda")
    live = refcount > 0
    n_live = live.sum()
    src, dst = torch.nonzero(live & (at >= n_live)).squeeze(1), torch.nonzero(~live & (at < n_live)).squeeze(1)
    page_map = torch.where(live, at, -1)
    page_map[src] = dst
    new_ref = refcount.clone()
    new_ref[dst] = refcount[src]
    new_ref[src] = 0
    table = torch.where(s["table"] >= 0, page_map[s["table"].clamp(min=0).long()].to(torch.int32), s["table"])
    for pool in (s["k"], s["v"]):
        pool[:, dst] = pool[:, src]
    return [table, new_ref, page_map.to(torch.int32), n_live.to(torch.int32).view(1), s["k"], s["v"]]


_OWN = {"window": _own_window, "decode": _own_decode, "rope": _own_rope, "fork": _own_fork, "step": _own_step, "compact": _own_compact}
_PLAIN = {"window": _plain_window, "decode": _plain_decode, "rope": _plain_rope, "fork": _plain_fork, "step": _plain_step, "compact": _plain_compact}


def run(state):
    op = state["case"]["op"]
    if own:
        return _OWN[op](state)
    return _PLAIN[op](state)


# ----------------------------------------------------------------------------------------------------------------------
# What a pass cannot do without
# ----------------------------------------------------------------------------------------------------------------------

def _seen_pairs(first, n, window, sinks):
    """Visible (query, key) pairs of n consecutive positions from `first`."""
    total = 0
    for p in range(first, first + n):
        low = max(0, p - window + 1)
        total += p + 1 - low + min(sinks, low)
    return total


def work(case):
    op = case["op"]
    if op == "window":
        W, S = case["window"], case["sinks"]
        pairs = tokens = keys = 0
        for n, prefix in _lengths(case):
            pairs += _seen_pairs(prefix, n, W, S)
            tokens += n
            low = max(0, prefix - W + 1)
            keys += prefix + n - low + min(S, low)
        return {"bytes": tokens * case["Hq"] * (4 * D + 4) + keys * case["Hkv"] * 4 * D, "flops": 4 * D * case["Hq"] * pairs}
    if op == "decode":
        W, S, n_q = case["window"] or NO_WINDOW, case["sinks"], case["n_q"]
        pairs = keys = 0
        for n in _lengths(case):
            new = min(n_q, n)
            pairs += _seen_pairs(n - new, new, W, S)
            low = max(0, n - new - W + 1)
            keys += n - low + min(S, low)
        elem = 1 if case["fp8"] else 2
        return {"bytes": keys * case["Hkv"] * 2 * D * elem + case["B"] * n_q * case["Hq"] * (4 * D + 4), "flops": 4 * D * case["Hq"] * pairs}
    if op == "rope":
        elem = 1 if case["fp8"] else 2
        return {"bytes": case["n"] * D * (case["Hq"] * 4 + case["Hkv"] * 2 * (2 + elem)), "flops": case["n"] * 3 * case["rot"] * (case["Hq"] + case["Hkv"])}
    if op == "fork":
        lens, parent = _lengths(case)
        rows = sum(lens[p] % case["page"] for p in parent)
        entries = sum(lens[p] // case["page"] + 1 for p in parent)
        return {"bytes": rows * case["layers"] * case["Hkv"] * D * 2 * 4 + entries * 16, "flops": 0}
    if op == "step":
        lens, _ = _lengths(case)
        return {"bytes": sum(-(-n // case["page"]) for n in lens) * 4 + case["pool"] * 4 + case["rows"] * 12, "flops": 0}
    # a uniform choice of live pages: (1 - live / pool) of them lie behind the first `live` ids
    moved = case["live"] * (1 - case["live"] / case["pool"])
    return {"bytes": moved * case["layers"] * case["page"] * case["Hkv"] * D * 2 * 4 + case["pool"] * 16, "flops": 0}


# ----------------------------------------------------------------------------------------------------------------------
# The definition in 64 bits
# ----------------------------------------------------------------------------------------------------------------------

def _exact_attention(q, k, v, p, W, S):
    """q [r, Hq, D], k and v [n, Hkv, D] (all keys of the sequence) in 64 bits, p [r] positions: every (row, key) pair is looked at."""
    r, Hq, _ = q.shape
    n, Hkv, _ = k.shape
    j = torch.arange(n, device=q.device)
    hidden = (j > p[:, None]) | ((p[:, None] - j >= W) & (j >= S))
    o = torch.zeros(r, Hq, D, dtype=torch.float64, device=q.device)
    lse = torch.full((Hq, r), -math.inf, dtype=torch.float64, device=q.device)
    some = ~hidden.all(1)
    for h in range(Hq):
        g = h // (Hq // Hkv)
        score = torch.einsum("rd,nd->rn", q[:, h], k[:, g]) / math.sqrt(D)
        score[hidden] = -math.inf
        z = torch.logsumexp(score, 1)
        lse[h] = z
        o[some, h] = torch.einsum("rn,nd->rd", torch.exp(score[some] - z[some, None]), v[:, g])
    return o, lse


def exact(case, seed):
    op = case["op"]
    if op in ("fork", "step", "compact"):
        return None                               # whole numbers and copies
    s = prepare(case, seed)
    page = case["page"]
    if op == "window":
        lens = s["lens"]
        cost = sum(n * (n + p) for n, p in lens) * case["Hq"]
        if cost > 6e10:
            return None
        outs, lses, row = [], [], 0
        for b, (n, prefix) in enumerate(lens):
            t = torch.arange(prefix + n, device="cuda")
            ids = s["table"][b, t // page].long()
            k, v = s["k"][ids, t % page].double(), s["v"][ids, t % page].double()
            for r0 in range(0, n, 1024):
                r1 = min(n, r0 + 1024)
                o, z = _exact_attention(s["q"][row + r0:row + r1].double(), k[:prefix + r1], v[:prefix + r1], prefix + torch.arange(r0, r1, device="cuda"),
                                        case["window"], case["sinks"])
                outs.append(o)
                lses.append(z)
            row += n
        return [torch.cat(outs), torch.cat(lses, 1)]
    if op == "decode":
        n_q = case["n_q"]
        outs, lses = [], []
        for b, n in enumerate(_lengths(case)):
            t = torch.arange(n, device="cuda")
            ids = s["table"][b, t // page].long().clamp(min=0)     # a page that was given back holds keys that nobody sees
            if case["fp8"]:
                k, v = (x.view(torch.float8_e4m3fn)[ids, t % page].double() * f.double()[:, None] for x, f in ((s["k"], s["k_scale"]), (s["v"], s["v_scale"])))
            else:
                k, v = s["k"][ids, t % page].double(), s["v"][ids, t % page].double()
            o, z = _exact_attention(s["q"][b].double(), k, v, n - n_q + torch.arange(n_q, device="cuda"), case["window"] or NO_WINDOW, case["sinks"])
            outs.append(o)
            lses.append(z)
        return [torch.stack(outs), torch.cat(lses, 1)]
    # rope: pair i of a head is a complex number, turned by exp(1j * angle)
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

    if case["fp8"]:
        return [turned(s["q"]), None, None]
    kp, vp = s["k"].double(), s["v"].double()
    ids = s["table"][s["seq"].long(), s["slot"].long() // page].long()
    kp[ids, s["slot"].long() % page] = turned(s["k_rows"])
    vp[ids, s["slot"].long() % page] = s["v_rows"].double()
    return [turned(s["q"]), kp, vp]
