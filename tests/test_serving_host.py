"""Host side of the serving calls: what is refused before anything reaches a device (addresses here are never read), and the rotary
description."""
import ctypes
import math

import pytest

from paper_2609_04774_b200 import binding, build

P = 0x10000          # an aligned address that a refused call never looks at


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


def cache(**kw):
    c = binding.cp_kv_cache()
    c.k = c.v = P
    c.num_pages, c.page_size, c.Hkv, c.D = 10, 16, 2, 128
    c.stride_page, c.stride_tok, c.stride_head = 16 * 256, 256, 128
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def pool(layers=2, **kw):
    p = binding.cp_page_pool()
    p._k = (ctypes.c_void_p * layers)(*[P] * layers)
    p.k = p.v = ctypes.addressof(p._k)
    p.n_layers, p.num_pages, p.page_size, p.Hkv, p.row_bytes = layers, 10, 16, 2, 256
    p.stride_page, p.stride_tok, p.stride_head = 16 * 512, 512, 256
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def test_rope_init():
    r = binding.make_rope([16, 24, 24], base=1e6, interleaved=True)
    assert (r.n_axes, r.rot_dims, r.interleaved) == (3, 128, 1)
    assert list(r.axis) == [0] * 16 + [1] * 24 + [2] * 24
    assert all(r.freq[i] == pytest.approx(1e6 ** (-2 * i / 128), rel=1e-15) for i in range(64))
    r = binding.make_rope([20])
    assert r.rot_dims == 40 and r.freq[19] == pytest.approx(10000.0 ** (-19 / 20), rel=1e-15)
    for sections, base in (([], 1e4), ([65], 1e4), ([0], 1e4), ([1] * 5, 1e4), ([70, -6], 1e4), ([64], 0.0), ([64], -1.0), ([64], math.inf), ([64], math.nan)):
        with pytest.raises(binding.CpError) as e:
            binding.make_rope(sections, base=base)
        assert e.value.code == binding.CP_ERR_INVALID_ARG


def rope_call(lib, rope=None, cache_=None, **kw):
    a = dict(q=P, k=P, v=P, n=4, Hq=4, pos=P, seq=P, slot=P, table=P, rows=3, stride=5, q_out=2 * P) | kw
    rope, cache_ = rope or binding.make_rope([64]), cache_ or cache()          # held while the call reads them
    return lib.cp_rope_append(None, ctypes.addressof(rope), a["q"], a["k"], a["v"], a["n"], a["Hq"], a["pos"], a["seq"], a["slot"],
                              ctypes.addressof(cache_), a["table"], a["rows"], a["stride"], a["q_out"], None)


def test_rope_refusals(lib):
    assert rope_call(lib) == binding.CP_ERR_INVALID_ARG and b"ctx is NULL" in lib.cp_last_error()      # all else is in order
    bad, uns = binding.CP_ERR_INVALID_ARG, binding.CP_ERR_UNSUPPORTED
    for kw, code, word in ((dict(q=None), bad, b"together"), (dict(q_out=None), bad, b"together"), (dict(k=None), bad, b"together"),
                           (dict(v=None), bad, b"together"), (dict(q=None, q_out=None, k=None, v=None), bad, b"neither"), (dict(pos=None), bad, b"null"),
                           (dict(seq=None), bad, b"null"), (dict(slot=None), bad, b"token_slot"), (dict(table=None), bad, b"table"),
                           (dict(rows=0), bad, b"table"), (dict(stride=0), bad, b"table"), (dict(n=-1), bad, b"negative"), (dict(Hq=0), bad, b"Hq"),
                           (dict(q=P + 8), bad, b"aligned"), (dict(k=P + 2), bad, b"aligned"), (dict(q_out=P + 1024), bad, b"overlaps"),
                           (dict(n=1 << 40), uns, b"tokens"), (dict(Hq=5000), uns, b"heads")):
        assert rope_call(lib, **kw) == code and word in lib.cp_last_error(), kw
    assert rope_call(lib, q_out=P) == bad and b"ctx is NULL" in lib.cp_last_error()                     # in place is fine
    for field, value, code in (("n_axes", 0, bad), ("n_axes", 5, bad), ("rot_dims", 0, bad), ("rot_dims", 130, bad), ("rot_dims", 40, uns)):
        r = binding.make_rope([64])
        setattr(r, field, value)
        assert rope_call(lib, rope=r) == code, field
    r = binding.make_rope([64])
    r.axis[5] = 1
    assert rope_call(lib, rope=r) == bad and b"axis" in lib.cp_last_error()
    r = binding.make_rope([64])
    r.freq[63] = math.nan
    assert rope_call(lib, rope=r) == bad and b"finite" in lib.cp_last_error()
    for kw, code in ((dict(page_size=48), uns), (dict(D=64), uns), (dict(stride_tok=4), uns), (dict(k=P + 8), uns), (dict(Hkv=0), bad), (dict(k=None), bad)):
        assert rope_call(lib, cache_=cache(**kw)) == code, kw


def page_calls(lib, p, ref=P, table=P, rows=3, stride=5, kv=P, other=P, n=2, ws=P, ws_bytes=1 << 20, window=5, sinks=0):
    a = ctypes.addressof(p)
    return {
        "extend": lib.cp_pages_extend(None, a, ref, table, rows, stride, kv, other, ws, ws_bytes, None),
        "evict": lib.cp_pages_evict(None, a, ref, table, rows, stride, kv, window, sinks, None),
        "free": lib.cp_pages_free(None, a, ref, table, rows, stride, kv, other, n, None),
        "fork": lib.cp_pages_fork(None, a, ref, table, rows, stride, kv, other, other, n, ws, ws_bytes, None),
        "compact": lib.cp_pages_compact(None, a, ref, table, rows, stride, kv, other, ws, ws_bytes, None),
        "copy": lib.cp_pages_copy(None, a, other, kv, n, ws, ws_bytes, None),
    }


def test_page_refusals(lib):
    bad, uns, wsp = binding.CP_ERR_INVALID_ARG, binding.CP_ERR_UNSUPPORTED, binding.CP_ERR_WORKSPACE
    assert set(page_calls(lib, pool()).values()) == {bad} and b"ctx is NULL" in lib.cp_last_error()
    copies = {"fork", "compact", "copy"}
    for p, codes in ((pool(num_pages=0), {k: bad for k in page_calls(lib, pool())}), (pool(page_size=8), {k: uns for k in page_calls(lib, pool())}),
                     (pool(num_pages=1 << 32), {k: uns for k in page_calls(lib, pool())}), (pool(row_bytes=64), {k: uns for k in copies}),
                     (pool(stride_tok=500), {k: uns for k in copies}), (pool(stride_page=0), {k: uns for k in copies}), (pool(n_layers=0), {k: bad for k in copies}),
                     (pool(layers=129), {k: uns for k in copies}), (pool(Hkv=0), {k: bad for k in copies})):
        got = page_calls(lib, p)
        assert all(got[k] == c for k, c in codes.items()), (got, codes)
    q = pool()
    q._k[1] = P + 8
    assert page_calls(lib, q)["copy"] == uns
    q._k[1] = None
    assert page_calls(lib, q)["fork"] == bad
    tables = {"extend", "evict", "free", "fork", "compact"}
    for kw, names, code in ((dict(ref=None), tables, bad), (dict(table=None), tables, bad), (dict(rows=0), tables, bad), (dict(stride=0), tables, bad),
                            (dict(stride=1 << 30), tables, uns), (dict(kv=None), tables | {"copy"}, bad), (dict(other=None), {"extend", "free", "fork", "compact", "copy"}, bad),
                            (dict(n=-1), {"free", "fork", "copy"}, bad), (dict(ws=None), {"extend", "fork", "compact", "copy"}, wsp),
                            (dict(ws=P + 16), {"extend", "fork", "compact", "copy"}, wsp), (dict(ws_bytes=255), {"extend", "fork", "compact", "copy"}, wsp),
                            (dict(window=0), {"evict"}, bad), (dict(sinks=-1), {"evict"}, bad)):
        got = page_calls(lib, pool(), **kw)
        assert all(got[k] == code for k in names), (kw, got)
    big = page_calls(lib, pool(), n=100000, ws_bytes=binding.cp_workspace_bytes_pages(10, 90000))
    assert big["fork"] == big["copy"] == wsp


def test_workspace_bytes_pages():
    assert binding.cp_workspace_bytes_pages(0) == 0 and binding.cp_workspace_bytes_pages(10, -1) == 0
    a, b = binding.cp_workspace_bytes_pages(1000), binding.cp_workspace_bytes_pages(1000, 5000)
    assert a % 256 == 0 and 1000 * 20 <= a < 1000 * 20 + 1024 and b - a >= 4000 * 16 - 256


def test_decode_refusals(lib):
    bad, uns, wsp = binding.CP_ERR_INVALID_ARG, binding.CP_ERR_UNSUPPORTED, binding.CP_ERR_WORKSPACE

    def call(c=None, **kw):
        a = dict(q=P, table=P, stride=5, kv_len=P, B=3, n_q=1, Hq=4, window=9, sinks=0, scale=0.1, out=P, lse=P, ws=P, ws_bytes=1 << 30) | kw
        c = c or cache()                                     # held while the call reads it
        return lib.cp_decode_attn(None, a["q"], ctypes.addressof(c), a["table"], a["stride"], a["kv_len"], a["B"], a["n_q"], a["Hq"], a["window"],
                                  a["sinks"], a["scale"], a["out"], a["lse"], a["ws"], a["ws_bytes"], None)
    assert call() == bad and b"ctx is NULL" in lib.cp_last_error()
    for kw, code, word in ((dict(q=None), bad, b"null"), (dict(table=None), bad, b"null"), (dict(kv_len=None), bad, b"null"), (dict(out=None), bad, b"null"),
                           (dict(lse=None), bad, b"null"), (dict(stride=0), bad, b"table_stride"), (dict(B=-1), bad, b"B=-1"), (dict(n_q=0), bad, b"n_q=0"),
                           (dict(Hq=0), bad, b"Hq"), (dict(Hq=5), bad, b"multiple"), (dict(window=0), bad, b"window"), (dict(sinks=-1), bad, b"sinks"),
                           (dict(scale=0.0), bad, b"scale"), (dict(scale=math.nan), bad, b"scale"), (dict(scale=math.inf), bad, b"scale"), (dict(q=P + 8), bad, b"aligned"),
                           (dict(out=P + 2), bad, b"aligned"), (dict(n_q=65), uns, b"n_q"), (dict(Hq=4096), uns, b"rows"), (dict(B=65537), uns, b"B="),
                           (dict(stride=1 << 30), uns, b"entries"), (dict(ws=None), wsp, b"workspace"), (dict(ws=P + 128), wsp, b"workspace"),
                           (dict(ws_bytes=binding.cp_workspace_bytes_decode(3, 1, 4, 2) - 1), wsp, b"workspace")):
        assert call(**kw) == code and word in lib.cp_last_error(), kw
    assert call(B=0, q=None, table=None, kv_len=None, out=None, lse=None) == bad and b"ctx is NULL" in lib.cp_last_error()
    for kw, code in ((dict(page_size=48), uns), (dict(D=64), uns), (dict(stride_tok=4), uns), (dict(k=P + 8), uns), (dict(Hkv=0), bad), (dict(k=None), bad)):
        assert call(cache(**kw)) == code, kw
    for args in ((-1, 1, 4, 2), (1, 0, 4, 2), (1, 1, 0, 2), (1, 1, 4, 0), (1, 1, 5, 2)):
        assert binding.cp_workspace_bytes_decode(*args) == 0


def test_struct_layouts():
    assert ctypes.sizeof(binding.cp_rope) == 16 + 256 + 512
    assert ctypes.sizeof(binding.cp_page_pool) == 64
