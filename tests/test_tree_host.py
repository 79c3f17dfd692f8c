"""Host side of the tree calls and the 4-bit cache calls: what is refused before anything reaches a device (addresses here are never read)."""
import ctypes
import math

import pytest

from paper_2609_04774_b200 import binding, build
from test_serving_host import P, cache, pool

BAD, UNS, WSP = binding.CP_ERR_INVALID_ARG, binding.CP_ERR_UNSUPPORTED, binding.CP_ERR_WORKSPACE


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


def cache_fp8(**kw):
    c = binding.cp_kv_cache_fp8()
    c.k = c.v = c.k_scale = c.v_scale = P
    c.num_pages, c.page_size, c.Hkv, c.D = 10, 16, 2, 128
    c.stride_page, c.stride_tok, c.stride_head = 16 * 256, 256, 128
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def cache_mx4(**kw):
    c = binding.cp_kv_cache_mx4()
    c.k = c.v = P
    c.num_pages, c.page_size, c.Hkv, c.D = 10, 16, 2, 128
    c.stride_page, c.stride_tok = 16 * 144, 144
    for k, v in kw.items():
        setattr(c, k, v)
    return c


KINDS = {"cp_tree_attn": cache, "cp_tree_attn_fp8": cache_fp8, "cp_tree_attn_mx4": cache_mx4}
BAD_MX4 = ((dict(page_size=48), UNS), (dict(D=64), UNS), (dict(stride_tok=128), BAD), (dict(stride_tok=152), UNS), (dict(stride_page=16 * 144 + 8), UNS),
           (dict(stride_page=0), BAD), (dict(k=P + 8), UNS), (dict(v=P + 4), UNS), (dict(Hkv=0), BAD), (dict(Hkv=4097, stride_tok=1 << 20), UNS), (dict(k=None), BAD),
           (dict(v=None), BAD), (dict(num_pages=0), BAD))


def attn_call(lib, name, c=None, **kw):
    a = dict(q=P, table=P, stride=5, kv_len=P, tree_len=P, mask=P, B=3, n_q=4, Hq=4, window=9, sinks=0, scale=0.1, out=P, lse=P, ws=P, ws_bytes=1 << 30) | kw
    c = c or KINDS[name]()                                   # held while the call reads it
    return getattr(lib, name)(None, a["q"], ctypes.addressof(c), a["table"], a["stride"], a["kv_len"], a["tree_len"], a["mask"], a["B"], a["n_q"], a["Hq"],
                              a["window"], a["sinks"], a["scale"], a["out"], a["lse"], a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("name", KINDS)
def test_tree_attention_refusals(lib, name):
    for kw in (dict(), dict(tree_len=None), dict(n_q=64, Hq=32), dict(B=0, q=None, table=None, kv_len=None, mask=None, out=None, lse=None)):
        assert attn_call(lib, name, **kw) == BAD and b"ctx is NULL" in lib.cp_last_error(), kw
    small, wide = (binding.cp_workspace_bytes_tree(3, n_q, Hq, 2) for n_q, Hq in ((4, 4), (64, 4)))
    for kw, code, word in ((dict(q=None), BAD, b"null"), (dict(table=None), BAD, b"null"), (dict(kv_len=None), BAD, b"null"), (dict(mask=None), BAD, b"null"),
                           (dict(out=None), BAD, b"null"), (dict(lse=None), BAD, b"null"), (dict(mask=P + 4), BAD, b"aligned"), (dict(stride=0), BAD, b"table_stride"),
                           (dict(B=-1), BAD, b"B=-1"), (dict(n_q=0), BAD, b"n_q=0"), (dict(Hq=0), BAD, b"Hq"), (dict(Hq=5), BAD, b"multiple"),
                           (dict(window=0), BAD, b"window"), (dict(sinks=-1), BAD, b"sinks"), (dict(scale=0.0), BAD, b"scale"), (dict(scale=math.nan), BAD, b"scale"),
                           (dict(q=P + 8), BAD, b"aligned"), (dict(out=P + 2), BAD, b"aligned"), (dict(n_q=65), UNS, b"n_q"), (dict(Hq=4096), UNS, b"rows"),
                           (dict(B=65537), UNS, b"B="), (dict(stride=1 << 30), UNS, b"entries"), (dict(ws=None), WSP, b"workspace"), (dict(ws=P + 128), WSP, b"workspace"),
                           (dict(ws_bytes=small - 1), WSP, b"workspace"), (dict(n_q=64, ws_bytes=wide - 1), WSP, b"workspace")):
        assert attn_call(lib, name, **kw) == code and word in lib.cp_last_error(), (kw, lib.cp_last_error())
    make = KINDS[name]
    for kw, code in ((dict(page_size=48), UNS), (dict(D=64), UNS), (dict(k=P + 8), UNS), (dict(Hkv=0), BAD), (dict(k=None), BAD)):
        assert attn_call(lib, name, make(**kw)) == code, kw
    if name == "cp_tree_attn_mx4":
        for kw, code in BAD_MX4:
            assert attn_call(lib, name, make(**kw)) == code, kw


def test_workspace_bytes_tree():
    for args in ((-1, 1, 4, 2), (1, 0, 4, 2), (1, 1, 0, 2), (1, 1, 4, 0), (1, 1, 5, 2), (1, 65, 4, 2), (1, 64, 64, 2), (65537, 1, 4, 2)):
        assert binding.cp_workspace_bytes_tree(*args) == 0 == binding.cp_workspace_bytes_decode(*args), args
    for n_q, Hq in ((1, 2), (8, 4), (9, 4), (16, 4), (17, 4), (64, 32)):
        n = binding.cp_workspace_bytes_tree(5, n_q, Hq, 2)
        assert n % 256 == 0 and n >= binding.cp_workspace_bytes_decode(5, n_q, Hq, 2) > 0


def test_plan_refusals(lib):
    def call(**kw):
        a = dict(parent=P, tree_len=P, kv_len=P, B=3, n_q=8, axes=1, mask=P, pos=P, seq=P, slot=P) | kw
        return lib.cp_tree_plan(None, a["parent"], a["tree_len"], a["kv_len"], a["B"], a["n_q"], a["axes"], a["mask"], a["pos"], a["seq"], a["slot"], None)
    for kw in (dict(), dict(tree_len=None), dict(B=0, parent=None, kv_len=None, mask=None, pos=None, seq=None, slot=None), dict(B=65536, n_q=64, axes=4)):
        assert call(**kw) == BAD and b"ctx is NULL" in lib.cp_last_error(), kw
    for kw, code in ((dict(parent=None), BAD), (dict(kv_len=None), BAD), (dict(mask=None), BAD), (dict(pos=None), BAD), (dict(seq=None), BAD), (dict(slot=None), BAD),
                     (dict(mask=P + 4), BAD), (dict(B=-1), BAD), (dict(n_q=0), BAD), (dict(axes=0), BAD), (dict(axes=5), BAD), (dict(n_q=65), UNS), (dict(B=65537), UNS)):
        assert call(**kw) == code and b"ctx is NULL" not in lib.cp_last_error(), kw


def test_commit_refusals(lib):
    def call(p=None, **kw):
        a = dict(table=P, stride=5, kv_len=P, tree_len=P, parent=P, accepted=P, B=3, n_q=8, path=P) | kw
        p = p or pool()                                      # held while the call reads it
        return lib.cp_tree_commit(None, ctypes.addressof(p), a["table"], a["stride"], a["kv_len"], a["tree_len"], a["parent"], a["accepted"], a["B"], a["n_q"],
                                  a["path"], None)
    for p, kw in ((None, dict()), (None, dict(B=0, table=None, kv_len=None, parent=None, accepted=None, path=None)), (pool(row_bytes=16, stride_head=16, Hkv=9, stride_tok=144), dict()),
                  (pool(row_bytes=128, stride_head=128), dict(tree_len=None, B=65535))):
        assert call(p, **kw) == BAD and b"ctx is NULL" in lib.cp_last_error(), kw
    for kw, code in ((dict(B=-1), BAD), (dict(n_q=0), BAD), (dict(n_q=65), UNS), (dict(B=65536), UNS)):
        assert call(**kw) == code and b"ctx is NULL" not in lib.cp_last_error(), kw
    for kw, code in ((dict(num_pages=0), BAD), (dict(page_size=8), UNS), (dict(row_bytes=64), UNS), (dict(row_bytes=32), UNS), (dict(stride_tok=500), UNS), (dict(n_layers=0), BAD),
                     (dict(layers=129), UNS), (dict(Hkv=0), BAD), (dict(stride_head=8), UNS)):
        assert call(pool(**kw)) == code and b"ctx is NULL" not in lib.cp_last_error(), kw
    for kw in (dict(kv_len=None), dict(parent=None), dict(accepted=None), dict(path=None), dict(table=None), dict(stride=0)):
        assert call(**kw) == BAD, kw


def test_mx4_refusals(lib):
    rope = binding.make_rope([64])

    def append(c=None, **kw):
        a = dict(q=P, k=P, v=P, n=4, Hq=4, pos=P, seq=P, slot=P, table=P, rows=3, stride=5, q_out=2 * P) | kw
        c = c or cache_mx4()
        return lib.cp_rope_append_mx4(None, ctypes.addressof(rope), a["q"], a["k"], a["v"], a["n"], a["Hq"], a["pos"], a["seq"], a["slot"], ctypes.addressof(c),
                                      a["table"], a["rows"], a["stride"], a["q_out"], None)

    def gather(c=None, **kw):
        a = dict(table=P, begin=0, n=5, k=P, v=P) | kw
        c = c or cache_mx4()
        return lib.cp_kv_gather_mx4(None, ctypes.addressof(c), a["table"], a["begin"], a["n"], a["k"], a["v"], None)

    def decode(c=None, **kw):
        a = dict(q=P, table=P, stride=5, kv_len=P, B=3, n_q=1, Hq=4, window=9, sinks=0, scale=0.1, out=P, lse=P, ws=P, ws_bytes=1 << 30) | kw
        c = c or cache_mx4()
        return lib.cp_decode_attn_mx4(None, a["q"], ctypes.addressof(c), a["table"], a["stride"], a["kv_len"], a["B"], a["n_q"], a["Hq"], a["window"], a["sinks"],
                                      a["scale"], a["out"], a["lse"], a["ws"], a["ws_bytes"], None)

    for call in (append, gather, decode):
        assert call() == BAD and b"ctx is NULL" in lib.cp_last_error(), call
        for kw, code in BAD_MX4:
            assert call(cache_mx4(**kw)) == code and b"ctx is NULL" not in lib.cp_last_error(), (call, kw)
    for kw, code in ((dict(k=None), BAD), (dict(q_out=None), BAD), (dict(slot=None), BAD), (dict(q=P + 8), BAD), (dict(n=-1), BAD), (dict(pos=None), BAD), (dict(Hq=0), BAD)):
        assert append(**kw) == code and b"ctx is NULL" not in lib.cp_last_error(), kw
    for kw, code in ((dict(table=None), BAD), (dict(begin=-1), BAD), (dict(n=-1), BAD), (dict(k=P + 8), BAD), (dict(v=P + 8), BAD), (dict(n=1 << 41), UNS), (dict(begin=1 << 41), UNS)):
        assert gather(**kw) == code and b"ctx is NULL" not in lib.cp_last_error(), kw
    for kw, code in ((dict(q=None), BAD), (dict(Hq=5), BAD), (dict(n_q=65), UNS), (dict(ws=None), WSP), (dict(ws_bytes=binding.cp_workspace_bytes_decode(3, 1, 4, 2) - 1), WSP),
                     (dict(scale=math.inf), BAD), (dict(window=0), BAD)):
        assert decode(**kw) == code and b"ctx is NULL" not in lib.cp_last_error(), kw


def test_mx4_layout():
    assert ctypes.sizeof(binding.cp_kv_cache_mx4) == 56
    assert [binding.mx4_token_bytes(h) for h in (1, 2, 3, 4, 8)] == [80, 144, 208, 272, 544]
