"""Workspaces of the sizes that bf16 and E4M3 decode calls took before there were 4-bit caches are still enough for them."""
import ctypes

import pytest

from paper_2609_04774_b200 import binding, build
from test_serving_host import P, cache
from test_tree_host import cache_fp8, cache_mx4

# 2 pieces x 384 CTAs x 2 heads x rows of a unit, 130 floats each, and 16 bytes a CTA
KEPT = {8: 6395904, 16: 12785664, 32: 25565184}


@pytest.mark.parametrize("Hkv", [1, 2, 3, 4, 8])
@pytest.mark.parametrize("rows", [1, 8, 9, 16, 17, 40])
def test_sizes(Hkv, rows):
    build.build()
    lib = binding.load()
    kept = KEPT[8 if rows <= 8 else (16 if rows <= 16 else 32)]

    def call(name, make, ws_bytes):
        c = make(Hkv=Hkv, stride_tok=1 << 14, stride_page=1 << 18)
        rc = getattr(lib, name)(None, P, ctypes.addressof(c), P, 5, P, 3, 1, rows * Hkv, 9, 0, 0.1, P, P, P, ws_bytes, None)
        if rc == binding.CP_ERR_WORKSPACE:
            return False
        assert rc == binding.CP_ERR_INVALID_ARG and b"ctx is NULL" in lib.cp_last_error()
        return True

    for name, make in (("cp_decode_attn", cache), ("cp_decode_attn_fp8", cache_fp8)):
        assert call(name, make, kept) and not call(name, make, kept - 1)
    size = binding.cp_workspace_bytes_decode(3, 1, rows * Hkv, Hkv)
    assert size >= kept
    for name, make in (("cp_decode_attn", cache), ("cp_decode_attn_fp8", cache_fp8), ("cp_decode_attn_mx4", cache_mx4)):
        assert call(name, make, size)
    assert not call("cp_decode_attn_mx4", cache_mx4, size - 1)
    assert binding.cp_workspace_bytes_tree(3, 1, rows * Hkv, Hkv) >= size
