"""cp_workspace_bytes_decode gives 0 exactly where the call refuses its sizes."""
import ctypes

import pytest

from paper_2609_04774_b200 import binding, build
from tests.test_serving_host import P, cache


@pytest.mark.parametrize("B,n_q,Hq,Hkv", [(65536, 64, 32, 2), (65537, 1, 32, 2), (1, 64, 2, 2), (1, 65, 2, 2), (1, 1, 2048, 2), (1, 1, 2050, 2),
                                          (1, 64, 32, 2), (1, 64, 34, 2), (0, 1, 2, 2), (2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 2, 2)])
def test_zero_where_the_call_refuses(B, n_q, Hq, Hkv):
    build.build()
    lib, c = binding.load(), cache(Hkv=Hkv)
    rc = lib.cp_decode_attn(None, P, ctypes.addressof(c), P, 5, P, B, n_q, Hq, 9, 0, 0.1, P, P, P, 1 << 40, None)
    taken = rc == binding.CP_ERR_INVALID_ARG and b"ctx is NULL" in lib.cp_last_error()       # all but the context is in order
    assert taken or rc == binding.CP_ERR_UNSUPPORTED
    assert (binding.cp_workspace_bytes_decode(B, n_q, Hq, Hkv) > 0) == taken
