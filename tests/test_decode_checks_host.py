"""What the speculative decode step's calls refuse before any device call: memory that its kernels could not read."""
import ctypes
import os

import pytest

from paper_2609_05228_gb300 import ace, build

INVALID = 1


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(ace.LIBPATH):
        build.build()
    ace._lib = None
    return ace.lib()


@pytest.mark.parametrize("head_dim,dtype", [(64, ace.ACE_BF16), (128, ace.ACE_BF16), (80, ace.ACE_F32)])
@pytest.mark.parametrize("ks,vs", [(17, 16), (16, 33), (24, 16), (16, 20), (18, 18)])
def test_create_refuses_scales_that_are_not_aligned(L, head_dim, dtype, ks, vs):
    out = ctypes.c_void_p(7)
    d = ace.ace_kv_desc(1, 4, 16, 2, head_dim, dtype, ace.ACE_KV_FP8)
    assert L.ace_kv_create(ctypes.byref(d), 16, 16, ks, vs, None, ctypes.byref(out)) == INVALID
    assert out.value is None and b"scales" in L.ace_last_error_message()
