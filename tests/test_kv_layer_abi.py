"""What hero_layer_fwd_kv refuses before anything is launched (no GPU needed), beside tests/test_kv_cache_abi.py."""
import ctypes as C

import pytest

from paper_2310_17723_amd import binding as HB
from test_kv_cache_abi import P, UNSUPPORTED, _cache, lib  # noqa: F401


@pytest.mark.parametrize("mask", [-1, 3, 7])
def test_a_mask_that_is_none(lib, mask):  # noqa: F811
    """(Any but the causal one was taken for no mask.)"""
    d = HB.LayerDesc(HB.ARCH_PRE_LN, 128, 2, 64, 256, 1e-5, mask, HB.MODE_M1)
    io = HB._LAYER_IO.pack(3, 1, 0, 0, 0, 0, P, P, 0, 0, 0, 0, 0, 0, 0)
    assert lib.hero_layer_fwd_kv(d, HB.LayerWeights(), io, _cache(), None, C.c_void_p(P), 1 << 30, None) == UNSUPPORTED
