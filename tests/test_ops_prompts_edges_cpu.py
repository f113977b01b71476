"""What the operators that bring prompts into the paged cache refuse besides, before they touch a GPU: memory that a call writes over what it reads or writes elsewhere."""

import ctypes as C

import pytest

from test_ops_prompts_cpu import E, _ops, _rotary

K = E * 4                                                                        # the keys' cache of _rotary: 50 pages of 16 tokens, 2 heads of 64, 2 bytes a number
TURN = dict(k_cache_page=4096, k_cache_token=256, k_cache_head=128, v_cache_page=4096, v_cache_token=256, v_cache_head=128)   # (places between the heads for the other cache's)


@pytest.mark.parametrize("bad", [dict(v_cache=K + 2), dict(v_cache=K - 2), dict(v_cache=K + 128), dict(v_cache=K + 256), dict(v_cache=K + 4096), dict(v_cache=K + 4096 * 50 - 2), dict(v_cache=K - 4096 * 49),
                                 dict(TURN, v_cache=K + 126), dict(TURN, v_cache=K + 130), dict(TURN, v_cache=K + 256), dict(TURN, v_cache=K + 8192 * 49 + 254),
                                 dict(v_cache=K + 256, v_cache_token=64, v_cache_head=1024),   # heads' tokens together, in the keys' pages
                                 # a cache over itself: heads at the next token's, a token's at the next page's
                                 dict(k_cache_token=64), dict(v_cache_head=128), dict(k_cache_page=2047), dict(v_cache_page=128, v_cache_token=100)])
def test_rotary_refuses_caches_over_each_other(bad):
    L, ops = _ops()
    assert L.tbs_rotary(C.byref(_rotary(ops, **bad)), None) == -1
