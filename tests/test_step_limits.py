"""What the host refuses of the calls over an 8-bit cache, of drafted trees and of the norms with rotation because no launch takes it, and the
entry that tells tests how a batch runs."""
import ctypes as C

import numpy as np
import pytest

from paper_2505_03756_amd import flpool
from test_step_host import pool_of

AT = 1 << 20                                               # an address that no check reads


def route(pool, n_q_heads, cu=(0, 3), prefix=(5,), kv8=0):
    b, keep = pool._attn_batch(np.array(cu, np.int32), np.array(prefix, np.int32), AT, 4, n_q_heads, None, None, None, None, 0.0)
    f = flpool.load().flp_step_attention_route
    f.argtypes = [C.c_void_p, C.c_void_p, C.c_int32]
    return f(pool._h, C.byref(b), kv8)


def test_route_of_bad_batches():
    p = pool_of()
    assert route(p, 4) > 0 and route(p, 4, kv8=1) > 0 and route(p, 4, cu=(0, 0)) == 0
    for heads in (0, -2, 3):
        assert route(p, heads) == -1
    assert route(p, 4, cu=(0, 500)) == -1
    p.close()
