"""What the host refuses of the calls over an 8-bit cache, of drafted trees and of the norms with rotation because no launch takes it, and the
entry that tells tests how a batch runs."""
import ctypes as C

import numpy as np
import pytest

from paper_2505_03756_amd import fllayer, flpool
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


def refused(text, f, *args, **kw):
    with pytest.raises(flpool.FlpError) as e:
        f(*args, **kw)
    assert e.value.code == flpool.FLP_ERANGE and text in str(e.value), str(e.value)


def test_more_new_tokens_than_an_append_takes():
    """The runtime counts a launch's threads in 32 bits: 2^24 runs of 32 positions."""
    p = pool_of(nkv=1)
    n = 1 << 29
    where = dict(cu_new=np.array([0, n, n + n], np.int32), prefix_len=np.zeros(2, np.int32), block_tables=AT, max_blocks=n // 32, stream=0)
    refused("new tokens", p.kv_append8, AT, AT, AT, AT, **where)
    where["cu_new"][2] = n
    refused("new tokens", p.kv_append8, AT, AT, AT, AT, **where)
    refused("new tokens", p.paged_prefix_attention8, AT, AT, AT, AT, n_q_heads=1, k_new=AT, v_new=AT, **where)
    p.close()


@pytest.mark.parametrize("dtype,T,nq,nkv,d", [("f16", 1 << 28, 1, 0, 64), ("bf16", 1 << 27, 0, 33, 128), ("f32", 2**31 - 1, 4, 4, 64)])
def test_more_heads_than_a_norm_takes(dtype, T, nq, nkv, d):
    q, k = AT if nq else None, AT if nkv else None
    refused("more heads", fllayer.qk_norm_rope, dtype, q, k, AT, AT, AT, q, k, T, nq, nkv, d, stream=0)
