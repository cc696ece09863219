"""Refusals of the calls over an 8-bit cache, of drafted trees and of accepted paths, and of the norms with rotation: found on the
host, before anything touches a GPU."""
import ctypes as C

import numpy as np
import pytest

from paper_2505_03756_amd import fllayer, flpool
from paper_2505_03756_amd.flpool import FLP_EINVAL, FLP_ENOTSUP, FLP_ERANGE

AT = 1 << 20                                               # addresses that no check reads


def pool_of(dtype="f16", nkv=2, d=64, bt=16):
    buf = np.zeros(4 * 2 * bt * nkv * d * 4 + 256, np.uint8)
    p = flpool.Pool(dtype, nkv, d, 4, 0, block_tokens=bt, dev=(buf.ctypes.data + 255) & ~255)
    p._buf = buf
    return p


def call(name, pool, cu=(0, 3), prefix=(5,), mb=4, nq=4, q=AT, out=AT, k=None, v=None, ks=AT, vs=AT, mask=AT, taken=AT, path=AT):
    cu, prefix = np.array(cu, np.int32), np.array(prefix, np.int32)
    where = dict(cu_new=cu, prefix_len=prefix, block_tables=AT, max_blocks=mb, stream=0)
    if name == "append8":
        return pool.kv_append8(AT if k is None else k, AT if v is None else v, ks, vs, **where)
    if name == "attn8":
        return pool.paged_prefix_attention8(q, out, ks, vs, n_q_heads=nq, k_new=k, v_new=v, **where)
    if name == "tree":
        return pool.paged_tree_attention(q, out, mask, n_q_heads=nq, k_new=k, v_new=v, **where)
    if name == "tree8":
        return pool.paged_tree_attention(q, out, mask, n_q_heads=nq, k_new=k, v_new=v, k_scale=ks, v_scale=vs, **where)
    return pool.kv_accept(taken, path, kv8=name == "accept8", **where)


def refused(code, text, name, pool, **kw):
    with pytest.raises(flpool.FlpError) as e:
        call(name, pool, **kw)
    assert e.value.code == code and text in str(e.value), str(e.value)


ALL = ("append8", "attn8", "tree", "tree8", "accept", "accept8")


@pytest.mark.parametrize("name", ALL)
def test_sequences(name):
    p = pool_of()
    refused(FLP_EINVAL, "cu_new[0]", name, p, cu=(1, 3))
    refused(FLP_EINVAL, "negative", name, p, cu=(0, -1))
    refused(FLP_EINVAL, "negative", name, p, prefix=(-1,))
    per = 32 if name.endswith("8") else 16
    refused(FLP_ERANGE, "positions", name, p, prefix=(4 * per - 2,))
    refused(FLP_ERANGE, "positions", name, p, mb=0)
    call(name, p, cu=(0, 0), q=None, out=None, mask=None, taken=None, path=None)      # no new tokens: nothing to do
    call(name, p, cu=(0,), prefix=())
    p.close()


@pytest.mark.parametrize("name", [n for n in ALL if n.endswith("8")])
def test_fp32_pools_hold_no_8_bit_cache(name):
    p = pool_of("f32")
    assert p.kv8_block_tokens == 0
    refused(FLP_ENOTSUP, "fp32", name, p)
    p.close()
    for bt in (16, 32):
        p = pool_of("bf16", bt=bt)
        assert p.kv8_block_tokens == 2 * bt
        p.close()


@pytest.mark.parametrize("name", ["append8", "attn8", "tree8"])
def test_scales(name):
    p = pool_of()
    for bad in (None, AT + 2):
        refused(FLP_EINVAL, "scales", name, p, ks=bad)
        refused(FLP_EINVAL, "scales", name, p, vs=bad)
    p.close()


@pytest.mark.parametrize("name", ["attn8", "tree", "tree8"])
def test_attention_arguments(name):
    p = pool_of()
    refused(FLP_EINVAL, "multiple", name, p, nq=3)
    refused(FLP_EINVAL, "multiple", name, p, nq=0)
    for bad in (None, AT + 8):
        refused(FLP_EINVAL, "q/out", name, p, q=bad)
        refused(FLP_EINVAL, "q/out", name, p, out=bad)
    refused(FLP_EINVAL, "k_new", name, p, k=AT)
    refused(FLP_EINVAL, "k_new", name, p, k=AT, v=AT + 8)
    if name != "attn8":
        refused(FLP_EINVAL, "tree_mask", name, p, mask=None)
        refused(FLP_EINVAL, "tree_mask", name, p, mask=AT + 4)
        refused(FLP_ERANGE, "at most 64", name, p, cu=(0, 65), mb=40)
    p.close()


def test_other_arguments():
    p = pool_of()
    refused(FLP_EINVAL, "k_new", "append8", p, k=AT + 4)
    refused(FLP_EINVAL, "n_accept", "accept", p, taken=None)
    refused(FLP_EINVAL, "n_accept", "accept8", p, path=None)
    lib = flpool.load()
    b, keep = p._attn_batch([0, 1], [0], None, 4, 0, None, None, None, None, 0.0)
    b.block_tables = AT
    assert lib.flp_kv_accept(p._h, C.byref(b), AT, AT, 2, None) == FLP_EINVAL
    assert lib.flp_kv_append8(None, C.byref(b), None, None) == FLP_EINVAL
    assert lib.flp_paged_prefix_attention8(p._h, None, None, None) == FLP_EINVAL
    assert lib.flp_paged_tree_attention(p._h, None, None, None, None) == FLP_EINVAL
    assert lib.flp_pool_kv8_block_tokens(None) == 0
    p.close()
    p = pool_of(d=32)
    for name in ALL:
        refused(FLP_ENOTSUP, "head_dim", name, p)
    p.close()


def test_qk_norm_rope_arguments():
    def bad(code, dtype="f16", q=AT, k=AT, wq=AT, wk=AT, pos=AT, qo=AT, ko=AT, T=4, nq=4, nkv=2, d=128, eps=1e-5, theta=1e4, lq=None, lk=None):
        with pytest.raises(flpool.FlpError) as e:
            fllayer.qk_norm_rope(dtype, q, k, wq, wk, pos, qo, ko, T, nq, nkv, d, eps=eps, theta=theta, ld_q_in=lq, ld_k_in=lk, stream=0)
        assert e.value.code == code, str(e.value)
    for kw in (dict(dtype=7), dict(q=AT + 8), dict(k=AT + 4), dict(wq=None), dict(wk=None), dict(wk=AT + 2), dict(pos=None), dict(pos=AT + 1),
               dict(qo=None), dict(ko=AT + 8), dict(T=-1), dict(nq=0), dict(nkv=-1), dict(eps=-1.0), dict(eps=float("nan")),
               dict(theta=0.0), dict(theta=float("inf")), dict(lq=511), dict(lk=100)):
        bad(FLP_EINVAL, **kw)
    bad(FLP_ENOTSUP, d=96)
    bad(FLP_ENOTSUP, lq=4 * 128 + 4)
    fllayer.qk_norm_rope("f16", AT, AT, AT, AT, AT, AT, AT, 0, 4, 2, 128, stream=0)
    fllayer.qk_norm_rope("f16", None, None, None, None, AT, None, None, 4, 4, 2, 128, stream=0)
