"""Norms of queries and keys with rotation where the tensors exceed the L2 caches: every type and head size, head counts that end inside a
wave's last heads, in place, and either side alone (tolerance as in test_gpu_step.py)."""
import numpy as np
import pytest
import torch

from oracle import step_oracle as so
from paper_2505_03756_amd import fllayer
from paper_2505_03756_amd import workload as wl
from test_gpu_step import BYTES, TORCH, norm_tolerance, up

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("nq,nkv,d", [(64, 8, 128), (40, 40, 64), (37, 5, 128), (3, 33, 64), (1, 1, 64)])
def test_qk_norm_rope_past_the_caches(dtype, nq, nkv, d):
    T = (32 << 20) // (2 * max(nq, nkv) * d * BYTES[dtype]) + 3        # one side alone exceeds them too
    r = np.random.default_rng(80)
    row, far = (nq + 2 * nkv) * d, 1 << 20
    g = torch.Generator("cuda").manual_seed(81)
    qkv = (torch.randn(T, row, device="cuda", generator=g) * torch.exp(torch.rand(T, 1, device="cuda", generator=g) * 8 - 4)).to(TORCH[dtype])
    wq, wk = (wl.quantize(r.uniform(0.5, 1.5, d).astype(np.float32), dtype) for _ in range(2))
    pos = r.integers(0, far, T).astype(np.int32)
    twq, twk, tp = up(wq), up(wk), up(pos)
    q, k = (torch.full((T + 1, n, d), 7.0, dtype=TORCH[dtype], device="cuda") for n in (nq, nkv))
    fllayer.qk_norm_rope(dtype, qkv, qkv[:, nq * d:], twq, twk, tp, q, k, T, nq, nkv, d, theta=50000.0, ld_q_in=row, ld_k_in=row)
    torch.cuda.synchronize()
    some = np.unique(np.concatenate([np.arange(min(T, 40)), r.integers(0, T, 200), np.arange(max(0, T - 40), T)]))
    at = torch.from_numpy(some).cuda()
    for got, lo, n, w in ((q, 0, nq, wq), (k, nq * d, nkv, wk)):
        xs = qkv[at, lo:lo + n * d].double().cpu().numpy().reshape(len(some), n, d)
        w = wl.dequantize(w, dtype)
        ref = so.qk_norm_rope(xs, w, pos[some], float(np.float32(1e-5)), 50000.0)
        over = np.abs(got[at].double().cpu().numpy() - ref) - norm_tolerance(ref, xs, w, dtype, far)
        assert over.max() <= 0, float(over.max())
        assert bool((got[T:] == 7).all())
    # dense rows in place, and one side alone: the same bits, in every row
    dq, dk = (qkv[:, lo:lo + n * d].clone() for lo, n in ((0, nq), (nq * d, nkv)))
    fllayer.qk_norm_rope(dtype, dq, dk, twq, twk, tp, dq, dk, T, nq, nkv, d, theta=50000.0)
    q2, k2 = torch.zeros_like(q), torch.zeros_like(k)
    fllayer.qk_norm_rope(dtype, qkv, None, twq, None, tp, q2, None, T, nq, 0, d, theta=50000.0, ld_q_in=row)
    fllayer.qk_norm_rope(dtype, None, qkv[:, nq * d:], None, twk, tp, None, k2, T, 0, nkv, d, theta=50000.0, ld_k_in=row)
    torch.cuda.synchronize()
    assert torch.equal(dq.view(T, nq, d), q[:T]) and torch.equal(dk.view(T, nkv, d), k[:T])
    assert torch.equal(q2[:T], q[:T]) and torch.equal(k2[:T], k[:T])
