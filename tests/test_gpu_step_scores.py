"""Attention over an 8-bit cache and of drafted trees where scores are as large as K's scales and sm_scale may make them: the result is V of the
one largest, the first position's, which every row sees."""
import numpy as np
import pytest
import torch

from oracle import step_oracle as so
from paper_2505_03756_amd import workload as wl
from test_gpu_step import Setup, spread

pytestmark = pytest.mark.gpu

WAYS = [("few", (8, 2, 128), [(300, 3), (2500, 2)]), ("few, of 64", (16, 4, 64), spread(24, 0, 50, [33, 64, 13, 50, 1])),
        ("tiles", (64, 4, 128), [(0, 64)] + spread(7, 400, 700, [64, 57])), ("tiles, cut", (64, 2, 128), [(6001, 64), (500, 19)])]


@pytest.mark.parametrize("size", [2.0 ** 20, 2.0 ** 34], ids=["2^20", "2^34"])
@pytest.mark.parametrize("kind", ["f32", "f16 8", "bf16 8", "f16", "bf16"])
@pytest.mark.parametrize("way", WAYS, ids=lambda w: w[0])
def test_scores_of_any_size(way, kind, size):
    _, (nq, nkv, d), seqs = way
    dtype, kv8 = kind.split()[0], kind.endswith("8")
    s = Setup(dtype, nq, nkv, d, seqs, kv8=kv8, seed=90)
    r = np.random.default_rng(91)
    if kv8:
        s.vs[:] = 64.0
    unit = 32.0 * s.ks.astype(np.float64) if kv8 else np.ones(nkv)       # a value of K that is stored as it is
    for i, (p, n) in enumerate(seqs):
        k, v = np.zeros((2, p + n, nkv, d))
        k[1:, :, 1] = r.integers(-16, 17, (p + n - 1, nkv)) / 16.0
        k[0, :, 0] = 1.0
        v[0] = 28672.0                                     # exact in every type, and as 448 times 64
        k, v = (s.elements(x * u[:, None], sc) for x, u, sc in ((k, unit, s.ks), (v, np.ones(nkv), s.vs)))
        so.store(s.image, s.tables[i], 0, k, v, nkv, d, s.pb)
    q = np.zeros((s.T, nq, d), np.float32)
    q[..., 0], q[..., 1] = 1.37, 0.31                      # products of a score and the scale have more bits than a float
    s.q = wl.quantize(q, dtype).reshape(q.shape)
    s.device()
    s.tree([[(2 << j) - 1 for j in range(n)] for _, n in seqs], sm_scale=size / float(unit.max()))
    torch.cuda.synchronize()
    got = s.out[:s.T].double().cpu().numpy()
    assert np.array_equal(got, np.full_like(got, 28672.0)), (float(got.min()), float(got.max()))
