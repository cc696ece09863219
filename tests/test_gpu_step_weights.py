"""Attention over an 8-bit cache and of drafted trees where a few keys take nearly all of the weight and have V = 0: the result is what the many
small weights leave.

Tolerances, relative to the result, whose terms have one sign.  A weight is held to U of itself or to 2^-35 of the largest, whichever is more
(fp16: weights are 2^10 at the running maximum, so half the smallest step, 2^-25, is 2^-35 of it; bf16 has no such end): U is half a step
squared where it is held in two pieces, half a step where the tiled kernel has a part in the call.  Numerator and sum of the weights are both
off by that.  Scores are sums of d products in fp32, d 2^-24 of their terms' sizes; exponents up to 64 are rounded by 2^-19 a few times; sums of n
terms by n 2^-24; the result by half a step."""
import numpy as np
import pytest
import torch

from oracle import step_oracle as so
from paper_2505_03756_amd import workload as wl
from test_gpu_step import HALF, TINY, Setup, spread

pytestmark = pytest.mark.gpu

WAYS = [
    ("few, eight", (8, 2, 128), [(700, 2), (90, 20), (0, 3)], True),
    ("few, cut", (4, 2, 64), [(2300, 2), (40, 3)], True),
    ("few, heads", (10, 5, 64), spread(270, 0, 60, [1, 2, 0, 3, 1]), True),
    ("few, row tiles", (16, 4, 64), spread(24, 0, 50, [33, 64, 13, 50, 1]), True),
    ("tiles", (64, 4, 128), [(0, 64), (700, 19)] + spread(6, 400, 700, [64, 57]), True),
    ("tiles, cut", (64, 2, 128), [(6001, 64), (500, 19)], True),
    ("prompts", (16, 2, 128), spread(24, 0, 500, [350, 164, 397, 1]), False),
]


def concentrated(kind, heads, seqs, gap, wide, every, bt=16):
    """Every `every`-th position has V = 0 and a score `gap` above the others', which are spread over +-wide; their V is large, or the result
    would be below what fp16 holds."""
    dtype, kv8 = kind.split()[0], kind.endswith("8")
    nq, nkv, d = heads
    s = Setup(dtype, *heads, seqs, kv8=kv8, bt=bt, seed=50)
    r = np.random.default_rng(51)
    if kv8:
        s.vs[:] = 64.0
    unit = 32.0 * s.ks.astype(np.float64) if kv8 else np.ones(nkv)       # a value of K that is stored as it is
    for i, (p, n) in enumerate(seqs):
        sink = np.arange(p + n) % every == 0
        k, v = np.zeros((2, p + n, nkv, d))
        k[:, :, 1] = r.integers(-16, 17, (p + n, nkv)) / 16.0
        k[sink] = 0.0
        k[sink, :, 0] = 1.0
        v[:] = r.integers(8, 15, v.shape) * 2048.0                       # exact in every type, 8-bit ones times 64 too
        v[sink] = 0.0
        k, v = (s.elements(x * u[:, None], sc) for x, u, sc in ((k, unit, s.ks), (v, np.ones(nkv), s.vs)))
        so.store(s.image, s.tables[i], 0, k, v, nkv, d, s.pb)
    q = np.zeros((s.T, nq, d), np.float32)
    per = np.repeat(unit, nq // nkv) / np.sqrt(d)
    q[:, :, 0], q[:, :, 1] = gap / per, wide / per
    q[:, :, 2:] = r.standard_normal((s.T, nq, d - 2))                    # meets zeros
    s.q = wl.quantize(q, dtype).reshape(q.shape)
    return s


def check(s, sees, once, only=None):
    torch.cuda.synchronize()
    got = s.out.double().cpu().numpy()
    q = wl.dequantize(s.q, s.dtype)
    of = "f16" if s.kv8 else s.dtype
    u, a = HALF[of] ** (1 if once else 2), 2.0 ** -35 if of == "f16" else 0.0
    G, worst_of = s.nq // s.nkv, 0.0
    for i, (p, n) in enumerate(s.seqs[:only]):
        lo, hi, length = s.cu[i], s.cu[i + 1], p + n
        k, v = s.values(s.image, i)
        on = sees(i)
        for h in range(s.nq if n else 0):
            g = h // G
            mag = (np.abs(q[lo:hi, h]) @ np.abs(k[:, g]).T).max(-1) / np.sqrt(s.d)
            x = np.where(on, q[lo:hi, h] @ k[:, g].T / np.sqrt(s.d), -np.inf)
            w = np.exp(x - x.max(-1, keepdims=True))
            total = w.sum(-1, keepdims=True)
            ref = w @ v[:, g] / total
            held = a * (on @ np.abs(v[:, g]) + on.sum(-1, keepdims=True) * ref) / total
            rel = HALF[s.dtype] + 2 * (u + (s.d * 2.0 ** -24 * mag + 2.0 ** -17 + length * 2.0 ** -24)[:, None])
            far = np.abs(got[lo:hi, h] - ref) / (rel * ref + held + TINY[s.dtype] + 1e-300)
            assert np.isfinite(got[lo:hi, h]).all() and far.max() <= 1, (i, (p, n), h, float(far.max()))
            worst_of = max(worst_of, float(far.max()))
    return worst_of


@pytest.mark.parametrize("gap,wide", [(14.1, 0.0), (17.0, 1.5), (22.0, 0.0)])
@pytest.mark.parametrize("kind", ["f16", "bf16", "f16 8", "bf16 8"])
@pytest.mark.parametrize("way", WAYS, ids=lambda w: w[0])
def test_small_weights_by_every_launch(way, kind, gap, wide):
    """One position in 32 takes nearly all of the weight, so that every tile of every piece has one."""
    _, heads, seqs, trees = way
    if not trees and not kind.endswith("8"):
        pytest.skip("prompts over a 16-bit cache are flp_paged_prefix_attention's")
    s = concentrated(kind, heads, seqs, gap, wide, 32)
    s.device()
    once = any(x.startswith("tiles") for x in s.routes())
    assert once == (way[0].startswith(("tiles", "prompts")))
    if trees:                                              # drafts that are one branch each
        masks = [[(2 << j) - 1 for j in range(n)] for _, n in seqs]
        s.tree(masks)
    else:
        s.prefix8()
    check(s, lambda i: so.causal(*s.seqs[i]), once)


@pytest.mark.parametrize("kind", ["f16", "f16 8", "bf16 8"])
def test_one_key_above_a_long_context(kind):
    """The first of 16385 positions takes nearly all of the weight: a batch of single tokens over one shared context, not cut."""
    s = concentrated(kind, (8, 8, 64), [(16384, 1)], 14.1, 0.0, 1 << 20)
    S = 64
    s.seqs, s.T = s.seqs * S, S
    s.tables = np.repeat(s.tables, S, 0)
    s.cu, s.P = np.arange(S + 1, dtype=np.int32), np.repeat(s.P, S)
    s.q = np.repeat(s.q, S, 0)
    s.device()
    assert not any("cut" in x or "tiles" == x[:5] for x in s.routes()), s.routes()
    s.tree([[1]] * S)
    check(s, lambda i: so.causal(*s.seqs[i]), False, 1)
    assert bool((s.out[:S] == s.out[:1]).all())


@pytest.mark.parametrize("up", [100, -100])
@pytest.mark.parametrize("way", [("few", (8, 2, 128), [(300, 3), (2500, 2)]), ("tiles", (64, 4, 128), [(0, 64)] + spread(7, 400, 700, [64, 57])),
                                 ("tiles, cut", (64, 2, 128), [(6001, 64), (500, 19)])], ids=lambda w: w[0])
def test_scales_at_the_ends_of_their_range(way, up):
    """K's scale of 2^100 under queries of 2^-100 and the other way round, and V's scales of 2^100 and 2^-100."""
    _, heads, seqs = way
    s = Setup("bf16", *heads, seqs, kv8=True, seed=52)
    s.ks[:], s.vs[:] = 2.0 ** up, 2.0 ** up
    s.q = wl.quantize((wl.dequantize(s.q, "bf16") * 2.0 ** -up / 64).astype(np.float32).reshape(s.q.shape), "bf16").reshape(s.q.shape)
    s.device()
    s.tree([[(2 << j) - 1 for j in range(n)] for _, n in seqs])
    s.check(lambda i: so.causal(*s.seqs[i]))
