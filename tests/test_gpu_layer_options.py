"""A whole decoder layer with its options (norms of queries and keys, drafted trees, the cache in 8 bits, and all of them) against the
layer oracle with these steps of it replaced by the step oracle's."""
import numpy as np
import pytest
import torch

from oracle import layer_oracle as lo
from oracle import step_oracle as so
from paper_2505_03756_amd import fllayer, flpool
from paper_2505_03756_amd import workload as wl
from paper_2505_03756_amd.harness import GpuStep, resident_pool, to_dev, to_np
from test_gpu_layer import ULP, layer_cfg, make_weights

pytestmark = pytest.mark.gpu

CASES = {
    "f16_norms": (layer_cfg("f16", new_range=(1, 40), seed=61), ("norms",)),
    "f32_norms_and_tree": (layer_cfg("f32", n_seqs=3, prefix_range=(0, 60), new_range=(1, 20), hidden=256, n_q_heads=2, n_kv_heads=2,
                                     mlp_dim=512, n_dev_blocks=300, seed=62), ("norms", "tree")),
    "bf16_tree": (layer_cfg("bf16", n_q_heads=8, n_kv_heads=2, hidden=1024, new_range=(1, 64), seed=63), ("tree",)),
    "f16_cache8_prompts_and_tokens": (layer_cfg("f16", decode_frac=0.5, seed=64), ("cache8",)),
    "bf16_all": (layer_cfg("bf16", n_q_heads=8, n_kv_heads=2, hidden=1024, new_range=(1, 30), projections=("q", "k", "v", "o"),
                           seed=65), ("norms", "tree", "cache8")),
}


@pytest.mark.parametrize("name", list(CASES))
def test_layer_with_options(name, monkeypatch):
    cfg, has = CASES[name]
    step = wl.make_step(cfg)
    T, d, nkv, nh = step.n_tokens, cfg.head_dim, cfg.n_kv_heads, cfg.n_q_heads
    r = np.random.default_rng(66)
    new = np.diff(step.cu_new)
    pool0 = resident_pool(step)
    W = make_weights(cfg, np.random.default_rng(7))
    h0, _ = lo.round_store(np.random.default_rng(8).normal(0, 1, (T, cfg.hidden)), cfg.dtype)
    norms = [lo.round_store(r.uniform(0.7, 1.4, d), cfg.dtype)[0] for _ in range(2)]
    scales = [r.uniform(0.005, 0.02, nkv).astype(np.float32) for _ in range(2)]
    masks, depth = [], []
    for n in new:
        parent = [int(r.integers(-1, j)) if j else -1 for j in range(n)]
        m, dep = [], []
        for j, p in enumerate(parent):
            m.append((1 << j) | (m[p] if p >= 0 else 0))
            dep.append(dep[p] + 1 if p >= 0 else 0)
        masks.append(m)
        depth.append(dep if "tree" in has else list(range(n)))
    pos = np.concatenate([step.prefix_len[i] + np.array(depth[i]) for i in range(cfg.n_seqs)]).astype(np.int32)
    kv8 = "cache8" in has
    pb = 2 * cfg.block_tokens if kv8 else cfg.block_tokens
    cache = lambda image: image.view(np.uint8).reshape(len(image), -1) if kv8 else image

    def stored(x, scale):                                  # values [n, nkv, d] -> the cache's elements
        return so.quantise(x, scale) if kv8 else lo.round_store(x, cfg.dtype)[0]

    def values(x, scale):
        return so.E4M3[x] * scale[:, None].astype(np.float64) if kv8 else lo.load(x, cfg.dtype)

    if kv8:                                                # the prefixes' blocks hold 16-bit numbers: quantise some
        for i in range(cfg.n_seqs):
            k, v = (stored(r.standard_normal((step.prefix_len[i], nkv, d)), s) for s in scales)
            so.store(cache(pool0), step.kv_tables[i], 0, k, v, nkv, d, pb)

    # the oracle's layer with these steps in the place of its own
    if "norms" in has:
        turn = iter(norms)
        monkeypatch.setattr(lo, "rope", lambda x, p, theta: so.qk_norm_rope(x, lo.load(next(turn), cfg.dtype), p, 1e-5, theta))

    def append(image, dt, bt, n_kv, d_, cu, prefix, tables, k, v):
        for i in range(cfg.n_seqs):
            rows = slice(cu[i], cu[i + 1])
            ke, ve = (stored(lo.load(x[rows], cfg.dtype), s) for x, s in zip((k, v), scales))
            so.store(cache(image), tables[i], int(prefix[i]), ke, ve, nkv, d, pb)

    def attend(image, dt, bt, n_kv, d_, n_q, cu, prefix, tables, q):
        out = np.zeros((T, nh, d))
        for i in range(cfg.n_seqs):
            rows, n, p = slice(cu[i], cu[i + 1]), int(new[i]), int(prefix[i])
            k, v = (values(x, s) for x, s in zip(so.cache_of(cache(image), tables[i], p + n, nkv, d, pb), scales))
            out[rows] = so.attention(lo.load(q[rows], cfg.dtype), k, v, so.tree(p, n, masks[i]) if "tree" in has else so.causal(p, n))[0]
        return out

    monkeypatch.setattr(lo, "_kv_append", append)
    monkeypatch.setattr(lo, "_paged_attention", attend)
    image = pool0.copy()
    want_st, _ = lo.layer_forward(cfg, step, image, W, h0, pos)
    want = lo.load(want_st, cfg.dtype)

    g = GpuStep(step, pool0, np.zeros((1, cfg.block_elems), pool0.dtype))
    layer = fllayer.Layer(g.pool, cfg.hidden, nh, cfg.mlp_dim, {k: to_dev(v) for k, v in W.items()})
    batch = fllayer.Batch(step.cu_new, step.prefix_len, to_dev(pos), g.kv_tables, g.token_adapter, g.rank, g.scale, g.lora_tables, g.proj,
                          n_adapters=len(step.rank), max_rank=int(step.rank.max()), max_blocks_per_seq=step.kv_tables.shape[1])
    nbytes = layer.scratch_bytes(T)
    scratch = torch.zeros(nbytes + 256, dtype=torch.uint8, device="cuda")
    opt = {}
    if "norms" in has:
        opt.update(q_norm=to_dev(norms[0]), k_norm=to_dev(norms[1]))
    if "tree" in has:
        opt["tree_mask"] = to_dev(np.array([m for ms in masks for m in ms], np.uint64).view(np.int64))
    if kv8:
        opt.update(k_scale=to_dev(scales[0]), v_scale=to_dev(scales[1]))
    h = to_dev(h0)
    layer.forward(batch, h, (scratch.data_ptr() + 255) & ~255, nbytes, **opt)
    torch.cuda.synchronize()
    got = lo.load(to_np(h, h0.dtype), cfg.dtype)
    # As in the plain layer's test a tensor between two steps may land on a neighbouring number, which the steps behind it carry on:
    # 8 spacings at the value or at 1 (fp32: 512 of its own for its arithmetic, as 1e-4 and 1e-5 there).  In 8 bits a neighbouring K or V
    # may also lie on the other side of a border of e4m3; behind the output projection, a sum over all heads and channels, such a
    # spacing of one element is below the same bound.
    tol = 8 * ULP[cfg.dtype] * np.maximum(np.abs(want), 1.0) * (64 if cfg.dtype == "f32" else 1)
    assert (np.abs(got - want) <= tol).all(), float((np.abs(got - want) / tol).max())


def test_options_refused():
    cfg = layer_cfg("f32", n_seqs=2, prefix_range=(0, 20), new_range=(66, 70), hidden=256, n_q_heads=2, n_kv_heads=2, mlp_dim=512,
                    n_dev_blocks=300, seed=67)
    step = wl.make_step(cfg)
    g = GpuStep(step, resident_pool(step), np.zeros((1, cfg.block_elems), np.float32))
    W = make_weights(cfg, np.random.default_rng(7))
    layer = fllayer.Layer(g.pool, cfg.hidden, 2, cfg.mlp_dim, {k: to_dev(v) for k, v in W.items()})
    pos = to_dev(np.zeros(step.n_tokens, np.int32))
    batch = fllayer.Batch(step.cu_new, step.prefix_len, pos, g.kv_tables, g.token_adapter, g.rank, g.scale, g.lora_tables, g.proj,
                          n_adapters=len(step.rank), max_rank=int(step.rank.max()), max_blocks_per_seq=step.kv_tables.shape[1])
    nbytes = layer.scratch_bytes(step.n_tokens)
    scratch = torch.zeros(nbytes + 256, dtype=torch.uint8, device="cuda")
    h = to_dev(np.zeros((step.n_tokens, cfg.hidden), np.float32))
    at = h.data_ptr()
    for code, opt in ((flpool.FLP_EINVAL, dict(q_norm=at)), (flpool.FLP_EINVAL, dict(k_norm=at)), (flpool.FLP_EINVAL, dict(v_scale=at)),
                      (flpool.FLP_EINVAL, dict(q_norm=at, k_norm=at + 4)), (flpool.FLP_EINVAL, dict(tree_mask=at + 4)),
                      (flpool.FLP_ENOTSUP, dict(k_scale=at, v_scale=at)), (flpool.FLP_ERANGE, dict(tree_mask=at))):
        with pytest.raises(flpool.FlpError) as e:
            layer.forward(batch, h, (scratch.data_ptr() + 255) & ~255, nbytes, **opt)
        assert e.value.code == code
    torch.cuda.synchronize()
    assert not h.any()
