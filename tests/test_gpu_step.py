"""The calls over an 8-bit cache, of drafted trees and of accepted paths on the GPU, and the norms with rotation, against the
float64 oracle.

Tolerances.  A result is rounded once, by half a step: HALF * |value|.  Before that, attention's scores are sums of d products in fp32
(off by at most d 2^-24 times the sum of their sizes, `worst`), which moves a weight by as much relative to itself, exp2 by a few
2^-23, the sums of weights by length * 2^-24 and the pieces that a 16-bit weight is held in by 2^-16 (bf16) or less; a weighted mean
of values of size vmax moves by at most twice the weights' relative change times vmax.  In calls that the tiled kernel has a part in
weights may be rounded once to the type of V, fp16 over an 8-bit cache, and summed as rounded: with weights w (1 + e), |e| <= HALF, the
mean moves by at most 2 HALF vmax."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import step_oracle as so
from paper_2505_03756_amd import fllayer, flpool
from paper_2505_03756_amd import workload as wl

pytestmark = pytest.mark.gpu
HALF = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 0.0, "f16": 2.0 ** -25, "bf16": 0.0}           # half the smallest fp16 number
TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}


def up(a):
    a = np.ascontiguousarray(a)
    return torch.from_numpy(a.view(np.int16) if a.dtype == np.uint16 else a.view(np.int64) if a.dtype == np.uint64 else a).cuda()


def same(a, b):
    return np.array_equal(a.view(np.uint8), b.view(np.uint8))


def image_of(t, like):
    a = t.detach().cpu().numpy()
    return a.view(like.dtype)


class Setup:
    """Sequences of (prefix, new) tokens over a pool whose slots hold random K and V up to their lengths and, past them, NaN."""

    def __init__(self, dtype, nq, nkv, d, seqs, kv8=False, bt=16, seed=0, spare=3):
        r = np.random.default_rng(seed)
        self.dtype, self.nq, self.nkv, self.d, self.seqs, self.kv8, self.bt = dtype, nq, nkv, d, seqs, kv8, bt
        self.pb = bt * BYTES[dtype] if kv8 else bt
        P, N = np.array([s[0] for s in seqs]), np.array([s[1] for s in seqs])
        need = -(-(P + N) // self.pb)
        self.n_blocks, mb = int(need.sum()) + spare, max(1, int(need.max()) + 1)
        ids = r.permutation(self.n_blocks)[:need.sum()].astype(np.int32)
        self.tables = np.full((len(seqs), mb), -1, np.int32)
        self.tables[np.arange(mb)[None, :] < need[:, None]] = ids
        self.cu = np.concatenate([[0], np.cumsum(N)]).astype(np.int32)
        self.P = P.astype(np.int32)
        self.T = int(self.cu[-1])
        elems = 2 * self.pb * nkv * d
        if kv8:
            self.image = np.full((self.n_blocks, elems), 127, np.uint8)
            self.ks, self.vs = (r.uniform(0.01, 0.03, nkv).astype(np.float32) for _ in range(2))
        else:
            self.image = np.full((self.n_blocks, elems), np.nan, np.float32)
            self.image = wl.quantize(self.image, dtype).reshape(self.n_blocks, elems)
            self.ks = self.vs = None
        for i, (p, n) in enumerate(seqs):
            k, v = (self.elements(r.standard_normal((p + n, nkv, d)), x) for x in (self.ks, self.vs))
            so.store(self.image, self.tables[i], 0, k, v, nkv, d, self.pb)
        self.q = wl.quantize(r.standard_normal((self.T, nq, d)).astype(np.float32), dtype)
        self.k_new, self.v_new = (wl.quantize(r.standard_normal((self.T, nkv, d)).astype(np.float32), dtype) for _ in range(2))

    def elements(self, x, scale):
        return so.quantise(x, scale) if self.kv8 else wl.quantize(np.asarray(x, np.float32), self.dtype).reshape(np.shape(x))

    def device(self):
        self.t = {n: up(getattr(self, n)) for n in ("image", "tables", "q", "k_new", "v_new")}
        self.t["ks"], self.t["vs"] = (None if s is None else up(s) for s in (self.ks, self.vs))
        self.out = torch.full((self.T + 2, self.nq, self.d), 7.0, dtype=TORCH[self.dtype], device="cuda")
        self.pool = flpool.Pool(self.dtype, self.nkv, self.d, self.n_blocks, 0, block_tokens=self.bt, dev=self.t["image"])
        self.where = (self.cu, self.P, self.t["tables"])
        return self

    def now(self):
        torch.cuda.synchronize()
        return image_of(self.t["image"], self.image)

    def values(self, image, i):
        """K and V of sequence i as float64."""
        p, n = self.seqs[i]
        k, v = so.cache_of(image, self.tables[i], p + n, self.nkv, self.d, self.pb)
        if self.kv8:
            return so.E4M3[k] * self.ks[:, None].astype(np.float64), so.E4M3[v] * self.vs[:, None].astype(np.float64)
        return wl.dequantize(k, self.dtype), wl.dequantize(v, self.dtype)

    def check(self, sees, image=None, scale=None):
        """The rows of `out` against the oracle; sees(i): what the new tokens of sequence i see."""
        image = self.image if image is None else image
        torch.cuda.synchronize()
        got = self.out.double().cpu().numpy()
        assert (got[self.T:] == 7).all(), "rows behind the last sequence were written"
        q = wl.dequantize(self.q, self.dtype)
        once = any(x.startswith("tiles") for x in self.routes())
        for i, (p, n) in enumerate(self.seqs):
            lo, hi = self.cu[i], self.cu[i + 1]
            if lo == hi:
                continue
            k, v = self.values(image, i)
            ref, worst, vmax = so.attention(q[lo:hi], k, v, sees(i), scale)
            pieces = 0 if self.dtype == "f32" else 2 * HALF["f16" if self.kv8 else self.dtype] if once else 2.0 ** -16
            tol = HALF[self.dtype] * np.abs(ref) + TINY[self.dtype] + vmax * (
                2 * (self.d * 2.0 ** -24 * worst + 2.0 ** -20 + (p + n) * 2.0 ** -24) + pieces)[..., None]
            mine = got[lo:hi]
            fin = np.isfinite(ref)
            assert np.array_equal(np.isnan(mine), np.isnan(ref)) and np.array_equal(mine[~fin & ~np.isnan(ref)], ref[~fin & ~np.isnan(ref)]), i
            far = np.abs(mine[fin] - ref[fin])
            assert not far.size or (far - tol[fin]).max() <= 0, (i, (p, n), float((far - tol[fin]).max()), float(far.max()))

    def prefix8(self, append=False, **kw):
        more = dict(k_new=self.t["k_new"], v_new=self.t["v_new"]) if append else {}
        self.pool.paged_prefix_attention8(self.t["q"], self.out, self.t["ks"], self.t["vs"], *self.where, n_q_heads=self.nq, **more, **kw)

    def routes(self):
        """The launches of the batch's attention: kernel, what its waves are side by side on, whether contexts are cut, where the records are."""
        b, keep = self.pool._attn_batch(*self.where, self.tables.shape[1], self.nq, None, None, None, None, 0.0)
        code = flpool.load().flp_step_attention_route(self.pool._h, C.byref(b), int(self.kv8))
        return [" ".join(x for x in (("rows", "tiles")[i], ("", "heads", "row tiles", "eight")[c >> 4], "cut" * (c >> 1 & 1),
                                     ("", "long", "packed", "staged")[c >> 2 & 3]) if x) for i, c in enumerate((code & 255, code >> 8)) if c]

    def tree(self, masks, append=False, **kw):
        more = dict(k_new=self.t["k_new"], v_new=self.t["v_new"]) if append else {}
        if self.kv8:
            more.update(k_scale=self.t["ks"], v_scale=self.t["vs"])
        self.mask = up(np.concatenate([np.asarray(m, np.uint64) for m in masks] + [np.zeros(1, np.uint64)]))
        self.pool.paged_tree_attention(self.t["q"], self.out, self.mask, *self.where, n_q_heads=self.nq, **more, **kw)

    def append_oracle(self):
        image = self.image.copy()
        for i in range(len(self.seqs)):
            lo, hi = self.cu[i], self.cu[i + 1]
            k, v = (a[lo:hi] for a in (self.k_new, self.v_new))
            if self.kv8:
                k, v = so.quantise(wl.dequantize(k, self.dtype), self.ks), so.quantise(wl.dequantize(v, self.dtype), self.vs)
            so.store(image, self.tables[i], int(self.P[i]), k, v, self.nkv, self.d, self.pb)
        return image


HEADS = [(4, 4, 128), (8, 2, 128), (16, 1, 64), (6, 6, 64), (40, 2, 128)]
ENDS = [(0, 1), (0, 33), (1, 31), (15, 17), (31, 1), (32, 1), (33, 64), (63, 2), (0, 0), (64, 70), (100, 7), (127, 129)]


def random_tree(rng, n, prefix=True):
    """Ancestors and itself of every token; some without any bit."""
    seen = []
    for j in range(n):
        parent = int(rng.integers(-1, j)) if j else -1
        seen.append((1 << j) | (seen[parent] if parent >= 0 else 0))
    return [0 if rng.random() < 0.1 else s for s in seen]


# ---------------------------------------------------------------------------------------------------------- append
@pytest.mark.parametrize("bt", [16, 32])
@pytest.mark.parametrize("heads", HEADS[:4])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_append8(dtype, heads, bt):
    s = Setup(dtype, *heads, ENDS, kv8=True, bt=bt, seed=1)
    odd = wl.quantize(np.array([np.nan, np.inf, -np.inf, 1e-9, -0.0, 30000.0, -1e-3], np.float32), dtype)
    flat = s.k_new.reshape(-1)
    flat[::97] = np.resize(odd, flat[::97].shape)
    flat = s.v_new.reshape(-1)
    flat[::89] = np.resize(odd, flat[::89].shape)
    s.device()
    want = s.append_oracle()
    s.pool.kv_append8(s.t["k_new"], s.t["v_new"], s.t["ks"], s.t["vs"], *s.where)
    got = s.now()
    nan = (want & 127) == 127                              # either sign
    assert np.array_equal((got & 127) == 127, nan) and np.array_equal(got[~nan], want[~nan])


@pytest.mark.parametrize("bt", [16, 32])
@pytest.mark.parametrize("heads", [(8, 2, 128), (20, 20, 128), (5, 5, 64)])
def test_append8_of_large_batches(heads, bt):
    """Launches with a workgroup for every CU: runs that are whole and cut, single slots, rows that end inside a workgroup's channels."""
    s = Setup("bf16", *heads, ENDS * 14 + [(5, 1)] * 40 + [(31, 2)] * 9, kv8=True, bt=bt, seed=35).device()
    s.pool.kv_append8(s.t["k_new"], s.t["v_new"], s.t["ks"], s.t["vs"], *s.where)
    assert same(s.now(), s.append_oracle())


def test_append8_past_the_caches():
    """More than the caches hold: the last prompt's K and V against the oracle, and the first one's."""
    n, lens = 18, 2500
    seqs = [(i % 3 * 11, lens) for i in range(n)]
    s = Setup("f16", 50, 50, 64, [seqs[0], seqs[-1]], kv8=True, seed=36)
    one = np.concatenate([s.k_new[:lens], s.k_new[:lens]]), np.concatenate([s.v_new[:lens], s.v_new[:lens]])
    s.device()
    nb = -(-(22 + lens) // 32)
    image = torch.zeros((n * nb, s.image.shape[1]), dtype=torch.uint8, device="cuda")
    pool = flpool.Pool("f16", 50, 64, n * nb, 0, dev=image)
    tables = torch.arange(n * nb, dtype=torch.int32, device="cuda").view(n, nb)
    cu, P = np.arange(n + 1, dtype=np.int32) * lens, np.array([p for p, _ in seqs], np.int32)
    k, v = (up(x[:lens]).repeat(n, 1, 1) for x in one)
    pool.kv_append8(k, v, s.t["ks"], s.t["vs"], cu, P, tables)
    torch.cuda.synchronize()
    for i in (0, 1, n - 1):
        want = np.zeros((nb, s.image.shape[1]), np.uint8)
        kk, vv = (so.quantise(wl.dequantize(x[:lens], "f16"), sc) for x, sc in zip(one, (s.ks, s.vs)))
        so.store(want, np.arange(nb, dtype=np.int32), int(P[i]), kk, vv, 50, 64, 32)
        assert same(image[i * nb:(i + 1) * nb].cpu().numpy(), want), i


def test_append8_of_many_sequences_and_scales():
    """More sequences than travel in a launch's arguments; quotients of many scales, ties among them."""
    r = np.random.default_rng(5)
    s = Setup("f16", 2, 2, 64, [(int(r.integers(0, 90)), int(r.integers(0, 5))) for _ in range(300)], kv8=True, seed=2)
    s.ks, s.vs = np.array([0.015625, 1.0], np.float32), np.array([0.0117, 0.3], np.float32)
    s.k_new = wl.quantize((r.integers(-480, 481, s.k_new.shape) / 16.0 * 0.015625).astype(np.float32), "f16").reshape(s.k_new.shape)
    s.device()
    s.pool.kv_append8(s.t["k_new"], s.t["v_new"], s.t["ks"], s.t["vs"], *s.where)
    assert same(s.now(), s.append_oracle())


# ---------------------------------------------------------------------------------------------------------- 8-bit attention
@pytest.mark.parametrize("bt", [16, 32])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_prefix_attention8(dtype, heads, bt):
    s = Setup(dtype, *heads, ENDS, kv8=True, bt=bt, seed=3).device()
    s.prefix8()
    s.check(lambda i: so.causal(*s.seqs[i]))
    assert same(s.now(), s.image)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("seqs", [[(1, 1)], [(299, 1)], [(5000, 1)], [(4000, 1), (10, 1), (0, 1)], [(3000, 40)], [(2500, 200), (2100, 1)]])
@pytest.mark.parametrize("heads", [(4, 4, 128), (8, 1, 64)])
def test_prefix_attention8_lengths(dtype, seqs, heads):
    """Single tokens, contexts that are cut into pieces, prompts and single tokens together."""
    s = Setup(dtype, *heads, seqs, kv8=True, seed=4).device()
    s.prefix8(append=True)
    image = s.append_oracle()
    assert same(s.now(), image)
    s.check(lambda i: so.causal(*s.seqs[i]), image)


def test_prefix_attention8_of_many_sequences():
    r = np.random.default_rng(6)
    seqs = [(int(r.integers(0, 400)), int(r.integers(0, 3))) for _ in range(250)]
    s = Setup("bf16", 4, 2, 64, seqs, kv8=True, seed=7).device()
    s.prefix8(sm_scale=0.2)
    s.check(lambda i: so.causal(*s.seqs[i]), scale=float(np.float32(0.2)))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("heads", [(4, 4, 128), (16, 2, 128), (4, 4, 64)])
def test_nan_reaches_the_rows_that_see_it(dtype, heads):
    """NaN in K and V of a new token: the tokens before it are as if it were not there."""
    s = Setup(dtype, *heads, [(70, 30), (0, 40), (200, 1)], kv8=True, seed=8)
    for i, pos in ((0, 85), (1, 13)):
        idx = [so.pages(s.image, s.tables[i], [pos], s.nkv, s.d, s.pb, part) for part in (0, 1)]
        s.image.reshape(-1)[idx[1][0, :, 3:60:7]] = 127
        s.image.reshape(-1)[so.pages(s.image, s.tables[i], [pos + 5], s.nkv, s.d, s.pb, 0)[0, 0, :2]] = 255
    s.device()
    s.prefix8()
    s.check(lambda i: so.causal(*s.seqs[i]))


# ---------------------------------------------------------------------------------------------------------- trees
@pytest.mark.parametrize("bt", [16, 32])
@pytest.mark.parametrize("kind", ["f32", "f16", "bf16", "f16 8", "bf16 8"])
@pytest.mark.parametrize("heads", HEADS)
def test_tree_attention(kind, heads, bt):
    """Rows that see nothing, lengths at the ends of blocks and tiles, 64 tokens, masks with bits past the last token."""
    r = np.random.default_rng(9)
    seqs = [(0, 1), (0, 5), (3, 64), (31, 9), (64, 33), (0, 0), (100, 16), (57, 7), (0, 64), (130, 1)]
    s = Setup(kind.split()[0], *heads, seqs, kv8=kind.endswith("8"), bt=bt, seed=10).device()
    masks = [random_tree(r, n) for _, n in seqs]
    s.tree([[m | ~((1 << n) - 1) & (1 << 64) - 1 for m in ms] for ms, (_, n) in zip(masks, seqs)])
    s.check(lambda i: so.tree(*s.seqs[i], masks[i]))
    assert same(s.now(), s.image)


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16", "f16 8", "bf16 8"])
@pytest.mark.parametrize("seqs", [[(3500, 16)], [(2600, 64), (5, 3), (900, 20)]])
def test_tree_attention_long(kind, seqs):
    """Contexts that are cut into pieces, with the tree's K and V stored by the same call."""
    r = np.random.default_rng(11)
    s = Setup(kind.split()[0], 8, 2, 128, seqs, kv8=kind.endswith("8"), seed=12).device()
    masks = [random_tree(r, n) for _, n in seqs]
    s.tree(masks, append=True, sm_scale=0.07)
    image = s.append_oracle()
    assert same(s.now(), image)
    s.check(lambda i: so.tree(*s.seqs[i], masks[i]), image, scale=float(np.float32(0.07)))


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16", "f16 8"])
@pytest.mark.parametrize("heads", [(4, 4, 128), (32, 4, 128), (4, 4, 64)])
def test_tree_keeps_hidden_values_apart(kind, heads):
    """Infinities and NaN in V (and NaN in K) of drafted tokens, and infinities in V of the prefix, where each row sees others."""
    dtype, kv8 = kind.split()[0], kind.endswith("8")
    seqs = [(50, 20), (0, 30), (700, 9)]
    s = Setup(dtype, *heads, seqs, kv8=kv8, seed=13)
    r = np.random.default_rng(14)
    masks = [random_tree(r, n) for _, n in seqs]
    bits = {"f32": np.array([np.nan, np.inf, -np.inf], np.float32)}.get(dtype, wl.quantize(np.array([np.nan, np.inf, -np.inf], np.float32), dtype))
    for i, (p, n) in enumerate(seqs):
        for x, node in enumerate(r.choice(n, 5, replace=False)):
            at = so.pages(s.image, s.tables[i], [p + node], s.nkv, s.d, s.pb, 1)[0]
            s.image.reshape(-1)[at[:, x::9]] = 127 if kv8 else bits[x % 3]
        at = so.pages(s.image, s.tables[i], [p + n - 1], s.nkv, s.d, s.pb, 0)[0]
        s.image.reshape(-1)[at[0, 5]] = 127 if kv8 else bits[0]
        if p and not kv8:                                  # seen by every row, in a tile that all rows see whole
            s.image.reshape(-1)[so.pages(s.image, s.tables[i], [7], s.nkv, s.d, s.pb, 1)[0, :, 2]] = bits[1]
    s.device()
    s.tree(masks)
    s.check(lambda i: so.tree(*s.seqs[i], masks[i]))


# ---------------------------------------------------------------------------------------------------------- every way to run them
def spread(n, lo, hi, new, seed=0):
    """n sequences: prefixes of lo .. hi, the new tokens in turns."""
    r = np.random.default_rng(seed)
    return [(int(r.integers(lo, hi + 1)), new[i % len(new)]) for i in range(n)]


WAYS = [  # name, heads, sequences, the launches in 16 bits, and in 8
    ("few", (4, 4, 128), spread(80, 0, 300, [1]), ["rows packed"], ["rows packed"]),
    ("few, cut", (4, 2, 64), [(2300, 2), (40, 3)], ["rows cut"], ["rows cut"]),
    ("few, cut, long list", (1, 1, 128), [(4000, 1)] + spread(40, 0, 70, [1, 2]), ["rows cut long"], ["rows cut long"]),
    ("few, cut, staged", (2, 1, 128), [(4000, 3)] + spread(120, 0, 70, [1, 2, 0]) + spread(30, 0, 70, [1]), ["rows cut staged"], ["rows cut staged"]),
    ("heads", (10, 5, 64), spread(270, 0, 60, [1, 2, 0, 3, 1]), ["rows heads packed"], ["rows heads packed"]),
    ("heads, staged", (10, 5, 64), spread(250, 0, 90, [1]), ["rows heads staged"], ["rows heads staged"]),
    ("row tiles", (16, 4, 64), spread(24, 0, 50, [33, 64, 13, 50, 1]), ["rows row tiles packed"], ["rows row tiles packed"]),
    ("row tiles, few sequences", (64, 4, 64), spread(8, 0, 50, [33, 64, 13, 50]), ["rows row tiles"], ["rows row tiles"]),
    ("tiles", (64, 4, 128), [(0, 64), (700, 19)] + spread(6, 400, 700, [64, 57]), ["tiles"], ["tiles"]),
    ("tiles, packed", (32, 4, 128), [(0, 64), (0, 40), (1, 63)] + spread(27, 0, 500, [64, 40, 57, 1]), ["tiles packed"], ["tiles packed"]),
    ("tiles, staged", (8, 1, 128), spread(230, 0, 200, [64, 40]), ["tiles staged"], ["tiles staged"]),
    ("tiles, cut", (64, 2, 128), [(6001, 64), (500, 19)], ["tiles cut"], ["tiles cut"]),
    ("tiles, cut, long list", (16, 1, 128), spread(12, 1500, 2100, [64, 39]), ["tiles cut long"], ["tiles cut long"]),
    ("both", (32, 4, 128), spread(16, 300, 700, [64]) + spread(70, 300, 900, [1, 2]), ["rows packed", "tiles packed"], ["rows packed", "tiles packed"]),
]


@pytest.mark.parametrize("kind,bt", [("f16", 32), ("bf16", 16), ("f16 8", 16), ("bf16 8", 32)])
@pytest.mark.parametrize("way", WAYS, ids=lambda w: w[0])
def test_trees_every_way(way, kind, bt):
    """Trees by every launch that the plan knows, tokens without any bit and K and V that are not finite and hidden from some rows among them."""
    _, heads, seqs, in16, in8 = way
    dtype, kv8 = kind.split()[0], kind.endswith("8")
    s = Setup(dtype, *heads, seqs, kv8=kv8, bt=bt, seed=30)
    r = np.random.default_rng(31)
    masks = [random_tree(r, n) for _, n in seqs]
    bits = [127] * 3 if kv8 else wl.quantize(np.array([np.nan, np.inf, -np.inf], np.float32), dtype)
    flat = s.image.reshape(-1)
    for i, (p, n) in enumerate(seqs):
        if i % 3 == 0 and n > 1:
            for x in range(3):
                at = so.pages(s.image, s.tables[i], [p + int(r.integers(0, n))], s.nkv, s.d, s.pb, 1)[0]
                flat[at[:, 5 * x::31]] = bits[x]
        if i % 4 == 0 and n > 1:
            flat[so.pages(s.image, s.tables[i], [p + n - 1], s.nkv, s.d, s.pb, 0)[0, -1, 9]] = bits[0]
    s.device()
    assert s.routes() == (in8 if kv8 else in16)
    s.tree(masks)
    s.check(lambda i: so.tree(*s.seqs[i], masks[i]))
    assert same(s.now(), s.image)


PROMPTS = [
    ("tiles", (8, 8, 128), [(1000, 700), (0, 800), (333, 600), (77, 65), (10, 1)], ["tiles"]),
    ("tiles, packed", (16, 2, 128), spread(24, 0, 500, [350, 164, 397, 1]), ["tiles packed"]),
    ("tiles, cut", (16, 2, 128), [(3000, 300)], ["tiles cut"]),
    ("tiles, cut, from nothing", (16, 1, 128), [(0, 1500)], ["tiles cut"]),
    ("row tiles", (16, 4, 64), spread(24, 0, 100, [33, 64, 13, 90, 1]), ["rows row tiles packed"]),
]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("bt", [16, 32])
@pytest.mark.parametrize("way", PROMPTS, ids=lambda w: w[0])
def test_prompts_every_way(way, bt, dtype):
    """Prompts over the 8-bit cache, NaN in V of a few new tokens (the rows before them do not see it)."""
    _, heads, seqs, launches = way
    s = Setup(dtype, *heads, seqs, kv8=True, bt=bt, seed=32)
    for i, (p, n) in enumerate(seqs):
        if i % 2 == 0 and n > 30:
            for x, at in enumerate((n // 3, n - 2)):
                s.image.reshape(-1)[so.pages(s.image, s.tables[i], [p + at], s.nkv, s.d, s.pb, 1)[0, :, 3 + x::17]] = 127 + 128 * x
    s.device()
    assert s.routes() == launches
    s.prefix8()
    s.check(lambda i: so.causal(*s.seqs[i]))


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16 8"])
def test_blocks_far_into_a_large_pool(kind):
    """Blocks more than 2^32 bytes behind the pool's base: stored, read by both kernels and moved."""
    dtype, kv8 = kind.split()[0], kind.endswith("8")
    seqs = spread(8, 0, 700, [64, 41, 17])
    s = Setup(dtype, 32, 4, 128, seqs, kv8=kv8, seed=33)
    r = np.random.default_rng(34)
    masks = [random_tree(r, n) for _, n in seqs]
    image = s.append_oracle()
    s.device()
    block = s.image[0].nbytes
    before = (5 << 30) // block
    big = torch.zeros((before + s.n_blocks) * block, dtype=torch.uint8, device="cuda")
    big[before * block:] = s.t["image"].view(torch.uint8).reshape(-1)
    s.t["image"] = big[before * block:]
    far = np.where(s.tables >= 0, s.tables + before, -1).astype(np.int32)
    s.pool = flpool.Pool(dtype, 4, 128, before + s.n_blocks, 0, block_tokens=16, dev=big)
    s.where = (s.cu, s.P, up(far))
    s.tree(masks, append=True)
    assert same(s.now().reshape(-1), image.reshape(-1))
    s.check(lambda i: so.tree(*s.seqs[i], masks[i]), image)
    taken, path = np.zeros(len(seqs), np.int32), np.full(s.T, -1, np.int32)
    for i, (p, n) in enumerate(seqs):
        taken[i] = n // 2
        path[s.cu[i]:s.cu[i] + taken[i]] = np.sort(r.choice(n, taken[i], replace=False))
        so.accept(image, s.tables[i], p, n, int(taken[i]), path[s.cu[i]:s.cu[i + 1]], s.nkv, s.d, s.pb)
    s.pool.kv_accept(up(taken), up(path), *s.where, kv8=kv8)
    assert same(s.now().reshape(-1), image.reshape(-1)) and not bool(big[:before * block].any())


# ---------------------------------------------------------------------------------------------------------- accepted paths
@pytest.mark.parametrize("bt", [16, 32])
@pytest.mark.parametrize("kind", ["f32", "f16", "bf16", "f16 8"])
@pytest.mark.parametrize("heads", [(4, 4, 128), (3, 3, 64), (40, 40, 128)])
def test_accept(kind, heads, bt):
    r = np.random.default_rng(15)
    seqs = [(int(r.integers(0, 100)), int(r.integers(0, 65))) for _ in range(130)]
    s = Setup(kind.split()[0], *heads, seqs, kv8=kind.endswith("8"), bt=bt, seed=16)
    taken, path, want = np.zeros(len(seqs), np.int32), np.full(s.T, -5, np.int32), s.image.copy()
    for i, (p, n) in enumerate(seqs):
        m = int(r.integers(0, n + 1))
        path[s.cu[i]:s.cu[i] + m] = np.sort(r.choice(n, m, replace=False)) if n else []
        taken[i] = m
        if m > 3 and i % 5 == 0:                           # an entry that is none ends the path; more taken than there are
            path[s.cu[i] + 2] = n if i % 2 else -1
            taken[i] = n + 7
        so.accept(want, s.tables[i], p, n, int(taken[i]), path[s.cu[i]:s.cu[i + 1]], s.nkv, s.d, s.pb)
    s.device()
    s.pool.kv_accept(up(taken), up(path), *s.where, kv8=s.kv8)
    assert same(s.now(), want)


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16 8"])
def test_accept_of_long_paths(kind):
    """More tokens than a tree has: paths over many blocks, some of which the first 64 table entries do not hold."""
    r = np.random.default_rng(18)
    seqs = [(7, 300), (0, 2500), (30, 90), (5, 0)]
    s = Setup(kind.split()[0], 4, 2, 64, seqs, kv8=kind.endswith("8"), seed=19)
    taken, path, want = np.array([200, 1200, 90, 1], np.int32), np.full(s.T, -1, np.int32), s.image.copy()
    for i, (p, n) in enumerate(seqs):
        m = min(n, int(taken[i]))
        path[s.cu[i]:s.cu[i] + m] = np.sort(r.choice(n, m, replace=False)) if n else []
        so.accept(want, s.tables[i], p, n, int(taken[i]), path[s.cu[i]:s.cu[i + 1]], s.nkv, s.d, s.pb)
    s.device()
    s.pool.kv_accept(up(taken), up(path), *s.where, kv8=s.kv8)
    assert same(s.now(), want)


# ---------------------------------------------------------------------------------------------------------- norms and rotation
def norm_tolerance(ref, x, w, dtype, far):
    """Norm: the sum of squares and the factors are off by a few 2^-24; the angle's fraction by 2^-24 of a turn in fp32 (2 pi) and far
    2^-52 in fp64; sine and cosine by as much as the larger of the pair."""
    d = x.shape[-1]
    size = np.abs(so.qk_norm_rope(x, w, np.zeros(len(x)), 1e-5, 1e4))
    pair = np.maximum(size, np.roll(size, d // 2, -1))
    return HALF[dtype] * np.abs(ref) + TINY[dtype] + pair * (2 * (2 * np.pi + 8 + d / 8) * 2.0 ** -24 + far * 2.0 ** -50)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("nq,nkv,d", [(4, 4, 128), (64, 8, 128), (5, 3, 64), (1, 1, 128), (40, 40, 64)])
@pytest.mark.parametrize("T", [1, 7, 700])
def test_qk_norm_rope(dtype, nq, nkv, d, T):
    r = np.random.default_rng(17)
    row = (nq + 2 * nkv) * d
    x = wl.quantize(r.standard_normal((T, row)).astype(np.float32) * np.exp(r.uniform(-4, 4, (T, 1))).astype(np.float32), dtype).reshape(T, row)
    x[-1, :d] = 0                                          # a head of zeros
    wq, wk = (wl.quantize(r.uniform(0.5, 1.5, d).astype(np.float32), dtype) for _ in range(2))
    far = 1 << 20
    pos = r.integers(0, far, T).astype(np.int32)
    pos[0] = 0
    qkv, q, k = up(x), *(torch.full((T + 1, n, d), 7.0, dtype=TORCH[dtype], device="cuda") for n in (nq, nkv))
    twq, twk, tp = up(wq), up(wk), up(pos)
    fllayer.qk_norm_rope(dtype, qkv, qkv[:, nq * d:], twq, twk, tp, q, k, T, nq, nkv, d, theta=50000.0, ld_q_in=row, ld_k_in=row)
    torch.cuda.synchronize()
    assert same(image_of(qkv, x), x)
    xd = wl.dequantize(x, dtype)
    for got, lo, n, w in ((q, 0, nq, wq), (k, nq * d, nkv, wk)):
        xs, w = xd[:, lo:lo + n * d].reshape(T, n, d), wl.dequantize(w, dtype)
        ref = so.qk_norm_rope(xs, w, pos, float(np.float32(1e-5)), 50000.0)
        g = got.double().cpu().numpy()
        assert (g[T:] == 7).all()
        over = np.abs(g[:T] - ref) - norm_tolerance(ref, xs, w, dtype, far)
        assert over.max() <= 0, float(over.max())
    # dense rows in place, and one side alone: the same bits
    dq, dk = (qkv[:, lo:lo + n * d].clone() for lo, n in ((0, nq), (nq * d, nkv)))
    fllayer.qk_norm_rope(dtype, dq, dk, twq, twk, tp, dq, dk, T, nq, nkv, d, theta=50000.0)
    k2 = torch.zeros_like(k)
    fllayer.qk_norm_rope(dtype, None, qkv[:, nq * d:], None, twk, tp, None, k2, T, 0, nkv, d, theta=50000.0, ld_k_in=row)
    torch.cuda.synchronize()
    assert torch.equal(dq.view(TORCH[dtype]).view(T, nq, d), q[:T]) and torch.equal(dk.view(TORCH[dtype]).view(T, nkv, d), k[:T])
    assert torch.equal(k2[:T], k[:T])
    fllayer.qk_norm_rope(dtype, qkv, None, twq, None, tp, k2, None, 0, nq, 0, d)      # no tokens


# ---------------------------------------------------------------------------------------------------------- together
@pytest.mark.parametrize("kv8", [False, True])
def test_a_speculative_step(kv8):
    """Norms and rotation of a draft's fused rows, its K and V stored, the tree verified, the accepted path kept, and the next token's
    attention over what was kept: as if the accepted tokens had been decoded one after the other."""
    dtype, nq, nkv, d = "f16", 8, 2, 128
    seqs = [(37, 12), (0, 7), (250, 30), (64, 1)]
    s = Setup(dtype, nq, nkv, d, seqs, kv8=kv8, seed=20)
    s.device()
    r = np.random.default_rng(21)
    parents = [[int(r.integers(-1, j)) if j else -1 for j in range(n)] for _, n in seqs]
    masks, depth, paths = [], [], []
    for par in parents:
        m, dep = [], []
        for j, p in enumerate(par):
            m.append((1 << j) | (m[p] if p >= 0 else 0))
            dep.append(dep[p] + 1 if p >= 0 else 0)
        j, path = int(r.integers(0, len(par))), []
        while j >= 0:
            path.insert(0, j)
            j = par[j]
        masks.append(m), depth.append(dep), paths.append(path)
    row = (nq + 2 * nkv) * d
    qkv = torch.randn(s.T, row, device="cuda", generator=torch.Generator("cuda").manual_seed(3)).to(TORCH[dtype])
    w = torch.ones(d, device="cuda", dtype=TORCH[dtype])
    pos = up(np.concatenate([p + np.array(dep) for (p, _), dep in zip(seqs, depth)]).astype(np.int32))
    q, k = (torch.empty(s.T, n, d, device="cuda", dtype=TORCH[dtype]) for n in (nq, nkv))
    v = qkv[:, (nq + nkv) * d:].contiguous()
    fllayer.qk_norm_rope(dtype, qkv, qkv[:, nq * d:], w, w, pos, q, k, s.T, nq, nkv, d, ld_q_in=row, ld_k_in=row)
    s.t["q"], s.t["k_new"], s.t["v_new"] = q, k, v
    s.q, s.k_new, s.v_new = (image_of(x, np.zeros(1, np.uint16)) for x in (q, k, v.view(s.T, nkv, d)))
    s.tree(masks, append=True)
    image = s.append_oracle()
    assert same(s.now(), image)
    s.check(lambda i: so.tree(*seqs[i], masks[i]), image)
    path, taken = np.full(s.T, -1, np.int32), np.array([len(p) for p in paths], np.int32)
    for i, p in enumerate(paths):
        path[s.cu[i]:s.cu[i] + len(p)] = p
        so.accept(image, s.tables[i], seqs[i][0], seqs[i][1], len(p), p, nkv, d, s.pb)
    s.pool.kv_accept(up(taken), up(path), *s.where, kv8=kv8)
    assert same(s.now(), image)
    # the last accepted token again, as the one new token of its sequence: its row is the one that the tree gave it
    tree_out = s.out.clone()
    last = np.array([s.cu[i] + p[-1] for i, p in enumerate(paths)])
    P2, cu2 = s.P + taken - 1, np.arange(len(seqs) + 1)
    q2, out2 = q[up(last)].contiguous(), torch.zeros(len(seqs), nq, d, device="cuda", dtype=TORCH[dtype])
    if kv8:
        s.pool.paged_prefix_attention8(q2, out2, s.t["ks"], s.t["vs"], cu2, P2, s.t["tables"], n_q_heads=nq)
    else:
        s.pool.paged_prefix_attention(q2, out2, cu2, P2, s.t["tables"], nq)
    torch.cuda.synchronize()
    a, b = out2.double(), tree_out[up(last)].double()
    assert float((a - b).abs().max()) <= 2 * HALF[dtype] * float(b.abs().max()) + 1e-4


def test_capture_and_replay():
    """Calls without staging and without pieces in a HIP graph; others are refused under capture and enqueue nothing."""
    seqs = [(100, 8), (0, 5), (333, 3)]
    s = Setup("f16", 8, 2, 128, seqs, kv8=True, seed=22).device()
    r = np.random.default_rng(23)
    masks = [random_tree(r, n) for _, n in seqs]
    taken, path = up(np.array([2, 1, 0], np.int32)), up(np.array([1, 4, 0, 0, 0, 0, 0, 0, 3, 0, 0, 0, 0, 0, 0, 0], np.int32))
    s.tree(masks, append=True)
    s.pool.kv_accept(taken, path, *s.where, kv8=True)
    torch.cuda.synchronize()
    want_out, want_image, start = s.out.clone(), s.t["image"].clone(), up(s.image)
    g = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.graph(g, stream=side):
        more = dict(k_new=s.t["k_new"], v_new=s.t["v_new"], k_scale=s.t["ks"], v_scale=s.t["vs"])
        s.pool.paged_tree_attention(s.t["q"], s.out, s.mask, *s.where, n_q_heads=8, **more)
        s.pool.kv_accept(taken, path, *s.where, kv8=True)
        long = np.array([0, 1], np.int32), np.array([300000], np.int32), torch.zeros(1, 10000, dtype=torch.int32, device="cuda")
        with pytest.raises(flpool.FlpError) as e:
            s.pool.paged_prefix_attention8(s.t["q"], s.out, s.t["ks"], s.t["vs"], *long, n_q_heads=8)
        assert e.value.code == flpool.FLP_ENOTSUP
    for _ in range(3):
        s.t["image"].copy_(start)
        s.out.fill_(7)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(s.t["image"], want_image) and torch.equal(s.out, want_out)


def test_two_streams_share_the_pieces_workspace():
    """Two calls whose contexts are cut into pieces, on two streams of one pool, one behind the other."""
    s = Setup("bf16", 8, 2, 128, [(4000, 2), (3000, 3)], kv8=True, seed=24).device()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.full_like(s.out, 7.0) for _ in range(8)]
    torch.cuda.synchronize()
    for i, out in enumerate(outs):
        s.pool.paged_prefix_attention8(s.t["q"], out, s.t["ks"], s.t["vs"], *s.where, n_q_heads=8, stream=streams[i % 2])
    torch.cuda.synchronize()
    s.out = outs[0]
    s.check(lambda i: so.causal(*s.seqs[i]))
    assert all(torch.equal(o, outs[0]) for o in outs)


def test_replays_between_eager_calls():
    """A captured step of more sequences than the short list holds, replayed between eager calls that cut contexts on the same pool."""
    seqs = spread(40, 0, 300, [1, 4, 0, 9])
    s = Setup("bf16", 8, 2, 128, seqs, kv8=True, seed=40).device()
    r = np.random.default_rng(41)
    masks = [random_tree(r, n) for _, n in seqs]
    s.tree(masks, append=True)
    torch.cuda.synchronize()
    want_out, want_image, start = s.out.clone(), s.t["image"].clone(), up(s.image)
    long = np.array([0, 2], np.int32), np.array([4000], np.int32)
    blocks = torch.randint(0, s.n_blocks, (1, 200), dtype=torch.int32, device="cuda")
    q, eager = s.t["q"][:2].contiguous(), torch.zeros(2, 8, 128, dtype=torch.bfloat16, device="cuda")
    cut = lambda: s.pool.paged_prefix_attention8(q, eager, s.t["ks"], s.t["vs"], *long, blocks, n_q_heads=8)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        more = dict(k_new=s.t["k_new"], v_new=s.t["v_new"], k_scale=s.t["ks"], v_scale=s.t["vs"])
        s.pool.paged_tree_attention(s.t["q"], s.out, s.mask, *s.where, n_q_heads=8, **more)
    first = None
    for i in range(5):
        s.t["image"].copy_(start)
        s.out.fill_(7)
        g.replay()
        cut()
        torch.cuda.synchronize()
        first = eager.clone() if first is None else first
        assert torch.equal(s.t["image"], want_image) and torch.equal(s.out, want_out), i
        assert same(eager.view(torch.int16).cpu().numpy(), first.view(torch.int16).cpu().numpy()), i


def test_threads_share_a_pool():
    """Two threads, each with a stream and calls of its own kind on one pool: cut contexts, staged lists and single launches."""
    import threading
    s = Setup("f16", 8, 2, 128, [(4000, 2), (3000, 3)] + spread(230, 0, 40, [1]), kv8=True, seed=42).device()
    single = Setup("f16", 8, 2, 128, [(50, 1)], kv8=True, seed=43).device()
    want = []
    for x in (s, single):
        x.prefix8()
        x.check(lambda i: so.causal(*x.seqs[i]))
        want.append(x.out.clone())
    failures = []

    def run(mine):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                for i in range(60):
                    x, w = ((s, want[0]), (single, want[1]))[(i + mine) % 3 == 0]
                    out = torch.full_like(w, 3.0)
                    out[x.T:] = 7
                    x.pool.paged_prefix_attention8(x.t["q"], out, x.t["ks"], x.t["vs"], *x.where, n_q_heads=8, stream=stream)
                    stream.synchronize()
                    if not torch.equal(out, w):
                        failures.append((mine, i))
        except Exception as e:                             # a thread's own would be lost
            failures.append(repr(e))

    torch.cuda.synchronize()
    threads = [threading.Thread(target=run, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failures


@pytest.mark.parametrize("kind", ["f16", "f16 8"])
def test_sequences_that_share_blocks(kind):
    """Drafts of several sequences over one shared prefix, and one sequence that is listed three times."""
    s = Setup(kind.split()[0], 8, 2, 128, [(96, 7), (96, 12), (96, 1), (96, 7), (96, 7)], kv8=kind.endswith("8"), seed=44)
    whole = 96 // s.pb
    s.tables[:, :whole] = s.tables[0, :whole]
    s.tables[3:] = s.tables[0]
    r = np.random.default_rng(45)
    masks = [random_tree(r, n) for _, n in s.seqs]
    s.device()
    s.tree(masks)
    s.check(lambda i: so.tree(*s.seqs[i], masks[i]))
    assert same(s.now(), s.image)
