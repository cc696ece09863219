"""Infinities and NaN in V that a token sees give the channel that value however small their weight (an infinity that infinity, infinities of
both signs or a NaN a NaN), by every launch of trees over a cache of the pool's type."""
import numpy as np
import pytest

from oracle import step_oracle as so
from paper_2505_03756_amd import workload as wl
from test_gpu_step import Setup, random_tree, same, spread

pytestmark = pytest.mark.gpu

WAYS = [  # name, heads, sequences, launches
    ("few, eight", (8, 2, 128), [(110, 3), (50, 20)], ["rows eight"]),
    ("few, channels apart", (4, 4, 128), [(120, 1)], ["rows eight"]),
    ("few, cut", (8, 2, 128), [(4000, 2), (70, 5)], ["rows cut"]),
    ("few", (4, 4, 128), spread(80, 0, 300, [1]), ["rows packed"]),
    ("row tiles", (16, 4, 64), spread(24, 0, 50, [33, 64, 13, 50, 1]), ["rows row tiles packed"]),
    ("tiles", (64, 4, 128), [(0, 64), (700, 19)] + spread(6, 400, 700, [64, 57]), ["tiles"]),
    ("tiles, packed", (32, 4, 128), [(0, 64), (0, 40), (1, 63)] + spread(27, 0, 500, [64, 40, 57, 1]), ["tiles packed"]),
    ("tiles, cut", (64, 2, 128), [(6001, 64), (500, 19)], ["tiles cut"]),
]


@pytest.mark.parametrize("below", [0.0, 45.0, 115.0])
@pytest.mark.parametrize("kind,bt", [("f32", 16), ("f16", 32), ("bf16", 16)])
@pytest.mark.parametrize("way", WAYS, ids=lambda w: w[0])
def test_infinities_of_any_weight(way, kind, bt, below):
    """The first half of every prefix scores `below` under the rest: 45, a weight that 16 bits do not hold; 115, one that 32 do not."""
    _, heads, seqs, launches = way
    nq, nkv, d = heads
    s = Setup(kind, *heads, seqs, bt=bt, seed=60)
    if kind == "f32" and launches[0].startswith("tiles"):
        pytest.skip("fp32 has no tiled kernel")
    r = np.random.default_rng(61)
    inf, low, nan = wl.quantize(np.array([np.inf, -np.inf, np.nan], np.float32), kind)
    masks = [random_tree(r, n) for _, n in seqs]
    flat = s.image.reshape(-1)
    q = wl.dequantize(s.q, kind).astype(np.float32).reshape(s.T, nq, d)
    q[..., 0] = 8.0
    s.q = wl.quantize(q, kind).reshape(q.shape)
    for i, (p, n) in enumerate(seqs):
        k0 = np.zeros(p + n, np.float32)
        k0[:p // 2] = -below * np.sqrt(d) / 8.0
        at = so.pages(s.image, s.tables[i], np.arange(p + n), nkv, d, s.pb, 0)
        flat[at[:, :, 0]] = wl.quantize(np.repeat(k0[:, None], nkv, 1), kind).reshape(-1, nkv)
        if p < 4:
            continue
        first, last = (so.pages(s.image, s.tables[i], [x], nkv, d, s.pb, 1)[0] for x in (1, p // 2 - 1))
        flat[first[:, 2]], flat[last[:, 3]], flat[last[:, 60]] = inf, low, nan
        flat[first[:, 5]], flat[last[:, 5]] = inf, low
        if n > 1:                                          # and among the drafted tokens, where rows see others: beside those of the prefix
            new = so.pages(s.image, s.tables[i], [p + n // 2], nkv, d, s.pb, 1)[0]
            flat[new[:, 2]], flat[new[:, 3]], flat[new[:, 9]] = low, low, inf
    s.device()
    assert kind == "f32" or s.routes() == launches
    s.tree(masks)
    s.check(lambda i: so.tree(*s.seqs[i], masks[i]))
    assert same(s.now(), s.image)
