"""CPU oracle of the calls over an 8-bit cache, of drafted trees and of accepted paths (TEST INFRASTRUCTURE ONLY), each the
definition of include/flpool.h and include/fllayer.h written out with numpy in float64:

  e4m3           a sign, 4 bits of exponent (bias 7), 3 of mantissa; no infinities, 0x7f and 0xff are NaN, largest value 448
  append8        byte = e4m3(x / scale of the kv head), the quotient in fp32 and limited to [-448, 448], to nearest even
  attention      out_r = sum_k w_rk V_k, w_r = softmax over the k that r sees of sm_scale q_r . K_k; zeros where it sees nothing
  accept         K and V of position prefix + path[j] move to position prefix + j
  qk_norm_rope   x / sqrt(mean(x^2) + eps) * w, then the pairs (i, i + d/2) turned by pos * theta^(-2i/d)

Caches are lists of per-sequence arrays K, V [length, n_kv, d]; `pages` and `cache_of` go between them and a pool's image.
"""
import numpy as np


def _table():
    b = np.arange(256)
    e, m = (b >> 3) & 15, b & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    v[(b & 127) == 127] = np.nan
    return np.where(b & 128, -v, v)


E4M3 = _table()


def to_e4m3(x):
    """Bytes of the e4m3 numbers nearest to x (ties to the even mantissa), limited to +-448."""
    x = np.asarray(x, dtype=np.float64)
    a = np.minimum(np.abs(x), 448.0)
    grid = E4M3[:127]                                     # ascending; a byte's parity is its mantissa's
    hi = np.clip(np.searchsorted(grid, a), 1, 126)
    lo = hi - 1
    down, up = a - grid[lo], grid[hi] - a
    pick = np.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)
    b = np.where(np.isnan(x), 127, pick) | np.where(np.signbit(x), 128, 0)
    return b.astype(np.uint8)


def quantise(x, scale):
    """x [..., n_kv, d] as float64 values of the element type, scale [n_kv]: bytes."""
    with np.errstate(over="ignore", invalid="ignore"):
        q = np.asarray(x, dtype=np.float32) / np.asarray(scale, dtype=np.float32)[:, None]
    return to_e4m3(q)


def pages(image, table, positions, n_kv, d, pb, part):
    """Flat indices into one tier's image [blocks, elements] of K (part 0) or V (part 1) of the positions: [len, n_kv, d]."""
    pos = np.asarray(positions)
    base = table[pos // pb].astype(np.int64) * image.shape[1]
    s = (pos % pb)[:, None, None]
    g, c = np.arange(n_kv)[None, :, None], np.arange(d)[None, None, :]
    inside = (g * pb + s) * d + c if part == 0 else n_kv * pb * d + (g * d + c) * pb + s
    return base[:, None, None] + inside


def cache_of(image, table, length, n_kv, d, pb):
    """The stored K and V elements of positions 0 .. length - 1."""
    return tuple(image.reshape(-1)[pages(image, table, np.arange(length), n_kv, d, pb, part)] for part in (0, 1))


def store(image, table, first, k, v, n_kv, d, pb):
    pos = first + np.arange(len(k))
    flat = image.reshape(-1)
    flat[pages(image, table, pos, n_kv, d, pb, 0)] = k
    flat[pages(image, table, pos, n_kv, d, pb, 1)] = v


def accept(image, table, prefix, n, taken, path, n_kv, d, pb):
    """In place; an entry outside [0, n) ends the path."""
    k, v = cache_of(image, table, prefix + n, n_kv, d, pb)
    keep = []
    for j in range(min(taken, n)):
        if not 0 <= path[j] < n:
            break
        keep.append(prefix + path[j])
    store(image, table, prefix, k[keep], v[keep], n_kv, d, pb)


def causal(prefix, n):
    return np.arange(prefix + n)[None, :] <= prefix + np.arange(n)[:, None]


def tree(prefix, n, masks):
    """masks: ints, bit j: the token sees new token j."""
    new = np.array([[(int(m) >> j) & 1 for j in range(n)] for m in masks], dtype=bool).reshape(n, n)
    return np.concatenate([np.ones((n, prefix), bool), new], axis=1)


def attention(q, k, v, sees, scale=None):
    """q [n, n_q, d]; k, v [length, n_kv, d]; sees bool [n, length].  Returns the result and, for tolerances, the largest
    sum of |scale q_c K_c| over the keys that a row sees and the largest |V| among finite ones."""
    n, nq, d = q.shape
    nkv = k.shape[1]
    scale = 1 / np.sqrt(d) if scale is None else scale
    out = np.zeros((n, nq, d))
    worst = np.zeros((n, nq))
    for h in range(nq):
        g = h // (nq // nkv)
        with np.errstate(all="ignore"):
            s = q[:, h] @ k[:, g].T * scale
            mag = np.abs(q[:, h]) @ np.abs(k[:, g]).T * scale
        for r in range(n):
            on = sees[r]
            if not on.any():
                continue
            with np.errstate(all="ignore"):
                w = np.exp(s[r, on] - s[r, on].max())
                out[r, h] = w @ v[on, g] / w.sum()
            worst[r, h] = mag[r, on].max()
    fin = np.abs(v[np.isfinite(v)])
    return out, worst, float(fin.max()) if fin.size else 0.0


def qk_norm_rope(x, w, positions, eps, theta):
    """x [T, heads, d], w [d]."""
    d = x.shape[-1]
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w
    ang = np.asarray(positions, np.float64)[:, None] * theta ** (-2.0 * np.arange(d // 2) / d)
    c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
    a, b = y[..., :d // 2], y[..., d // 2:]
    return np.concatenate([a * c - b * s, b * c + a * s], -1)
