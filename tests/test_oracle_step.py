"""Pins of the step oracle: e4m3's numbers, rounding and limits, and attention's masks, from values worked out by hand."""
import numpy as np
import pytest

from oracle import step_oracle as so


def test_e4m3_numbers():
    assert so.E4M3[0x00] == 0 and so.E4M3[0x01] == 2.0 ** -9 and so.E4M3[0x07] == 7 * 2.0 ** -9
    assert so.E4M3[0x08] == 2.0 ** -6 and so.E4M3[0x38] == 1.0 and so.E4M3[0x39] == 1.125 and so.E4M3[0x7e] == 448
    assert np.isnan(so.E4M3[0x7f]) and np.isnan(so.E4M3[0xff]) and so.E4M3[0xb8] == -1.0
    assert np.all(np.diff(so.E4M3[:127]) > 0)
    finite = np.delete(np.arange(256), [127, 255])
    back = so.to_e4m3(so.E4M3[finite])
    assert np.array_equal(so.E4M3[back], so.E4M3[finite]) and np.array_equal(back, finite)      # -0.0 keeps its sign


@pytest.mark.parametrize("x,want", [(1.0625, 0x38), (1.1875, 0x3a), (1.07, 0x39), (2.0 ** -10, 0x00), (3 * 2.0 ** -10, 0x02),
                                    (2.1 ** -9, 0x01), (449.0, 0x7e), (1e9, 0x7e), (np.inf, 0x7e), (-np.inf, 0xfe), (464.0, 0x7e),
                                    (np.nan, 0x7f), (-0.0, 0x80)])
def test_e4m3_rounding(x, want):
    assert so.to_e4m3(x) == want


def test_e4m3_agrees_with_torch():
    import torch
    x = torch.cat([torch.randn(20000) * s for s in (0.003, 0.1, 3.0, 100.0)] + [torch.arange(-448, 449) / 16.0])
    want = x.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(so.to_e4m3(x.numpy()), want)


def test_attention_by_hand():
    """Equal scores: the mean of what a row sees; one score ln 3 above the other: three quarters and a quarter."""
    v = np.array([[1.0, 0], [2, 0], [4, 8]]).reshape(3, 1, 2)
    k = np.zeros((3, 1, 2))
    q = np.ones((2, 1, 2))
    out, _, _ = so.attention(q, k, v, so.causal(1, 2))
    assert np.allclose(out[:, 0], [[1.5, 0], [7 / 3, 8 / 3]])
    out, _, _ = so.attention(q, k, v, so.tree(1, 2, [0b10, 0b01]))
    assert np.allclose(out[:, 0], [[2.5, 4], [1.5, 0]])
    out, _, _ = so.attention(q, k[1:], v[1:], so.tree(0, 2, [0, 0b10]))
    assert np.array_equal(out[0, 0], [0, 0]) and np.allclose(out[1, 0], [4, 8])
    k[2, 0] = [np.log(3), 0]
    out, _, _ = so.attention(q, k, v, np.array([[True, False, True]] * 2), scale=1.0)
    assert np.allclose(out[0, 0], [0.25 + 3, 6])


def test_accept_and_layout():
    image = np.arange(3 * 2 * 2 * 4 * 3).reshape(3, -1)       # 2 kv heads, 3 channels, 4 positions per block
    table = np.array([2, 0])
    k, v = so.cache_of(image, table, 6, 2, 3, 4)
    assert k[0, 0, 0] == 96 and k[1, 0, 0] == 99 and k[0, 1, 0] == 108 and v[0, 0, 0] == 120 and v[1, 0, 0] == 121 and k[4, 0, 0] == 0
    before = image.copy()
    so.accept(image, table, 1, 5, 3, [0, 2, 4, -1, -1], 2, 3, 4)
    k2, v2 = so.cache_of(image, table, 6, 2, 3, 4)
    assert np.array_equal(k2, k[[0, 1, 3, 5, 4, 5]]) and np.array_equal(v2, v[[0, 1, 3, 5, 4, 5]])
    assert np.array_equal(image[1], before[1])


def test_norm_rope_by_hand():
    x = np.array([3.0, 4.0]).reshape(1, 1, 2)
    y = so.qk_norm_rope(x, np.array([1.0, 2.0]), [0], 0.0, 10000.0)
    assert np.allclose(y, np.array([3, 8]) / np.sqrt(12.5))
    y = so.qk_norm_rope(np.tile(x, (2, 1, 1)), np.ones(2), [0, 1], 0.0, 10000.0)
    assert np.allclose(y[1, 0], np.array([3 * np.cos(1) - 4 * np.sin(1), 4 * np.cos(1) + 3 * np.sin(1)]) / np.sqrt(12.5))
