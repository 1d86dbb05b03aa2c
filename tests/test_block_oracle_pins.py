"""The 64-bit statements of the cast to 8-bit blocks, the block-scaled product and attention to an encoder's states, pinned by examples
worked by hand and by torch's own 8-bit type."""
import math

import numpy as np
import torch

from oracle import block_oracle as blk


def test_codes_are_those_of_the_type():
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(blk.e4m3_values(), want, equal_nan=True)


def test_cast_by_hand():
    x = np.zeros((1, 130))
    x[0, :4] = [448, -224, 17, 0.01]                  # scale 1: 17 lies between 16 and 18, a tie; 0.01 is 5.12 steps of 2^-9
    x[0, 128:] = [449, 15]                            # scale 2: 224.5 -> 224, 7.5 exactly
    y, s = blk.quantize(x)
    assert s.tolist() == [[1.0, 2.0]]
    assert y[0, :4].tolist() == [448, -224, 16, 5 * 2.0 ** -9] and y[0, 128:].tolist() == [224, 7.5]
    assert blk.quantize(np.zeros((3, 5)))[1].tolist() == [[1.0]] * 3


def test_cast_rounds_as_torch_does_and_fills_the_range():
    x = np.random.default_rng(0).standard_normal((64, 300)) * np.exp(np.random.default_rng(1).standard_normal((64, 1)) * 5)
    x = x.astype(np.float32)
    for rows in (1, 128):
        y, s = blk.quantize(x, rows)
        each = np.repeat(np.repeat(s, rows, 0)[:64], 128, 1)[:, :300]
        want = torch.from_numpy(x.astype(np.float64) / each).float().to(torch.float8_e4m3fn).double().numpy()
        assert np.array_equal(y, want)
        top = np.abs(x / each)
        assert top.max() <= 448 and all(top[:, i:i + 128].max(1 if rows == 1 else None).min() > 224 for i in (0, 128, 256))


def test_cast_of_what_is_not_finite():
    x = np.ones((1, 6))
    x[0, :3] = [math.inf, -math.inf, math.nan]
    y, s = blk.quantize(x)
    assert np.isnan(y[0, :3]).all() and s[0, 0] == 2.0 ** -8 and (y[0, 3:] == 256).all()


def test_product_by_hand():
    a, w = np.ones((1, 129)), np.ones((130, 129))
    a[0, 128] = 4
    out, size = blk.scaled_matmul(a, [[2, -1]], w, [[1, 3], [0.5, 1]], bias=np.full(130, 7.0), add=np.full((1, 130), -1.0))
    assert out[0, 0] == 128 * 2 - 4 * 3 + 7 - 1 and out[0, 128] == 128 - 4 + 6 and size[0, 0] == 256 + 12 + 8


def test_attention_by_hand():
    q = np.array([[[1.0, 0.0], [0.0, 1.0]]])                       # one query, two heads on one key head
    k = np.array([[[math.log(3), 0.0]], [[0.0, 0.0]], [[5.0, 5.0]]])
    v = np.array([[[1.0, 2.0]], [[5.0, -2.0]], [[99.0, math.nan]]])
    out, lse, _, _ = blk.cross_attention(q, k, v, 1.0, [1, 1, 0])
    assert np.allclose(out[0], [[2.0, 1.0], [3.0, 0.0]]) and np.allclose(lse[0], np.log([4.0, 2.0]))
    out, lse, _, _ = blk.cross_attention(q, k, v, 1.0, [0, 0, 0])
    assert (out == 0).all() and (lse == -math.inf).all()
