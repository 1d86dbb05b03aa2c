"""64-bit statements of the operators around the layer: the cast to 8 bits (e4m3) with a scale for each block of 128, the product of
such operands, and attention to an encoder's states.  numpy only; shares no code with the CUDA library."""
from __future__ import annotations

import math

import numpy as np

BLOCK = 128


def e4m3_values():
    """The number that each of the 256 codes stands for: sign, 4 exponent bits (bias 7), 3 mantissa bits; 0x7F and 0xFF are NaN."""
    out = np.zeros(256)
    for code in range(256):
        e, m = (code >> 3) & 15, code & 7
        x = m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        out[code] = math.nan if code & 127 == 127 else x
        if code & 128:
            out[code] = -out[code]
    return out


def quantize(x, block_rows=1):
    """x [rows, cols] -> (values in 8 bits, scales [ceil(rows / block_rows), ceil(cols / 128)])."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    numbers = e4m3_values()[:127]                                        # 0 .. 448, in order
    scale = np.ones((-(-rows // block_rows), -(-cols // BLOCK)))
    out = np.empty_like(x)
    for i in range(scale.shape[0]):
        for j in range(scale.shape[1]):
            w = (slice(i * block_rows, (i + 1) * block_rows), slice(j * BLOCK, (j + 1) * BLOCK))
            b = x[w]
            some = np.abs(b[np.isfinite(b)])
            if some.size and some.max() > 0:
                s = 2.0 ** -126
                while some.max() > 448 * s:
                    s *= 2
                scale[i, j] = s
            y = np.abs(b) / scale[i, j]
            hi = np.searchsorted(numbers, np.where(np.isfinite(y), y, 0.0)).clip(1, 126)
            lo = hi - 1
            up, down = numbers[hi] - y, y - numbers[lo]
            near = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)      # ties to the even code
            out[w] = np.where(np.isfinite(y), np.copysign(numbers[near], b), math.nan)
    return out, scale


def scaled_matmul(a, a_scale, w, w_scale, bias=None, add=None):
    """a [M, K], w [N, K] (values in 8 bits), a_scale [M, blocks], w_scale [ceil(N / 128), blocks] -> (out, sizes): sizes [M, N] is the
    sum of the magnitudes of all terms, what roundings are relative to."""
    a, w = np.asarray(a, np.float64), np.asarray(w, np.float64)
    k = a.shape[1]
    x = a * np.repeat(np.asarray(a_scale, np.float64), BLOCK, 1)[:, :k]
    y = w * np.repeat(np.repeat(np.asarray(w_scale, np.float64), BLOCK, 0)[: w.shape[0]], BLOCK, 1)[:, :k]
    out, size = x @ y.T, np.abs(x) @ np.abs(y).T
    for more in (bias, add):
        if more is not None:
            out, size = out + np.asarray(more, np.float64), size + np.abs(np.asarray(more, np.float64))
    return out, size


def cross_attention(q, k, v, scale, counts=None):
    """One batch row.  q [L, H, d], k, v [n, Hk, d], counts [n] (which keys count) -> out [L, H, d], lse [L, H], and for error bounds
    spread [L, H] = the largest scale sum_c |q_c| |k_c| over the keys, weight [L, H, d] = sum_j p_j |v_j|."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    L, H, d = q.shape
    if counts is not None:
        k, v = k[np.asarray(counts, bool)], v[np.asarray(counts, bool)]
    out, lse = np.zeros((L, H, d)), np.full((L, H), -math.inf)
    spread, weight = np.zeros((L, H)), np.zeros((L, H, d))
    if k.shape[0] == 0:
        return out, lse, spread, weight
    for h in range(H):
        kh, vh = k[:, h // (H // k.shape[1])], v[:, h // (H // k.shape[1])]
        z = scale * q[:, h] @ kh.T
        spread[:, h] = abs(scale) * (np.abs(q[:, h]) @ np.abs(kh).T).max(1)
        top = z.max(1, keepdims=True)
        e = np.exp(z - top)
        lse[:, h] = (top + np.log(e.sum(1, keepdims=True)))[:, 0]
        p = e / e.sum(1, keepdims=True)
        out[:, h], weight[:, h] = p @ vh, p @ np.abs(vh)
    return out, lse, spread, weight
