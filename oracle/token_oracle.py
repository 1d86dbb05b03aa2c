"""64-bit statements of the token-wise operators: the gated delta rule (Eq. 2) token by token, and rotary positions on three
axes.  numpy only; shares no code with the CUDA library."""
from __future__ import annotations

import numpy as np


def unit(x, eps):
    return x / np.sqrt((x * x).sum(-1, keepdims=True) + eps) if eps > 0 else x


def delta_rule(q, k, v, beta, log_alpha=None, s0=None, scale=1.0, l2_eps=0.0, sizes=None):
    """One sequence.  q, k [N,Hk,d], v [N,H,d], beta, log_alpha [N,H], s0 [H,dv,dk] -> out [N,H,d], state [H,dv,dk].
    `sizes`, a list, receives [N,H]: the root of the summed squares of the terms S_ij q_j of a token's read-out, what
    independent roundings of those terms are relative to.

    Eq. 2:  S_bar = alpha S,   S = S_bar + beta (v - S_bar k) k^T,   o = scale S q;  value head h reads key head h // (H/Hk).
    """
    q, k, v, beta = (np.asarray(x, np.float64) for x in (q, k, v, beta))
    n, h, d = v.shape
    r = h // q.shape[1]
    q, k = np.repeat(unit(q, l2_eps), r, 1), np.repeat(unit(k, l2_eps), r, 1)
    s = np.zeros((h, d, d)) if s0 is None else np.array(s0, np.float64)
    alpha = np.ones((n, h)) if log_alpha is None else np.exp(np.asarray(log_alpha, np.float64))
    out = np.zeros((n, h, d))
    for t in range(n):
        s = alpha[t][:, None, None] * s
        u = beta[t][:, None] * (v[t] - np.einsum("hij,hj->hi", s, k[t]))
        s = s + u[:, :, None] * k[t][:, None, :]
        out[t] = scale * np.einsum("hij,hj->hi", s, q[t])
        if sizes is not None:
            sizes.append(np.abs(scale) * np.sqrt(np.einsum("hij,hj->h", s * s, q[t] * q[t])))
    return out, s


def packed(q, k, v, beta, lens, log_alpha=None, s0=None, scale=1.0, l2_eps=0.0, sizes=None):
    """delta_rule for sequences of `lens` tokens packed one behind another -> out [sum(lens),H,d], state [S,H,dv,dk]."""
    at, outs, states = 0, [], []
    for i, n in enumerate(lens):
        w = slice(at, at + n)
        o, s = delta_rule(q[w], k[w], v[w], beta[w], None if log_alpha is None else log_alpha[w],
                          None if s0 is None else s0[i], scale, l2_eps, sizes)
        outs.append(o)
        states.append(s)
        at += n
    return np.concatenate(outs), np.stack(states)


def rotary(x, positions, freq, axis, half=False, inverse=False, weight=None, norm_eps=0.0):
    """x [tokens, heads, d], positions [3, tokens]: pair p turned by positions[axis[p]] * freq[p]; pairs with another axis
    and channels beyond the pairs stay."""
    x = np.array(x, np.float64)
    if norm_eps > 0:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + norm_eps)
        if weight is not None:
            x = x * np.asarray(weight, np.float64)
    y = x.copy()
    n = len(freq)
    for p in range(n):
        if axis[p] not in (0, 1, 2):
            continue
        angle = np.asarray(positions[axis[p]], np.float64) * float(freq[p])
        c, s = np.cos(angle)[:, None], np.sin(angle)[:, None] * (-1 if inverse else 1)
        i, j = (p, p + n) if half else (2 * p, 2 * p + 1)
        y[..., i] = x[..., i] * c - x[..., j] * s
        y[..., j] = x[..., i] * s + x[..., j] * c
    return y


def grid_positions(B, T, Y, X, t0=0):
    n = np.arange(B * T * Y * X)
    u = n % (Y * X)
    return np.stack([t0 + n // (Y * X) % T, u // X, u % X])
