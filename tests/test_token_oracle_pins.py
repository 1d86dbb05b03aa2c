"""The 64-bit statements of the token-wise operators, pinned by hand-worked numbers, invariants and the frame-wise oracle."""
import numpy as np
import pytest

from oracle import token_oracle as tok
from oracle import vda_oracle as orc


def draw(n, h, d, seed=0, hk=None):
    r = np.random.default_rng(seed)
    f = lambda *s: r.standard_normal(s)
    k = tok.unit(f(n, hk or h, d), 1e-30)
    return tok.unit(f(n, hk or h, d), 1e-30), k, f(n, h, d), 1 / (1 + np.exp(-f(n, h))), -np.exp(f(n, h) - 2)


def test_two_tokens_by_hand():
    """d = 2, keys e1 then (e1 + e2)/sqrt 2, alpha = 1 then 1/2, beta = 1 then 1/2, v = (2, 0) then (0, 4).
    S1 = [[2,0],[0,0]];  decayed [[1,0],[0,0]];  S_bar k = (1/sqrt2, 0);  u = ((0 - .7071)/2, 2) = (-.35355, 2);
    S2 = [[1,0],[0,0]] + u k^T = [[1 - .25, -.25], [1.41421, 1.41421]]."""
    h = 1 / np.sqrt(2)
    q = np.array([[[1.0, 0]], [[0, 1.0]]])
    k = np.array([[[1.0, 0]], [[h, h]]])
    v = np.array([[[2.0, 0]], [[0, 4.0]]])
    out, s = tok.delta_rule(q, k, v, np.array([[1.0], [0.5]]), np.array([[0.0], [np.log(0.5)]]), scale=3.0)
    np.testing.assert_allclose(s[0], [[0.75, -0.25], [2 * h, 2 * h]], atol=1e-15)
    np.testing.assert_allclose(out[:, 0], [[6.0, 0.0], [-0.75, 6 * h]], atol=1e-15)


def test_orthonormal_keys_store_their_values():
    d = 8
    k = np.eye(d)[:, None]
    v = np.random.default_rng(1).standard_normal((d, 1, d))
    out, s = tok.delta_rule(k, k, v, np.ones((d, 1)))
    np.testing.assert_allclose(s[0], v[:, 0].T, atol=1e-14)
    np.testing.assert_allclose(out, v, atol=1e-14)


def test_a_frame_of_one_token_is_the_frame_update():
    """With one token per frame the joint update (S + B)(I + A)^-1 is the token rule with beta / (1 + beta |k|^2)."""
    q, k, v, beta, _ = draw(6, 1, 8, seed=2)
    k = 1.7 * k
    s = np.zeros((8, 8))
    for t in range(6):
        A, B = orc.frame_statistics(k[t], v[t], beta[t])
        s = orc.frame_update(s, np.ones(8), A, B)
    eff = beta / (1 + beta * (k * k).sum(-1))
    np.testing.assert_allclose(tok.delta_rule(q, k, v, eff)[1][0], s, atol=1e-12)


def test_sequences_do_not_see_each_other_and_split_anywhere():
    q, k, v, beta, g = draw(20, 4, 8, seed=3, hk=2)
    out, s = tok.packed(q, k, v, beta, [7, 0, 13], g)
    for w, i in ((slice(0, 7), 0), (slice(7, 20), 2)):
        o1, s1 = tok.delta_rule(q[w], k[w], v[w], beta[w], g[w])
        np.testing.assert_array_equal(out[w], o1)
        np.testing.assert_array_equal(s[i], s1)
    assert not s[1].any()
    o1, s1 = tok.delta_rule(q[:9], k[:9], v[:9], beta[:9], g[:9])
    o2, s2 = tok.delta_rule(q[9:], k[9:], v[9:], beta[9:], g[9:], s0=s1)
    np.testing.assert_allclose(np.concatenate([o1, o2]), tok.delta_rule(q, k, v, beta, g)[0], atol=1e-13)


def test_minus_infinity_forgets():
    q, k, v, beta, g = draw(5, 2, 8, seed=4)
    g[3] = -np.inf
    a = tok.delta_rule(q, k, v, beta, g)[1]
    b = tok.delta_rule(q[3:], k[3:], v[3:], beta[3:], g[3:])[1]
    np.testing.assert_allclose(a, b, atol=1e-14)


def test_rotary_by_hand_and_as_relative_positions():
    x = np.array([[[1.0, 0, 0, 2]]])
    y = tok.rotary(x, np.array([[2], [0], [5]]), [np.pi / 4, np.pi / 10], [0, 2])
    np.testing.assert_allclose(y[0, 0], [0, 1, -2, 0], atol=1e-12)
    y = tok.rotary(x, np.array([[2], [0], [5]]), [np.pi / 4, np.pi / 10], [0, 2], half=True)      # pairs (0,2), (1,3)
    np.testing.assert_allclose(y[0, 0], [0, -2, 1, 0], atol=1e-12)
    r = np.random.default_rng(5)
    q, k = r.standard_normal((1, 1, 12)), r.standard_normal((1, 1, 12))
    freq, axis = [1.0, 0.3, 0.5, 0.1, 0.7, 0.2], [0, 0, 1, 1, 2, 2]
    rot = lambda x, p: tok.rotary(x, np.array(p)[:, None], freq, axis)
    dot = lambda p, c: float((rot(q, p) * rot(k, c)).sum())
    assert dot([4, 7, 9], [1, 5, 2]) == pytest.approx(dot([13, 2, 7], [10, 0, 0]), abs=1e-12)


def test_rotary_inverse_undoes_and_other_axes_stay():
    r = np.random.default_rng(6)
    x, pos = r.standard_normal((7, 3, 10)), r.integers(0, 1000, (3, 7))
    freq, axis = [1.0, 0.1, 0.01, 0.5], [0, 7, 2, 1]
    y = tok.rotary(x, pos, freq, axis)
    np.testing.assert_allclose(tok.rotary(y, pos, freq, axis, inverse=True), x, atol=1e-12)
    np.testing.assert_array_equal(y[..., [2, 3, 8, 9]], x[..., [2, 3, 8, 9]])
    np.testing.assert_array_equal(tok.grid_positions(2, 2, 2, 3, t0=4)[:, [0, 5, 6, 11, 12]],
                                  [[4, 4, 5, 5, 4], [0, 1, 0, 1, 0], [0, 2, 0, 2, 0]])
