"""The fp64 oracle of the gated-delta layer, pinned by closed forms and by
library routines on special cases (no GPU)."""
import numpy as np
import scipy.signal
import scipy.special
import scipy.stats

import oracle


def _rand(seed, *shape):
    return np.random.default_rng(seed).standard_normal(shape)


def test_delta_is_the_product_of_its_transitions():
    """S_T = sum_t (prod_{s>t} M_s) beta_t k_t v_t^T + (prod M_s) S_0, M = a (I - beta k k^T)."""
    T, K, V = 7, 5, 3
    q, k, v = _rand(1, T, 1, K), _rand(2, T, 1, K) * 0.4, _rand(3, T, 1, V)
    g, beta, h0 = -np.abs(_rand(4, T, 1)), np.random.default_rng(5).random((T, 1)), _rand(6, 1, K, V)
    S = h0[0].copy()
    want = []
    for t in range(T):
        kt = k[t, 0][:, None]
        S = np.exp(g[t, 0]) * (np.eye(K) - beta[t, 0] * kt @ kt.T) @ S + beta[t, 0] * kt @ v[t]
        want.append(0.3 * q[t, 0] @ S)
    o, hT = oracle.delta(q, k, v, g, beta, h0, scale=0.3)
    assert np.allclose(hT[0], S, rtol=1e-12, atol=1e-13)
    assert np.allclose(o[:, 0], np.stack(want), rtol=1e-12, atol=1e-13)


def test_delta_special_cases():
    K, V = 6, 4
    eye, v = np.eye(K)[:, None], _rand(7, K, 1, V)
    _, S = oracle.delta(eye, eye, v)                     # orthonormal keys, beta 1: the values by rows
    assert np.allclose(S[0], v[:, 0])
    o, S = oracle.delta(eye[[0, 0]], eye[[0, 0]], v[:2], scale=1.0)  # the same key: the last value
    assert np.allclose(o[:, 0], v[:2, 0]) and np.allclose(S[0, 0], v[1, 0])
    h0 = _rand(8, 1, K, V)
    _, S = oracle.delta(eye, eye, v, np.full((K, 1), -0.25), np.zeros((K, 1)), h0)  # beta 0: only decay
    assert np.allclose(S, h0 * np.exp(-0.25 * K))
    # a prefix's state continues the sequence, and normalised keys have no length
    q, k, v = _rand(9, 9, 2, K), _rand(10, 9, 2, K), _rand(11, 9, 4, V)
    o, S = oracle.delta(q, k, v, qk_norm=True, eps=0.0)
    o1, S1 = oracle.delta(q[:4], k[:4] * 7, v[:4], qk_norm=True, eps=0.0)
    o2, S2 = oracle.delta(q[4:] * 3, k[4:], v[4:], h0=S1, qk_norm=True, eps=0.0)
    assert np.allclose(np.concatenate([o1, o2]), o, rtol=1e-12, atol=1e-13) and np.allclose(S2, S, atol=1e-13)
    # value heads share the key heads in order
    alone, _ = oracle.delta(q[:, 1:], k[:, 1:], v[:, 2:], qk_norm=True, eps=0.0)
    assert np.allclose(alone, o[:, 2:])


def test_conv_is_a_filter():
    T, D, W = 20, 3, 4
    x, w, b, tail = _rand(12, T, D), _rand(13, D, W), _rand(14, D), _rand(15, W - 1, D)
    y, t = oracle.conv(x, w, b, tail, silu=False)
    ext = np.concatenate([tail, x])
    for d in range(D):
        full = scipy.signal.lfilter(w[d, ::-1], [1.0], ext[:, d])
        assert np.allclose(y[:, d], full[W - 1:] + b[d])
    assert np.array_equal(t, x[-3:])
    s, _ = oracle.conv(x, w, b, tail)
    assert np.allclose(s, y * scipy.special.expit(y))
    y2, t2 = oracle.conv(x[:1], w, b, tail)
    y3, t3 = oracle.conv(x[1:], w, b, t2)
    assert np.allclose(np.concatenate([y2, y3]), s) and np.array_equal(t3, t)


def test_score_matches_library_routines():
    x = _rand(16, 500) * 3
    lp, ent, ids, tops = oracle.score(x, 17, 5)
    ref = scipy.special.log_softmax(x)
    assert np.isclose(lp, ref[17]) and np.isclose(ent, scipy.stats.entropy(np.exp(ref)))
    assert np.array_equal(ids, np.argsort(-x)[:5]) and np.allclose(tops, ref[ids])
    x[:] = 1.0
    lp, ent, ids, _ = oracle.score(x, 3, 4)
    assert np.isclose(lp, -np.log(500)) and np.isclose(ent, np.log(500)) and np.array_equal(ids, [0, 1, 2, 3])
    x[2:] = -np.inf
    lp, ent, ids, tops = oracle.score(x, 3, 4)
    assert lp == -np.inf and np.isclose(ent, np.log(2)) and np.array_equal(ids, [0, 1, -1, -1]) and tops[2] == -np.inf
