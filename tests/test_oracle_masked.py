"""CPU pins of the oracle for layer norm, rotary embedding over several axes and masked attention: closed forms on small inputs, the
operators they generalise, and every gradient against central differences."""
import numpy as np
import pytest

from oracle import block_oracle as bo


def differences(f, x, d, eps=1e-6):
    """sum(d * df/dx) along each entry of x, by central differences."""
    g = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        y = x.copy()
        y[i] += eps
        up = (d * f(y)).sum()
        y[i] -= 2 * eps
        g[i] = (up - (d * f(y)).sum()) / (2 * eps)
    return g


def test_layernorm_and_its_gradients():
    rng = np.random.default_rng(1)
    x, g, b, d = rng.standard_normal((3, 10)) + 4.0, rng.uniform(0.5, 1.5, 10), rng.standard_normal(10), rng.standard_normal((3, 10))
    h, mean, r = bo.layernorm(x, g, b, 1e-5)
    xh = (h - b) / g
    assert np.allclose(xh.mean(axis=1), 0.0, atol=1e-12) and np.allclose((xh ** 2).mean(axis=1), 1.0, atol=1e-4)
    assert np.allclose(bo.layernorm(x, g, None, 1e-5)[0], h - b)
    zero_mean = x - x.mean(axis=1, keepdims=True)
    assert np.allclose(bo.layernorm(zero_mean, g, None, 1e-5)[0], bo.rmsnorm(zero_mean, g, 1e-5)[0])
    dx, dg, db = bo.layernorm_backward(d, x, g, mean, r)
    assert np.allclose(dx, differences(lambda t: bo.layernorm(t, g, b, 1e-5)[0], x, d), atol=1e-7)
    assert np.allclose(dg, differences(lambda t: bo.layernorm(x, t, b, 1e-5)[0], g, d), atol=1e-7)
    assert np.allclose(db, differences(lambda t: bo.layernorm(x, g, t, 1e-5)[0], b, d), atol=1e-7)


@pytest.mark.parametrize("pairs", [False, True])
def test_rope_axes(pairs):
    rng = np.random.default_rng(2)
    T, H, dh, half = 5, 3, 32, 8
    x, d = rng.standard_normal((T, H * dh)), rng.standard_normal((T, H * dh))
    pos, axis, freq = rng.integers(-9, 100, (2, T)), [0, 1, 1, 0, 0, 1, 0, 1], [10.0 ** (-i / 3) for i in range(half)]
    y = bo.rope_axes(x, pos, axis, freq, dh, pairs)
    assert np.allclose(bo.rope_axes(y, pos, axis, freq, dh, pairs, inverse=True), x)
    assert np.array_equal(y.reshape(T, H, dh)[..., 2 * half:], x.reshape(T, H, dh)[..., 2 * half:])
    # orthogonal: the gradient of sum(d * y) with respect to x is the inverse rotation of d
    assert np.allclose((d * y).sum(), (bo.rope_axes(d, pos, axis, freq, dh, pairs, inverse=True) * x).sum())
    if not pairs:                                         # one axis, everything rotated: the one-axis embedding with its tables
        p = np.arange(T)
        f = np.array([10.0 ** (-i / 3) for i in range(dh // 2)])
        ang = p[:, None] * f[None, :]
        assert np.allclose(bo.rope_axes(x, p[None], [0] * (dh // 2), f, dh), bo.rope(x, np.cos(ang), np.sin(ang), p, dh))


def test_allowed_keys():
    assert bo.allowed_keys(3, 3).astype(int).tolist() == [[1, 0, 0], [1, 1, 0], [1, 1, 1]]
    assert bo.allowed_keys(3, 3, prefix=2).astype(int).tolist() == [[1, 1, 0], [1, 1, 0], [1, 1, 1]]
    assert bo.allowed_keys(1, 4, window=2).astype(int).tolist() == [[0, 0, 1, 1]]
    assert bo.allowed_keys(3, 2).astype(int).tolist() == [[0, 0], [1, 0], [1, 1]]           # the first query stands before every key
    assert bo.allowed_keys(2, 3, causal=False, window=2).astype(int).tolist() == [[1, 1, 1], [0, 1, 1]]
    assert bo.allowed_keys(2, 4, prefix=4, window=1).astype(int).tolist() == [[0, 0, 1, 0], [0, 0, 0, 1]]


def test_masked_attention_generalises_the_causal_one():
    rng = np.random.default_rng(3)
    n_seq, S, n_q, n_kv, dh = 2, 6, 4, 2, 8
    T = n_seq * S
    q, k, v, d = (rng.standard_normal((T, h * dh)) for h in (n_q, n_kv, n_kv, n_q))
    o, P = bo.attention(q, k, v, n_seq, n_q, n_kv, dh, 0.3)
    seqs = [(b * S, S, b * S, S, 0) for b in range(n_seq)]
    got = bo.masked_attention(q, k, v, seqs, n_q, n_kv, dh, 0.3, d_o=d)
    assert np.allclose(got[0], o)
    for a, b in zip(got[2:], bo.attention_backward(d, q, k, v, P, n_seq, n_q, n_kv, dh, 0.3)):
        assert np.allclose(a, b)
    # a cap far above the scores and a bias of nothing change nothing
    assert np.allclose(bo.masked_attention(q, k, v, seqs, n_q, n_kv, dh, 0.3, cap=1e5, slopes=np.zeros(n_q))[0], o, atol=1e-8)


@pytest.mark.parametrize("causal,window,cap,biased", [(True, 0, 2.0, False), (True, 3, 0.0, True), (False, 0, 1.5, True), (False, 2, 0.0, False)])
def test_masked_attention_gradients(causal, window, cap, biased):
    rng = np.random.default_rng(4)
    n_q, n_kv, dh = 2, 1, 3
    # rows 0 and 8 belong to no sequence; the second sequence has more queries than keys (its first query sees nothing), the third no keys
    seqs = [(1, 4, 0, 5, 3), (5, 2, 6, 1, 0), (7, 1, 8, 0, 0)]
    q, k, v, d = (rng.standard_normal((9, h * dh)) for h in (n_q, n_kv, n_kv, n_q))
    slopes = [0.5, 0.1] if biased else None
    f = lambda q_, k_, v_: bo.masked_attention(q_, k_, v_, seqs, n_q, n_kv, dh, 0.7, causal, window, cap, slopes)[0]
    o, lse, dq, dk, dv = bo.masked_attention(q, k, v, seqs, n_q, n_kv, dh, 0.7, causal, window, cap, slopes, d_o=d)
    assert not o[[0, 7, 8]].any() and np.isnan(lse[:, [0, 8]]).all() and np.isneginf(lse[:, 7]).all()
    if causal:
        assert np.isneginf(lse[:, 5]).all() and not o[5].any()
    assert np.allclose(dq, differences(lambda t: f(t, k, v), q, d), atol=1e-7)
    assert np.allclose(dk, differences(lambda t: f(q, t, v), k, d), atol=1e-7)
    assert np.allclose(dv, differences(lambda t: f(q, k, t), v, d), atol=1e-7)
