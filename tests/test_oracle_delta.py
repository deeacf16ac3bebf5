"""Pins of the fp64 checkers of the gated delta rule, the norms with rotation and the slot copies; none re-uses their loops."""
import numpy as np
import pytest

from oracle import dsla_oracle as orc


def _inputs(T, Hq, H, d, seed):
    r = np.random.default_rng(seed)
    k = r.standard_normal((T, Hq, d))
    k /= np.linalg.norm(k, axis=-1, keepdims=True)
    return (r.standard_normal((T, Hq, d)), k, r.standard_normal((T, H, d)), r.uniform(0.5, 1, (T, H)), r.uniform(0, 1, (T, H)))


def test_hand_example():
    """d = 1: S = 0.5 * 2 = 1; u = 0.25 (3 - 2 * 1) = 0.25; S = 1 + 2 * 0.25 = 1.5; o = 4 * 1.5."""
    one = lambda x: np.full((1, 1, 1), float(x))  # noqa: E731
    o, S = orc.delta_prefill(one(4), one(2), one(3), np.full((1, 1), .5), np.full((1, 1), .25), state=np.full((1, 1, 1, 1, 1), 2.0))
    assert o.item() == 6.0 and S.item() == 1.5


def test_transition_matrices():
    """S_t = g (I - beta k^T k) S_{t-1} + beta k^T v, with the products of the matrices formed explicitly."""
    q, k, v, g, b = _inputs(9, 1, 2, 4, 0)
    o, S = orc.delta_prefill(q, k, v, g, b, scale=0.7)
    for h in range(2):
        M = [g[t, h] * (np.eye(4) - b[t, h] * np.outer(k[t, 0], k[t, 0])) for t in range(9)]
        for t in range(9):
            want = np.zeros((4, 4))
            for s in range(t + 1):
                term = b[s, h] * np.outer(k[s, 0], v[s, h])
                for r in range(s + 1, t + 1):
                    term = M[r] @ term
                want += term
            np.testing.assert_allclose(o[t, h], 0.7 * q[t, 0] @ want, rtol=1e-12, atol=1e-13)
        np.testing.assert_allclose(S[0, 0, h], want, rtol=1e-12, atol=1e-13)


@pytest.mark.parametrize("C", [1, 5, 16])
def test_chunked_form(C):
    """The triangular system of a chunk, solved by numpy: what the kernels compute."""
    T, d = 33, 8
    q, k, v, g, b = _inputs(T, 1, 1, d, 1)
    S0 = np.random.default_rng(2).standard_normal((1, 1, 1, d, d))
    o, S1 = orc.delta_prefill(q, k, v, g, b, state=S0.copy())
    S, got = S0[0, 0, 0], []
    for c in range(0, T, C):
        Q, K, V, G, B = q[c:c + C, 0], k[c:c + C, 0], v[c:c + C, 0], g[c:c + C, 0], b[c:c + C, 0]
        n = len(Q)
        Dm = np.array([[np.prod(G[i + 1:j + 1]) if i <= j else 0.0 for i in range(n)] for j in range(n)])
        Gc = np.cumprod(G)
        A = np.eye(n) + np.tril(B[:, None] * Dm * (K @ K.T), -1)
        U = np.linalg.solve(A, B[:, None] * (V - Gc[:, None] * (K @ S)))
        got.append(Gc[:, None] * (Q @ S) + (np.tril(Q @ K.T) * Dm) @ U)
        S = Gc[-1] * S + K.T @ (Dm[-1][:, None] * U)
    np.testing.assert_allclose(np.concatenate(got), o[:, 0], rtol=1e-11, atol=1e-12)
    np.testing.assert_allclose(S, S1[0, 0, 0], rtol=1e-11, atol=1e-12)


def test_limits():
    q, k, v, g, b = _inputs(6, 2, 2, 6, 3)
    S0 = np.random.default_rng(4).standard_normal((1, 1, 2, 6, 6))
    _, S = orc.delta_prefill(q, k, v, g, np.zeros_like(b), state=S0.copy())      # beta = 0: decay alone
    np.testing.assert_allclose(S[0, 0], g.prod(0)[:, None, None] * S0[0, 0], rtol=1e-13)
    e = np.eye(6)[:, None].repeat(2, 1)                                            # orthonormal keys, g = 1, beta = 1: plain linear attention
    o, S = orc.delta_prefill(q, e, v, np.ones_like(g), np.ones_like(b))
    np.testing.assert_allclose(S[0, 0], v.transpose(1, 0, 2), atol=1e-14)
    o, S = orc.delta_prefill(q, np.repeat(k[:1], 6, 0), v, np.ones_like(g), np.ones_like(b))     # one key, beta = 1: the last value replaces the others
    np.testing.assert_allclose(np.einsum("hk,hkv->hv", k[0], S[0, 0]), v[-1], atol=1e-13)


def test_packing_groups_and_slots():
    q, k, v, g, b = _inputs(12, 2, 6, 5, 5)
    cu, slots = np.array([0, 3, 3, 12]), np.array([2, 0, 1])
    o, S = orc.delta_prefill(q, k, v, g, b, cu, slots=slots)
    wide = [np.repeat(x, 3, 1) for x in (q, k)]
    for n in range(3):
        a, e = cu[n], cu[n + 1]
        o1, S1 = orc.delta_prefill(wide[0][a:e], wide[1][a:e], v[a:e], g[a:e], b[a:e])
        np.testing.assert_array_equal(o[a:e], o1)
        np.testing.assert_array_equal(S[slots[n]], S1[0])


def test_norms_and_rotation():
    r = np.random.default_rng(6)
    x, w, pos, f = r.standard_normal((3, 2, 8)), r.standard_normal(8), np.array([0, 5, -3]), np.array([1.0, 0.25])
    for inter in (False, True):
        y = orc.qk_norm_rope(x, w, pos, f, eps=0.0, norm="l2", interleaved=inter)
        base = x / np.linalg.norm(x, axis=-1, keepdims=True) * w
        np.testing.assert_allclose(y[0], base[0], rtol=1e-13)                        # position 0 turns nothing
        a, c = ([0, 2], [1, 3]) if inter else ([0, 1], [2, 3])
        z = (base[..., a] + 1j * base[..., c]) * np.exp(1j * pos[:, None, None] * f)
        np.testing.assert_allclose(y[..., a] + 1j * y[..., c], z, rtol=1e-12)
        np.testing.assert_array_equal(y[..., 4:], base[..., 4:])
    np.testing.assert_allclose((orc.qk_norm_rope(x, eps=0.0) ** 2).mean(-1), 1.0)
    np.testing.assert_array_equal(orc.qk_norm_rope(x, norm="none"), x)


def test_copies():
    s = np.arange(5.0)[:, None]
    assert orc.state_copy(s.copy(), [0, 1, 2], [1, 2, 3]).ravel().tolist() == [0, 0, 0, 0, 4]      # a chain passes slot 0 on
    assert orc.state_copy(s.copy(), [4, -1, 7, 3, -2], [0, 4, 1, 9, 2]).ravel().tolist() == [4, 1, 2, 3, 0]
