"""Pins of the oracle of the selective scan: against the SSD oracle where decays are equal, against a closed form, and against a
sum over all pairs of tokens."""
import numpy as np
import pytest

from oracle import mixer_oracle, ssd_oracle


def draw(tokens, C, N, seed):
    r = np.random.default_rng(seed)
    return (r.standard_normal((tokens, C)), r.uniform(0.01, 0.4, (tokens, C)), -r.uniform(0.3, 4.0, (C, N)), r.standard_normal((tokens, N)),
            r.standard_normal((tokens, N)), r.standard_normal(C))


def test_equal_decays_are_the_ssd_core():
    """One decay for all states of a head and one step size for its channels: heads of one channel each."""
    x, d, A, B, C, D = draw(23, 5, 6, 0)
    A = np.repeat(A[:, :1], 6, axis=1)
    y, h = mixer_oracle.selective_scan(x, d, A, B, C, D, [0, 23])
    y_ref, h_ref = ssd_oracle.prefill(x[None, :, :, None], d[None].astype(np.float32), A[:, 0], B[None, :, None], C[None, :, None], D)
    y2, h2 = mixer_oracle.selective_scan(x, d.astype(np.float32), A, B, C, D, [0, 23])
    assert np.allclose(y2, y_ref[0, :, :, 0], rtol=1e-6, atol=1e-6) and np.allclose(h2[0], h_ref[0, :, 0], rtol=1e-6, atol=1e-6)
    assert np.allclose(y, y2, rtol=1e-5, atol=1e-5) and np.allclose(h, h2, rtol=1e-5, atol=1e-5)


def test_closed_form_of_constant_inputs():
    """Constant d, x, B: h after t tokens is d x B (1 - a^t) / (1 - a)."""
    T, a = 17, np.exp(-0.25 * np.array([[1.0, 2.0, 3.0]]))
    one = np.ones((T, 1))
    y, h = mixer_oracle.selective_scan(2.0 * one, 0.25 * one, np.log(a) / 0.25, np.tile([1.0, -1.0, 0.5], (T, 1)), np.ones((T, 3)), None, [0, T])
    t = np.arange(1, T + 1)[:, None]
    states = 0.5 * np.array([1.0, -1.0, 0.5]) * (1 - a ** t) / (1 - a)
    assert np.allclose(y[:, 0], states.sum(1), rtol=1e-12) and np.allclose(h[0, 0], states[-1], rtol=1e-12)


def test_sum_over_pairs():
    x, d, A, B, C, D = draw(9, 3, 4, 1)
    z = np.random.default_rng(2).standard_normal((9, 3))
    h0 = np.random.default_rng(3).standard_normal((1, 3, 4))
    y, _ = mixer_oracle.selective_scan(x, d, A, B, C, D, [0, 9], z, h0)
    cs = np.cumsum(d, axis=0)
    for t in range(9):
        want = D * x[t] + np.einsum("n,cn->c", C[t], np.exp(cs[t][:, None] * A) * h0[0])
        for s in range(t + 1):
            want = want + np.exp((cs[t] - cs[s])[:, None] * A) @ (C[t] * B[s]) * d[s] * x[s]
        assert np.allclose(y[t], want * z[t] / (1 + np.exp(-z[t])), rtol=1e-10, atol=1e-12)


def test_packed_sequences_are_their_own():
    x, d, A, B, C, D = draw(30, 3, 4, 4)
    cu = [2, 2, 11, 12, 28]
    h0 = np.random.default_rng(5).standard_normal((4, 3, 4))
    y, h = mixer_oracle.selective_scan(x, d, A, B, C, D, cu, h0=h0)
    assert np.isnan(y[:2]).all() and np.isnan(y[28:]).all() and np.array_equal(h[0], h0[0])
    for q in range(1, 4):
        rows = slice(cu[q], cu[q + 1])
        yq, hq = mixer_oracle.selective_scan(x[rows], d[rows], A, B[rows], C[rows], D, [0, cu[q + 1] - cu[q]], h0=h0[q:q + 1])
        assert np.array_equal(y[rows], yq) and np.array_equal(h[q], hq[0])


@pytest.mark.parametrize("interleaved", [False, True])
def test_normed_heads_keep_their_length_under_rotation(interleaved):
    r = np.random.default_rng(6)
    q, k, v = r.standard_normal((3, 2, 8)), r.standard_normal((3, 1, 8)), r.standard_normal((3, 1, 8))
    angle = r.uniform(0, 6, (8, 4))
    cache = np.zeros((2, 1, 4, 8))
    out, kc, vc = mixer_oracle.append_norm(q, k, v, np.ones(8), np.ones(8), cache, cache, np.array([[1, 0]]), np.array([5]), np.array([0, 3]),
                                           (np.cos(angle), np.sin(angle)), interleaved, eps=0.0)
    assert np.allclose((out ** 2).mean(2), 1.0) and np.allclose((kc[[1, 1, 0], 0, [2, 3, 0]] ** 2).mean(1), 1.0)
    assert np.array_equal(vc[[1, 1, 0], 0, [2, 3, 0]], v[:, 0])
