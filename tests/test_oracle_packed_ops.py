"""Pins of the oracle of the operations on packed sequences: gradients against central differences, special cases in closed form, and
equivalence with the oracle's attention of one length."""
import numpy as np
import pytest

from oracle import packed_ops as P
from oracle import transformer as OT


def differences(f, x, eps=1e-5):
    g = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        hi, lo = x.copy(), x.copy()
        hi[i] += eps
        lo[i] -= eps
        g[i] = (f(hi) - f(lo)) / (2 * eps)
    return g


def test_attention_of_equal_lengths_is_the_layers():
    rng = np.random.default_rng(0)
    b, s, a, d = 3, 7, 2, 4
    qkv = rng.standard_normal((b * s, 3 * a * d))
    q, k, v = (qkv[:, i * a * d:(i + 1) * a * d].reshape(b, s, a * d) for i in range(3))
    o, prob = OT.causal_attention_fwd(q, k, v, a)
    do = rng.standard_normal((b, s, a * d))
    got, lse = P.packed_attention_fwd(qkv, np.arange(b + 1) * s, a, a, d, 1 / np.sqrt(d))
    assert np.allclose(got, o.reshape(b * s, -1), rtol=1e-12) and np.isfinite(lse).all()
    grads = np.concatenate([g.reshape(b * s, -1) for g in OT.causal_attention_bwd(do, q, k, v, prob, a)], axis=1)
    assert np.allclose(P.packed_attention_bwd(qkv, do.reshape(b * s, -1), np.arange(b + 1) * s, a, a, d, 1 / np.sqrt(d)), grads, rtol=1e-10, atol=1e-12)


def test_attention_gradient_of_shared_heads():
    rng = np.random.default_rng(1)
    heads, kv, d, off = 4, 2, 3, [1, 1, 5, 8]
    qkv, w = rng.standard_normal((9, (heads + 2 * kv) * d)), rng.standard_normal((9, heads * d))
    inside = np.zeros(9, bool)
    inside[1:8] = True

    def f(x):
        return np.sum((P.packed_attention_fwd(x, off, heads, kv, d, 0.7)[0] * w)[inside])

    got = P.packed_attention_bwd(qkv, w, off, heads, kv, d, 0.7)
    assert np.isnan(got[~inside]).all()
    assert np.allclose(got[inside], differences(f, qkv)[inside], rtol=1e-6, atol=1e-8)


def test_sequences_of_disordered_offsets():
    assert P.sequences([3, 1, 5, 4, 99], 9) == [(3, 3), (3, 5), (5, 5), (5, 9)]
    assert P.sequences([-4, 2, 2], 9) == [(0, 2), (2, 2)]


def test_logprobs_gradient():
    rng = np.random.default_rng(2)
    z, t, c = rng.standard_normal((5, 6)), np.array([0, 5, -100, 6, 2]), rng.standard_normal(5)
    logp, lse = P.token_logprobs(z, t)
    assert np.allclose(lse[[0, 1, 4]], np.log(np.exp(z).sum(axis=1))[[0, 1, 4]]) and not logp[2:4].any() and not lse[2:4].any()
    assert np.allclose(P.token_logprobs_bwd(z, t, c), differences(lambda x: np.sum(P.token_logprobs(x, t)[0] * c), z), atol=1e-8)


@pytest.mark.parametrize("kl", [0.0, 0.3])
def test_policy_gradient(kl):
    rng = np.random.default_rng(3)
    T, V = 12, 5
    z, t = rng.standard_normal((T, V)), rng.integers(-1, V, T)
    logp = P.token_logprobs(z, t)[0]
    # ratios on both sides of both limits, advantages of both signs
    old, A, w = logp - np.tile([-0.5, -0.1, 0.1, 0.5], 3), np.repeat([1.3, -0.8, 0.0], 4), np.where(np.arange(T) == 3, 0.0, 0.2)
    ref = logp + 0.3 * rng.standard_normal(T) if kl else None

    def f(x):
        return P.policy_loss(x, t, old, ref, A, w, 0.2, 0.25, kl)[2]

    out = P.policy_loss(z, t, old, ref, A, w, 0.2, 0.25, kl)
    assert np.allclose(out[3], differences(f, z), atol=1e-8) and not out[1][(w == 0) | (t < 0)].any()
    if not kl:     # by hand: clipped above at A > 0, below at A < 0
        assert np.allclose(out[1][[0, 4]][(t >= 0)[[0, 4]]], np.array([-1.3 * np.exp(-0.5), 0.8 * 0.8])[(t >= 0)[[0, 4]]])


@pytest.mark.parametrize("smoothing", [0.0, 0.2])
def test_preference_gradient(smoothing):
    rng = np.random.default_rng(4)
    off = [1, 4, 6, 6, 9]
    logp, ref, live = -rng.random(11), -rng.random(11), rng.random(11) < 0.8
    pair, loss, d = P.preference_loss(logp, ref, off, live, 0.5, smoothing, 0.7)
    assert np.isclose(loss, 0.7 * pair.sum()) and len(pair) == 2 and not d[[0, 9, 10]].any()
    assert np.allclose(d, differences(lambda x: P.preference_loss(x, ref, off, live, 0.5, smoothing, 0.7)[1], logp), atol=1e-9)
    same = P.preference_loss(logp, logp, off, live, 0.5, smoothing, 1.0)
    assert np.allclose(same[0], np.log(2))
    # a rejected token without probability: nothing left to prefer, unless the labels are smoothed
    logp[4], live = -np.inf, np.ones(11, bool)
    pair, _, d = P.preference_loss(logp, ref, off, live, 0.5, smoothing, 0.7)
    assert pair[0] == (np.inf if smoothing else 0.0) and np.allclose(d[1:6], 0.35 * smoothing * np.array([1, 1, 1, -1, -1]))


@pytest.mark.parametrize("tail", [False, True])
def test_distillation_gradient(tail):
    rng = np.random.default_rng(5)
    T, V, K = 5, 9, 4
    z, u, ids, w = rng.standard_normal((T, V)), rng.standard_normal((T, K)), np.argsort(rng.random((T, V)))[:, :K], rng.random(T)
    ids[1, 2:], ids[2], w[3], ids[4, 1] = -1, V, 0.0, ids[4, 0]
    lse = np.log(np.exp(u / 1.5).sum(axis=1)) + 0.4 if tail else None
    loss, total, dz = P.distill_loss(z, u, ids, lse, 1.5, w)
    assert np.isclose(total, np.sum(w * loss)) and not loss[2:4].any() and not dz[2:4].any()
    assert np.allclose(dz, differences(lambda x: P.distill_loss(x, u, ids, lse, 1.5, w)[1], z), atol=1e-8)
    # all tokens named by a teacher that is the student: nothing to learn
    ids = np.tile(np.arange(V), (T, 1))
    loss, _, dz = P.distill_loss(z, z, ids, np.log(np.exp(z / 1.5).sum(axis=1)) if tail else None, 1.5, w)
    assert np.allclose(loss, 0, atol=1e-7) and np.allclose(dz, 0, atol=1e-12)
    # all tokens named with a log-sum-exp that is a little too large: the rest's mass is nobody's
    lse = np.log(np.exp(u / 1.5).sum(axis=1))
    few = [P.distill_loss(z[:, :K], u, ids[:, :K], x, 1.5, w)[0] for x in (None, lse + 1e-7)]
    assert np.allclose(few[0], few[1], atol=1e-5)
