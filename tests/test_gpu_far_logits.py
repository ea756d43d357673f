"""GPU parity of the losses over logits with their float64 definitions where logits lie far from 0: masks by large finite values, rows
that are one such value, rows with an offset.  A log-sum-exp is then known to its own rounding only, or the product of a logit and the
exponent's factor is; the softmax of the row is as well known as any.

Bounds: fp32 arithmetic is off by U = 2^-24 of the magnitudes that go into it, counted along the formulas; a 16-bit result is rounded once
more (`within`)."""
import numpy as np
import pytest

from oracle import packed_ops as P
from paper_2110_13005_amd import binding as B
from paper_2110_13005_amd.inputs import snap_elem
from helpers import dev_i32, host
from test_gpu_distillation import Distillation, student
from test_gpu_losses import empty, f32
from test_gpu_step_ops import Padded, U, within

pytestmark = [pytest.mark.gpu, pytest.mark.parametrize("axonn_elem", ["bf16", "fp16"], indirect=True)]
VOCABULARIES = [2100, 12289, 40000, 140001]          # 256, 512 and 1024 threads a row, and more columns than registers hold


def far_values():
    """Masks of this type: the largest is the type's lowest value."""
    lowest = {"bf16": -float(2 - 2 ** -7) * 2.0 ** 127, "fp16": -65504.0}[B.ELEM]
    return [float(v) for v in snap_elem(np.array({"bf16": [-1e4, -1e6, -1e8, -1e9, -1e10, -1e15, -1e30], "fp16": [-1e4, -3e4]}[B.ELEM], np.float32))] + [lowest]


def softmax_bounds(z):
    """Of a row's log-sum-exp counted from its maximum, and of every element of its softmax, relative."""
    z = np.asarray(z, np.float64)
    V = z.shape[1]
    gap = np.where(np.isfinite(z), z.max(axis=1, keepdims=True) - z, 0.0)
    row = U * (60 + V / 512 + 4 * np.sum(np.exp(P.log_softmax(z)) * gap, axis=1) + 4 * np.log(V + 1))
    return row, row[:, None] + U * (8 + 6 * np.minimum(gap, 1e4))


@pytest.mark.parametrize("mass", [None, 0.7, 1.0])
@pytest.mark.parametrize("tau", [0.5, 1.0, 2.0, 8.0, 2.0 ** -12, 2.0 ** 14])
def test_distillation_with_all_but_the_named_masked(tau, mass):
    T, V, K = 3, 2100, 40
    for i, value in enumerate(far_values()):
        rng = np.random.default_rng(i)
        ids = np.argsort(rng.random((T, V)), axis=1)[:, :K]
        named = student(rng, T, V, ids) * min(tau, 1.0)
        z = np.full((T, V), value, np.float32)
        np.put_along_axis(z, ids, snap_elem(np.take_along_axis(named, ids, axis=1).astype(np.float32)), axis=1)
        u = rng.standard_normal((T, K)) * tau
        if mass is not None:
            u -= tau * np.log(np.exp(u / tau).sum(axis=1, keepdims=True) / mass)
        # a power of two: the products by 1 / temperature are exact, and so is the division
        d = Distillation(z, u.astype(np.float32), ids, None if mass is None else np.zeros(T, np.float32), tau, np.full(T, tau if tau < 1 else 1.0, np.float32))
        d.run()
        d.check()


def rows_of(value, V, lower):
    """Half of the columns at `value`, the others below it; a row of nothing but it; one that holds it once."""
    rng = np.random.default_rng(V)
    z = np.full((3, V), value, np.float32)
    z[0, rng.random(V) < 0.5] = lower
    z[2] = lower
    targets = np.array([int(np.flatnonzero(z[0] == value)[3]), V // 3, V - 2])
    z[2, V - 2] = value
    return z, targets


@pytest.mark.parametrize("lower", ["masked", "lowest"])
@pytest.mark.parametrize("V", VOCABULARIES)
def test_rows_whose_maximum_is_far(V, lower):
    for value in far_values():
        below = -np.inf if lower == "masked" else far_values()[-1]
        z, targets = rows_of(value, V, below)
        T = len(z)
        buf, grad = Padded(T, V, values=z), Padded(T, V)
        t, ones = dev_i32(targets), f32(np.ones(T))
        logp, lse, token = empty(T), empty(T), empty(T)
        want, want_lse = P.token_logprobs(z, targets)
        row, rel = softmax_bounds(z)
        B.axonn_token_logprobs_fwd(T, V, buf.t, V, t, logp, lse)
        assert (np.abs(host(logp) - want) <= row + 3 * U * np.abs(want)).all(), value
        assert (np.abs(host(lse) - want_lse) <= row + 2 * U * np.abs(want_lse)).all(), value
        # a ratio of about 1, which no limit clips
        old = want.astype(np.float32)
        B.axonn_policy_loss(T, V, buf.t, V, t, f32(old), None, ones, ones, 0.2, 0.2, 0.0, 1.0, logp, token, None, grad.t, V)
        _, r_token, _, r_d = P.policy_loss(z, targets, old, None, np.ones(T), np.ones(T), 0.2, 0.2, 0.0)
        e = 2 * row + U * (16 + 8 * np.abs(want))
        assert (np.abs(host(logp) - want) <= row + 3 * U * np.abs(want)).all(), value
        assert (np.abs(host(token) - r_token) <= 2 * e).all(), value
        q, onehot = np.exp(P.log_softmax(z)), np.arange(V) == targets[:, None]
        within(grad.result(), r_d, q * rel + 4 * e[:, None] * (q + onehot), label=("policy", value))
        # a teacher that names the target and another one
        ids = np.stack([targets, (targets + 7) % V], axis=1)
        z[np.arange(T), ids[:, 1]] = value
        d = Distillation(z, np.zeros((T, 2), np.float32), ids, np.full(T, 1.0, np.float32), 1.0, np.ones(T, np.float32))
        d.run()
        d.check()


@pytest.mark.parametrize("V", VOCABULARIES)
def test_gradient_of_rows_with_an_offset(V):
    """The softmax of a row does not change with an offset, although its log-sum-exp is rounded ever more coarsely; in place too."""
    rng = np.random.default_rng(V)
    offsets = np.array([0.0, 900.0, -900.0, 1500.0, -3000.0, 20000.0, -20000.0] + far_values())
    T = len(offsets) + 3
    z = snap_elem((np.maximum(np.append(offsets, [0, 5000.0, 5000.0])[:, None] + 2 * rng.standard_normal((T, V)), far_values()[-1])).astype(np.float32))
    z = np.asarray(z, np.float32).reshape(T, V)
    targets = rng.integers(0, V, T)
    targets[:-3] = z[:-3].argmax(axis=1)
    d = rng.standard_normal(T).astype(np.float32)
    targets[-2], d[-1] = -100, 0.0
    buf, grad, t = Padded(T, V, V + 3, 1, z), Padded(T, V, V + 5, 3), dev_i32(targets)
    logp, lse = empty(T), empty(T)
    B.axonn_token_logprobs_fwd(T, V, buf.t, V + 3, t, logp, lse)
    B.axonn_token_logprobs_bwd(T, V, buf.t, V + 3, t, lse, f32(d), grad.t, V + 5)
    row, rel = softmax_bounds(z)
    q, slope = np.exp(P.log_softmax(z)), np.where(P.has_target(targets, V), np.abs(d), 0.0)[:, None]
    # up to 2^10 the softmax goes by the rounded log-sum-exp
    rel = rel + row[:, None] + 4 * U * np.minimum(np.abs(P.token_logprobs(z, np.abs(targets))[1]), 1024.0)[:, None]
    within(grad.result(), P.token_logprobs_bwd(z, targets, d), slope * (q * rel + 4 * U * (q + (np.arange(V) == targets[:, None]))))
    assert not grad.result()[-2:].any()
    B.axonn_token_logprobs_bwd(T, V, buf.t, V + 3, t, lse, f32(d), buf.t, V + 3)
    assert (buf.result() == grad.result()).all()


@pytest.mark.parametrize("tau", [0.5, 1.0])
@pytest.mark.parametrize("lse", [None, 3.0])
def test_distillation_of_named_tokens_without_probability(lse, tau):
    """The student masks all that the teacher names: the loss is infinite, its gradient is not; wherever the others' logits lie."""
    T, V, K = 5, 2100, 3
    rng = np.random.default_rng(1)
    z = np.asarray(normal_at([0.0, -30.0, -100.0, -3000.0, 60.0], rng, V), np.float32)
    ids = np.argsort(rng.random((T, V)), axis=1)[:, :K]
    np.put_along_axis(z, ids, -np.inf, axis=1)
    d = Distillation(z, np.zeros((T, K), np.float32), ids, None if lse is None else np.full(T, lse, np.float32), tau, np.ones(T, np.float32))
    d.run()
    with np.errstate(all="ignore"):
        token, _, dz = P.distill_loss(z, d.u, ids, d.lse, tau, d.w)
    assert (token == np.inf).all() and (host(d.token) == np.inf).all()
    row, rel = softmax_bounds(z / tau)
    q, p = np.exp(P.log_softmax(z / tau)), np.zeros((T, V))
    np.put_along_axis(p, ids, 1 / 3 if lse is None else np.exp(-lse), axis=1)
    rest = 1 - p.sum(axis=1, keepdims=True)
    # of the others: q (1 - rest / Q), Q = 1: of both parts and of the rest's mass
    within(d.grad.result() / d.scale, dz, (q * (rel + row[:, None]) * (1 + rest) + 32 * U * (q + p)) / tau)


def normal_at(offsets, rng, V):
    return snap_elem((np.array(offsets)[:, None] + rng.standard_normal((len(offsets), V))).astype(np.float32)).reshape(len(offsets), V)


@pytest.mark.parametrize("tau", [0.25, 1.0])
def test_distillation_of_entries_without_mass(tau):
    """The teacher gives what it names no mass, and the student masks it by its type's lowest value: all that counts are the others."""
    T, V, K = 4, 2100, 3
    rng = np.random.default_rng(2)
    z = np.asarray(normal_at([0.0, 3.0, -40.0, 40.0], rng, V), np.float32)
    ids = np.argsort(rng.random((T, V)), axis=1)[:, :K]
    np.put_along_axis(z, ids, far_values()[-1], axis=1)
    d = Distillation(z, np.full((T, K), -500.0 * tau, np.float32), ids, np.zeros(T, np.float32), tau, np.ones(T, np.float32))
    d.run()
    scaled = z.astype(np.float64) / tau
    row, rel = softmax_bounds(scaled)
    # all mass is the others', of both: log 1 - log 1, and no gradient
    assert (np.abs(host(d.token)) <= 2 * row + 8 * U).all()
    q = np.exp(P.log_softmax(scaled))
    within(d.grad.result() / d.scale, np.zeros((T, V)), (2 * q * (rel + row[:, None]) + 8 * U * q) / tau)


@pytest.mark.parametrize("tau", [0.25, 1.0])
@pytest.mark.parametrize("lse", [None, 0.5])
def test_distillation_of_a_masked_entry_of_little_mass(lse, tau):
    """The student masks one of the teacher's entries by its type's lowest value: its mass times the distance counts, however far that is."""
    T, V, K = 4, 2100, 3
    rng = np.random.default_rng(3)
    z = np.asarray(normal_at([0.0, 3.0, -40.0, 40.0], rng, V), np.float32)
    ids = np.argsort(rng.random((T, V)), axis=1)[:, :K]
    z[np.arange(T), ids[:, 1]] = far_values()[-1]
    u = np.tile(np.array([0.0, -20.0, -1.0]) * tau, (T, 1)).astype(np.float32)
    d = Distillation(z, u, ids, None if lse is None else np.full(T, lse, np.float32), tau, np.ones(T, np.float32))
    d.run()
    d.check()
    assert np.isfinite(host(d.token)).all()
