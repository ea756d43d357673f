"""GPU parity of distillation with its float64 definition where the teacher's named tokens hold any mass: less than 1 with no other tokens
left for the rest, or more.

Bounds: fp32 arithmetic is off by U = 2^-24 of the magnitudes that go into it, counted along the formulas (`bounds`); a 16-bit result is
rounded once more (`within`)."""
import numpy as np
import pytest

from oracle import packed_ops as P
from paper_2110_13005_amd import binding as B
from helpers import dev_i32, host
from test_gpu_losses import empty, f32
from test_gpu_step_ops import Padded, U, normal, within

pytestmark = [pytest.mark.gpu, pytest.mark.parametrize("axonn_elem", ["bf16", "fp16"], indirect=True)]
LARGEST = float(np.finfo(np.float32).max)


def bounds(z, u, ids, lse, tau):
    """-> of a token's loss; of the gradient's elements by logits / tau.  z may hold -inf, ids name tokens of the vocabulary alone."""
    z = np.asarray(z, np.float64)
    T, V = z.shape
    K = ids.shape[1]
    logq = P.log_softmax(z / tau)
    E_loss, E_grad = np.zeros(T), np.zeros((T, V))
    for t in range(T):
        x, lq, q = u[t].astype(np.float64) / tau, logq[t], np.exp(logq[t])
        sums = (K / 64 + 24) * U                                       # of the entries: a lane's share, then over the wave
        if lse is None:
            norm = x.max() + np.log(np.exp(x - x.max()).sum())
            e_norm = sums + U * (4 * (x.max() - x).max() + 4 * np.abs(x).max() + 4 * abs(norm))
        else:
            norm, e_norm = float(lse[t]), 0.0
        logp = x - norm
        p = np.exp(logp)
        e_p = e_norm + U * (8 + 4 * np.abs(x) + 2 * np.abs(logp))      # of a p, relative; of a logp
        named = np.zeros(V, bool)
        named[ids[t]] = True
        gap = np.where(np.isfinite(z[t]), z[t].max() - z[t], 0.0) / tau
        mean = np.sum(q * gap)
        row = U * (60 + V / 512 + 4 * mean + 4 * np.log(V + 1))        # of the student's log-sum-exp, from the maximum
        e_q = row + U * (8 + 6 * gap)                                  # of a q, relative; of its logarithm, with U |log q|
        top = z[t][named].max()
        size = np.abs(logp) + (top - z[t][ids[t]]) / tau + (z[t].max() - top) / tau + np.abs(lq[ids[t]]) + 1
        mass, e_mass = p.sum(), np.sum(p * e_p) + sums * p.sum()
        E_loss[t] = np.sum(p * ((2 * e_p + sums + 8 * U) * size + row))
        full, e_full = np.zeros(V), np.zeros(V)
        np.add.at(full, ids[t], p)
        np.add.at(e_full, ids[t], p * (e_p + (K + 4) * U))
        total, rest, e_rest, share, e_share = 1.0 if lse is None else mass, 0.0, 0.0, 0.0, 0.0
        if lse is not None and np.isfinite(lq[~named]).any():
            z_far = z[t][~named].max()
            far = P.log_softmax(z[t][~named] / tau)
            logQ = lq[~named].max() - far.max()
            rest, e_rest = max(1.0 - mass, 0.0), e_mass + 2 * U
            total = max(mass, 1.0)
            E_loss[t] += 2 * e_rest * (2 + abs(np.log(max(rest, 1e-12))) + abs(logQ)) + rest * (2 * row + 8 * U * (abs(logQ) + abs(np.log(max(rest, 1e-12)))))
            # of the others' share P softmax(z over them)
            share = np.zeros(V)
            share[~named] = np.exp(far)
            gap_far = np.where(np.isfinite(z[t]) & ~named, z_far - z[t], 0.0) / tau
            e_share = U * (60 + V / 512 + 4 * np.sum(share * gap_far) + 4 * np.log(V + 1) + 8 + 6 * gap_far)
        E_grad[t] = q * (total * e_q + 2 * e_mass) + e_full + share * (e_rest + rest * e_share) + 4 * U * (q * total + full + share * rest)
    return E_loss, E_grad


class Distillation:
    """Operands of a call; out: the marks around its gradient."""

    def __init__(self, z, u, ids, lse, tau, w, ld=None, shift=0):
        self.z, self.u, self.ids, self.lse, self.tau, self.w = z, u, ids, lse, tau, w
        self.T, self.V = z.shape
        self.ld, self.K = ld or self.V, ids.shape[1]
        self.scale = 1.0 if B.ELEM == "bf16" else 64.0
        self.logits, self.grad = Padded(self.T, self.V, self.ld, shift, z), Padded(self.T, self.V, self.ld, shift)
        self.token, self.loss = empty(self.T), empty(1)

    def run(self, in_place=False):
        out = self.logits if in_place else self.grad
        B.axonn_distill_loss(self.T, self.V, self.K, self.logits.t, self.ld, f32(self.u), dev_i32(self.ids), self.K,
                             None if self.lse is None else f32(self.lse), self.tau, f32(self.w), self.scale, self.token, self.loss, out.t, self.ld)

    def check(self):
        with np.errstate(invalid="ignore", divide="ignore"):
            token, loss, dz = P.distill_loss(self.z, self.u, self.ids, self.lse, self.tau, self.w)
            E_loss, E_grad = bounds(self.z, self.u, self.ids, self.lse, self.tau)
        got = host(self.token)
        small = np.abs(token) < LARGEST
        assert (np.abs(got - token) <= E_loss + 2 * U * np.abs(token))[small].all(), (np.abs(got - token) / E_loss)[small].max()
        assert (got[~small] == np.sign(token[~small]) * np.inf).all()
        if small.all() and abs(loss) < LARGEST:
            assert abs(host(self.loss)[0] - loss) <= np.sum(self.w * E_loss) + 4 * U * np.sum(self.w * np.abs(token))
        g = (self.w / self.tau)[:, None]
        result = self.grad.result() / self.scale
        within(result, dz, g * E_grad + 4 * U * np.abs(dz), label="distillation")
        return result


def student(rng, T, V, ids):
    """Logits of which the first named one is likely."""
    z = normal(rng, T, V, std=2.0)
    z[np.arange(T), ids[:, 0]] = normal(rng, 1, T, mean=5.0)[0]
    return z


SIZES = [(9, 4, 12, 3), (300, 150, 300, 0), (2049, 64, 2050, 1), (12289, 700, 12289, 0), (140001, 20, 140008, 0)]  # vocabulary, entries, rows, first element
NAMED = [(*size, others) for others in ("there", "masked") for size in SIZES] + [(9, 9, 12, 3, "none"), (300, 300, 300, 0, "none"), (1001, 1001, 1002, 1, "none")]


@pytest.mark.parametrize("mass", [None, 0.3, 0.7, 1.0, 1.04, 1.3])
@pytest.mark.parametrize("twice", [False, True])
@pytest.mark.parametrize("V,K,ld,shift,others", NAMED)
def test_any_mass(V, K, ld, shift, others, twice, mass):
    T, tau = 4, 1.5
    rng = np.random.default_rng(V + K)
    ids = np.argsort(rng.random((T, V)), axis=1)[:, :K]
    z = student(rng, T, V, ids)
    if twice:
        ids = np.concatenate([ids, ids[:, -2:]], axis=1)
    u = rng.standard_normal(ids.shape)
    if mass is not None:
        u -= tau * np.log(np.exp(u / tau).sum(axis=1, keepdims=True) / mass)
    if others == "masked":
        free = np.ones((T, V), bool)
        np.put_along_axis(free, ids, False, axis=1)
        z[free] = -np.inf
    lse = None if mass is None else np.zeros(T, np.float32)
    d = Distillation(z, u.astype(np.float32), ids, lse, tau, (rng.random(T) + 0.1).astype(np.float32), ld, shift)
    d.run()
    result = d.check()
    assert (result[~np.isfinite(z)] == 0).all()
    before = d.grad.t.clone()
    d.run(in_place=True)
    assert (d.logits.t == before).all()
