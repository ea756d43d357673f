"""GPU parity of the losses over logits (log-probabilities of tokens, policy, preference, distillation) with their float64 definitions,
element by element, at the sizes, strides, masks and values where they can go wrong.

Bounds: fp32 arithmetic is off by U = 2^-24 of the magnitudes that go into it, counted along the formulas; a 16-bit result is rounded
once more (`within`)."""
import numpy as np
import pytest

from oracle import packed_ops as P
from paper_2110_13005_amd import binding as B
from paper_2110_13005_amd.inputs import snap_elem
from helpers import dev_i32, host
from test_gpu_step_ops import Padded, U, half_step, normal, within

pytestmark = [pytest.mark.gpu, pytest.mark.parametrize("axonn_elem", ["bf16", "fp16"], indirect=True)]
# rows, vocabulary, leading dimension, first element
SIZES = [(1, 1, 1, 0), (3, 2, 5, 1), (4, 7, 7, 0), (5, 8, 8, 0), (6, 9, 12, 3), (3, 255, 255, 1), (9, 1000, 1000, 0), (4, 2047, 2050, 1), (4, 2049, 2049, 0),
         (3, 4100, 4104, 8), (5, 8191, 8191, 0), (2, 16392, 16392, 0), (3, 12289, 12289, 0), (3, 32003, 32003, 1), (2, 40968, 40968, 0), (2, 51200, 51200, 0), (2, 65536, 65536, 0), (2, 70001, 70004, 1), (1, 81921, 81921, 0), (1, 106497, 106497, 3), (1, 131071, 131071, 0),
         (2, 131080, 131080, 0), (1, 262144, 262144, 0), (1, 300007, 300007, 1), (1, 393216, 393216, 0)]


def f32(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).cuda()


def empty(n):
    import torch
    return torch.full((n,), 7.0, device="cuda")


class Logits:
    """Logits of which a row's target is likely, with rows that have none and hold NaN."""

    def __init__(self, T, V, ld=None, shift=0, seed=0, std=2.0, masked=0.2):
        rng = self.rng = np.random.default_rng(1000 * T + V + seed)
        self.T, self.V, self.ld = T, V, ld or V
        self.targets = rng.integers(0, V, T)
        z = normal(rng, T, V, std=std)
        z[np.arange(T), self.targets] = snap_elem((5 + rng.standard_normal(T)).astype(np.float32))
        self.out = rng.random(T) < masked if T > 1 else np.zeros(T, bool)
        self.z = z
        held = z.copy()
        held[self.out] = np.nan
        self.buf = Padded(T, V, self.ld, shift, held)
        self.labels = np.where(self.out, rng.choice([-100, -1, V, V + 5], T), self.targets)
        self.grad = Padded(T, V, self.ld, shift)

    def slack_logp(self):
        """Of a row's log-probability; and per element, of the softmax relative to itself."""
        logq = P.log_softmax(self.z)
        gap = np.abs(self.z - self.z.max(axis=1, keepdims=True))
        mean = np.sum(np.exp(logq) * gap, axis=1)
        log_sum = np.abs(self.z.max(axis=1) - (self.z - logq)[:, 0])
        row = U * (40 + self.V / 512 + 4 * mean + 4 * log_sum)
        at = np.arange(self.T), self.targets
        return row + 3 * U * (gap[at] + np.abs(logq[at])), row[:, None] + U * (8 + 6 * gap)

    def check_gradient(self, got, ref, slope, slack_slope, label):
        """ref = slope (onehot - q); slack_slope: of the slope."""
        q, rel = np.exp(P.log_softmax(self.z)), self.slack_logp()[1]
        onehot = np.zeros_like(q)
        onehot[np.arange(self.T), self.targets] = 1
        slope, slack = np.abs(slope)[:, None], slack_slope[:, None]
        within(got, ref, (slope + slack) * q * rel + slack * (q + onehot) + 2 * U * slope * (q + onehot), label=label)
        assert (got[slope[:, 0] == 0] == 0).all()


@pytest.mark.parametrize("T,V,ld,shift", SIZES)
def test_token_logprobs(T, V, ld, shift):
    L = Logits(T, V, ld, shift)
    logp, lse, d = empty(T), empty(T), np.where(L.rng.random(T) < 0.2, 0.0, L.rng.standard_normal(T)).astype(np.float32)
    t = dev_i32(L.labels)
    B.axonn_token_logprobs_fwd(T, V, L.buf.t, ld, t, logp, lse)
    ref_p, ref_l = P.token_logprobs(L.z, L.labels)
    slack = L.slack_logp()[0]
    assert (np.abs(host(logp) - ref_p) <= np.where(L.out, 0, slack)).all()
    assert (np.abs(host(lse) - ref_l) <= np.where(L.out, 0, slack + 2 * U * np.abs(ref_l))).all()
    B.axonn_token_logprobs_bwd(T, V, L.buf.t, ld, t, lse, f32(d), L.grad.t, ld)
    slope = np.where(L.out, 0.0, d)
    # the softmax goes by the rounded log-sum-exp here
    L.check_gradient(L.grad.result(), P.token_logprobs_bwd(L.z, L.labels, d), slope, np.abs(slope) * (slack + 4 * U * np.abs(ref_l)), "logprobs")
    # in place
    before = L.grad.t.clone()
    B.axonn_token_logprobs_bwd(T, V, L.buf.t, ld, t, lse, f32(d), L.buf.t, ld)
    assert (L.buf.t == before).all()
    L.buf.result()


def policy_operands(L, kl):
    rng, T = L.rng, L.T
    logp = P.token_logprobs(L.z, np.where(L.out, -1, L.targets))[0]
    old = (logp - (np.round(rng.standard_normal(T) * 12) + 0.5) / 64).astype(np.float32)      # no ratio at a limit
    ref = (logp + 0.3 * rng.standard_normal(T)).astype(np.float32) if kl else None
    A = np.where(rng.random(T) < 0.1, 0.0, rng.standard_normal(T)).astype(np.float32)
    w = np.where(rng.random(T) < (0.1 if T > 1 else 0), 0.0, rng.random(T) + 0.1).astype(np.float32)
    return old, ref, A, w


@pytest.mark.parametrize("kl,lo,hi", [(0.0, 0.2, 0.2), (0.1, 0.2, 0.28)])
@pytest.mark.parametrize("T,V,ld,shift", SIZES)
def test_policy_loss(T, V, ld, shift, kl, lo, hi):
    L = Logits(T, V, ld, shift, seed=int(kl * 10))
    old, ref, A, w = policy_operands(L, kl)
    scale = 1.0 if B.ELEM == "bf16" else 64.0
    logp, token, loss, t = empty(T), empty(T), empty(1), dev_i32(L.labels)
    ops = (t, f32(old), None if ref is None else f32(ref), f32(A), f32(w), lo, hi, kl, scale)
    B.axonn_policy_loss(T, V, L.buf.t, ld, *ops, logp, token, loss, L.grad.t, ld)
    r_logp, r_token, r_loss, r_d = P.policy_loss(L.z, L.labels, old, ref, A, w, lo, hi, kl)
    live = (w != 0) & ~L.out
    e = np.where(live, L.slack_logp()[0], 0.0)
    x = np.where(live, r_logp - old, 0.0)
    ratio, y = np.exp(x), (ref - r_logp if kl else np.zeros(T))
    e_ratio = ratio * (2 * e + U * (8 + 2 * np.abs(x)))
    e_kl = kl * (np.exp(np.abs(y)) * (2 * e + U * (8 + 4 * np.abs(y))))
    e_token = np.where(live, np.abs(A) * e_ratio + e_kl + 4 * U * (np.abs(A * ratio) + np.abs(r_token)), 0.0)
    assert (np.abs(host(logp) - r_logp) <= e).all()
    assert (np.abs(host(token) - r_token) <= e_token).all(), np.max(np.abs(host(token) - r_token))
    assert abs(host(loss)[0] - r_loss) <= np.sum(w * e_token) + 2 * U * np.sum(w * np.abs(r_token)) + 1e-30
    at = np.arange(T), L.targets
    slope = np.where(live, r_d[at] / np.where(live, 1 - np.exp(P.log_softmax(L.z)[at]), 1.0), 0.0) if V > 1 else np.zeros(T)
    e_slope = np.where(live, w * (np.abs(A) * e_ratio + e_kl + 4 * U * (np.abs(A) * ratio + kl * np.abs(np.expm1(y)))), 0.0)
    got = L.grad.result()
    assert (got[~live] == 0).all()
    L.check_gradient(got / scale, r_d, slope, e_slope + (1e-9 if V == 1 else 0.0), "policy")
    # losses alone; in place
    token2, loss2, before = empty(T), empty(1), L.grad.t.clone()
    B.axonn_policy_loss(T, V, L.buf.t, ld, *ops, None, token2, loss2, None, 0)
    assert (token2 == token).all() and (loss2 == loss).all()
    B.axonn_policy_loss(T, V, L.buf.t, ld, *ops, None, token2, None, L.buf.t, ld)
    assert (L.buf.t == before).all() and (token2 == token).all()
    L.buf.result()


@pytest.mark.parametrize("lens,front,pad", [([1, 1], 0, 0), ([0, 3], 2, 1), ([5, 0, 0, 0, 7, 300], 0, 9), ([700, 1300, 255, 257, 256, 1], 3, 0), ([3] * 200, 0, 5)])
@pytest.mark.parametrize("smoothing", [0.0, 0.15])
def test_preference_loss(lens, front, pad, smoothing):
    rng = np.random.default_rng(sum(lens))
    off = front + np.concatenate([[0], np.cumsum(lens)])
    T, V, n = int(off[-1]) + pad, 50, len(lens) // 2
    labels = np.where(rng.random(T) < 0.2, rng.choice([-100, V], T), rng.integers(0, V, T))
    live = P.has_target(labels, V)
    logp, ref = (-3 * rng.random(T)).astype(np.float32), (-3 * rng.random(T)).astype(np.float32)
    ref[~live] = np.nan
    beta, scale, loss_scale = 0.1, 0.5 / n, 8.0
    for r in (ref, None):
        pair, loss, d = empty(n), empty(1), empty(T)
        B.axonn_preference_loss(T, n, V, dev_i32(off), dev_i32(labels), f32(logp), None if r is None else f32(r), beta, smoothing, scale, loss_scale,
                                pair, loss, d)
        r_pair, r_loss, r_d = P.preference_loss(logp, r, off, live, np.float32(beta), np.float32(smoothing), np.float32(scale))
        x = np.abs(np.where(live, logp - (0 if r is None else r), 0.0))
        m = np.array([beta * x[a:b].sum() for a, b in zip(off[0:-1:2], off[2::2])])
        e_m = 4 * U * np.minimum(m, 40) + 2 * U                                    # the margin, rounded once
        assert (np.abs(host(pair) - r_pair) <= e_m + 8 * U * (1 + np.abs(r_pair))).all()
        assert abs(host(loss)[0] - r_loss) <= scale * np.sum(e_m + 8 * U * (1 + np.abs(r_pair)))
        e = np.zeros(T)
        for i in range(n):
            e[off[2 * i]:off[2 * i + 2]] = e_m[i] + 16 * U
        assert (np.abs(host(d) - loss_scale * r_d) <= loss_scale * scale * beta * e).all()
        assert not host(d)[~live].any() and not host(d)[:front].any() and not host(d)[T - pad:].any()


@pytest.mark.parametrize("rows", [4, 2000])                       # one workgroup, and one per pair
@pytest.mark.parametrize("smoothing,want", [(0.0, [0.0, np.inf]), (1.0, [np.inf, 0.0]), (0.25, [np.inf, np.inf])])
def test_preference_of_a_token_without_probability(rows, smoothing, want):
    """A log-probability of -inf in the rejected or the chosen answer: an infinite margin, saturated gradients."""
    logp = np.full(rows, -1.0, np.float32)
    off = np.array([0, 1, rows // 2, rows - 1, rows])                # pair 0: rejected has it; pair 1: chosen
    logp[1] = logp[rows // 2] = -np.inf
    pair, loss, d = empty(2), empty(1), empty(rows)
    B.axonn_preference_loss(rows, 2, 9, dev_i32(off), dev_i32(np.zeros(rows)), f32(logp), None, 0.5, smoothing, 1.0, 1.0, pair, loss, d)
    assert host(pair).tolist() == want and host(loss)[0] == np.inf
    # d loss / dm: smoothing - (1 - smoothing) 0 at +inf, smoothing 0 - (1 - smoothing) at -inf
    slope = np.where(np.arange(rows) < rows // 2, 0.5 * smoothing, -0.5 * (1 - smoothing))
    chosen = (np.arange(rows) < 1) | ((np.arange(rows) >= rows // 2) & (np.arange(rows) < rows - 1))
    assert (host(d) == np.where(chosen, slope, -slope)).all()


class Teacher:
    def __init__(self, L, K, tail, how):
        rng, T, V = L.rng, L.T, L.V
        ids = np.stack([rng.choice(V, K, replace=False) if how != "twice" else rng.integers(0, max(V // 2, 1), K) for _ in range(T)])
        u = (4 - 0.5 * np.arange(K) + rng.standard_normal((T, K)) * 0.5).astype(np.float32)
        if how == "fewer":
            ids = np.where(np.arange(K) >= rng.integers(0, K + 1, (T, 1)), rng.choice([-1, V, 1 << 30], (T, K)), ids)
            u[ids < 0] = np.nan
        self.K, self.temperature = K, 1.5
        self.ids, self.u = ids, u
        named = (ids >= 0) & (ids < V)
        mass = np.log(np.sum(np.where(named, np.exp(u.astype(np.float64) / self.temperature), 0), axis=1) + 1e-30)
        self.lse = (mass - np.log(0.4 + 0.59 * rng.random(T))).astype(np.float32) if tail else None


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("how", ["all", "fewer", "twice"])
@pytest.mark.parametrize("T,V,ld,shift", SIZES)
def test_distill_loss(T, V, ld, shift, how, tail):
    L = Logits(T, V, ld, shift, seed=3 * tail + len(how))
    K = {1: 1, 2: 1, 7: 7, 8: 3, 9: 4, 255: 100, 1000: 300, 2047: 1024, 8191: 257}.get(V, 64)
    A = Teacher(L, K, tail, how)
    if tail and K == V:
        pytest.skip("no token is left for the rest's mass: the loss has none")
    w = np.where(L.out, 0.0, L.rng.random(T) + 0.1).astype(np.float32)
    scale = 1.0 if B.ELEM == "bf16" else 64.0
    token, loss = empty(T), empty(1)
    ops = (f32(A.u), dev_i32(A.ids), K, None if A.lse is None else f32(A.lse), A.temperature, f32(w), scale)
    B.axonn_distill_loss(T, V, K, L.buf.t, ld, *ops, token, loss, L.grad.t, ld)
    r_token, r_loss, r_d = P.distill_loss(L.z, A.u, A.ids, A.lse, A.temperature, w)
    # per entry: p (log p - log q), with errors of the exponents, the sums and the two logarithms
    named = (A.ids >= 0) & (A.ids < V)
    tau = A.temperature
    logq = P.log_softmax(L.z / tau)
    top = np.where(named, A.u.astype(np.float64), -1e30).max(axis=1) / tau
    lse_u = np.array([np.log(np.sum(np.exp(A.u[t].astype(np.float64)[named[t]] / tau - top[t]))) + top[t] if named[t].any() else 0.0 for t in range(T)]) \
        if A.lse is None else A.lse.astype(np.float64)
    logp = np.where(named, A.u.astype(np.float64) / tau - lse_u[:, None], 0.0)
    p = np.where(named, np.exp(logp), 0.0)
    gap = np.abs(L.z - L.z.max(axis=1, keepdims=True)) / tau
    mean = np.sum(np.exp(logq) * gap, axis=1)
    row = U * (60 + V / 512 + 4 * mean + 4 * np.log(V + 1) + 4 * np.abs(lse_u) + 4 * np.abs(top))          # of the two log-sum-exps
    at = np.where(named, A.ids, 0)
    lq = np.take_along_axis(logq, at, axis=1)
    e_p = row[:, None] + U * (8 + 4 * np.abs(A.u) / tau * named)
    e_token = np.sum(np.where(named, p * ((2 + np.abs(logp - lq)) * np.nan_to_num(e_p) + 4 * U * (np.abs(logp) + np.abs(lq) + np.take_along_axis(gap, at, axis=1))), 0.0), axis=1)
    e_token = e_token + K * U * np.abs(r_token)
    e_share = np.zeros(T)
    if tail:
        mass = np.array([sum(p[t]) for t in range(T)])
        rest = np.maximum(1 - mass, 0)
        e_rest = np.sum(np.nan_to_num(p * e_p), axis=1) + K * U
        others = np.ones((T, V), bool)
        for t in range(T):
            others[t, at[t][named[t]]] = False
        Q = np.array([np.exp(logq[t][others[t]]).sum() for t in range(T)])
        e_token = e_token + 2 * e_rest * (2 + np.abs(np.log(np.maximum(rest, 1e-12))) + np.abs(np.log(Q))) + 4 * rest * row + 16 * U
        e_share = (e_rest + 4 * rest * row) / Q
    live = (w != 0) & named.any(axis=1)
    assert (np.abs(host(token) - r_token) <= np.where(live, e_token, 0)).all(), (np.abs(host(token) - r_token) / np.maximum(e_token, 1e-30)).max()
    assert abs(host(loss)[0] - r_loss) <= np.sum(w * e_token) + 2 * U * np.sum(np.abs(w * r_token)) + 1e-30
    got, g = L.grad.result() / scale, (w / tau)[:, None]
    q = np.exp(logq)
    full = np.zeros((T, V))
    for t in range(T):
        np.add.at(full[t], at[t][named[t]], p[t][named[t]] * (2 * np.nan_to_num(e_p[t][named[t]]) + (K + 4) * U))
    slack = g * (q * (row[:, None] + U * (8 + 6 * gap)) * 2 + full + q * e_share[:, None] * 2 + 4 * U * np.abs(r_d / np.maximum(g, 1e-30)))
    within(got, r_d, slack, label="distill")
    assert (got[~live] == 0).all()
    token2, before = empty(T), L.grad.t.clone()
    B.axonn_distill_loss(T, V, K, L.buf.t, ld, *ops, token2, None, None, 0)
    assert (token2 == token).all()
    B.axonn_distill_loss(T, V, K, L.buf.t, ld, *ops, token2, loss, L.buf.t, ld)
    assert (L.buf.t == before).all() and (token2 == token).all()
    L.buf.result()


@pytest.mark.parametrize("V", [1, 7, 64, 300, 1024])
@pytest.mark.parametrize("masked", [False, True])
def test_distill_of_all_tokens(V, masked):
    """All tokens that have a probability are named: with the teacher's own log-sum-exp, however it is rounded, as without one."""
    import torch
    T, W, tau = 6, V + 77 * masked, 1.5
    L = Logits(T, V, masked=0.0)
    buf = torch.full((T, W), float("-inf"), dtype=L.buf.t.dtype, device="cuda")
    buf[:, :V] = L.buf.t
    ids = np.stack([L.rng.permutation(V) for _ in range(T)])
    u = L.rng.standard_normal((T, V)).astype(np.float32)
    top = u.max(axis=1).astype(np.float64) / tau
    lse = top + np.log(np.sum(np.exp(u.astype(np.float64) / tau - top[:, None]), axis=1))
    w = f32(np.ones(T))
    got = []
    for x in (None, *(f32(lse.astype(np.float32) + i * np.spacing(np.abs(lse).astype(np.float32))) for i in (-1, 0, 1))):
        token, grad = empty(T), torch.zeros_like(buf)
        B.axonn_distill_loss(T, W, V, buf, W, f32(u), dev_i32(ids), V, x, tau, w, 1.0, token, None, grad, W)
        got.append((host(token), host(grad)))
    # the two log-sum-exps: one and a half steps of the given one; the formed one's exponents, sum and logarithm
    delta = U * (3 * np.abs(lse) + 4 * np.abs(top) + V / 64 + 20 + 3 * (top[:, None] - u / tau).max(axis=1))[:, None]
    p, logp = np.exp(u / tau - lse[:, None]), u / tau - lse[:, None]
    logq = np.take_along_axis(P.log_softmax(L.z / tau), ids, axis=1)
    gap = np.abs(np.take_along_axis(L.z, ids, axis=1) - L.z.max(axis=1, keepdims=True)) / tau
    slack = np.sum(p * (delta * (np.abs(logp - logq) + 1) + 2 * U * (V / 64 + 24) * (np.abs(logp) + gap + np.abs(logq) + 1)), axis=1)
    full = np.zeros((T, W))
    np.put_along_axis(full, ids, p * delta / tau, axis=1)
    for token, grad in got[1:]:
        assert (np.abs(token - got[0][0]) <= 2 * slack).all()
        assert (np.abs(grad - got[0][1]) <= 2 * full * (1 + half_step()) + 2 * half_step() * np.abs(got[0][1]) + 4 * U).all()
        assert not grad[:, V:].any()


def test_infinite_and_lowest_logits():
    """Tokens that the vocabulary's mask leaves out (-inf, or the type's lowest value) have probability 0 and gradient 0."""
    import torch
    T, V = 4, 5000
    low = torch.finfo(B.torch_elem_dtype()).min
    for value in (-float("inf"), low):
        L = Logits(T, V, masked=0.0)
        drop = np.random.default_rng(1).random((T, V)) < 0.5
        drop[0, :2500] = True                                     # whole chunks and whole threads' shares
        drop[np.arange(T), L.targets] = False
        L.z[drop] = -1e30
        L.buf.t[torch.from_numpy(drop).cuda()] = value
        t, ones, zeros = dev_i32(L.targets), f32(np.ones(T)), f32(np.zeros(T))
        logp, lse, token, loss = empty(T), empty(T), empty(T), empty(1)
        B.axonn_token_logprobs_fwd(T, V, L.buf.t, V, t, logp, lse)
        ref = P.token_logprobs(L.z, L.targets)[0]
        assert (np.abs(host(logp) - ref) <= 1e-5).all()
        B.axonn_token_logprobs_bwd(T, V, L.buf.t, V, t, lse, ones, L.grad.t, V)
        assert (L.grad.result()[drop] == 0).all() and np.isfinite(L.grad.result()).all()
        B.axonn_policy_loss(T, V, L.buf.t, V, t, logp, None, ones, ones, 0.2, 0.2, 0.0, 1.0, logp, token, loss, L.grad.t, V)
        assert (L.grad.result()[drop] == 0).all() and np.isfinite(L.grad.result()).all()
        ids = dev_i32(L.targets[:, None])
        B.axonn_distill_loss(T, V, 1, L.buf.t, V, f32(np.zeros((T, 1))), ids, 1, f32(np.full(T, 0.5)), 1.0, ones, 1.0, token, loss, L.grad.t, V)
        assert (L.grad.result()[drop] == 0).all() and np.isfinite(L.grad.result()).all() and np.isfinite(host(token)).all()
        # nothing but the named token is left of the student's distribution
        L.buf.t.fill_(-float("inf"))
        L.buf.t[torch.arange(T), torch.from_numpy(L.targets).cuda()] = 1.0
        B.axonn_distill_loss(T, V, 1, L.buf.t, V, f32(np.zeros((T, 1))), ids, 1, None, 1.0, ones, 1.0, token, loss, L.grad.t, V)
        assert (host(token) == 0).all() and (L.grad.result() == 0).all()


def test_rows_of_nothing_but_masked_logits():
    """They have no softmax: NaN in the row's results, whichever way they are formed, and in no other row's."""
    import torch
    T, V = 3, 2100
    L = Logits(T, V, masked=0.0)
    L.buf.t[1] = -float("inf")
    t, ones, fine = dev_i32(L.targets), f32(np.ones(T)), torch.tensor([True, False, True]).cuda()
    logp, lse, token = empty(T), empty(T), empty(T)
    B.axonn_token_logprobs_fwd(T, V, L.buf.t, V, t, logp, lse)
    assert (torch.isfinite(logp) == fine).all() and lse[1] == -float("inf")
    B.axonn_token_logprobs_bwd(T, V, L.buf.t, V, t, lse, ones, L.grad.t, V)
    assert torch.isfinite(L.grad.t[fine]).all() and torch.isnan(L.grad.t[1]).all()
    B.axonn_policy_loss(T, V, L.buf.t, V, t, f32(np.full(T, -8)), None, ones, ones, 0.2, 0.2, 0.0, 1.0, None, token, None, L.grad.t, V)
    assert (torch.isfinite(token) == fine).all() and torch.isfinite(L.grad.t[fine]).all() and torch.isnan(L.grad.t[1]).all()
    ids = dev_i32(np.tile(np.arange(3), (T, 1)))
    B.axonn_distill_loss(T, V, 3, L.buf.t, V, f32(np.zeros((T, 3))), ids, 3, None, 1.0, ones, 1.0, token, None, L.grad.t, V)
    assert (torch.isfinite(token) == fine).all() and torch.isfinite(L.grad.t[fine]).all() and torch.isnan(L.grad.t[1, :3]).all()


def test_nan_reaches_its_own_row_alone():
    import torch
    T, V = 6, 3001
    L = Logits(T, V, masked=0.0)
    L.buf.t[2, 77] = float("nan")
    L.buf.t[4, :] = float("nan")
    L.buf.t[5, 9] = float("inf")
    t, ones = dev_i32(L.targets), f32(np.ones(T))
    logp, lse, token, loss = empty(T), empty(T), empty(T), empty(1)
    bad = torch.tensor([False, False, True, False, True, True]).cuda()
    B.axonn_token_logprobs_fwd(T, V, L.buf.t, V, t, logp, lse)
    assert (torch.isfinite(logp) == ~bad).all()
    B.axonn_token_logprobs_bwd(T, V, L.buf.t, V, t, lse, ones, L.grad.t, V)
    assert (torch.isfinite(L.grad.t).all(dim=1) == ~bad).all()
    B.axonn_policy_loss(T, V, L.buf.t, V, t, f32(np.zeros(T)), None, ones, ones, 0.2, 0.2, 0.0, 1.0, None, token, loss, L.grad.t, V)
    assert (torch.isfinite(token) == ~bad).all() and (torch.isfinite(L.grad.t).all(dim=1) == ~bad).all() and not torch.isfinite(loss).any()
    ids = dev_i32((L.targets[:, None] + np.arange(3)) % V)
    B.axonn_distill_loss(T, V, 3, L.buf.t, V, f32(np.zeros((T, 3))), ids, 3, f32(np.full(T, 2.0)), 1.0, ones, 1.0, token, loss, L.grad.t, V)
    assert (torch.isfinite(token) == ~bad).all() and (torch.isfinite(L.grad.t).all(dim=1) == ~bad).all()
    # tokens without a part: NaN in their rows and in what comes with them reaches nothing
    labels, w = dev_i32(np.where(bad.cpu().numpy(), -100, L.targets)), torch.where(bad, float("nan"), 1.0)
    B.axonn_policy_loss(T, V, L.buf.t, V, labels, w, w, w, w, 0.2, 0.2, 0.1, 1.0, logp, token, loss, L.grad.t, V)
    assert all(torch.isfinite(x).all() for x in (logp, token, loss, L.grad.t)) and (L.grad.t[bad] == 0).all() and (L.grad.t[~bad] != 0).any()
    none = torch.where(bad[:, None], -1, ids).contiguous()
    B.axonn_distill_loss(T, V, 3, L.buf.t, V, w[:, None].repeat(1, 3).contiguous(), none, 3, w + 2, 1.0, torch.ones_like(w), 1.0, token, loss, L.grad.t, V)
    assert all(torch.isfinite(x).all() for x in (token, loss, L.grad.t)) and (L.grad.t[bad] == 0).all()


def test_losses_captured():
    """One graph of all of them, replayed with other operands, eager work and synchronizations between."""
    import torch
    T, V, K = 40, 5003, 16
    sets = [Logits(T, V, seed=i) for i in range(3)]
    teachers = [Teacher(L, K, True, "all") for L in sets]
    off = np.array([0, 10, 25, 30, 38])
    z, labels, u, ids, tlse = torch.zeros_like(sets[0].buf.t), dev_i32(sets[0].labels), f32(teachers[0].u), dev_i32(teachers[0].ids), f32(teachers[0].lse)
    weight = f32(np.where(sets[0].out, 0, 1.0))
    zeros, ones, offsets = f32(np.full(T, -8.0)), f32(np.ones(T)), dev_i32(off)

    def results():
        out = dict(logp=empty(T), lse=empty(T), dlogp=empty(T), pair=empty(2), loss=empty(1), token=empty(T), loss2=empty(1), token2=empty(T), loss3=empty(1))
        out.update({k: torch.zeros_like(z) for k in ("d1", "d2", "d3")})
        return out

    def run(r, s):
        B.axonn_token_logprobs_fwd(T, V, z, V, labels, r["logp"], r["lse"], s)
        B.axonn_preference_loss(T, 2, V, offsets, labels, r["logp"], zeros, 0.1, 0.1, 0.5, 1.0, r["pair"], r["loss"], r["dlogp"], s)
        B.axonn_token_logprobs_bwd(T, V, z, V, labels, r["lse"], r["dlogp"], r["d1"], V, s)
        B.axonn_policy_loss(T, V, z, V, labels, zeros, zeros, ones, weight, 0.2, 0.2, 0.1, 1.0, None, r["token"], r["loss2"], r["d2"], V, s)
        B.axonn_distill_loss(T, V, K, z, V, u, ids, K, tlse, 1.5, weight, 1.0, r["token2"], r["loss3"], r["d3"], V, s)

    stream = torch.cuda.Stream()
    captured = results()
    stream.wait_stream(torch.cuda.current_stream())
    run(captured, stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        run(captured, stream)
    for i in (0, 1, 2, 0, 1):
        z.copy_(sets[i].buf.t)
        labels.copy_(dev_i32(sets[i].labels))
        weight.copy_(f32(np.where(sets[i].out, 0, 1.0)))
        u.copy_(f32(teachers[i].u)); ids.copy_(dev_i32(teachers[i].ids)); tlse.copy_(f32(teachers[i].lse))
        eager = results()
        run(eager, torch.cuda.current_stream())
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for k, x in eager.items():
            assert (x == captured[k]).all(), (i, k)
