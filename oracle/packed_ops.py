"""Operations on packed sequences from their definitions, in float64 numpy: causal attention inside sequences of different lengths with
shared key / value heads, log-probabilities of tokens, the clipped policy loss, the preference loss of pairs of sequences, distillation
from a teacher's top logits.  Shares no code with the GPU path."""
import numpy as np


# ---------------------------------------------------------------------------------------------------------- attention
def sequences(offsets, T):
    """[(first row, row behind the last)]: offsets are clamped to [0, T] and to what is in front of them."""
    ends = np.maximum.accumulate(np.clip(np.asarray(offsets, np.int64), 0, T))
    return list(zip(ends[:-1].tolist(), ends[1:].tolist()))


def _split(x, heads, kv, d):
    return [x[:, a * d:b * d].reshape(len(x), b - a, d) for a, b in ((0, heads), (heads, heads + kv), (heads + kv, heads + 2 * kv))]


def attention_probabilities(q, k, scale):
    """One head of one sequence: [n, d] each -> P [n, n], log-sum-exp [n]."""
    s = scale * (q @ k.T)
    s[np.triu_indices(len(q), 1)] = -np.inf
    m = s.max(axis=1, keepdims=True)
    e = np.exp(s - m)
    return e / e.sum(axis=1, keepdims=True), m[:, 0] + np.log(e.sum(axis=1))


def packed_attention_fwd(qkv, offsets, heads, kv, d, scale):
    """-> o [T, heads d], lse [heads, T]; NaN in rows of no sequence."""
    T = len(qkv)
    q, k, v = _split(np.asarray(qkv, np.float64), heads, kv, d)
    o, lse = np.full((T, heads, d), np.nan), np.full((heads, T), np.nan)
    for a, b in sequences(offsets, T):
        for h in range(heads if b > a else 0):
            j = h // (heads // kv)
            P, lse[h, a:b] = attention_probabilities(q[a:b, h], k[a:b, j], scale)
            o[a:b, h] = P @ v[a:b, j]
    return o.reshape(T, -1), lse


def packed_attention_bwd(qkv, dout, offsets, heads, kv, d, scale):
    """-> dqkv; NaN in rows of no sequence."""
    T = len(qkv)
    q, k, v = _split(np.asarray(qkv, np.float64), heads, kv, d)
    do = np.asarray(dout, np.float64).reshape(T, heads, d)
    g = np.full((T, heads + 2 * kv, d), np.nan)
    for a, b in sequences(offsets, T):
        g[a:b] = 0.0
        for h in range(heads if b > a else 0):
            j = h // (heads // kv)
            P, _ = attention_probabilities(q[a:b, h], k[a:b, j], scale)
            dP = do[a:b, h] @ v[a:b, j].T
            dS = scale * P * (dP - (P * dP).sum(axis=1, keepdims=True))
            g[a:b, h] = dS @ k[a:b, j]
            g[a:b, heads + j] += dS.T @ q[a:b, h]
            g[a:b, heads + kv + j] += P.T @ do[a:b, h]
    return g.reshape(T, -1)


# ------------------------------------------------------------------------------------------------------------- losses
def log_softmax(z):
    z = np.asarray(z, np.float64)
    m = z.max(axis=-1, keepdims=True)
    return z - m - np.log(np.exp(z - m).sum(axis=-1, keepdims=True))


def has_target(targets, V):
    t = np.asarray(targets)
    return (t >= 0) & (t < V)


def token_logprobs(logits, targets):
    """-> logp, lse; 0 where there is no target."""
    live = has_target(targets, logits.shape[1])
    at = np.where(live, targets, 0)[:, None]
    logp = np.take_along_axis(log_softmax(logits), at, axis=1)[:, 0]
    return np.where(live, logp, 0.0), np.where(live, np.take_along_axis(np.asarray(logits, np.float64), at, axis=1)[:, 0] - logp, 0.0)


def token_logprobs_bwd(logits, targets, dlogp):
    V = logits.shape[1]
    slope = np.where(has_target(targets, V), np.asarray(dlogp, np.float64), 0.0)
    d = -slope[:, None] * np.exp(log_softmax(logits))
    rows = np.flatnonzero(slope)
    d[rows, np.asarray(targets)[rows]] += slope[rows]
    d[slope == 0] = 0.0
    return d


def policy_loss(logits, targets, old_logp, ref_logp, advantage, weight, clip_low, clip_high, kl_coef):
    """-> logp, token_loss, loss, dlogits."""
    w = np.where(has_target(targets, logits.shape[1]), np.asarray(weight, np.float64), 0.0)
    live, A = w != 0, np.asarray(advantage, np.float64)
    logp = np.where(live, token_logprobs(logits, targets)[0], 0.0)
    r = np.exp(logp - old_logp)
    plain, clipped = r * A, np.clip(r, 1 - clip_low, 1 + clip_high) * A
    x = (0.0 if ref_logp is None else np.asarray(ref_logp, np.float64)) - logp
    loss = -np.minimum(plain, clipped) + (kl_coef * (np.exp(x) - x - 1) if kl_coef else 0.0)
    slope = np.where(plain <= clipped, -plain, 0.0) + (kl_coef * (1 - np.exp(x)) if kl_coef else 0.0)
    loss = np.where(live, loss, 0.0)
    return logp, loss, float(np.sum(w * loss)), token_logprobs_bwd(logits, targets, np.where(live, w * slope, 0.0))


def preference_loss(logp, ref_logp, offsets, live, beta, smoothing, scale):
    """-> pair_loss, loss, dlogp."""
    x = np.where(live, np.asarray(logp, np.float64) - (0.0 if ref_logp is None else np.asarray(ref_logp, np.float64)), 0.0)
    spans, dlogp, losses = sequences(offsets, len(x)), np.zeros(len(x)), []
    for (a, b), (c, d) in zip(spans[0::2], spans[1::2]):
        m = beta * (x[a:b].sum() - x[c:d].sum())
        sigma = 1 / (1 + np.exp(-m))
        losses.append(sum(share * np.logaddexp(0, side) for share, side in ((1 - smoothing, -m), (smoothing, m)) if share > 0))
        slope = scale * beta * (smoothing * sigma - (1 - smoothing) * (1 - sigma))
        dlogp[a:b], dlogp[c:d] = slope, -slope
    return np.array(losses), scale * float(np.sum(losses)), np.where(live, dlogp, 0.0)


def distill_loss(logits, teacher, ids, teacher_lse, temperature, weight):
    """-> token_loss, loss, dlogits.  One token after the other, one entry after the other."""
    T, V = logits.shape
    logq_all = log_softmax(np.asarray(logits, np.float64) / temperature)
    loss, dz = np.zeros(T), np.zeros((T, V))
    for t in range(T):
        entries = [(int(i), float(u) / temperature) for i, u in zip(ids[t], teacher[t]) if 0 <= i < V]
        if not entries or weight[t] == 0:
            continue
        u = np.array([e[1] for e in entries])
        m = u.max()
        norm = m + np.log(np.exp(u - m).sum()) if teacher_lse is None else float(teacher_lse[t])
        logq = logq_all[t]
        others, p = np.ones(V, bool), np.zeros(V)
        for (i, x) in entries:
            e = np.exp(x - norm)
            loss[t] += e * (x - norm - logq[i]) if e else 0.0
            p[i] += e
            others[i] = False
        if teacher_lse is not None:
            P = max(1.0 - p.sum(), 0.0)
            if P > 0 and np.isfinite(logq[others]).any():              # else the student has no other tokens
                share = log_softmax(np.asarray(logits[t][others], np.float64) / temperature)
                likely = share.argmax()
                loss[t] += P * (np.log(P) - (logq[others][likely] - share[likely]))
                p[others] = P * np.exp(share)
        # of sum_i p_i (log p_i - log q_i), whatever the p_i sum up to
        g = p.sum() * np.exp(logq) - p
        dz[t] = weight[t] / temperature * g
    return loss, float(np.sum(np.asarray(weight, np.float64) * loss)), dz
