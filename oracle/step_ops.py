"""Operations of a training step around the layer's own, from their definitions, in float64 numpy: scaled embedding lookup,
norms of queries and keys per head with the position rotation, dropout from the Philox4x32-10 generator, and matrices in 8-bit
floating point (e4m3) with a power-of-two scale for each block of 128.  Shares no code with the GPU path."""
import numpy as np


# ---------------------------------------------------------------------------------------------------------- embedding
def embedding_fwd(tokens, table, scale):
    ids = np.clip(np.asarray(tokens, np.int64), 0, len(table) - 1)
    return np.asarray(table, np.float64)[ids] * scale


def embedding_bwd(tokens, dout, vocab, scale):
    ids = np.clip(np.asarray(tokens, np.int64), 0, vocab - 1)
    out = np.zeros((vocab, dout.shape[1]))
    np.add.at(out, ids, np.asarray(dout, np.float64))
    return out * scale


# ------------------------------------------------------------------------------------- norms of queries and keys, rotation
def _pairs(d, rot, interleaved):
    i = np.arange(rot // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)


def _rotate(z, angle, pairs):
    """z [T, heads, d], angle [T, pairs]."""
    a, b = pairs
    c, s = np.cos(angle)[:, None, :], np.sin(angle)[:, None, :]
    out = z.copy()
    out[..., a] = z[..., a] * c - z[..., b] * s
    out[..., b] = z[..., a] * s + z[..., b] * c
    return out


def qk_norm_rope_fwd(qkv, heads, kv, d, rot, interleaved, gamma_q, gamma_k, eps, positions, inv_freq):
    """qkv [T, (heads + 2 kv) d] -> the same with queries and keys normalised and rotated."""
    T = len(qkv)
    x = np.asarray(qkv, np.float64).reshape(T, heads + 2 * kv, d)
    angle = np.asarray(positions, np.float64)[:, None] * np.asarray(inv_freq, np.float64)[None, :rot // 2]
    out = x.copy()
    for lo, hi, g in ((0, heads, gamma_q), (heads, heads + kv, gamma_k)):
        h = x[:, lo:hi]
        z = np.asarray(g, np.float64) * h / np.sqrt(np.mean(h * h, axis=-1, keepdims=True) + eps)
        out[:, lo:hi] = _rotate(z, angle, _pairs(d, rot, interleaved))
    return out.reshape(T, -1)


def qk_norm_rope_bwd(dout, qkv, heads, kv, d, rot, interleaved, gamma_q, gamma_k, eps, positions, inv_freq):
    """-> dqkv, dgamma_q, dgamma_k."""
    T = len(qkv)
    x = np.asarray(qkv, np.float64).reshape(T, heads + 2 * kv, d)
    dy = np.asarray(dout, np.float64).reshape(x.shape)
    angle = np.asarray(positions, np.float64)[:, None] * np.asarray(inv_freq, np.float64)[None, :rot // 2]
    dx, gains = dy.copy(), []
    for lo, hi, g in ((0, heads, gamma_q), (heads, heads + kv, gamma_k)):
        h, g = x[:, lo:hi], np.asarray(g, np.float64)
        rms = np.sqrt(np.mean(h * h, axis=-1, keepdims=True) + eps)
        dz = _rotate(dy[:, lo:hi], -angle, _pairs(d, rot, interleaved))
        gains.append(np.sum(dz * h / rms, axis=(0, 1)))
        w = dz * g
        dx[:, lo:hi] = w / rms - h * np.mean(w * h, axis=-1, keepdims=True) / rms ** 3
    return dx.reshape(T, -1), gains[0], gains[1]


# ------------------------------------------------------------------------------------------------------------- dropout
def philox4x32(counter, key, rounds=10):
    """Salmon et al. 2011: counter, key: sequences of 4 and 2 arrays of 32-bit words -> 4 arrays of words."""
    m = np.uint64(0xFFFFFFFF)
    c = [np.asarray(v, np.uint64) & m for v in counter]
    k = [int(v) & 0xFFFFFFFF for v in key]
    for _ in range(rounds):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), p1 & m, (p0 >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), p0 & m]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def dropout_threshold(p):
    return int(np.rint(float(np.float32(p)) * 65536.0))


def dropout_keep(T, h, p, seed, offset):
    """Which elements of a [T, h] matrix are kept (bool)."""
    groups = -(-h // 8)
    r, g = np.meshgrid(np.arange(T), np.arange(groups), indexing="ij")
    offset &= (1 << 64) - 1
    w = philox4x32((g, r, np.full_like(g, offset & 0xFFFFFFFF), np.full_like(g, offset >> 32)), (seed, seed >> 32))
    halves = np.stack([half for word in w for half in (word & np.uint64(0xFFFF), word >> np.uint64(16))], axis=-1)
    return halves.reshape(T, groups * 8)[:, :h] >= dropout_threshold(p)


def dropout(x, p, seed, offset, res=None):
    T, h = x.shape
    thr = dropout_threshold(p)
    y = np.where(dropout_keep(T, h, p, seed, offset), np.asarray(x, np.float64), 0.0) * (65536.0 / (65536 - thr) if thr < 65536 else 0.0)
    return y if res is None else y + res


# ------------------------------------------------------------------------------------------------- 8-bit floating point
BLOCK = 128


def e4m3_values():
    """The 256 values of the format, by code (NaN for 0x7f and 0xff)."""
    code = np.arange(256)
    ex, man = code >> 3 & 15, code & 7
    v = np.where(ex == 0, man / 512.0, (1 + man / 8.0) * 2.0 ** (ex - 7))
    v = np.where(code & 128, -v, v)
    v[[0x7f, 0xff]] = np.nan
    return v


def fp8_quantize(x):
    """[R, K] -> codes [R, Kp], scale bytes [R, S]: the nearest of the format's values, ties to the even code."""
    x = np.asarray(x, np.float64)
    R, K = x.shape
    nb = -(-K // BLOCK)
    v = np.zeros((R, nb * BLOCK))
    v[:, :K] = x
    v = v.reshape(R, nb, BLOCK)
    finite = np.isfinite(v)
    amax = np.max(np.where(finite, np.abs(v), 0.0), axis=2)
    e = np.full(amax.shape, -127)
    for step in range(-126, 128):                       # the least exponent that is large enough
        e = np.where(amax > 448.0 * 2.0 ** (step - 1), step, e)
    u = np.where(finite, v / 2.0 ** e[:, :, None].astype(np.float64), 0.0)
    positive = e4m3_values()[:0x7f]
    at = np.searchsorted(positive, np.abs(u))           # positive[at - 1] < |u| <= positive[at]
    hi = np.minimum(at, 0x7e)
    lo = np.maximum(hi - 1, 0)
    mid = (positive[lo] + positive[hi]) / 2
    code = np.where(np.abs(u) > mid, hi, np.where(np.abs(u) < mid, lo, np.where(lo % 2 == 0, lo, hi)))
    code = np.where(np.signbit(v), code | 128, code)
    code = np.where(finite, code, 0x7f)
    scales = np.zeros((R, -(-nb // 4) * 4), np.uint8)
    scales[:, :nb] = e + 127
    return code.reshape(R, -1).astype(np.uint8), scales


def fp8_values(codes, scales):
    """What codes and scales stand for, [R, Kp]."""
    nb = codes.shape[1] // BLOCK
    v = e4m3_values()[codes].reshape(len(codes), nb, BLOCK)
    return (v * 2.0 ** (scales[:, :nb, None].astype(np.float64) - 127)).reshape(codes.shape)
