"""Norms of queries and keys with the position rotation, where values and sizes are out of the ordinary: rotated parts that fill no
chunk of 8 while the LDS still holds what earlier kernels left there, and heads whose squares do not fit into 32 bits.  Bounds as in
test_gpu_step_ops.py: half a step of the result's type, and fp32 arithmetic counted in units of U of what went into it."""
import numpy as np
import pytest

from oracle import step_ops as O
from paper_2110_13005_amd import binding as B
from paper_2110_13005_amd.inputs import snap_elem
from helpers import dev_i32
from test_gpu_step_ops import EPS, Padded, U, normal, within, workspace

pytestmark = [pytest.mark.gpu, pytest.mark.parametrize("axonn_elem", ["bf16", "fp16"], indirect=True)]


def leave_nan_in_lds():
    """Every CU's LDS (132 KB of it from its start) filled with numbers that are NaN in 32 bits: an 8-bit product of 256 tiles of 128 x 128,
    one workgroup per CU, whose codes and scales are all 0xff, and which copies whole tiles to its end."""
    import torch
    n, k = 2048, 512
    codes = torch.full((n, k), 0xff, dtype=torch.uint8, device="cuda")
    scales = torch.full((n, 4), 0xff, dtype=torch.uint8, device="cuda")
    out = torch.zeros(n, n, dtype=B.torch_elem_dtype(), device="cuda")
    B.axonn_gemm_fp8(B.EPI_BIAS, n, n, k, codes, scales, codes, scales, out, n)
    return out


def both_passes(T, heads, kv, d, rot, inter, x, dy, gq, gk, pos, before=lambda: None, eps=EPS):
    """-> forward result, dqkv, dgamma_q, dgamma_k of the device (float64), each checked for writes around it."""
    import torch
    width = (heads + 2 * kv) * d
    X, Y, DY, DX = Padded(T, width, values=x), Padded(T, width), Padded(T, width, values=dy), Padded(T, width)
    GQ, GK = Padded(1, d, values=gq[None]), Padded(1, d, values=gk[None])
    inv = 10000.0 ** (-2.0 * np.arange(rot // 2) / max(rot, 1))
    INV = torch.from_numpy(inv).cuda() if rot else None
    POS, shape = dev_i32(pos), (T, T, heads, kv, d, rot, inter)
    dg = [Padded(1, d, dtype=torch.float32) for _ in range(2)]
    ws = workspace(B.axonn_qk_norm_rope_bwd_workspace(T, heads, kv, d))
    norm = (GQ.t, GK.t, eps, POS, INV)
    left = [before()]
    B.axonn_qk_norm_rope_fwd(*shape, X.t, X.ld, *norm, Y.t, Y.ld)
    left.append(before())
    B.axonn_qk_norm_rope_bwd(*shape, DY.t, DY.ld, X.t, X.ld, *norm, DX.t, DX.ld, dg[0].t, dg[1].t, ws)
    assert all(t is None or bool(t.isnan().all()) for t in left)
    eps = float(np.float32(eps))
    ref = (O.qk_norm_rope_fwd(x, heads, kv, d, rot, inter, gq, gk, eps, pos, inv),
           *O.qk_norm_rope_bwd(dy, x, heads, kv, d, rot, inter, gq, gk, eps, pos, inv))
    return (Y.result(), DX.result(), dg[0].result()[0], dg[1].result()[0]), ref


def compare(got, ref, T, heads, kv, d, x, dy, gq, gk, eps=EPS):
    width = (heads + 2 * kv) * d
    eps = float(np.float32(eps))
    # sums of d squares, the root, the gain, an angle off by up to 4 U of a turn's 2 pi, the turn: 80 U of the head's largest
    top = np.abs(ref[0].reshape(T, -1, d)).max(axis=2, keepdims=True)
    slack = np.broadcast_to(80 * U * top, (T, width // d, d)).copy()
    slack[:, heads + kv:] = 0
    within(got[0], ref[0], slack.reshape(T, width), label="forward")
    xs, dys = x.reshape(T, -1, d).astype(np.float64), np.abs(dy.reshape(T, -1, d).astype(np.float64))
    rms = np.sqrt((xs ** 2).mean(axis=2, keepdims=True) + eps)
    g_top = max(np.abs(gq).max(), np.abs(gk).max())
    # dz is off by 8 U of the head's largest dy (times sqrt 2 for a turned pair), the products and sums add their own
    big = np.sqrt(2) * dys.max(axis=2, keepdims=True)
    slack = 160 * U * g_top * big * (1 + np.abs(xs) / rms * np.minimum(1, np.abs(xs).max(axis=2, keepdims=True) / rms)) / rms
    slack[:, heads + kv:] = 0
    within(got[1], ref[1], slack.reshape(T, width), label="dqkv")
    for k, (lo, hi) in enumerate(((0, heads), (heads, heads + kv))):
        terms = (big[:, lo:hi] * np.abs(xs[:, lo:hi]) / rms[:, lo:hi]).sum(axis=(0, 1))
        within(got[2 + k], ref[2 + k], (T * (hi - lo) + 64) * U * terms, U, "gain")


# d, rotated, pair by pair: parts of 1 to 7 elements (rotated halves, rotated pairs, the rest), and of whole and overlapping chunks
@pytest.mark.parametrize("d,rot,inter", [(2, 2, 0), (2, 2, 1), (10, 6, 0), (10, 6, 1), (20, 14, 0), (20, 18, 1), (44, 40, 0), (44, 40, 1),
                                         (128, 2, 0), (128, 6, 1), (256, 254, 0), (256, 254, 1), (100, 60, 0), (36, 20, 1), (64, 64, 0)])
def test_angles_of_no_pair_take_no_part(d, rot, inter):
    rng = np.random.default_rng(d + rot)
    T, heads, kv = 300, 3, 2
    width = (heads + 2 * kv) * d
    x, dy = normal(rng, T, width, std=1.5), normal(rng, T, width)
    gq, gk = normal(rng, d, std=0.3, mean=1.0), normal(rng, d, std=0.3, mean=1.0)
    pos = rng.integers(0, 1 << 16, T)
    got, ref = both_passes(T, heads, kv, d, rot, inter, x, dy, gq, gk, pos, before=leave_nan_in_lds)
    compare(got, ref, T, heads, kv, d, x, dy, gq, gk)


@pytest.mark.parametrize("d,rot,inter", [(128, 128, 0), (64, 32, 1), (10, 6, 0), (100, 60, 0), (256, 256, 1)])
def test_heads_of_huge_values(d, rot, inter):
    """Magnitudes up to the element type's largest: squares of bfloat16 values beyond 2^64 are infinite in 32 bits, the norm is not.
    A head each of 2^40, 2^60, 2^63, 2^64, 2^100, and of values up to the largest, in turn over the tokens (half precision: up to 65504)."""
    rng = np.random.default_rng(d)
    T, heads, kv = 37, 4, 2
    width = (heads + 2 * kv) * d
    dy = normal(rng, T, width)
    gq, gk = normal(rng, d, std=0.3, mean=1.0), normal(rng, d, std=0.3, mean=1.0)
    base = rng.uniform(-1, 1, (T, heads + 2 * kv, d))
    if B.ELEM == "bf16":
        sizes = 2.0 ** np.array([0, 40, 58, 60, 61, 62, 63, 64, 66, 80, 100, 120, 126, 127])
    else:
        sizes = 2.0 ** np.array([0, 8, 12, 15])
    base *= sizes[rng.integers(0, len(sizes), (T, heads + 2 * kv, 1))]
    base[3, 0, d // 2] = base[5, 1, 0] = (2.0 - 2.0 ** -7) * 2.0 ** 127 if B.ELEM == "bf16" else 65504.0
    x = snap_elem(base.astype(np.float32)).reshape(T, width)
    pos = rng.integers(0, 1 << 16, T)
    got, ref = both_passes(T, heads, kv, d, rot, inter, x, dy, gq, gk, pos)
    compare(got, ref, T, heads, kv, d, x, dy, gq, gk)


@pytest.mark.parametrize("eps", [1e-30, 2.0 ** -126, 2.0 ** -149])
def test_heads_of_tiny_values(eps):
    """Squares that vanish in 32 bits, beside an epsilon as small; heads of ordinary values next to them."""
    rng = np.random.default_rng(7)
    T, heads, kv, d, rot = 37, 4, 2, 128, 128
    width = (heads + 2 * kv) * d
    dy = normal(rng, T, width, std=2.0 ** -20)                                # (the gradient is that over the root mean square)
    gq, gk = normal(rng, d, std=0.3, mean=1.0), normal(rng, d, std=0.3, mean=1.0)
    base = rng.uniform(-1, 1, (T, heads + 2 * kv, d))
    sizes = 2.0 ** np.array([0, -30, -48, -50, -52, -60, -63, -70, -75, -90] if B.ELEM == "bf16" else [0, -8, -13])
    x = snap_elem((base * sizes[rng.integers(0, len(sizes), (T, heads + 2 * kv, 1))]).astype(np.float32)).reshape(T, width)
    pos = rng.integers(0, 1 << 16, T)
    got, ref = both_passes(T, heads, kv, d, rot, 0, x, dy, gq, gk, pos, eps=eps)
    if B.ELEM == "bf16":
        compare(got, ref, T, heads, kv, d, x, dy, gq, gk, eps)
    else:                                                                     # the gradient of a small head may pass 65504
        ref = (ref[0], np.where(np.abs(ref[1]) < 65504 / 2, ref[1], 0.0), *ref[2:])
        compare((got[0], np.where(ref[1] != 0, got[1], 0.0), *got[2:]), ref, T, heads, kv, d, x, dy, gq, gk, eps)


def test_infinities_and_nan_stay_in_their_heads():
    rng = np.random.default_rng(1)
    T, heads, kv, d = 9, 2, 1, 64
    width = (heads + 2 * kv) * d
    x, dy = normal(rng, T, width), normal(rng, T, width)
    gq = gk = np.ones(d, np.float32)
    x[2, 5], x[4, d + 1], x[7, 2 * d + 3] = np.inf, np.nan, -np.inf
    hit = np.zeros((T, heads + 2 * kv), bool)
    hit[2, 0] = hit[4, 1] = hit[7, 2] = True
    clean = np.where(np.isfinite(x), x, 0.0).astype(np.float32)
    got, _ = both_passes(T, heads, kv, d, d, 0, x, dy, gq, gk, np.arange(T))
    want, _ = both_passes(T, heads, kv, d, d, 0, clean, dy, gq, gk, np.arange(T))
    for g, w in zip(got[:2], want[:2]):
        g, w = g.reshape(T, -1, d), w.reshape(T, -1, d)
        assert np.array_equal(g[~hit], w[~hit])
        assert np.isnan(g[hit]).any(axis=1).all()


def test_the_smallest_epsilon():
    """The least normal number: heads of zeros come out as zeros, not as 0 * infinity."""
    import torch
    T, d = 5, 16
    x = torch.zeros(T, 3 * d, dtype=B.torch_elem_dtype(), device="cuda")
    x[3, :d] = 1.0
    one, y = torch.ones(d, dtype=x.dtype, device="cuda"), torch.full_like(x, 7.0)
    B.axonn_qk_norm_rope_fwd(T, T, 1, 1, d, 0, 0, x, 3 * d, one, one, 2.0 ** -126, None, None, y, 3 * d)
    assert torch.equal(y, x)
