"""Norms of queries and keys with the position rotation, where values and sizes are out of the ordinary: rotated parts that fill no
chunk of 8 while the LDS still holds what earlier kernels left there.  Bounds as in
test_gpu_step_ops.py: half a step of the result's type, and fp32 arithmetic counted in units of U of what went into it."""
import numpy as np
import pytest

from oracle import step_ops as O
from paper_2110_13005_amd import binding as B
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


def both_passes(T, heads, kv, d, rot, inter, x, dy, gq, gk, pos, before=lambda: None):
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
    norm = (GQ.t, GK.t, EPS, POS, INV)
    left = [before()]
    B.axonn_qk_norm_rope_fwd(*shape, X.t, X.ld, *norm, Y.t, Y.ld)
    left.append(before())
    B.axonn_qk_norm_rope_bwd(*shape, DY.t, DY.ld, X.t, X.ld, *norm, DX.t, DX.ld, dg[0].t, dg[1].t, ws)
    assert all(t is None or bool(t.isnan().all()) for t in left)
    eps = float(np.float32(EPS))
    ref = (O.qk_norm_rope_fwd(x, heads, kv, d, rot, inter, gq, gk, eps, pos, inv),
           *O.qk_norm_rope_bwd(dy, x, heads, kv, d, rot, inter, gq, gk, eps, pos, inv))
    return (Y.result(), DX.result(), dg[0].result()[0], dg[1].result()[0]), ref


def compare(got, ref, T, heads, kv, d, x, dy, gq, gk):
    width = (heads + 2 * kv) * d
    eps = float(np.float32(EPS))
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
