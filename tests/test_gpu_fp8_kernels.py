"""The kernels of the 8-bit product, each at sizes that the launcher is known to send to it (test_fp8_choice.py checks that on the
host), with every epilogue: ragged edges, workgroups that take several tiles one after the other, contractions of 2 to 10 blocks of
128.  Results against float64 sums of what the codes stand for."""
import math

import numpy as np
import pytest

from oracle import step_ops as O
from paper_2110_13005_amd import binding as B
from test_gpu_step_ops import Padded, U, _product_slack, half_step

pytestmark = [pytest.mark.gpu, pytest.mark.parametrize("axonn_elem", ["bf16", "fp16"], indirect=True)]

# M, N, K -> width of the tiles with 16-bit and with 32-bit results.  256 x 256 tiles, 16-bit: 225 tiles (one each, no share per XCD),
# 256 with ragged edges, 506 (two each, the last ones alone), 728 (two or three each), 1024 (four each); 2, 3, 4, 6, 7, 8 and 9 blocks.
TILES = {(3800, 3800, 1000): (256, 256), (3841, 4090, 480): (256, 256), (5500, 5800, 300): (256, 256), (5500, 5800, 500): (256, 256),
         (5500, 5800, 700): (256, 256), (5500, 5800, 860): (256, 256), (5500, 5800, 1100): (256, 256), (5500, 5800, 1250): (256, 256),
         (7000, 6600, 1150): (256, 256), (8190, 8180, 250): (256, 128), (2047, 2049, 1900): (128, 128), (1700, 1812, 136): (128, 64),
         (5500, 5800, 130): (128, 128), (513, 130, 2000): (64, 64)}


def codes_of(rng, rows, K, low=-9, high=-4):
    """Codes and scales of random values (normal, with the scale of a block anywhere in 2^low .. 2^high) on the device, and the
    values in float64."""
    import torch
    nb = -(-K // 128)
    codes = (torch.randn(rows, 128 * nb, generator=rng, device="cuda") * 64).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    codes[:, K:] = 0
    scales = torch.zeros(rows, -(-nb // 4) * 4, dtype=torch.uint8, device="cuda")
    scales[:, :nb] = torch.randint(127 + low, 128 + high, (rows, nb), generator=rng, device="cuda").to(torch.uint8)
    return codes, scales, stands_for(codes, scales)


def stands_for(codes, scales):
    import torch
    values = torch.from_numpy(O.e4m3_values()).cuda()
    e = scales[:, :codes.shape[1] // 128].double() - 127.0
    return values[codes.long()] * torch.exp2(e).repeat_interleave(128, dim=1)


def near(out, ref, slack, half, label):
    """Half a step of the result's type, and `slack`."""
    tiny = 2.0 ** -25 if B.ELEM == "fp16" and half > U else 2.0 ** -134
    err = (out.t.double() - ref).abs()
    bad = ~(err <= half * (ref.abs() + slack) + slack + tiny)
    assert not bool(bad.any()), (label, int(bad.sum()), bad.nonzero()[0].tolist(), float(out.t.double()[bad][0]), float(ref[bad][0]))
    edge = out.buf.clone()
    edge.as_strided((out.rows, out.cols), (out.ld, 1), out.t.storage_offset()).fill_(out.MARK)
    assert bool((edge == out.MARK).all()), (label, "written outside the matrix")


@pytest.mark.parametrize("M,N,K", list(TILES))
def test_every_epilogue(M, N, K):
    import torch
    rng = torch.Generator(device="cuda")
    rng.manual_seed(M + N + K)
    qa, sa, a = codes_of(rng, M, K)
    qb, sb, b = codes_of(rng, N, K)
    y, mags = a @ b.t(), a.abs() @ b.abs().t()
    narrow, wide, half = _product_slack(mags, K, False), _product_slack(mags, K, True), half_step()
    dt = B.torch_elem_dtype()
    bias = torch.randn(N, generator=rng, device="cuda").to(dt)
    side = torch.randn(M, N, generator=rng, device="cuda").to(dt)
    args = (M, N, K, qa, sa, qb, sb)

    def result(values=None, pad=3, shift=1, dtype=None):
        out = Padded(M, N, N + pad, shift, dtype=dtype)
        if values is not None:
            out.t.copy_(values)
        return out

    C = result()
    B.axonn_gemm_fp8(B.EPI_BIAS, *args, C.t, C.ld, bias=bias)
    z = y + bias.double()
    near(C, z, narrow + U * z.abs(), half, "bias")
    again = result()
    B.axonn_gemm_fp8(B.EPI_BIAS, *args, again.t, again.ld, bias=bias)
    assert torch.equal(again.t, C.t)                                          # the same bits
    C, S = result(), result(side, 5, 0)
    B.axonn_gemm_fp8(B.EPI_BIAS_RES, *args, C.t, C.ld, bias=bias, res=S.t, ld_res=S.ld)
    near(C, z + side.double(), narrow + 2 * U * (z.abs() + side.double().abs()), half, "residual")
    C, X = result(), result(pad=4, shift=0)
    B.axonn_gemm_fp8(B.EPI_BIAS_GELU, *args, C.t, C.ld, bias=bias, aux=X.t, ld_aux=X.ld)
    # Phi is off by 1.5e-7 and some roundings; |GeLU'| <= 1.13 and |GeLU''| <= 0.8
    cdf, dz = 0.5 * torch.erfc(-z / math.sqrt(2.0)), narrow + U * z.abs()
    near(C, z * cdf, 1.13 * dz + 4e-7 * (1 + z.abs()), half, "gelu")
    near(X, cdf + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi), 0.8 * dz + 8e-7 * (1 + z.abs()), half, "gelu derivative")
    S = result(side)
    B.axonn_gemm_fp8(B.EPI_DGELU, *args, S.t, S.ld, aux=S.t, ld_aux=S.ld)       # the result over the factor
    near(S, y * side.double(), (narrow + U * y.abs()) * side.double().abs(), half, "times the derivative")
    for epi, dtype, slack, step in ((B.EPI_ACC_BF16, None, narrow, half), (B.EPI_ACC_F32, torch.float32, wide, U)):
        C = result(side, dtype=dtype)
        B.axonn_gemm_fp8(epi, *args, C.t, C.ld, accumulate=1)
        near(C, y + side.double(), slack + U * (y.abs() + side.double().abs()), step, "added to %d" % epi)
        C = result(dtype=dtype)
        B.axonn_gemm_fp8(epi, *args, C.t, C.ld)
        near(C, y, slack, step, "overwritten %d" % epi)
        again = result(dtype=dtype)
        B.axonn_gemm_fp8(epi, *args, again.t, again.ld)
        assert torch.equal(again.t, C.t)


@pytest.mark.parametrize("M,N,K", [(513, 130, 2000), (2047, 2049, 1900), (5500, 5800, 500)])
def test_sums_that_cancel(M, N, K):
    """Every block has products of 2^16 of both signs beside small ones.  16-bit results keep to what is documented of them, 7 * 2^-13 of
    the products' magnitudes, and 32-bit results to a sum in fp32, however much cancels."""
    import torch
    rng = torch.Generator(device="cuda")
    rng.manual_seed(K)
    (qa, sa, _), (qb, sb, _) = codes_of(rng, M, K), codes_of(rng, N, K)
    qa[:, ::16], qb[:, ::16], qa[:, 1::16], qb[:, 1::16] = 0x78, 0x78, 0xf8, 0x78     # 256 * 256 and -256 * 256
    qa[:, K:], qb[:, K:] = 0, 0
    sa.clamp_(max=120)                                                              # of one size over a row, so that they cancel
    sa[sa > 0], sb[sb > 0] = 120, 120
    a, b = stands_for(qa, sa), stands_for(qb, sb)
    y, mags = a @ b.t(), a.abs() @ b.abs().t()
    for epi, dtype, half in ((B.EPI_BIAS, None, half_step()), (B.EPI_ACC_F32, torch.float32, U)):
        C = Padded(M, N, dtype=dtype)
        B.axonn_gemm_fp8(epi, M, N, K, qa, sa, qb, sb, C.t, N)
        near(C, y, _product_slack(mags, K, dtype is not None), half, epi)


def test_values_at_the_ends_of_the_range():
    """Blocks of 2^-127 and of 2^119 times the codes, whose products with blocks of the other end are ordinary numbers: nothing of them is
    lost on the way to 16-bit or 32-bit results."""
    import torch
    rng = torch.Generator(device="cuda")
    rng.manual_seed(3)
    M, N, K = 70, 90, 512
    (qa, sa, _), (qb, sb, _) = codes_of(rng, M, K), codes_of(rng, N, K)
    for k, (ea, eb) in enumerate(((-127, 115), (119, -124), (-120, 112), (-126, 119))):
        sa[:, k], sb[:, k] = 127 + ea, 127 + eb
    # what the quantiser makes of bfloat16 numbers, all multiples of 2^-133: at 2^-127 (2^-126) every code from 2^-3 (2^-4) on, of the
    # smaller ones not all, and none of them is needed here
    for q, k, least in ((qa, 0, 0x20), (qa, 3, 0x18)):
        block = q[:, 128 * k:128 * k + 128]
        block[(block & 0x7f) < least] = 0
    a, b = stands_for(qa, sa), stands_for(qb, sb)
    y, mags = a @ b.t(), a.abs() @ b.abs().t()
    for epi, dtype, half in ((B.EPI_BIAS, None, half_step()), (B.EPI_ACC_F32, torch.float32, U)):
        C = Padded(M, N, dtype=dtype)
        B.axonn_gemm_fp8(epi, M, N, K, qa, sa, qb, sb, C.t, N)
        near(C, y, _product_slack(mags, K, dtype is not None), half, epi)
