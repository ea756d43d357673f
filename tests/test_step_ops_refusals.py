"""What the single operations of step_ops.py's kind refuse, and with which status: checked on the host, in front of any launch."""
import ctypes

import pytest

from paper_2110_13005_amd import binding as B

A = 1 << 20         # an address that is never read: every call below is refused first
INV, UNS = B.AXONN_EINVAL, B.AXONN_EUNSUPPORTED


def refused(status, fn, *args, **kw):
    with pytest.raises(B.AxonnError) as e:
        fn(*args, **kw)
    assert e.value.status == status, e.value


def with_args(base, **changes):
    """Arguments of a call with some replaced by position."""
    out = list(base)
    for k, v in changes.items():
        out[int(k[1:])] = v
    return out


def test_embedding():
    ok = [4, 8, 10, A, A, 1.0, A, 8]
    for pos in (3, 4, 6):
        refused(INV, B.axonn_embedding_fwd, *with_args(ok, **{"_%d" % pos: None}))
    for pos in (0, 1, 2):
        refused(INV, B.axonn_embedding_fwd, *with_args(ok, **{"_%d" % pos: 0}))
    refused(INV, B.axonn_embedding_fwd, *with_args(ok, _7=7))
    refused(UNS, B.axonn_embedding_fwd, *with_args(ok, _0=(1 << 24) + 1))
    refused(UNS, B.axonn_embedding_fwd, *with_args(ok, _1=65536, _7=65536))
    refused(UNS, B.axonn_embedding_fwd, *with_args(ok, _1=1024, _2=1 << 25, _7=1024))
    ok = [4, 8, 10, A, A, 8, 1.0, A, 0, 0, A]
    for pos in (3, 4, 7, 10):
        refused(INV, B.axonn_embedding_bwd, *with_args(ok, **{"_%d" % pos: None}))
    refused(INV, B.axonn_embedding_bwd, *with_args(ok, _5=7))
    refused(INV, B.axonn_embedding_bwd, *with_args(ok, _10=A + 8))
    refused(INV, B.axonn_embedding_bwd, *with_args(ok, _7=A + 2, _8=1))
    refused(UNS, B.axonn_embedding_bwd, *with_args(ok, _2=(1 << 24) + 1))
    refused(INV, B.axonn_embedding_bwd_workspace, 0, 8, 10)
    assert B.load().axonn_embedding_bwd_workspace(4, 8, 10, None) == INV
    assert B.axonn_embedding_bwd_workspace(4, 8, 10) >= 16
    assert B.axonn_embedding_bwd_workspace(1 << 24, 65535, 1 << 18) > 0


def test_qk_norm_rope():
    ok = [6, 3, 4, 2, 16, 8, 0, A, 128, A, A, 1e-6, None, A, A, 128]
    for pos in (7, 9, 10, 13, 14):
        refused(INV, B.axonn_qk_norm_rope_fwd, *with_args(ok, **{"_%d" % pos: None}))
    for pos in (0, 1, 2, 3, 4):
        refused(INV, B.axonn_qk_norm_rope_fwd, *with_args(ok, **{"_%d" % pos: 0}))
    for rot in (-2, 7, 18):
        refused(INV, B.axonn_qk_norm_rope_fwd, *with_args(ok, _5=rot))
    for eps in (0.0, -1e-6, float("nan"), float("inf")):
        refused(INV, B.axonn_qk_norm_rope_fwd, *with_args(ok, _11=eps))
    refused(INV, B.axonn_qk_norm_rope_fwd, *with_args(ok, _13=A + 4))
    refused(INV, B.axonn_qk_norm_rope_fwd, *with_args(ok, _8=127))
    refused(INV, B.axonn_qk_norm_rope_fwd, *with_args(ok, _15=127, _14=2 * A))
    refused(INV, B.axonn_qk_norm_rope_fwd, *with_args(ok, _15=136))                # in place, another leading dimension
    refused(UNS, B.axonn_qk_norm_rope_fwd, *with_args(ok, _4=15, _5=0))
    refused(UNS, B.axonn_qk_norm_rope_fwd, *with_args(ok, _4=258, _8=4096, _15=4096))
    refused(UNS, B.axonn_qk_norm_rope_fwd, *with_args(ok, _0=(1 << 24) + 1))
    ok = [6, 3, 4, 2, 16, 8, 0, A, 128, 2 * A, 128, A, A, 1e-6, None, A, 3 * A, 128, A, A, A]
    for pos in (7, 9, 11, 12, 15, 16, 18, 19, 20):
        refused(INV, B.axonn_qk_norm_rope_bwd, *with_args(ok, **{"_%d" % pos: None}))
    for pos in (8, 10, 17):
        refused(INV, B.axonn_qk_norm_rope_bwd, *with_args(ok, **{"_%d" % pos: 127}))
    refused(INV, B.axonn_qk_norm_rope_bwd, *with_args(ok, _16=A, _17=136))
    refused(INV, B.axonn_qk_norm_rope_bwd, *with_args(ok, _16=2 * A, _17=136))
    refused(INV, B.axonn_qk_norm_rope_bwd, *with_args(ok, _20=A + 4))
    refused(INV, B.axonn_qk_norm_rope_bwd_workspace, 6, 4, 0, 16)
    assert B.axonn_qk_norm_rope_bwd_workspace(6, 4, 2, 16) > 0


def test_dropout():
    ok = [4, 8, A, 8, None, 0, 0.1, 1, 2, None, 2 * A, 8]
    for pos in (2, 10):
        refused(INV, B.axonn_dropout_fwd, *with_args(ok, **{"_%d" % pos: None}))
    for pos in (0, 1):
        refused(INV, B.axonn_dropout_fwd, *with_args(ok, **{"_%d" % pos: 0}))
    for p in (-0.1, 1.1, float("nan")):
        refused(INV, B.axonn_dropout_fwd, *with_args(ok, _6=p))
    for pos in (3, 11):
        refused(INV, B.axonn_dropout_fwd, *with_args(ok, **{"_%d" % pos: 7}))
    refused(INV, B.axonn_dropout_fwd, *with_args(ok, _4=A, _5=7))
    refused(INV, B.axonn_dropout_fwd, *with_args(ok, _10=A, _11=9))
    refused(INV, B.axonn_dropout_fwd, *with_args(ok, _4=2 * A, _5=16))
    refused(INV, B.axonn_dropout_fwd, *with_args(ok, _9=A + 4))
    refused(UNS, B.axonn_dropout_fwd, *with_args(ok, _0=(1 << 24) + 1))
    refused(UNS, B.axonn_dropout_fwd, *with_args(ok, _0=1 << 24, _1=1 << 14, _3=1 << 14, _11=1 << 14))
    ok = [4, 8, A, 8, 0.1, 1, 2, None, 2 * A, 8]
    refused(INV, B.axonn_dropout_bwd, *with_args(ok, _2=None))
    refused(INV, B.axonn_dropout_bwd, *with_args(ok, _4=2.0))
    refused(INV, B.axonn_dropout_bwd, *with_args(ok, _9=7))


def test_fp8():
    ok = [4, 8, A, 8, A, A, None, None]
    refused(INV, B.axonn_fp8_quantize, *with_args(ok, _2=None))
    refused(INV, B.axonn_fp8_quantize, *with_args(ok, _4=None))
    refused(INV, B.axonn_fp8_quantize, *with_args(ok, _4=None, _5=None))
    refused(INV, B.axonn_fp8_quantize, *with_args(ok, _6=A))
    refused(INV, B.axonn_fp8_quantize, *with_args(ok, _3=7))
    refused(INV, B.axonn_fp8_quantize, *with_args(ok, _4=A + 8))
    refused(INV, B.axonn_fp8_quantize, *with_args(ok, _5=A + 2))
    refused(INV, B.axonn_fp8_quantize, *with_args(ok, _0=0))
    refused(UNS, B.axonn_fp8_quantize, *with_args(ok, _0=(1 << 22) + 1))
    refused(UNS, B.axonn_fp8_quantize, *with_args(ok, _0=1 << 22, _1=1 << 15, _3=1 << 15))
    ok = [0, 16, 16, 16, A, A, A, A, A, 16]
    for pos in (4, 5, 6, 7, 8):
        refused(INV, B.axonn_gemm_fp8, *with_args(ok, **{"_%d" % pos: None}))
    for pos in (1, 2, 3):
        refused(INV, B.axonn_gemm_fp8, *with_args(ok, **{"_%d" % pos: 0}))
    for epi in (-1, 6):
        refused(INV, B.axonn_gemm_fp8, *with_args(ok, _0=epi))
    refused(INV, B.axonn_gemm_fp8, *with_args(ok, _9=15))
    refused(INV, B.axonn_gemm_fp8, *with_args(ok, _0=B.EPI_BIAS_RES))
    refused(INV, B.axonn_gemm_fp8, *with_args(ok, _0=B.EPI_BIAS_RES), res=A, ld_res=15)
    for epi in (B.EPI_BIAS_GELU, B.EPI_DGELU):
        refused(INV, B.axonn_gemm_fp8, *with_args(ok, _0=epi))
        refused(INV, B.axonn_gemm_fp8, *with_args(ok, _0=epi), aux=A, ld_aux=15)
    refused(INV, B.axonn_gemm_fp8, *with_args(ok, _4=A + 8))
    refused(INV, B.axonn_gemm_fp8, *with_args(ok, _7=A + 2))
    refused(INV, B.axonn_gemm_fp8, *with_args(ok, _0=B.EPI_ACC_F32, _8=A + 2))
    refused(INV, B.axonn_gemm_fp8, *with_args(ok, _0=B.EPI_BIAS_RES), res=A, ld_res=24)              # the result over its residual
    refused(INV, B.axonn_gemm_fp8, *with_args(ok, _0=B.EPI_DGELU), aux=A, ld_aux=24)
    refused(INV, B.axonn_gemm_fp8, *with_args(ok, _0=B.EPI_BIAS_GELU), aux=A, ld_aux=16)
    refused(UNS, B.axonn_gemm_fp8, *with_args(ok, _3=(1 << 22) + 1))
    refused(UNS, B.axonn_gemm_fp8, *with_args(ok, _1=1 << 20, _2=1 << 20, _9=1 << 20))


def test_both_builds_refuse_alike():
    for elem in ("bf16", "fp16"):
        lib = B.load(elem)
        assert lib.axonn_dropout_fwd(4, 8, None, 8, None, 0, ctypes.c_float(0.1), 0, 0, None, None, 8, None) == INV
        assert b"dropout_fwd" in lib.axonn_last_error()
