"""Dropout of matrices that take several chunks per lane, with rows of whole and of shorter last chunks, against the generator's float64
definition; the bounds are test_gpu_step_ops.py's."""
import numpy as np
import pytest

from oracle import step_ops as O
from paper_2110_13005_amd import binding as B
from test_gpu_step_ops import Padded, U, normal, within

pytestmark = [pytest.mark.gpu, pytest.mark.parametrize("axonn_elem", ["bf16", "fp16"], indirect=True)]


@pytest.mark.parametrize("T,h,ld,shift", [(4300, 1001, 1003, 1), (1, 4200000, 4200000, 0), (530000, 3, 5, 1), (66000, 64, 64, 0)])
def test_large_dropout(T, h, ld, shift):
    rng = np.random.default_rng(T + h)
    x, res, p, seed, offset = normal(rng, T, h), normal(rng, T, h), 0.3, 0xABCDEF0123456789, (1 << 40) + 3
    X, R, Y = Padded(T, h, ld, shift, x), Padded(T, h, ld, 0, res), Padded(T, h, ld + 1, shift)
    B.axonn_dropout_fwd(T, h, X.t, ld, R.t, ld, p, seed, offset, None, Y.t, ld + 1)
    ref = O.dropout(x, p, seed, offset, res)
    within(Y.result(), ref, 3 * U * (np.abs(ref - res) + np.abs(ref)))
    B.axonn_dropout_bwd(T, h, X.t, ld, p, seed, offset, None, X.t, ld)           # in place
    ref = O.dropout(x, p, seed, offset)
    got = X.result()
    within(got, ref, 2 * U * np.abs(ref))
    assert not got[ref == 0].any()
