"""Packed attention of heads above 128 columns, which has tiles and accumulators of its own: a sequence's results have the same bits wherever
it lies and whatever its neighbours hold, infinities and NaN too, in Q, K, V and in the gradient that comes in."""
import numpy as np
import pytest

from test_gpu_packed_ops import Attention

pytestmark = [pytest.mark.gpu, pytest.mark.parametrize("axonn_elem", ["bf16", "fp16"], indirect=True)]


@pytest.mark.parametrize("heads,kv,d", [(4, 2, 188), (3, 3, 192), (16, 2, 160), (2, 1, 132), (8, 8, 176), (4, 2, 128), (4, 1, 64)])
@pytest.mark.parametrize("bad", [[3], [1, 3, 6]])
def test_a_sequence_does_not_depend_on_its_neighbours(heads, kv, d, bad):
    import torch
    lens = [150, 31, 260, 97, 150, 1, 290, 260]
    same = [(0, 4), (2, 7)]
    a = Attention(np.random.default_rng(8), lens, heads, kv, d)
    off = a.offsets
    for m in (a.qkv, a.dout):
        for i, j in same:
            m.t[off[j]:off[j + 1]] = m.t[off[i]:off[i + 1]]
    good = torch.ones(a.T, dtype=torch.bool)
    for i in bad:
        good[off[i]:off[i + 1]] = False
    outs = []
    for value in (1.0, float("nan"), float("inf")):
        a.qkv.t[~good] = a.dout.t[~good] = value
        a.run()
        outs.append([x.clone() for x in (a.o.t, a.lse.t(), a.dqkv.t)])
    for out in outs:
        for x, y in zip(outs[0], out):
            assert torch.isfinite(x[good]).all() and (x[good] == y[good]).all()
            for i, j in same:
                assert (y[off[i]:off[i + 1]] == y[off[j]:off[j + 1]]).all()
