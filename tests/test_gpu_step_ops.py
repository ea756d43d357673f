"""GPU parity of the operations of a training step around the layer's own (scaled embedding, query / key norms with rotation,
dropout, 8-bit linear maps) with their float64 definitions, element by element, at the sizes, strides and values where they can
go wrong.

Bounds: a result is one rounding to its type of an fp32 value, so |got - ref| <= half a step of the result plus what fp32
arithmetic may have added: `slack`, counted for each operation in units of U = 2^-24 of the magnitudes that went into it."""
import numpy as np
import pytest

from oracle import step_ops as O
from oracle import transformer as OT
from paper_2110_13005_amd import binding as B
from paper_2110_13005_amd.inputs import snap_elem
from helpers import dev_i32, host, rel_fro

pytestmark = [pytest.mark.gpu, pytest.mark.parametrize("axonn_elem", ["bf16", "fp16"], indirect=True)]
U = 2.0 ** -24
EPS = 1e-5


def half_step():
    """Half a step of the element type, relative to the value."""
    return 2.0 ** -8 if B.ELEM == "bf16" else 2.0 ** -11


def within(got, ref, slack, half=None, label=""):
    """got: float64 array of the device's result; half: of its type (default: the element type)."""
    half = half_step() if half is None else half
    tiny = 2.0 ** -25 if B.ELEM == "fp16" and half > U else 2.0 ** -134       # half a step below the smallest normal number
    bound = half * (np.abs(ref) + slack) + slack + tiny
    err = np.abs(got - ref)
    bad = ~(err <= bound)
    assert not bad.any(), (label, int(bad.sum()), "first", np.argwhere(bad)[0], got[bad][0], np.broadcast_to(ref, got.shape)[bad][0])


def normal(rng, *shape, std=1.0, mean=0.0):
    return snap_elem((rng.standard_normal(shape) * std + mean).astype(np.float32)).reshape(shape)


class Padded:
    """A matrix inside a larger buffer: `shift` elements in front, rows of `ld` elements, everything else filled with a mark that
    must be there afterwards."""
    MARK = 7.0

    def __init__(self, rows, cols, ld=None, shift=0, values=None, dtype=None):
        import torch
        self.rows, self.cols, self.ld = rows, cols, ld or cols
        self.buf = torch.full((shift + rows * self.ld + 64,), self.MARK, dtype=dtype or B.torch_elem_dtype(), device="cuda")
        self.t = self.buf[shift:shift + rows * self.ld].view(rows, self.ld)[:, :cols]
        if values is not None:
            self.t.copy_(torch.from_numpy(np.ascontiguousarray(values, np.float32)))

    def result(self):
        """Values as float64; checks that nothing around them was written."""
        import torch
        out = host(self.t)
        outside = torch.ones_like(self.buf, dtype=torch.bool)
        torch.as_strided(outside, (self.rows, self.cols), (self.ld, 1), self.t.storage_offset()).zero_()
        assert bool((self.buf[outside] == self.MARK).all()), "written outside the matrix"
        return out


def workspace(nbytes):
    import torch
    return torch.full((nbytes,), 0xA5, dtype=torch.uint8, device="cuda")      # what a workspace holds does not matter


# ---------------------------------------------------------------------------------------------------------- embedding
@pytest.mark.parametrize("T,h,V,ld,shift", [(1, 1, 1, 1, 0), (1, 8, 5, 8, 0), (3, 7, 9, 11, 1), (70, 64, 33, 64, 0), (65, 129, 100, 130, 3),
                                            (130, 520, 7, 520, 0), (9, 2056, 50, 2064, 8), (33, 1000, 1000, 1003, 1), (5, 4100, 3, 4100, 2)])
def test_embedding_lookup(T, h, V, ld, shift):
    rng = np.random.default_rng(T + h)
    tokens = rng.integers(-2, V + 3, T)
    table = Padded(V, h, values=normal(rng, V, h), shift=shift)
    out, scale = Padded(T, h, ld, shift), np.float32(np.sqrt(h))
    B.axonn_embedding_fwd(T, h, V, dev_i32(tokens), table.t, float(scale), out.t, ld)
    ref = O.embedding_fwd(tokens, host(table.t), float(scale))
    within(out.result(), ref, 2 * U * np.abs(ref))


def _tokens(rng, how, T, V):
    if how == "one":
        return np.full(T, V // 2)
    if how == "distinct":
        return rng.permutation(V)[:T] if T <= V else rng.integers(0, V, T)
    if how == "outside":
        return rng.integers(-V, 2 * V, T)
    p = 1.0 / (np.arange(V) + 2.7) ** 1.07                                    # ordinary text
    return rng.permutation(V)[rng.choice(V, T, p=p / p.sum())]


@pytest.mark.parametrize("T,h,V,how,fp32,ld,shift", [
    (1, 1, 1, "one", 1, 1, 0), (1, 8, 3, "one", 0, 8, 0), (2, 5, 2, "distinct", 1, 9, 1), (31, 64, 40, "text", 0, 64, 0),
    (32, 64, 3, "text", 1, 64, 0), (33, 65, 40, "outside", 0, 67, 1), (64, 96, 1, "one", 0, 96, 0), (200, 384, 1000, "distinct", 1, 384, 0),
    (255, 136, 70, "text", 0, 136, 0), (257, 136, 70, "text", 1, 136, 0), (700, 520, 2000, "text", 0, 520, 0),
    (1023, 40, 1500, "outside", 1, 43, 1), (1025, 40, 1024, "text", 0, 40, 0), (2049, 264, 1025, "text", 1, 264, 0),
    (4100, 24, 70000, "text", 0, 24, 0), (5000, 17, 300000, "text", 1, 17, 0), (6000, 48, 5, "text", 0, 48, 0),
    (9000, 16, 2000000, "distinct", 0, 16, 0), (20000, 8, 100, "one", 1, 8, 0), (20000, 33, 60000, "text", 0, 33, 0),
    (70000, 9, 2000, "text", 1, 9, 0)])
def test_embedding_gradient(T, h, V, how, fp32, ld, shift):
    """Overwriting, then adding to the result; every size around a piece, a sort tile, a digit and the limits between the
    kernels; runs of one id over many pieces; ids outside the table."""
    import torch
    rng = np.random.default_rng(T + h + V)
    scale = float(np.float32(0.75))
    dt = torch.float32 if fp32 else B.torch_elem_dtype()
    half = 0.5 * torch.finfo(dt).eps
    dtable = Padded(V, h, shift=2 * shift if fp32 else shift, dtype=dt)
    ws = workspace(B.axonn_embedding_bwd_workspace(T, h, V))
    old, bits = np.zeros((V, h)), None
    for accumulate in (0, 1):
        tokens, dout = _tokens(rng, how, T, V), Padded(T, h, ld, shift, normal(rng, T, h))
        terms = O.embedding_bwd(tokens, np.abs(host(dout.t)), V, abs(scale))
        count = np.bincount(np.clip(tokens, 0, V - 1), minlength=V)[:, None]
        before = dtable.t.clone()
        B.axonn_embedding_bwd(T, h, V, dev_i32(tokens), dout.t, ld, scale, dtable.t, fp32, accumulate, ws)
        got = dtable.result()
        ref = old + O.embedding_bwd(tokens, host(dout.t), V, scale)
        within(got, ref, (count + 3) * U * (terms + np.abs(old)), half)
        if accumulate:
            assert torch.equal(dtable.t[torch.from_numpy(count[:, 0] == 0).cuda()], before[torch.from_numpy(count[:, 0] == 0).cuda()])
        else:
            assert not got[count[:, 0] == 0].any()
            again = Padded(V, h, dtype=dt)
            B.axonn_embedding_bwd(T, h, V, dev_i32(tokens), dout.t, ld, scale, again.t, fp32, 0, ws)
            assert torch.equal(again.t, dtable.t)                             # the same bits
        old = got


@pytest.mark.parametrize("T,V", [(5, 40), (5, 4000), (300, 4000), (17000, 300)])
def test_embedding_gradient_of_nan_and_infinity(T, V):
    """What is not a number in one token's gradient stays in its row, and rows without tokens are zeros whatever the scale."""
    import torch
    rng, h = np.random.default_rng(T), 72
    tokens = rng.integers(0, V // 2, T)
    dout = normal(rng, T, h)
    dout[T // 2] = np.nan
    named, hit = np.unique(tokens), tokens[T // 2]
    ws = workspace(B.axonn_embedding_bwd_workspace(T, h, V))
    for scale in (1.0, np.inf):
        for dt in (B.torch_elem_dtype(), torch.float32):
            out, x = Padded(V, h, dtype=dt), Padded(T, h, values=dout)
            B.axonn_embedding_bwd(T, h, V, dev_i32(tokens), x.t, h, scale, out.t, int(dt == torch.float32), 0, ws)
            got = out.result()
            assert np.isnan(got[hit]).all()
            assert not np.delete(got, named, axis=0).any()
            if scale == 1.0:
                assert np.isfinite(np.delete(got, hit, axis=0)).all()


# ------------------------------------------------------------------------------------- norms of queries and keys, rotation
def _qk_case(rng, T, heads, kv, d, rot, positions, big=False):
    width = (heads + 2 * kv) * d
    x = normal(rng, T, width, std=1.5)
    x[0, :d] = 0                                                              # a head of zeros
    if big:
        x[T // 2] = snap_elem(x[T // 2] * np.float32(1000.0))
    gq, gk = normal(rng, d, std=0.3, mean=1.0), normal(rng, d, std=0.3, mean=1.0)
    inv = 10000.0 ** (-2.0 * np.arange(rot // 2) / max(rot, 1))
    pos = {"none": None, "far": rng.integers(0, 1 << 20, T), "signed": rng.integers(-2 ** 31, 2 ** 31 - 1, T)}[positions]
    return width, x, gq, gk, inv, pos


QK = [  # T, seq, heads, kv, d, rot, interleaved, positions, padding, shift
    (1, 1, 1, 1, 2, 2, 0, "none", 0, 0), (1, 1, 4, 4, 64, 64, 0, "far", 0, 0), (5, 5, 16, 16, 64, 32, 1, "far", 0, 0),
    (7, 3, 4, 2, 128, 128, 0, "none", 8, 0), (6, 6, 3, 1, 128, 128, 1, "signed", 3, 1), (9, 4, 2, 2, 188, 188, 0, "none", 0, 0),
    (9, 4, 2, 2, 188, 188, 1, "none", 1, 1), (4, 4, 5, 5, 80, 48, 0, "far", 0, 0), (4, 2, 8, 1, 256, 256, 0, "none", 0, 0),
    (3, 3, 2, 1, 256, 254, 0, "far", 5, 0), (3, 3, 2, 1, 256, 2, 1, "far", 0, 0), (8, 8, 2, 1, 96, 0, 0, "none", 0, 0),
    (5, 5, 3, 3, 10, 6, 1, "signed", 1, 1), (2050, 1025, 2, 1, 64, 64, 0, "none", 0, 0), (2100, 2100, 1, 1, 20, 14, 0, "far", 0, 0),
    (700, 700, 12, 4, 128, 128, 0, "none", 0, 0), (33, 33, 5, 2, 100, 60, 0, "far", 0, 0), (33, 11, 5, 2, 100, 60, 1, "none", 1, 0),
    (20, 20, 3, 3, 36, 20, 1, "none", 0, 1), (20, 20, 3, 3, 46, 36, 0, "far", 0, 0), (70, 70, 40, 40, 128, 128, 0, "none", 0, 0)]


@pytest.mark.parametrize("T,seq,heads,kv,d,rot,inter,positions,pad,shift", QK)
def test_qk_norm_rope(T, seq, heads, kv, d, rot, inter, positions, pad, shift):
    import torch
    rng = np.random.default_rng(T + d + rot)
    width, x, gq, gk, inv, pos = _qk_case(rng, T, heads, kv, d, rot, positions, big=T > 1)
    X, Y = Padded(T, width, width + pad, shift, x), Padded(T, width, width + 2 * pad, shift)
    GQ, GK = Padded(1, d, shift=shift, values=gq[None]), Padded(1, d, shift=shift, values=gk[None])
    INV = torch.from_numpy(inv).cuda() if rot else None
    POS = None if pos is None else dev_i32(pos)
    shape = (T, seq, heads, kv, d, rot, inter)
    norm = (GQ.t, GK.t, EPS, POS, INV)
    B.axonn_qk_norm_rope_fwd(*shape, X.t, X.ld, *norm, Y.t, Y.ld)
    where = np.arange(T) % seq if pos is None else pos
    eps = float(np.float32(EPS))
    ref = O.qk_norm_rope_fwd(x, heads, kv, d, rot, inter, gq, gk, eps, where, inv)
    # sums of d squares, the root, the gain, an angle off by up to 4 U of a turn's 2 pi, the turn: 80 U of the head's largest
    top = np.abs(ref.reshape(T, -1, d)).max(axis=2, keepdims=True)
    slack = np.broadcast_to(80 * U * top, (T, width // d, d)).copy()
    slack[:, heads + kv:] = 0
    got = Y.result()
    within(got, ref, slack.reshape(T, width))
    v = (heads + kv) * d
    assert np.array_equal(got[:, v:], x[:, v:])
    B.axonn_qk_norm_rope_fwd(*shape, X.t, X.ld, *norm, X.t, X.ld)                # in place
    assert np.array_equal(X.result(), got)

    X = Padded(T, width, width + pad, shift, x)
    dy = normal(rng, T, width)
    DY, DX = Padded(T, width, width + 2 * pad, shift, dy), Padded(T, width, width + pad, shift)
    dg = [Padded(1, d, dtype=torch.float32) for _ in range(2)]
    ws = workspace(B.axonn_qk_norm_rope_bwd_workspace(T, heads, kv, d))
    B.axonn_qk_norm_rope_bwd(*shape, DY.t, DY.ld, X.t, X.ld, *norm, DX.t, DX.ld, dg[0].t, dg[1].t, ws)
    rdx, rgq, rgk = O.qk_norm_rope_bwd(dy, x, heads, kv, d, rot, inter, gq, gk, eps, where, inv)
    xs, dys = x.reshape(T, -1, d).astype(np.float64), np.abs(dy.reshape(T, -1, d).astype(np.float64))
    rms = np.sqrt((xs ** 2).mean(axis=2, keepdims=True) + eps)
    g_top = max(np.abs(gq).max(), np.abs(gk).max())
    # dz is off by 8 U of the head's largest dy (times sqrt 2 for a turned pair), the products and sums add their own
    big = np.sqrt(2) * dys.max(axis=2, keepdims=True)
    slack = 160 * U * g_top * big * (1 + np.abs(xs) / rms * np.minimum(1, np.abs(xs).max(axis=2, keepdims=True) / rms)) / rms
    slack[:, heads + kv:] = 0
    gdx = DX.result()
    within(gdx, rdx, slack.reshape(T, width))
    assert np.array_equal(gdx[:, v:], dy[:, v:])
    for k, (lo, hi, r) in enumerate(((0, heads, rgq), (heads, heads + kv, rgk))):
        terms = (big[:, lo:hi] * np.abs(xs[:, lo:hi]) / rms[:, lo:hi]).sum(axis=(0, 1))
        within(dg[k].result()[0], r, (T * (hi - lo) + 64) * U * terms, U, "gain")
    again = [torch.empty(d, device="cuda") for _ in range(2)]
    B.axonn_qk_norm_rope_bwd(*shape, DY.t, DY.ld, X.t, X.ld, *norm, DY.t, DY.ld, *again, ws)      # in place of the gradient
    assert np.array_equal(DY.result(), gdx)
    assert torch.equal(again[0], dg[0].t[0]) and torch.equal(again[1], dg[1].t[0])
    DY = Padded(T, width, values=dy)
    B.axonn_qk_norm_rope_bwd(*shape, DY.t, width, X.t, X.ld, *norm, X.t, X.ld, *again, ws)        # in place of the input
    assert np.array_equal(X.result(), gdx)


# ------------------------------------------------------------------------------------------------------------- dropout
@pytest.mark.parametrize("T,h,p,ld,shift", [(1, 1, 0.5, 1, 0), (1, 8, 0.1, 8, 0), (3, 7, 0.5, 9, 1), (7, 1001, 0.1, 1003, 1), (33, 64, 0.0, 64, 0),
                                            (33, 65, 1.0, 66, 0), (200, 520, 0.9, 520, 0), (1030, 24, 0.25, 24, 0), (5, 20000, 1e-5, 20000, 0),
                                            (2, 9, 1 - 2.0 ** -16, 9, 1)])
def test_dropout(T, h, p, ld, shift):
    import torch
    rng = np.random.default_rng(T + h)
    x, res = normal(rng, T, h), normal(rng, T, h)
    seed, offset = 0xFEDCBA9876543210 + T, (1 << 35) + 7 * h
    keep = O.dropout_keep(T, h, p, seed, offset)
    x[~keep] = np.where(rng.random((~keep).sum()) < 0.5, np.inf, np.nan)       # what is dropped does not matter
    clean = np.where(keep, x, 0.0).astype(np.float64)
    X, R, Y = Padded(T, h, ld, shift, x), Padded(T, h, ld + 1, shift, res), Padded(T, h, ld + 2, 0)
    B.axonn_dropout_fwd(T, h, X.t, ld, R.t, ld + 1, p, seed, offset, None, Y.t, ld + 2)
    ref = O.dropout(clean, p, seed, offset, res)
    within(Y.result(), ref, 3 * U * (np.abs(ref - res) + np.abs(ref)))
    Z = Padded(T, h, ld, shift)
    B.axonn_dropout_fwd(T, h, X.t, ld, None, 0, p, seed, offset, None, Z.t, ld)
    ref = O.dropout(clean, p, seed, offset)
    got = Z.result()
    within(got, ref, 2 * U * np.abs(ref))
    assert not got[~keep].any()
    # the same mask from an offset in device memory (64 bits, with carry), backward, in place
    low = 0xFFFFFFFFFFFFFFF0
    dev = torch.tensor([(offset - low) % 2 ** 64], dtype=torch.int64, device="cuda")
    B.axonn_dropout_bwd(T, h, X.t, ld, p, seed, low, dev, X.t, ld)
    assert np.array_equal(X.result(), got)
    B.axonn_dropout_fwd(T, h, X.t, ld, R.t, ld + 1, 0.0, 1, 2, None, R.t, ld + 1)     # p = 0 into the residual
    ref = got + res
    within(R.result(), ref, U * np.abs(ref))


def test_dropout_seeds_and_offsets_are_independent():
    import torch
    T, h, p = 64, 256, 0.5
    x = torch.ones(T, h, dtype=B.torch_elem_dtype(), device="cuda")
    masks = []
    for seed, offset in ((0, 0), (1, 0), (1 << 32, 0), (0, 1), (0, 1 << 32)):
        y = torch.empty_like(x)
        B.axonn_dropout_fwd(T, h, x, h, None, 0, p, seed, offset, None, y, h)
        assert np.array_equal(host(y) != 0, O.dropout_keep(T, h, p, seed, offset))
        masks.append(host(y) != 0)
    for i in range(len(masks)):
        for j in range(i):
            # agreement of independent masks: 1/2, five standard deviations
            assert abs((masks[i] == masks[j]).mean() - 0.5) < 5 * 0.5 / np.sqrt(T * h)


# ------------------------------------------------------------------------------------------------- 8-bit floating point
def quantised(x, rows=True, cols=True, ld=None, shift=0):
    """Device codes and scales of x's rows and of its transpose's, in buffers filled with marks."""
    import torch
    R, C = x.shape
    X = Padded(R, C, ld, shift, x)

    def form(r, k):
        kp = -(-k // 128) * 128
        return (torch.full((r + 1, kp), 0x55, dtype=torch.uint8, device="cuda"),
                torch.full((r + 1, -(-kp // 512) * 4), 0x55, dtype=torch.uint8, device="cuda"))
    a = form(R, C) if rows else (None, None)
    b = form(C, R) if cols else (None, None)
    B.axonn_fp8_quantize(R, C, X.t, X.ld, *a, *b)
    for f in a + b:
        assert f is None or bool((f[-1] == 0x55).all())                       # nothing behind the last row
    return tuple(None if f is None else f[:-1] for f in a + b)


@pytest.mark.parametrize("R,C,pad,shift", [(1, 1, 0, 0), (1, 128, 0, 0), (3, 7, 2, 1), (127, 129, 0, 0), (128, 128, 0, 0), (130, 520, 8, 0),
                                           (513, 200, 1, 3), (40, 1100, 0, 0), (1100, 40, 0, 0)])
def test_codes_and_scales(R, C, pad, shift):
    """Bit for bit, rows and transpose, together and each alone; blocks of zeros, of tiny and of huge values, block maxima at
    the border between two scales, values half way between two codes, infinities and NaN."""
    rng = np.random.default_rng(R + C)
    x = normal(rng, R, C) * np.exp2(rng.integers(-12, 9, (R, 1))).astype(np.float32)
    x = snap_elem(x).reshape(R, C)
    flat = x.reshape(-1)
    for k, v in enumerate((448.0, 450.0, 224.0, 17.0, 19.0, -17.0, 2.0 ** -10, 3 * 2.0 ** -10, 0.0, -0.0, 2.0 ** -14, 2.0 ** -24)):
        flat[(k * 37) % flat.size] = v
    if R > 100:
        x[5:100] = 0
        x[-1] = 1e-30 if B.ELEM == "bf16" else 2.0 ** -24
        x[-2, ::3] = 3e38 if B.ELEM == "bf16" else 65504.0
        x[-3, 0], x[-4, C // 2] = np.inf, -np.inf
        x[-5, -1] = np.nan
        x[-7] *= np.float32(2.0 ** -120 if B.ELEM == "bf16" else 2.0 ** -14)      # into the subnormal numbers
        x[-8], x[-8, 3] = 0, 2.0 ** -133 if B.ELEM == "bf16" else 2.0 ** -24
    x = snap_elem(x).reshape(R, C)
    q, s, qt, st = quantised(x, ld=C + pad, shift=shift)
    for got, want in zip((q, s, qt, st), O.fp8_quantize(x) + O.fp8_quantize(x.T)):
        got = got.cpu().numpy()
        assert np.array_equal(got, want), (np.argwhere(got != want)[:5], got[got != want][:5], want[got != want][:5])
    one = quantised(x, cols=False, ld=C + pad, shift=shift)[:2] + quantised(x, rows=False)[2:]
    for got, want in zip(one, (q, s, qt, st)):
        assert bool((got == want).all())


def _product(rng, M, N, K):
    a, b = normal(rng, M, K), normal(rng, N, K, std=0.05)
    a[M // 2] = 0
    (qa, sa), (qb, sb) = O.fp8_quantize(a), O.fp8_quantize(b)
    import torch
    dev = tuple(torch.from_numpy(t).cuda() for t in (qa, sa, qb, sb))
    va, vb = O.fp8_values(qa, sa), O.fp8_values(qb, sb)
    return dev, va @ vb.T, np.abs(va) @ np.abs(vb).T


# The matrix unit drops, in a group of 8 products, what lies 13 binary places below the largest: 7 times 2^-13 of it, which the
# sum of the magnitudes bounds.  32-bit results are sums in fp32.
def _product_slack(mags, K, wide):
    return (K + 8) * U * mags if wide else (7 * 2.0 ** -13 + (K + 8) * U) * mags


PRODUCTS = [(1, 1, 1, 0, 0), (1, 8, 128, 0, 0), (5, 3, 130, 2, 1), (64, 64, 512, 0, 0), (65, 66, 640, 1, 1), (200, 1000, 392, 0, 0), (129, 40, 1700, 4, 0),
            (1700, 1812, 136, 0, 0), (1999, 1601, 300, 3, 1), (4100, 4090, 136, 0, 0), (300, 16, 4100, 0, 0)]


@pytest.mark.parametrize("M,N,K,pad,shift", PRODUCTS)
def test_product_with_every_epilogue(M, N, K, pad, shift):
    import math
    import torch
    rng = np.random.default_rng(M + N + K)
    (qa, sa, qb, sb), y, mags = _product(rng, M, N, K)
    bias, side = normal(rng, N, std=0.5), normal(rng, M, N)
    BIAS = Padded(1, N, shift=shift, values=bias[None])
    narrow, wide = _product_slack(mags, K, False), _product_slack(mags, K, True)
    args = (M, N, K, qa, sa, qb, sb)
    erf = np.vectorize(math.erf) if M * N < 300000 else None

    def result(dtype=None, values=None):
        return Padded(M, N, N + pad, shift if dtype is None else 0, values, dtype)
    C = result()
    B.axonn_gemm_fp8(B.EPI_BIAS, *args, C.t, C.ld)
    got = C.result()
    within(got, y, narrow, label="plain")
    # rounding to nearest is at most a third of a step in the mean square; the matrix unit's part is far below that
    assert rel_fro(got, y) <= 0.64 * half_step() or np.linalg.norm(y) == 0
    B.axonn_gemm_fp8(B.EPI_BIAS, *args, C.t, C.ld, bias=BIAS.t)
    within(C.result(), y + bias, narrow + U * np.abs(y + bias), label="bias")
    S = result(values=side)
    B.axonn_gemm_fp8(B.EPI_BIAS_RES, *args, S.t, S.ld, bias=BIAS.t, res=S.t, ld_res=S.ld)          # the result over the residual
    within(S.result(), y + bias + side, narrow + 2 * U * (np.abs(y + bias) + np.abs(side)), label="residual")
    if erf is not None:
        z = y + bias
        cdf, pdf = 0.5 * (1 + erf(z / math.sqrt(2))), np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
        C, X = result(), Padded(M, N, N + 2 * pad, shift)
        B.axonn_gemm_fp8(B.EPI_BIAS_GELU, *args, C.t, C.ld, bias=BIAS.t, aux=X.t, ld_aux=X.ld)
        # Phi is off by 1.5e-7 and some roundings; |GeLU'| <= 1.13 and |GeLU''| <= 0.8
        dz = narrow + U * np.abs(z)
        within(C.result(), z * cdf, 1.13 * dz + 4e-7 * (1 + np.abs(z)), label="gelu")
        within(X.result(), cdf + z * pdf, 0.8 * dz + 8e-7 * (1 + np.abs(z)), label="gelu derivative")
    S = result(values=side)
    B.axonn_gemm_fp8(B.EPI_DGELU, *args, S.t, S.ld, aux=S.t, ld_aux=S.ld)                           # the result over the factor
    within(S.result(), y * side, (narrow + U * np.abs(y)) * np.abs(side), label="dgelu")
    for epi, dt, old, slack in ((B.EPI_ACC_F32, torch.float32, side, wide), (B.EPI_ACC_BF16, None, side, narrow)):
        C = result(dt, old)
        half = U if dt is not None else None
        B.axonn_gemm_fp8(epi, *args, C.t, C.ld, accumulate=1)
        within(C.result(), y + old, slack + U * (np.abs(y) + np.abs(old)), half, "accumulate %d" % epi)
        B.axonn_gemm_fp8(epi, *args, C.t, C.ld)
        got = C.result()
        within(got, y, slack, half, "overwrite %d" % epi)
        again = result(dt)
        B.axonn_gemm_fp8(epi, *args, again.t, again.ld)
        assert np.array_equal(again.result(), got)


def test_product_of_extreme_blocks():
    """Scales of 2^-127 and of 2^100, blocks of zeros beside large ones, a NaN that stays in its row, in 16 and in 32 bits."""
    import torch
    M, N, K = 20, 24, 384
    rng = np.random.default_rng(0)
    a, b = rng.standard_normal((M, K)), rng.standard_normal((N, K))
    a[:, :128] *= 2.0 ** 100
    b[:, :128] *= 2.0 ** -100
    a[:, 128:256] = 0
    b[:, 128:256] *= 2.0 ** 90
    a[3, 300] = np.nan
    (qa, sa), (qb, sb) = O.fp8_quantize(a), O.fp8_quantize(b)
    qb[5, 256:], sb[5, 2] = 1, 0                        # the smallest number the form has
    va, vb = O.fp8_values(qa, sa), O.fp8_values(qb, sb)
    dev = [torch.from_numpy(t).cuda() for t in (qa, sa, qb, sb)]
    ref, mags = va @ vb.T, np.abs(va) @ np.abs(vb).T
    live = np.arange(M) != 3
    for epi, dt in ((B.EPI_BIAS, None), (B.EPI_ACC_F32, torch.float32)):
        C = Padded(M, N, dtype=dt)
        B.axonn_gemm_fp8(epi, M, N, K, *dev, C.t, N)
        got = C.result()
        assert np.isnan(got[3]).all()
        within(got[live], ref[live], _product_slack(mags, K, dt is not None)[live], U if dt is not None else None)


# ------------------------------------------------------------------------------------------------------ used together
def test_captured_and_replayed():
    """Every operation in one captured graph, replayed with new inputs and a moving dropout offset, between eager calls on the
    same stream; each replay against the eager calls."""
    import torch
    dt = B.torch_elem_dtype()
    T, h, V, a, d = 300, 192, 500, 3, 64
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dt)
    tokens = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    table, gq, gk, w = rnd(V, h), 1 + 0.1 * rnd(d), 1 + 0.1 * rnd(d), rnd(3 * h, h)
    inv = torch.from_numpy(10000.0 ** (-np.arange(32) / 32.0)).cuda()
    offset = torch.zeros(1, dtype=torch.int64, device="cuda")
    qw, sw = torch.empty(3 * h, 256, dtype=torch.uint8, device="cuda"), torch.empty(3 * h, 4, dtype=torch.uint8, device="cuda")
    B.axonn_fp8_quantize(3 * h, h, w, h, qw, sw)
    ws_e = workspace(B.axonn_embedding_bwd_workspace(T, h, V))
    ws_q = workspace(B.axonn_qk_norm_rope_bwd_workspace(T, a, a, d))

    def buffers():
        e = lambda *s, dtype=dt: torch.empty(*s, dtype=dtype, device="cuda")
        return dict(x=e(T, h), y=e(T, h), qx=e(T, 256, dtype=torch.uint8), sx=e(T, 4, dtype=torch.uint8), qkv=e(T, 3 * h), rot=e(T, 3 * h),
                    back=e(T, 3 * h), dq=e(d, dtype=torch.float32), dk=e(d, dtype=torch.float32), dx=e(T, h), dt=e(V, h, dtype=torch.float32))

    def step(b, stream):
        B.axonn_embedding_fwd(T, h, V, tokens, table, 2.0, b["x"], h, stream)
        B.axonn_dropout_fwd(T, h, b["x"], h, table, h, 0.2, 5, 6, offset, b["y"], h, stream)
        B.axonn_fp8_quantize(T, h, b["y"], h, b["qx"], b["sx"], stream=stream)
        B.axonn_gemm_fp8(B.EPI_BIAS, T, 3 * h, h, b["qx"], b["sx"], qw, sw, b["qkv"], 3 * h, stream=stream)
        B.axonn_qk_norm_rope_fwd(T, 100, a, a, d, d, 0, b["qkv"], 3 * h, gq, gk, EPS, None, inv, b["rot"], 3 * h, stream)
        B.axonn_qk_norm_rope_bwd(T, 100, a, a, d, d, 0, b["rot"], 3 * h, b["qkv"], 3 * h, gq, gk, EPS, None, inv, b["back"], 3 * h, b["dq"],
                                 b["dk"], ws_q, stream)
        B.axonn_dropout_bwd(T, h, b["back"], 3 * h, 0.2, 5, 6, offset, b["dx"], h, stream)
        B.axonn_embedding_bwd(T, h, V, tokens, b["dx"], h, 2.0, b["dt"], 1, 0, ws_e, stream)

    graph, stream, made, eager = torch.cuda.CUDAGraph(), torch.cuda.Stream(), buffers(), buffers()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        step(made, stream)
    for i in range(4):
        tokens.copy_(torch.randint(-3, V + 3, (T,), generator=g, device="cuda", dtype=torch.int32))
        offset.fill_(i)
        torch.cuda.synchronize()
        for t in made.values():
            t.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        step(eager, None)
        torch.cuda.synchronize()
        for k in made:
            assert torch.equal(made[k], eager[k]), (i, k)


def test_calls_at_once_on_two_streams():
    """The same operations on other data, side by side with workspaces of their own."""
    import torch
    dt = B.torch_elem_dtype()
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    T, h, V, d = 2900, 256, 700, 64
    inv = torch.from_numpy(10000.0 ** (-np.arange(32) / 32.0)).cuda()
    one = torch.ones(d, dtype=dt, device="cuda")
    data = [(torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32), torch.randn(T, h, generator=g, device="cuda").to(dt),
             torch.randn(T, 4 * h, generator=g, device="cuda").to(dt)) for _ in range(2)]

    def step(k, stream):
        tokens, dout, qkv = data[k]
        out = [torch.empty(V, h, device="cuda"), torch.empty(T, 4 * h, dtype=dt, device="cuda"), torch.empty(d, device="cuda"), torch.empty(d, device="cuda"),
               torch.empty(h, h, device="cuda")]
        ws = [workspace(B.axonn_embedding_bwd_workspace(T, h, V)), workspace(B.axonn_qk_norm_rope_bwd_workspace(T, 8, 4, d))]
        q = [torch.empty(h, -(-T // 128) * 128, dtype=torch.uint8, device="cuda"), torch.empty(h, 24, dtype=torch.uint8, device="cuda")]
        torch.cuda.synchronize()

        def run():
            B.axonn_embedding_bwd(T, h, V, tokens, dout, h, 1.0, out[0], 1, 0, ws[0], stream)
            B.axonn_qk_norm_rope_bwd(T, T, 8, 4, d, d, 0, qkv, 4 * h, qkv, 4 * h, one, one, EPS, None, inv, out[1], 4 * h, out[2], out[3], ws[1],
                                     stream)
            B.axonn_fp8_quantize(T, h, dout, h, None, None, *q, stream=stream)
            B.axonn_gemm_fp8(B.EPI_ACC_F32, h, h, T, *q, *q, out[4], h, stream=stream)
        return run, out, (ws, q)
    alone = []
    for k in range(2):
        run, out, keep = step(k, None)
        run()
        torch.cuda.synchronize()
        alone.append(out)
    streams = [torch.cuda.Stream() for _ in range(2)]
    both = [step(k, streams[k]) for k in range(2)]
    for _ in range(3):
        for run, _, _ in both:
            run()
    torch.cuda.synchronize()
    for k in range(2):
        for a, b in zip(alone[k], both[k][1]):
            assert torch.equal(a, b)


def _layer_step(seed):
    """A small layer's attention half, forward and backward, through the operations as a training step would string them
    together; returns what every operation was given and what it gave."""
    import torch
    dt = B.torch_elem_dtype()
    rng = np.random.default_rng(seed)
    b, s, a, d, V, p = 2, 72, 4, 64, 300, 0.1
    h, T = a * d, b * s
    up = lambda x: torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(dt).cuda()
    e = lambda *shape, dtype=dt: torch.empty(*shape, dtype=dtype, device="cuda")
    f32 = torch.float32
    t = dict(tokens=rng.integers(0, V, T), table=normal(rng, V, h, std=0.06), w_qkv=normal(rng, h, 3 * h, std=0.06),
             w_o=normal(rng, h, h, std=0.06), gq=normal(rng, d, std=0.1, mean=1.0), gk=normal(rng, d, std=0.1, mean=1.0),
             ln_g=normal(rng, h, std=0.1, mean=1.0), ln_b=normal(rng, h, std=0.1), dy=normal(rng, T, h))
    D = {k: up(v) for k, v in t.items() if k != "tokens"}
    D["tokens"], inv = dev_i32(t["tokens"]), 10000.0 ** (-np.arange(d // 2) / (d / 2))
    INV = torch.from_numpy(inv).cuda()
    kp = lambda k: -(-k // 128) * 128
    form = lambda r, k: (e(r, kp(k), dtype=torch.uint8), e(r, -(-kp(k) // 512) * 4, dtype=torch.uint8))

    def both(x, r, c):
        rows, cols = form(r, c), form(c, r)
        B.axonn_fp8_quantize(r, c, x, c, *rows, *cols)
        return rows, cols
    wq, wq_t = both(D["w_qkv"], h, 3 * h)
    wo, wo_t = both(D["w_o"], h, h)
    ws_e, ws_q = workspace(B.axonn_embedding_bwd_workspace(T, h, V)), workspace(B.axonn_qk_norm_rope_bwd_workspace(T, a, a, d))
    qk = (T, s, a, a, d, d, 0)
    o = {k: e(T, h) for k in ("emb", "x", "u", "att", "proj", "y", "datt", "dproj", "du", "dx", "demb")}
    o.update({k: e(T, 3 * h) for k in ("qkv", "rot", "drot", "dqkv")})
    stats, lse, delta = e(T, 2, dtype=f32), e(b * a * s, dtype=f32), e(b * a * s, dtype=f32)
    o.update(dw_qkv=e(h, 3 * h, dtype=f32), dw_o=e(h, h, dtype=f32), dgq=e(d, dtype=f32), dgk=e(d, dtype=f32), dtable=e(V, h, dtype=f32))
    ln_dg, ln_db, ln_ws = e(h, dtype=f32), e(h, dtype=f32), e(2 * -(-T // 64) * h, dtype=f32)

    B.axonn_embedding_fwd(T, h, V, D["tokens"], D["table"], 16.0, o["emb"], h)
    B.axonn_dropout_fwd(T, h, o["emb"], h, None, 0, p, 1, 0, None, o["x"], h)
    B.axonn_layernorm_fwd(T, h, o["x"], D["ln_g"], D["ln_b"], EPS, o["u"], stats)
    u8, u8_t = both(o["u"], T, h)
    B.axonn_gemm_fp8(B.EPI_BIAS, T, 3 * h, h, *u8, *wq_t, o["qkv"], 3 * h)
    B.axonn_qk_norm_rope_fwd(*qk, o["qkv"], 3 * h, D["gq"], D["gk"], EPS, None, INV, o["rot"], 3 * h)
    B.axonn_attention_fwd(b, s, a, d, o["rot"], o["att"], lse)
    att8, att8_t = both(o["att"], T, h)
    B.axonn_gemm_fp8(B.EPI_BIAS, T, h, h, *att8, *wo_t, o["proj"], h)
    B.axonn_dropout_fwd(T, h, o["proj"], h, o["x"], h, p, 1, 1, None, o["y"], h)

    B.axonn_dropout_bwd(T, h, D["dy"], h, p, 1, 1, None, o["dproj"], h)
    dp8, dp8_t = both(o["dproj"], T, h)
    B.axonn_gemm_fp8(B.EPI_BIAS, T, h, h, *dp8, *wo, o["datt"], h)
    B.axonn_gemm_fp8(B.EPI_ACC_F32, h, h, T, *att8_t, *dp8_t, o["dw_o"], h)
    B.axonn_attention_bwd(b, s, a, d, o["rot"], o["att"], lse, o["datt"], o["drot"], delta)
    B.axonn_qk_norm_rope_bwd(*qk, o["drot"], 3 * h, o["qkv"], 3 * h, D["gq"], D["gk"], EPS, None, INV, o["dqkv"], 3 * h, o["dgq"], o["dgk"], ws_q)
    dq8, dq8_t = both(o["dqkv"], T, 3 * h)
    B.axonn_gemm_fp8(B.EPI_BIAS, T, h, 3 * h, *dq8, *wq, o["du"], h)
    B.axonn_gemm_fp8(B.EPI_ACC_F32, h, 3 * h, T, *u8_t, *dq8_t, o["dw_qkv"], 3 * h)
    B.axonn_layernorm_bwd(T, h, o["du"], o["x"], stats, D["ln_g"], D["dy"], o["dx"], ln_dg, ln_db, ln_ws)
    B.axonn_dropout_bwd(T, h, o["dx"], h, p, 1, 0, None, o["demb"], h)
    B.axonn_embedding_bwd(T, h, V, D["tokens"], o["demb"], h, 16.0, o["dtable"], 1, 0, ws_e)
    torch.cuda.synchronize()
    return t, {k: host(v) for k, v in o.items()}, (b, s, a, d, V, p, inv)


def test_a_training_step_of_a_layers_attention_half():
    """Against the whole computation in float64 without any 8-bit rounding.  A number of 4 significant bits is off by at most 2^-4
    of itself (at the start of a binade; 2^-5 at its end), uniformly, so by 2^-4 / sqrt(3) = 3.61 % at most in the mean square, and
    the sum of products of two such numbers by sqrt(2) * 3.61 % = 5.11 % of its root mean square.  A result that has passed n
    products may be n * 5.11 % off; a wrong mask, angle, transpose, scale or order is off by far more (1.0 or so)."""
    t, got, (b, s, a, d, V, p, inv) = _layer_step(11)
    h, T = a * d, b * s
    f = {k: np.asarray(v, np.float64) for k, v in t.items() if k != "tokens"}
    pos, one = np.arange(T) % s, 0.0511
    emb = O.embedding_fwd(t["tokens"], f["table"], 16.0)
    x = O.dropout(emb, p, 1, 0)
    u, xhat, rstd = OT.layernorm_fwd(x, f["ln_g"], f["ln_b"], EPS)
    qkv = u @ f["w_qkv"]
    rot = O.qk_norm_rope_fwd(qkv, a, a, d, d, False, f["gq"], f["gk"], EPS, pos, inv)
    # plain causal attention and its gradient, head by head
    att, probs = np.zeros((T, h)), {}
    for i in range(b):
        for j in range(a):
            q, k, v = (rot[i * s:(i + 1) * s, n * h + j * d:n * h + (j + 1) * d] for n in range(3))
            sc = q @ k.T / np.sqrt(d)
            sc[np.triu_indices(s, 1)] = -np.inf
            w = np.exp(sc - sc.max(axis=1, keepdims=True))
            probs[i, j] = w / w.sum(axis=1, keepdims=True)
            att[i * s:(i + 1) * s, j * d:(j + 1) * d] = probs[i, j] @ v
    proj = att @ f["w_o"]
    y = O.dropout(proj, p, 1, 1, x)
    dproj = O.dropout(f["dy"], p, 1, 1)
    datt, dw_o, drot = dproj @ f["w_o"].T, att.T @ dproj, np.zeros_like(rot)
    for (i, j), w in probs.items():
        r = slice(i * s, (i + 1) * s)
        q, k, v = (rot[r, n * h + j * d:n * h + (j + 1) * d] for n in range(3))
        do = datt[r, j * d:(j + 1) * d]
        dw = do @ v.T
        ds = w * (dw - (dw * w).sum(axis=1, keepdims=True)) / np.sqrt(d)
        for n, g in enumerate((ds @ k, ds.T @ q, w.T @ do)):
            drot[r, n * h + j * d:n * h + (j + 1) * d] = g
    dqkv, dgq, dgk = O.qk_norm_rope_bwd(drot, qkv, a, a, d, d, False, f["gq"], f["gk"], EPS, pos, inv)
    du, dw_qkv = dqkv @ f["w_qkv"].T, u.T @ dqkv
    dx, _, _ = OT.layernorm_bwd(du, xhat, rstd, f["ln_g"])
    dx = dx + f["dy"]
    demb = O.dropout(dx, p, 1, 0)
    dtable = O.embedding_bwd(t["tokens"], demb, V, 16.0)
    for name, ref, passed in (("emb", emb, 0), ("x", x, 0), ("u", u, 0), ("qkv", qkv, 1), ("rot", rot, 1), ("att", att, 2), ("proj", proj, 3),
                              ("y", y, 3), ("dproj", dproj, 0), ("datt", datt, 1), ("dw_o", dw_o, 3), ("drot", drot, 4), ("dqkv", dqkv, 4),
                              ("dgq", dgq, 5), ("dgk", dgk, 5), ("du", du, 5), ("dw_qkv", dw_qkv, 5), ("dx", dx, 5), ("demb", demb, 5),
                              ("dtable", dtable, 5)):
        assert rel_fro(got[name], ref) <= max(2 * half_step(), passed * one), (name, rel_fro(got[name], ref))


@pytest.mark.parametrize("M,N,K", [(4096, 4096, 100), (4096, 4096, 130), (3841, 4356, 300), (4096, 4096, 512), (4100, 4200, 600), (4096, 4096, 1030),
                                   (4352, 4096, 1500)])
def test_large_products_of_every_length(M, N, K):
    """Products that fill the chip, over contractions of one block of k and more, an odd number of them too; a result of each
    kind of rounding.  The float64 sums are formed on the GPU from the values that the oracle says the codes stand for."""
    import torch
    rng = np.random.default_rng(K)
    forms = []
    for rows in (M, N):
        codes = rng.integers(0, 256, (rows, -(-K // 128) * 128)).astype(np.uint8)
        codes[(codes & 0x7f) == 0x7f] = 0
        codes[:, K:] = 0
        scales = np.zeros((rows, -(-K // 512) * 4), np.uint8)
        nb = -(-K // 128)
        scales[:, :nb] = rng.integers(110, 140, (rows, nb))
        forms += [codes, scales]
    dev = [torch.from_numpy(f).cuda() for f in forms]
    values = torch.from_numpy(O.e4m3_values()).cuda().nan_to_num(0.0)

    def stands_for(codes, scales):
        e = scales[:, :codes.shape[1] // 128].double() - 127.0
        return values[codes.long()] * torch.exp2(e).repeat_interleave(128, dim=1)
    a, b = stands_for(*dev[:2]), stands_for(*dev[2:])
    # brought into half precision's range by the scales of A
    shift = int(torch.log2((a @ b.t()).abs().max()).item()) - 12
    dev[1].sub_((dev[1] > 0).to(torch.uint8) * shift if shift >= 0 else -(dev[1] > 0).to(torch.uint8) * (-shift))
    a = a * 2.0 ** -shift
    ref, mags = a @ b.t(), a.abs() @ b.abs().t()
    for epi, dt in ((B.EPI_BIAS, B.torch_elem_dtype()), (B.EPI_ACC_F32, torch.float32)):
        wide = dt == torch.float32
        C = torch.full((M + 1, N), 7.0, dtype=dt, device="cuda")
        B.axonn_gemm_fp8(epi, M, N, K, *dev, C, N)
        half = U if wide else half_step()
        slack = _product_slack(mags, K, wide)
        err = (C[:M].double() - ref).abs()
        assert bool((err <= half * (ref.abs() + slack) + slack + 2.0 ** -25).all()), float((err / (slack + half * ref.abs())).max())
        assert float(err.norm() / ref.norm()) <= 0.64 * half + (K + 8) * U
        assert bool((C[M] == 7.0).all())
