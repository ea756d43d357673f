"""GPU parity of attention over packed sequences with its float64 definition, element by element, at the lengths, head layouts, strides and
values where it can go wrong; the plan that it follows; and a training step of packed operations as they are used together.

Bounds: every rounding to 16 bits is off by half a step at most, fp32 arithmetic by U = 2^-24 of the magnitudes that go into it, counted
along the formula (`attention_bounds`); a result is within what these add up to at worst."""
import numpy as np
import pytest

from oracle import packed_ops as P
from paper_2110_13005_amd import binding as B
from helpers import dev_i32, host, rel_fro
from test_gpu_step_ops import Padded, U, half_step, normal, within, workspace

pytestmark = [pytest.mark.gpu, pytest.mark.parametrize("axonn_elem", ["bf16", "fp16"], indirect=True)]


def surrounded(rows, cols, ld, shift, values, inside):
    """A matrix among NaN: around it, and in its rows that belong to no sequence."""
    import torch
    m = Padded(rows, cols, ld, shift)
    m.buf.fill_(float("nan"))
    m.t[torch.from_numpy(inside).cuda()] = torch.from_numpy(np.ascontiguousarray(values[inside], np.float32)).cuda().to(m.buf.dtype)
    return m


def attention_bounds(qkv, dout, offsets, heads, kv, d, scale):
    """-> how far o, lse and dqkv may be from their definitions (`within` adds the last rounding of the 16-bit ones)."""
    h, T = half_step(), len(qkv)
    tiny = 2.0 ** -25 if B.ELEM == "fp16" else 0.0                # half a step below half precision's smallest normal number
    q, k, v = P._split(np.asarray(qkv, np.float64), heads, kv, d)
    do = np.asarray(dout, np.float64).reshape(T, heads, d)
    E_o, E_lse, E_g = np.zeros((T, heads, d)), np.zeros((heads, T)), np.zeros((T, heads + 2 * kv, d))
    for a, b in P.sequences(offsets, T):
        n = b - a
        for i in range(heads if n else 0):
            j = i // (heads // kv)
            Q, K, V, D = q[a:b, i], k[a:b, j], v[a:b, j], do[a:b, i]
            p, lse = P.attention_probabilities(Q, K, scale)
            keep = np.tril(np.ones((n, n), bool))
            s = np.where(keep, scale * (Q @ K.T), 0.0)
            e = np.where(keep, (d + 8) * U * scale * (np.abs(Q) @ np.abs(K.T)), 0.0)           # of a score
            far = 4 * U * (np.abs(s) + np.abs(s).max(axis=1, keepdims=True))                   # of an exponent
            total = (n / 8 + 32) * U                                                           # of a sum of exponentials
            E_lse[i, a:b] = (e + far).max(axis=1) + total + 4 * U * np.abs(lse)
            rp = e + far + (e + far).max(axis=1, keepdims=True) + total
            aV, aD, aK, aQ = np.abs(V), np.abs(D), np.abs(K), np.abs(Q)
            o = p @ V
            E_o[a:b, i] = (p * (h + 2 * rp) + tiny * keep) @ aV + (n + 8) * U * (p @ aV)
            E_out = E_o[a:b, i] * (1 + h) + h * np.abs(o) + tiny
            delta, dP = np.sum(D * o, axis=1, keepdims=True), D @ V.T
            E_delta = np.sum(aD * E_out, axis=1, keepdims=True) + (d + 8) * U * np.sum(aD * np.abs(o), axis=1, keepdims=True)
            E_dP = (d + 8) * U * (aD @ aV.T)
            rq = e + far + E_lse[i, a:b, None] + 4 * U * np.abs(lse)[:, None] + 8 * U
            dS = p * (dP - delta)
            E_dS = p * (1 + 2 * rq) * (E_dP + E_delta + U * (np.abs(dP) + np.abs(delta))) + 2 * rq * np.abs(dS)
            E_dS = np.where(keep, E_dS + h * (np.abs(dS) + E_dS) + tiny, 0.0)
            sums = (n * heads // kv + 8) * U
            E_g[a:b, i] += scale * (E_dS @ aK + sums * (np.abs(dS) @ aK))
            E_g[a:b, heads + j] += scale * (E_dS.T @ aQ + sums * (np.abs(dS).T @ aQ))
            E_g[a:b, heads + kv + j] += (p * (h + 2 * rq) + tiny * keep).T @ aD + sums * (p.T @ aD)
    return E_o.reshape(T, -1), E_lse, E_g.reshape(T, -1)


class Attention:
    """Operands of a call on sequences of `lens` rows with `front` rows of nobody's in front of them and `pad` behind."""

    def __init__(self, rng, lens, heads, kv, d, front=0, pad=0, extra=0, shift=0, std=1.0, scale=None):
        import torch
        self.heads, self.kv, self.d, self.n = heads, kv, d, len(lens)
        self.offsets = front + np.concatenate([[0], np.cumsum(lens)])
        self.T = T = int(self.offsets[-1]) + pad
        self.scale = float(np.float32(d ** -0.5 if scale is None else scale))
        self.width, self.width_o = (heads + 2 * kv) * d, heads * d
        self.ld, self.ld_o = self.width + extra, self.width_o + extra
        self.inside = np.zeros(T, bool)
        self.inside[front:self.offsets[-1]] = True
        self.values, self.dvalues = normal(rng, T, self.width, std=std), normal(rng, T, self.width_o)
        self.qkv = surrounded(T, self.width, self.ld, shift, self.values, self.inside)
        self.dout = surrounded(T, self.width_o, self.ld_o, shift, self.dvalues, self.inside)
        self.o, self.dqkv = Padded(T, self.width_o, self.ld_o, shift), Padded(T, self.width, self.ld, shift)
        self.lse = torch.full((heads, T), 7.0, device="cuda")
        self.off_dev = dev_i32(self.offsets)
        self.plan = workspace(B.axonn_attention_packed_plan_bytes(T, self.n))
        self.ws = workspace(B.axonn_attention_packed_bwd_workspace(T, self.n, heads, kv, d))

    def run(self, stream=None, backward=True):
        shape = (self.T, self.n, self.heads, self.kv, self.d, self.scale, self.plan, self.qkv.t, self.ld)
        B.axonn_attention_packed_plan(self.T, self.n, self.off_dev, self.plan, stream)
        B.axonn_attention_packed_fwd(*shape, self.o.t, self.ld_o, self.lse, stream)
        if backward:
            B.axonn_attention_packed_bwd(*shape, self.o.t, self.ld_o, self.lse, self.dout.t, self.ld_o, self.dqkv.t, self.ld, self.ws, stream)

    def results(self):
        """o, lse, dqkv on the host; checks that rows of nobody's are as they were."""
        o, lse, g = self.o.result(), host(self.lse), self.dqkv.result()
        assert (o[~self.inside] == 7).all() and (lse[:, ~self.inside] == 7).all() and (g[~self.inside] == 7).all()
        return o[self.inside], lse[:, self.inside], g[self.inside]

    def check(self):
        args = (self.offsets, self.heads, self.kv, self.d, self.scale)
        x, dy = (np.where(self.inside[:, None], a, 0.0) for a in (self.values, self.dvalues))
        o_ref, lse_ref = P.packed_attention_fwd(x, *args)
        g_ref = P.packed_attention_bwd(x, dy, *args)
        E_o, E_lse, E_g = attention_bounds(x, dy, *args)
        o, lse, g = self.results()
        keep = self.inside
        within(o, o_ref[keep], E_o[keep], label="o")
        assert (np.abs(lse - lse_ref[:, keep]) <= E_lse[:, keep]).all(), np.abs(lse - lse_ref[:, keep]).max()
        within(g, g_ref[keep], E_g[keep], label="dqkv")


CASES = [
    # lens, heads, kv, d, front, pad, extra columns, first element
    ([1], 1, 1, 4, 0, 0, 0, 0), ([1, 2, 3], 2, 1, 8, 0, 0, 0, 0), ([5], 3, 3, 64, 2, 3, 5, 1),
    ([64, 65, 127, 128, 129, 1], 2, 1, 64, 0, 0, 0, 0), ([0, 5, 0, 300, 0], 4, 2, 128, 0, 7, 0, 0), ([200, 31], 3, 3, 188, 1, 0, 3, 1),
    ([257, 33], 4, 1, 192, 0, 0, 0, 0), ([130, 1, 1, 62], 8, 8, 80, 3, 3, 3, 1), ([513], 4, 2, 128, 0, 0, 8, 0), ([700], 2, 2, 64, 0, 1, 0, 0),
    ([33] * 9, 6, 3, 36, 0, 0, 1, 3), ([1] * 70, 4, 4, 32, 0, 0, 0, 0),
    # more tiles than the one-launch backward takes
    ([140] * 9 + [3], 16, 4, 128, 0, 5, 0, 0), ([140] * 9 + [300], 16, 16, 64, 0, 0, 0, 0), ([129] * 9, 16, 2, 188, 0, 0, 0, 0),
    ([131] * 9, 16, 8, 92, 0, 0, 2, 1), ([400, 300, 200, 100, 50, 20, 10, 1] * 2, 8, 1, 64, 0, 0, 0, 0), ([90] * 18, 24, 24, 40, 0, 0, 0, 0),
    # tiles of keys shared out over workgroups, in one launch with dQ and in one of their own
    ([600, 200], 16, 1, 64, 1, 1, 0, 0), ([500], 12, 1, 128, 0, 0, 0, 0), ([450, 90], 8, 1, 160, 0, 3, 4, 0), ([1000, 400, 290], 32, 1, 64, 0, 0, 0, 0),
    ([900, 380, 130], 32, 2, 100, 0, 9, 0, 0),
]


@pytest.mark.parametrize("lens,heads,kv,d,front,pad,extra,shift", CASES)
def test_attention(lens, heads, kv, d, front, pad, extra, shift):
    a = Attention(np.random.default_rng(sum(lens) + d), lens, heads, kv, d, front, pad, extra, shift)
    a.run()
    a.check()
    first = [x.clone() for x in (a.o.t, a.lse, a.dqkv.t)]
    a.dqkv.t[:] = 7
    a.run()
    a.results()
    assert all((x == y).all() for x, y in zip(first, (a.o.t, a.lse, a.dqkv.t))), "another result the second time"


@pytest.mark.parametrize("d,heads,kv", [(64, 4, 2), (128, 2, 1), (188, 2, 2)])
@pytest.mark.parametrize("std,scale", [(4.0, None), (1.0, 3.0), (0.01, 1e-3)])
def test_attention_of_steep_and_flat_scores(d, heads, kv, std, scale):
    a = Attention(np.random.default_rng(5), [300, 77, 1], heads, kv, d, std=std, scale=scale)
    a.run()
    a.check()


@pytest.mark.parametrize("heads,kv,d", [(4, 2, 128), (16, 8, 64)])
def test_a_sequence_does_not_depend_on_its_neighbours(heads, kv, d):
    """The same bits wherever a sequence lies and whatever the others hold, infinities and NaN too."""
    import torch
    rng = np.random.default_rng(8)
    lens = [150, 260, 150, 97, 260]
    a = Attention(rng, lens, heads, kv, d)
    off = a.offsets
    same = [(0, 2), (1, 4)]
    for m in (a.qkv, a.dout):
        for i, j in same:
            m.t[off[j]:off[j + 1]] = m.t[off[i]:off[i + 1]]
    m = a.qkv.t
    bad = slice(int(off[3]), int(off[4]))
    outs = []
    for value in (1.0, float("nan"), float("inf")):
        m[bad] = value
        a.run()
        outs.append([x.clone() for x in (a.o.t, a.lse.t(), a.dqkv.t)])
    good = torch.ones(a.T, dtype=torch.bool)
    good[bad] = False
    for out in outs:
        for x, y in zip(outs[0], out):
            assert (x[good] == y[good]).all() and torch.isfinite(x[good]).all()
            for i, j in same:
                assert (y[off[i]:off[i + 1]] == y[off[j]:off[j + 1]]).all()


def test_attention_rows_beyond_32_bit_offsets():
    """Sequences whose rows lie more than 2^31 elements behind the first row."""
    import torch
    heads, kv, d, T, ld = 2, 1, 64, 1200, 1 << 21
    rng = np.random.default_rng(11)
    lens = [20, 900, 150, 130]
    a = Attention(rng, lens, heads, kv, d)
    big = torch.empty(T * ld, dtype=B.torch_elem_dtype(), device="cuda").view(T, ld)
    out = torch.empty(T * ld, dtype=B.torch_elem_dtype(), device="cuda").view(T, ld)
    big[:, :a.width], big[:, 4096:4096 + a.width_o] = a.qkv.t, a.dout.t
    a.run()
    shape = (T, a.n, heads, kv, d, a.scale, a.plan, big, ld)
    o, dout, dqkv, lse = out[:, 4096:], big[:, 4096:], out, torch.zeros_like(a.lse)
    B.axonn_attention_packed_fwd(*shape, o, ld, lse)
    B.axonn_attention_packed_bwd(*shape, o, ld, lse, dout, ld, dqkv, ld, a.ws)
    assert (o[:, :a.width_o] == a.o.t).all() and (lse == a.lse).all() and (dqkv[:, :a.width] == a.dqkv.t).all()


@pytest.mark.parametrize("T,offsets", [
    (1, [0, 1]), (300, [0, 300]), (1000, [0, 0, 128, 256, 257, 1000, 1000]), (900, [5, 3, 400, 200, 901, 7]), (900, [-7, 20, 2000]),
    (100000, "many"), (5000, "200"), (70000, "256"), (70000, "257"), (1 << 24, [0, 1 << 24]), (1 << 24, [0, 1 << 20, 1 << 23, (1 << 24) - 5]), (70, [70, 70])])
def test_plan(T, offsets):
    """Every tile of every sequence once, those with the most tiles in front of them first (as far as these are told apart)."""
    rng = np.random.default_rng(3)
    if isinstance(offsets, str):
        offsets = np.sort(rng.integers(0, T + 1, 1 + (5000 if offsets == "many" else int(offsets))))
    n = len(offsets) - 1
    plan = workspace(B.axonn_attention_packed_plan_bytes(T, n))
    B.axonn_attention_packed_plan(T, n, dev_i32(offsets), plan)
    got = plan.cpu().numpy().view(np.int32)
    want = [(a, b - a, t, 0) for a, b in P.sequences(offsets, T) for t in range((b - a + 127) // 128)]
    assert got[0] == len(want) <= T // 128 + n
    items = got[4:4 + 4 * len(want)].reshape(-1, 4)
    assert sorted(map(tuple, items.tolist())) == sorted(want)
    assert (np.diff(np.minimum(items[:, 2], 4095)) <= 0).all()


def test_attention_with_disordered_offsets():
    """Offsets that do not ascend: the sequences that the header says they stand for, nothing written elsewhere."""
    rng = np.random.default_rng(2)
    a = Attention(rng, [100, 0, 60, 40], 2, 2, 64, pad=10)
    a.off_dev = dev_i32([0, 100, 30, 160, 200])            # the third is taken as the second
    a.run()
    a.check()


def test_a_list_that_is_no_plan_leaves_the_rows():
    """Whatever the plan's memory holds, no workgroup reads or writes outside the T rows."""
    import torch
    rng = np.random.default_rng(2)
    a = Attention(rng, [100, 60], 2, 2, 64)
    a.run()
    items = a.plan.view(torch.int32)
    items[4:] = torch.tensor([150, 60, 0, 0, -5, 20, 0, 0, 10, -1, 0, 0], dtype=torch.int32, device="cuda")
    shape = (a.T, a.n, a.heads, a.kv, a.d, a.scale, a.plan, a.qkv.t, a.ld)
    a.o.t[:] = 7
    B.axonn_attention_packed_fwd(*shape, a.o.t, a.ld_o, a.lse)
    B.axonn_attention_packed_bwd(*shape, a.o.t, a.ld_o, a.lse, a.dout.t, a.ld_o, a.dqkv.t, a.ld, a.ws)
    assert (a.o.result() == 7).all()


def test_attention_captured_with_other_sequences_at_each_replay():
    import torch
    rng = np.random.default_rng(9)
    packs = [Attention(rng, lens, 4, 2, 64, pad=pad) for lens, pad in (([100, 200, 84], 16), ([1, 300, 99], 0), ([0, 0, 390], 10), ([133, 133, 133], 1))]
    a = packs[0]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        a.run(stream)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        a.run(stream)
    for p in packs + packs[:2]:
        p.run()
        a.qkv.t.copy_(p.qkv.t)
        a.dout.t.copy_(p.dout.t)
        a.off_dev.copy_(p.off_dev)
        graph.replay()
        torch.cuda.synchronize()
        keep = torch.from_numpy(p.inside).cuda()
        assert all((x[keep] == y[keep]).all() for x, y in zip((a.o.t, a.lse.t(), a.dqkv.t), (p.o.t, p.lse.t(), p.dqkv.t)))


def test_attention_on_two_streams_at_once():
    import torch
    rng = np.random.default_rng(10)
    calls = [Attention(rng, [300, 500, 90], 16, 4, 128), Attention(rng, [200] * 6, 8, 8, 64)]
    want = []
    for a in calls:
        a.run()
        want.append([x.clone() for x in (a.o.t, a.lse, a.dqkv.t)])
        for x in (a.o.t, a.lse, a.dqkv.t):
            x[:] = 0
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(5):
        for a, s in zip(calls, streams):
            a.run(s)
    torch.cuda.synchronize()
    for a, w in zip(calls, want):
        assert all((x == y).all() for x, y in zip((a.o.t, a.lse, a.dqkv.t), w))


@pytest.mark.parametrize("loss", ["policy", "prefer", "distill"])
def test_a_training_step_on_packed_sequences(loss):
    """Embedding, projection, query / key norms with positions inside the sequences, packed attention, residual, LayerNorm, head and loss,
    and all of it backwards, against the same step written out in float64 with automatic differentiation."""
    import torch
    rng = np.random.default_rng(12)
    lens, heads, kv, d, V, h = [40, 23, 0, 17, 1, 30], 8, 2, 32, 200, 256
    off = np.concatenate([[0], np.cumsum(lens)])
    T, n, width = 120, len(lens), (heads + 2 * kv) * d              # nine rows behind the last sequence
    eps, scale, S = 1e-5, d ** -0.5, 64.0
    inside = np.arange(T) < off[-1]
    pos = np.concatenate([np.arange(m) for m in lens] + [np.zeros(T - off[-1], int)])
    tokens = rng.integers(0, V, T)
    targets = np.where(inside & (rng.random(T) < 0.8), rng.integers(0, V, T), -100)
    W = dict(table=normal(rng, V, h, std=0.5), wqkv=normal(rng, h, width, std=h ** -0.5), gq=normal(rng, 1, d, std=0.1, mean=1.0)[0],
             gk=normal(rng, 1, d, std=0.1, mean=1.0)[0], wo=normal(rng, heads * d, h, std=(heads * d) ** -0.5), lng=normal(rng, 1, h, std=0.1, mean=1.0)[0],
             lnb=normal(rng, 1, h, std=0.1)[0], head=normal(rng, h, V, std=h ** -0.5))
    inv_freq = 100.0 ** (-2.0 * np.arange(d // 2) / d)
    old, ref = -5.3 + 0.3 * rng.standard_normal(T), -5.3 + 0.3 * rng.standard_normal(T)
    A, weight = rng.standard_normal(T), np.where(targets >= 0, 1 / 64, 0.0)
    K = 12
    ids, teacher = np.stack([rng.choice(V, K, replace=False) for _ in range(T)]), rng.standard_normal((T, K))
    teacher_lse = np.log(np.exp(teacher).sum(axis=1)) + 0.3

    # the step in float64
    P64 = {k: torch.tensor(np.asarray(v, np.float64), requires_grad=True) for k, v in W.items()}
    x = P64["table"][torch.tensor(tokens)] * 2.0
    qkv = (x @ P64["wqkv"]).view(T, heads + 2 * kv, d)
    ang = torch.tensor(pos[:, None] * inv_freq)[:, None]

    def rotated(z, gain):
        z = gain * z / torch.sqrt((z * z).mean(dim=-1, keepdim=True) + eps)
        a, b = z[..., :d // 2], z[..., d // 2:]
        return torch.cat((a * torch.cos(ang) - b * torch.sin(ang), a * torch.sin(ang) + b * torch.cos(ang)), dim=-1)

    q, k, v = rotated(qkv[:, :heads], P64["gq"]), rotated(qkv[:, heads:heads + kv], P64["gk"]), qkv[:, heads + kv:]
    rows = []
    for a, b in zip(off, off[1:]):
        for i in range(heads if b > a else 0):
            j = i // (heads // kv)
            s = (scale * q[a:b, i] @ k[a:b, j].T).masked_fill(torch.ones(b - a, b - a, dtype=torch.bool).triu(1), -torch.inf)
            rows.append((a, b, i, torch.softmax(s, dim=1) @ v[a:b, j]))
    o = torch.zeros(T, heads, d, dtype=torch.float64)
    for a, b, i, r in rows:
        o[a:b, i] = r
    y = o.view(T, -1) @ P64["wo"] + x
    logits = torch.nn.functional.layer_norm(y, (h,), P64["lng"], P64["lnb"], eps) @ P64["head"]
    logq = torch.log_softmax(logits, dim=1)
    live = torch.tensor(targets >= 0)
    logp = torch.where(live, logq[torch.arange(T), torch.tensor(np.maximum(targets, 0))], 0.0)
    if loss == "policy":
        r, x_ref = torch.exp(logp - torch.tensor(old)), torch.tensor(ref) - logp
        each = -torch.minimum(r * torch.tensor(A), r.clamp(0.8, 1.2) * torch.tensor(A)) + 0.1 * (torch.exp(x_ref) - x_ref - 1)
        total = (torch.where(live, each, 0.0) * torch.tensor(weight)).sum()
    elif loss == "prefer":
        gain = torch.where(live, logp - torch.tensor(ref), 0.0)
        m = 0.5 * torch.stack([gain[off[2 * i]:off[2 * i + 1]].sum() - gain[off[2 * i + 1]:off[2 * i + 2]].sum() for i in range(n // 2)])
        total = -torch.nn.functional.logsigmoid(m).sum() / (n // 2)
    else:
        lp = torch.tensor(teacher - teacher_lse[:, None])
        rest, at = 1 - torch.exp(lp).sum(dim=1), torch.tensor(ids)
        others = torch.logsumexp(logq.scatter(1, at, -torch.inf), dim=1)
        each = (torch.exp(lp) * (lp - logq.gather(1, at))).sum(dim=1) + rest * (torch.log(rest) - others)
        total = (each * torch.tensor(weight)).sum()
    total.backward()

    # the same on the GPU
    dt = B.torch_elem_dtype()

    def up(a, dtype=dt):
        return torch.from_numpy(np.ascontiguousarray(a)).to(dtype).cuda()

    def zeros(*shape, dtype=dt):
        return torch.zeros(*shape, dtype=dtype, device="cuda")

    f32 = torch.float32
    G = {name: up(w) for name, w in W.items()}
    offsets, tok, tgt = dev_i32(off), dev_i32(tokens), dev_i32(targets)
    positions, freq = dev_i32(pos), up(inv_freq, torch.float64)
    X, QKV, R, O, Y, N, Z = zeros(T, h), zeros(T, width), zeros(T, width), zeros(T, heads * d), zeros(T, h), zeros(T, h), zeros(T, V)
    lse, stats = zeros(heads, T, dtype=f32), zeros(T, 2, dtype=f32)
    plan = workspace(B.axonn_attention_packed_plan_bytes(T, n))
    B.axonn_embedding_fwd(T, h, V, tok, G["table"], 2.0, X, h)
    B.axonn_gemm_bf16(1, 0, B.EPI_BIAS, T, width, h, X, h, G["wqkv"], width, QKV, width)
    norm = (T, T, heads, kv, d, d, 0)
    B.axonn_qk_norm_rope_fwd(*norm, QKV, width, G["gq"], G["gk"], eps, positions, freq, R, width)
    B.axonn_attention_packed_plan(T, n, offsets, plan)
    shape = (T, n, heads, kv, d, scale, plan, R, width)
    B.axonn_attention_packed_fwd(*shape, O, heads * d, lse)
    B.axonn_gemm_bf16(1, 0, B.EPI_BIAS_RES, T, h, heads * d, O, heads * d, G["wo"], h, Y, h, res=X, ld_res=h)
    B.axonn_layernorm_fwd(T, h, Y, G["lng"], G["lnb"], eps, N, stats)
    B.axonn_gemm_bf16(1, 0, B.EPI_BIAS, T, V, h, N, h, G["head"], V, Z, V)
    token_loss, out, lp_dev = zeros(T, dtype=f32), zeros(1, dtype=f32), zeros(T, dtype=f32)
    w_dev = up(weight, f32)
    if loss == "policy":
        B.axonn_policy_loss(T, V, Z, V, tgt, up(old, f32), up(ref, f32), up(A, f32), w_dev, 0.2, 0.2, 0.1, S, lp_dev, token_loss, out, Z, V)
    elif loss == "prefer":
        lse_z, dlogp, pair = zeros(T, dtype=f32), zeros(T, dtype=f32), zeros(n // 2, dtype=f32)
        B.axonn_token_logprobs_fwd(T, V, Z, V, tgt, lp_dev, lse_z)
        B.axonn_preference_loss(T, n // 2, V, offsets, tgt, lp_dev, up(ref, f32), 0.5, 0.0, 1 / (n // 2), S, pair, out, dlogp)
        B.axonn_token_logprobs_bwd(T, V, Z, V, tgt, lse_z, dlogp, Z, V)
    else:
        B.axonn_distill_loss(T, V, K, Z, V, up(teacher, f32), dev_i32(ids), K, up(teacher_lse, f32), 1.0, w_dev, S, token_loss, out, Z, V)
    dN, dY, dO, dR, dX = zeros(T, h), zeros(T, h), zeros(T, heads * d), zeros(T, width), zeros(T, h)
    grads = {name: zeros(*W[name].shape, dtype=f32) for name in ("head", "wo", "wqkv", "gq", "gk", "lng", "lnb", "table")}
    B.axonn_gemm_bf16(0, 0, B.EPI_ACC_F32, h, V, T, N, h, Z, V, grads["head"], V)
    B.axonn_gemm_bf16(1, 1, B.EPI_BIAS, T, h, V, Z, V, G["head"], V, dN, h)
    B.axonn_layernorm_bwd(T, h, dN, Y, stats, G["lng"], None, dY, grads["lng"], grads["lnb"], zeros(2 * ((T + 63) // 64) * h, dtype=f32))
    B.axonn_gemm_bf16(0, 0, B.EPI_ACC_F32, heads * d, h, T, O, heads * d, dY, h, grads["wo"], h)
    B.axonn_gemm_bf16(1, 1, B.EPI_BIAS, T, heads * d, h, dY, h, G["wo"], h, dO, heads * d)
    ws = workspace(B.axonn_attention_packed_bwd_workspace(T, n, heads, kv, d))
    B.axonn_attention_packed_bwd(*shape, O, heads * d, lse, dO, heads * d, dR, width, ws)
    ws = workspace(B.axonn_qk_norm_rope_bwd_workspace(T, heads, kv, d))
    B.axonn_qk_norm_rope_bwd(*norm, dR, width, QKV, width, G["gq"], G["gk"], eps, positions, freq, dR, width, grads["gq"], grads["gk"], ws)
    B.axonn_gemm_bf16(0, 0, B.EPI_ACC_F32, h, width, T, X, h, dR, width, grads["wqkv"], width)
    B.axonn_gemm_bf16(1, 1, B.EPI_BIAS, T, h, width, dR, width, G["wqkv"], width, dX, h)
    dX += dY
    ws = workspace(B.axonn_embedding_bwd_workspace(T, h, V))
    B.axonn_embedding_bwd(T, h, V, tok, dX, h, 2.0, grads["table"], 1, 0, ws)
    # the bounds of the framework's own layers: outputs 2e-2, gradients 3e-2
    assert rel_fro(host(O)[inside], o.detach().view(T, -1).numpy()[inside]) <= 2e-2
    assert abs(host(out)[0] - total.item()) <= 2e-2 * abs(total.item()) + 1e-3
    for name, g in grads.items():
        want = P64[name].grad.numpy()
        assert rel_fro(host(g) / S, want) <= 3e-2, (name, rel_fro(host(g) / S, want))
