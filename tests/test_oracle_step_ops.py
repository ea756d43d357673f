"""The float64 definitions of oracle/step_ops.py against pins of their own: the generator's published known answers, difference
quotients, torch's 8-bit conversions, and hand-computed cases."""
import numpy as np
import pytest

from oracle import step_ops as O


def test_generator_known_answers():
    """Philox4x32-10, the known-answer vectors published with the generator (Random123)."""
    def words(c, k):
        return [int(w[0]) for w in O.philox4x32([np.array([v]) for v in c], k)]
    assert words([0] * 4, [0] * 2) == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]
    assert words([0xffffffff] * 4, [0xffffffff] * 2) == [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]
    assert words([0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344], [0xa4093822, 0x299f31d0]) == \
        [0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1]


@pytest.mark.parametrize("p", [0.1, 0.5, 0.9])
def test_dropout_keeps_the_expected_share(p):
    T, h = 200, 1000
    keep = O.dropout_keep(T, h, p, 0x1234567890ABCDEF, 7)
    # five standard deviations of a binomial mean
    assert abs(keep.mean() - (1 - p)) < 5 * np.sqrt(p * (1 - p) / (T * h))
    assert not np.array_equal(keep, O.dropout_keep(T, h, p, 0x1234567890ABCDEF, 8))
    assert np.array_equal(keep[:7, :33], O.dropout_keep(7, 33, p, 0x1234567890ABCDEF, 7))     # a function of the place alone


@pytest.mark.parametrize("rot,interleaved", [(8, False), (8, True), (4, False), (0, False), (6, True)])
def test_qk_gradient_against_differences(rot, interleaved):
    rng = np.random.default_rng(rot)
    T, heads, kv, d, eps = 3, 4, 2, 8, 1e-3
    x = rng.standard_normal((T, (heads + 2 * kv) * d))
    gq, gk, inv = 1 + 0.3 * rng.standard_normal(d), 1 + 0.3 * rng.standard_normal(d), rng.random(rot // 2)
    pos, w = np.array([0, 5, -3]), rng.standard_normal(x.shape)

    def loss(x, gq, gk):
        return float((O.qk_norm_rope_fwd(x, heads, kv, d, rot, interleaved, gq, gk, eps, pos, inv) * w).sum())

    grads = O.qk_norm_rope_bwd(w, x, heads, kv, d, rot, interleaved, gq, gk, eps, pos, inv)
    args = [x, gq, gk]
    for k in range(3):
        flat = args[k].reshape(-1)
        for i in rng.choice(flat.size, min(flat.size, 40), replace=False):
            keep, step = flat[i], 1e-6
            flat[i] = keep + step
            up = loss(*args)
            flat[i] = keep - step
            down = loss(*args)
            flat[i] = keep
            assert abs((up - down) / (2 * step) - grads[k].reshape(-1)[i]) < 1e-6 * (1 + abs(grads[k].reshape(-1)[i]))


def test_rotation_depends_on_distance_alone():
    """Products of a rotated query and a rotated key are those of their distance."""
    rng = np.random.default_rng(1)
    d, inv = 16, 10000.0 ** (-np.arange(8) / 8)
    row = rng.standard_normal((1, 3 * d)).repeat(4, 0)
    out = O.qk_norm_rope_fwd(row, 1, 1, d, d, False, np.ones(d), np.ones(d), 1e-6, [3, 10, 1003, 1010], inv)
    q, k = out[:, :d], out[:, d:2 * d]
    assert abs(q[0] @ k[1] - q[2] @ k[3]) < 1e-12 * d


def test_embedding_gradient_is_the_transpose_of_the_lookup():
    rng = np.random.default_rng(2)
    V, h, tokens = 7, 5, np.array([3, 3, -2, 9, 0, 3])
    table, dout = rng.standard_normal((V, h)), rng.standard_normal((6, h))
    assert np.isclose((O.embedding_fwd(tokens, table, 2.5) * dout).sum(), (O.embedding_bwd(tokens, dout, V, 2.5) * table).sum())


def test_codes_against_torch():
    torch = pytest.importorskip("torch")
    rng = np.random.default_rng(3)
    for spread in (1.0, 1e3, 1e-30, 1e30):
        x = (rng.standard_normal((9, 300)) * spread * np.exp(rng.standard_normal((9, 1)) * 5)).astype(np.float32)
        codes, scales = O.fp8_quantize(x)
        e = scales[:, :3].astype(np.int64) - 127
        u = np.zeros((9, 384))
        u[:, :300] = x
        u = (u.reshape(9, 3, 128) / 2.0 ** e[:, :, None].astype(np.float64)).astype(np.float32)
        assert np.abs(u).max() <= 448 and (np.abs(u).max(axis=2) > 224).all()
        want = torch.from_numpy(u).to(torch.float8_e4m3fn).view(torch.uint8).numpy().reshape(9, -1)
        assert np.array_equal(codes, want)


def test_scales_at_their_borders():
    x = np.zeros((6, 128))
    x[0, 5], x[1, 5], x[2, 5], x[4, 0], x[5, :2] = 448.0, np.nextafter(448.0, 1e3), 2.0 ** -150, np.inf, (np.nan, 3.0)
    codes, scales = O.fp8_quantize(x)
    assert scales[:, 0].tolist() == [127, 128, 0, 0, 0, 127 - 7] and not scales[:, 1:].any()
    assert codes[0, 5] == 0x7e and codes[4, 0] == 0x7f and codes[5, 0] == 0x7f
    assert O.fp8_values(codes, scales)[5, 1] == 3.0


def test_codes_round_ties_to_even():
    # scale 1: the block holds 448; 17 lies between 16 and 18, 19 between 18 and 20, 2^-10 between 0 and 2^-9
    x = np.zeros((1, 128))
    x[0, :7] = [448.0, 17.0, 19.0, -17.0, 2.0 ** -10, 3 * 2.0 ** -10, 464.0 - 48]
    codes, scales = O.fp8_quantize(x)
    assert O.fp8_values(codes, scales)[0, :7].tolist() == [448.0, 16.0, 20.0, -16.0, 0.0, 2.0 ** -8, 416.0]
