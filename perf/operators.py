"""What the performance of the training step's single operators is measured on: the scaled embedding lookup and its gradient,
norms of queries and keys with the position rotation, dropout with the residual addition, and linear maps in 8-bit floating
point with a scale for each block of 128.

A case is a plain dict.  `kind` says what one pass is:

  embed_fwd    rows of a [vocab, hidden] table, scaled
  embed_bwd    the table's gradient from the gradient of the looked-up rows (the whole table is written)
  qk_fwd       packed [Q | K | V] rows: every query and key head normalised (RMS) and rotated by its position, V copied
  qk_bwd       the gradient of the packed rows and of the two gains
  dropout_fwd  residual + dropout(x), or dropout(x) alone; the mask is a function of (seed, offset, row, column)
  dropout_bwd  dropout's gradient: the same mask again
  fp8_fwd      a linear map y = epilogue(x W): x is quantised, W is kept quantised
  fp8_bwd      its backward pass: dy is quantised along both dimensions, dx = dy W^T and dW = x^T dy (32-bit)

`run` computes the operators in plain torch where `own` is false, and calls the library's operators where it is true.
"""
import math
import random

import numpy as np
import torch

own = False

FP8_BLOCK = 128          # elements that share a scale
EPS = 1e-6
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


# ------------------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # the lookup in front of a 12B-shape model's first layer (hidden 5120, vocabulary 51200), eight sequences of 2048
        dict(name="embed_fwd_12b", kind="embed_fwd", elem="bf16", T=16384, hidden=5120, vocab=51200, zipf=True),
        # the gradient of a microbatch of ordinary text (few tokens take most of the places), a table of 51200 rows
        dict(name="embed_bwd_text", kind="embed_bwd", elem="bf16", T=16384, hidden=2048, vocab=51200, zipf=True, fp32=False),
        # a small model's step in half precision with 32-bit gradients: short, ragged sequence, launches and latency
        dict(name="embed_bwd_small", kind="embed_bwd", elem="fp16", T=200, hidden=384, vocab=1000, zipf=False, fp32=True),
        # in front of attention in a 12B-shape layer: 40 heads of 128, four sequences of 2048
        dict(name="qk_fwd_12b", kind="qk_fwd", elem="bf16", T=8192, seq=2048, heads=40, kv=40, d=128, rot=128,
             interleaved=False, far=False),
        # its backward pass with 8 shared key / value heads, two sequences
        dict(name="qk_bwd_shared", kind="qk_bwd", elem="bf16", T=4096, seq=2048, heads=32, kv=8, d=128, rot=128,
             interleaved=False, far=False),
        # a few tokens at far positions, head dim 64, half of it rotated pair by pair, in half precision
        dict(name="qk_fwd_few", kind="qk_fwd", elem="fp16", T=5, seq=5, heads=16, kv=16, d=64, rot=32, interleaved=True,
             far=True),
        # behind the output projection of a 12B-shape layer: eight sequences of 2048
        dict(name="dropout_fwd_12b", kind="dropout_fwd", elem="bf16", T=16384, hidden=5120, p=0.1, residual=True),
        # the gradient in the 4512-wide layer of the paper's 12B model, microbatch of 8 x 512 tokens, half precision
        dict(name="dropout_bwd_table1", kind="dropout_bwd", elem="fp16", T=4096, hidden=4512, p=0.1, residual=False),
        # a few rows of an odd width
        dict(name="dropout_fwd_odd", kind="dropout_fwd", elem="bf16", T=7, hidden=1001, p=0.5, residual=True),
        # FC1 of a 12B-shape layer, four sequences of 2048
        dict(name="fp8_fwd_12b", kind="fp8_fwd", elem="bf16", M=8192, K=5120, N=20480, epilogue="bias"),
        # the backward pass of a linear map in a model of one to two billion parameters, ragged tokens
        dict(name="fp8_bwd_ragged", kind="fp8_bwd", elem="bf16", M=2047, K=2048, N=8192, epilogue="none"),
        # a small layer's FC1 with GeLU and its stored derivative, sizes that fill no block, half precision
        dict(name="fp8_fwd_small", kind="fp8_fwd", elem="fp16", M=200, K=392, N=1000, epilogue="gelu"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_once(rng):
    kind = rng.choice(["embed_fwd", "embed_bwd", "qk_fwd", "qk_bwd", "dropout_fwd", "dropout_bwd", "fp8_fwd", "fp8_bwd"])
    c = dict(kind=kind, elem=rng.choice(["bf16", "bf16", "fp16"]))
    if kind.startswith("embed"):
        hidden = _log_uniform(rng, 64, 8192)
        c.update(T=_log_uniform(rng, 1, 32768), hidden=hidden if rng.random() < 0.2 else -(-hidden // 8) * 8,
                 vocab=_log_uniform(rng, 100, 262144), zipf=rng.random() < 0.6)
        if kind == "embed_bwd":
            c.update(fp32=rng.random() < 0.5)
    elif kind.startswith("qk"):
        d = rng.choice([64, 64, 128, 128, 128, 80, 96, 188, 192, 256, 2 * rng.randint(4, 96)])
        kv = rng.choice([1, 2, 4, 8, 12, 16])
        T = _log_uniform(rng, 1, 8192)
        c.update(T=T, seq=rng.choice([T, max(1, T // 2), max(1, T // 3)]), heads=kv * rng.choice([1, 1, 2, 4]), kv=kv, d=d,
                 rot=d if rng.random() < 0.7 else 2 * rng.randint(0, d // 2), interleaved=rng.random() < 0.3,
                 far=rng.random() < 0.3)
    elif kind.startswith("dropout"):
        hidden = _log_uniform(rng, 8, 8192)
        c.update(T=_log_uniform(rng, 1, 16384), hidden=hidden if rng.random() < 0.3 else -(-hidden // 8) * 8,
                 p=rng.choice([0.05, 0.1, 0.1, 0.2, 0.5, round(rng.random(), 3)]),
                 residual=kind == "dropout_fwd" and rng.random() < 0.7)
    else:
        c.update(M=_log_uniform(rng, 1, 8192), K=_log_uniform(rng, 64, 8192), N=8 * _log_uniform(rng, 8, 2048),
                 epilogue=rng.choice(["bias", "gelu", "residual"]) if kind == "fp8_fwd" else "none")
    return c


def draw(rng):
    flops = max(work(c)["flops"] for c in listed())
    moved = max(work(c)["bytes"] for c in listed())
    while True:
        c = _draw_once(rng)
        w = work(c)
        if w["flops"] <= flops and w["bytes"] <= moved:
            return c


# -------------------------------------------------------------------------------------------------------------- work
def _zipf_weights(vocab):
    return 1.0 / (np.arange(vocab) + 2.7) ** 1.07


def _expected_rows(case):
    """Rows of the table that the tokens are expected to name."""
    if not case["zipf"]:
        return case["vocab"] * -math.expm1(case["T"] * math.log1p(-1.0 / case["vocab"]))
    p = _zipf_weights(case["vocab"])
    return float(-np.expm1(case["T"] * np.log1p(-p / p.sum())).sum())


def work(case):
    c = case
    if c["kind"] == "embed_fwd":
        n = c["T"] * c["hidden"]
        return {"bytes": int(4 * c["T"] + 2 * _expected_rows(c) * c["hidden"] + 2 * n), "flops": n}
    if c["kind"] == "embed_bwd":
        n = c["T"] * c["hidden"]
        return {"bytes": 4 * c["T"] + 2 * n + (4 if c["fp32"] else 2) * c["vocab"] * c["hidden"], "flops": n}
    if c["kind"].startswith("qk"):
        rotated, rest = c["T"] * (c["heads"] + c["kv"]) * c["d"], c["T"] * c["kv"] * c["d"]
        small = (4 * c["T"] if c["far"] else 0) + 4 * c["rot"] + 4 * c["d"]
        if c["kind"] == "qk_fwd":
            return {"bytes": 4 * (rotated + rest) + small, "flops": 8 * rotated}
        return {"bytes": 6 * rotated + 4 * rest + small + 8 * c["d"], "flops": 18 * rotated}
    if c["kind"].startswith("dropout"):
        n = c["T"] * c["hidden"]
        return {"bytes": (6 if c["residual"] else 4) * n, "flops": 2 * n}
    M, K, N = c["M"], c["K"], c["N"]
    if c["kind"] == "fp8_fwd":
        outputs = {"bias": 2, "residual": 4, "gelu": 4}[c["epilogue"]]
        return {"bytes": 2 * M * K + N * K + outputs * M * N, "flops": 2 * M * N * K}
    return {"bytes": 2 * M * N + M * K + N * K + 2 * M * K + 4 * K * N, "flops": 4 * M * N * K}


# ------------------------------------------------------------------------------------------------------------- state
def _ceil(n, to):
    return -(-n // to) * to


def _quantise(x):
    """[R, C] -> codes (uint8, [R, C padded to blocks of 128]) and scale exponents + 127 (uint8, [R, blocks padded to 4]):
    the least power of two with which a block's largest magnitude stays within e4m3's 448."""
    R, C = x.shape
    Cp = _ceil(C, FP8_BLOCK)
    v = torch.zeros(R, Cp, device=x.device)
    v[:, :C] = x.float()
    blocks = v.view(R, Cp // FP8_BLOCK, FP8_BLOCK)
    mant, exp = torch.frexp(blocks.abs().amax(dim=2))                      # amax = mant * 2^exp, mant in [0.5, 1)
    e = torch.where(mant > 0.875, exp - 8, exp - 9).clamp(-127, 127)       # 448 = 0.875 * 2^9
    e = torch.where(mant == 0, torch.full_like(e, -127), e)
    codes = torch.ldexp(blocks, -e[:, :, None]).to(torch.float8_e4m3fn).view(torch.uint8).view(R, Cp)
    scales = torch.zeros(R, _ceil(Cp // FP8_BLOCK, 4), dtype=torch.uint8, device=x.device)
    scales[:, :Cp // FP8_BLOCK] = (e + 127).to(torch.uint8)
    return codes, scales


def _values(codes, scales):
    """What the codes and scales stand for, 32-bit, [R, padded C]."""
    R, Cp = codes.shape
    e = scales[:, :Cp // FP8_BLOCK].int() - 127
    return torch.ldexp(codes.view(torch.float8_e4m3fn).float().view(R, -1, FP8_BLOCK), e[:, :, None]).view(R, Cp)


def prepare(case, seed):
    c, dt = case, DTYPES[case["elem"]]
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rng = random.Random(seed)

    def normal(*shape, std=1.0, mean=0.0):
        return (torch.randn(*shape, generator=g, device="cuda") * std + mean).to(dt)

    s = dict(case=c)
    if c["kind"].startswith("embed"):
        T, h, V = c["T"], c["hidden"], c["vocab"]
        if c["zipf"]:
            cdf = torch.from_numpy(np.cumsum(_zipf_weights(V))).cuda()
            u = torch.rand(T, generator=g, device="cuda", dtype=torch.float64) * cdf[-1]
            ids = torch.searchsorted(cdf, u).clamp(max=V - 1)
            s["tokens"] = torch.randperm(V, generator=g, device="cuda")[ids].int()
        else:
            s["tokens"] = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
        s["scale"] = math.sqrt(h)
        if c["kind"] == "embed_fwd":
            s["table"] = normal(V, h, std=0.02)
        else:
            s["dout"] = normal(T, h, std=0.05)
    elif c["kind"].startswith("qk"):
        width = (c["heads"] + 2 * c["kv"]) * c["d"]
        s["qkv"] = normal(c["T"], width, std=1.5)
        s["gamma_q"], s["gamma_k"] = normal(c["d"], std=0.2, mean=1.0), normal(c["d"], std=0.2, mean=1.0)
        i = torch.arange(c["rot"] // 2, dtype=torch.float64, device="cuda")
        s["inv_freq"] = 10000.0 ** (-2.0 * i / max(c["rot"], 1))
        s["positions"] = None
        if c["far"]:
            s["positions"] = torch.randint(0, 1 << 20, (c["T"],), generator=g, device="cuda", dtype=torch.int32)
        if c["kind"] == "qk_bwd":
            s["dout"] = normal(c["T"], width)
    elif c["kind"].startswith("dropout"):
        s["x"] = normal(c["T"], c["hidden"])
        s["res"] = normal(c["T"], c["hidden"]) if c["residual"] else None
        s["seed"], s["offset"] = rng.getrandbits(64), rng.getrandbits(40)
    else:
        M, K, N = c["M"], c["K"], c["N"]
        w = normal(K, N, std=0.02)
        if c["kind"] == "fp8_fwd":
            s["x"], s["bias"] = normal(M, K), normal(N, std=0.02)
            s["w"], s["w_scale"] = _quantise(w.t())                        # rows of outputs, blocks along K
            s["res"] = normal(M, N) if c["epilogue"] == "residual" else None
        else:
            s["dy"] = normal(M, N)
            s["x_t"], s["x_t_scale"] = _quantise(normal(M, K).t())         # kept by the forward pass, blocks along tokens
            s["w"], s["w_scale"] = _quantise(w)                            # rows of inputs, blocks along N
    return s


# --------------------------------------------------------------------------------------------------------- plain forms
def _angles(s, c):
    pos = s["positions"]
    if pos is None:
        pos = torch.arange(c["T"], device="cuda") % c["seq"]
    return pos.double()[:, None, None] * s["inv_freq"]


def _pair(x, rot, interleaved):
    """Views of the first and second elements of the rotated pairs in the last dimension."""
    if interleaved:
        return x[..., 0:rot:2], x[..., 1:rot:2]
    return x[..., :rot // 2], x[..., rot // 2:rot]


def _rotate(x, cos, sin, rot, interleaved):
    out = x.clone()
    a, b = _pair(x, rot, interleaved)
    oa, ob = _pair(out, rot, interleaved)
    oa.copy_(a * cos - b * sin)
    ob.copy_(a * sin + b * cos)
    return out


def _plain_qk(s, c):
    dt, T, d = DTYPES[c["elem"]], c["T"], c["d"]
    ang = _angles(s, c)
    cos, sin = torch.cos(ang).float(), torch.sin(ang).float()
    src = s["qkv"].view(T, -1, d)
    out = (s["qkv"] if c["kind"] == "qk_fwd" else s["dout"]).view(T, -1, d).clone()          # V passes through
    gains = []
    for lo, hi, gamma in ((0, c["heads"], s["gamma_q"]), (c["heads"], c["heads"] + c["kv"], s["gamma_k"])):
        x, gam = src[:, lo:hi].float(), gamma.float()
        r = torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS)
        if c["kind"] == "qk_fwd":
            out[:, lo:hi] = _rotate(gam * (x * r), cos, sin, c["rot"], c["interleaved"]).to(dt)
            continue
        dz = _rotate(out[:, lo:hi].float(), cos, -sin, c["rot"], c["interleaved"])
        xh = x * r
        gains.append((dz * xh).sum(dim=(0, 1), dtype=torch.float64).float())
        dxh = dz * gam
        out[:, lo:hi] = (r * (dxh - xh * (dxh * xh).mean(dim=-1, keepdim=True))).to(dt)
    out = out.view(T, -1)
    return out if c["kind"] == "qk_fwd" else (out, *gains)


def _philox(c0, c1, offset, seed):
    """Philox4x32-10 (Salmon et al. 2011): counters (c0, c1, offset), int64 tensors that hold 32-bit words -> 4 words."""
    mask = 0xFFFFFFFF
    x = [c0, c1, torch.full_like(c0, offset & mask), torch.full_like(c0, offset >> 32 & mask)]
    k0, k1 = seed & mask, seed >> 32 & mask
    for _ in range(10):
        p0, p1 = x[0] * 0xD2511F53, x[2] * 0xCD9E8D57                      # modulo 2^64: the low 64 bits are those wanted
        x = [p1 >> 32 & mask ^ x[1] ^ k0, p1 & mask, p0 >> 32 & mask ^ x[3] ^ k1, p0 & mask]
        k0, k1 = k0 + 0x9E3779B9 & mask, k1 + 0xBB67AE85 & mask
    return x


def _keep_threshold(p):
    return int(round(p * 65536.0))


def _plain_dropout(s, c):
    T, h, thr = c["T"], c["hidden"], _keep_threshold(c["p"])
    groups = (h + 7) // 8
    parts = []
    for r0 in range(0, T, 1024):
        rows = torch.arange(r0, min(r0 + 1024, T), device="cuda")[:, None].expand(-1, groups)
        cols = torch.arange(groups, device="cuda")[None, :].expand_as(rows)
        words = torch.stack(_philox(cols, rows, s["offset"], s["seed"]), dim=-1)
        parts.append(torch.stack((words & 0xFFFF, words >> 16), dim=-1).flatten(1)[:, :h] >= thr)
    y = torch.zeros(T, h, device="cuda")
    if thr < 65536:
        y = torch.where(torch.cat(parts), s["x"].float() * (65536.0 / (65536 - thr)), y)
    if s["res"] is not None:
        y = s["res"].float() + y
    return y.to(DTYPES[c["elem"]])


def _gelu_and_derivative(z, erf):
    cdf = 0.5 * (1.0 + erf(z * math.sqrt(0.5)))
    return z * cdf, cdf + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)


def _plain(s, c):
    dt = DTYPES[c["elem"]]
    if c["kind"] == "embed_fwd":
        return (s["table"][s["tokens"].long()].float() * s["scale"]).to(dt)
    if c["kind"] == "embed_bwd":
        # long sums: a frequent token's row collects thousands of terms
        total = torch.zeros(c["vocab"], c["hidden"], dtype=torch.float64, device="cuda")
        total.index_add_(0, s["tokens"].long(), s["dout"].double())
        return (total * s["scale"]).to(torch.float32 if c["fp32"] else dt)
    if c["kind"].startswith("qk"):
        return _plain_qk(s, c)
    if c["kind"].startswith("dropout"):
        return _plain_dropout(s, c)
    if c["kind"] == "fp8_fwd":
        z = _values(*_quantise(s["x"])) @ _values(s["w"], s["w_scale"]).t() + s["bias"].float()
        if c["epilogue"] == "gelu":
            return tuple(t.to(dt) for t in _gelu_and_derivative(z, torch.erf))
        return (z if s["res"] is None else z + s["res"].float()).to(dt)
    dx = _values(*_quantise(s["dy"])) @ _values(s["w"], s["w_scale"]).t()
    dw = _values(s["x_t"], s["x_t_scale"]) @ _values(*_quantise(s["dy"].t())).t()
    return dx.to(dt), dw


# ------------------------------------------------------------------------------------------------------- the operators
def _library(s, c):
    from paper_2110_13005_amd import binding as B
    B.select_elem(c["elem"])
    dt = DTYPES[c["elem"]]
    stream = torch.cuda.current_stream()

    def empty(*shape, dtype=dt):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    if c["kind"].startswith("embed"):
        T, h, V = c["T"], c["hidden"], c["vocab"]
        if c["kind"] == "embed_fwd":
            out = empty(T, h)
            B.axonn_embedding_fwd(T, h, V, s["tokens"], s["table"], s["scale"], out, h, stream)
            return out
        dtable = empty(V, h, dtype=torch.float32 if c["fp32"] else dt)
        ws = empty(B.axonn_embedding_bwd_workspace(T, h, V), dtype=torch.uint8)
        B.axonn_embedding_bwd(T, h, V, s["tokens"], s["dout"], h, s["scale"], dtable, int(c["fp32"]), 0, ws, stream)
        return dtable
    if c["kind"].startswith("qk"):
        T, ld = c["T"], s["qkv"].shape[1]
        shape = (T, c["seq"], c["heads"], c["kv"], c["d"], c["rot"], int(c["interleaved"]))
        norm = (s["gamma_q"], s["gamma_k"], EPS, s["positions"], s["inv_freq"])
        out = torch.empty_like(s["qkv"])
        if c["kind"] == "qk_fwd":
            B.axonn_qk_norm_rope_fwd(*shape, s["qkv"], ld, *norm, out, ld, stream)
            return out
        dgq, dgk = empty(c["d"], dtype=torch.float32), empty(c["d"], dtype=torch.float32)
        ws = empty(B.axonn_qk_norm_rope_bwd_workspace(T, c["heads"], c["kv"], c["d"]), dtype=torch.uint8)
        B.axonn_qk_norm_rope_bwd(*shape, s["dout"], ld, s["qkv"], ld, *norm, out, ld, dgq, dgk, ws, stream)
        return out, dgq, dgk
    if c["kind"].startswith("dropout"):
        T, h = c["T"], c["hidden"]
        out = empty(T, h)
        if c["kind"] == "dropout_fwd":
            B.axonn_dropout_fwd(T, h, s["x"], h, s["res"], h, c["p"], s["seed"], s["offset"], None, out, h, stream)
        else:
            B.axonn_dropout_bwd(T, h, s["x"], h, c["p"], s["seed"], s["offset"], None, out, h, stream)
        return out
    M, K, N = c["M"], c["K"], c["N"]

    def quantised(rows, cols):
        return (empty(rows, _ceil(cols, FP8_BLOCK), dtype=torch.uint8),
                empty(rows, _ceil(_ceil(cols, FP8_BLOCK) // FP8_BLOCK, 4), dtype=torch.uint8))

    if c["kind"] == "fp8_fwd":
        xq, y = quantised(M, K), empty(M, N)
        B.axonn_fp8_quantize(M, K, s["x"], K, *xq, None, None, stream)
        aux = empty(M, N) if c["epilogue"] == "gelu" else None
        B.axonn_gemm_fp8({"bias": B.EPI_BIAS, "gelu": B.EPI_BIAS_GELU, "residual": B.EPI_BIAS_RES}[c["epilogue"]], M, N, K,
                         *xq, s["w"], s["w_scale"], y, N, bias=s["bias"], res=s["res"], ld_res=N, aux=aux, ld_aux=N,
                         stream=stream)
        return y if aux is None else (y, aux)
    dyq, dyq_t = quantised(M, N), quantised(N, M)
    dx, dw = empty(M, K), empty(K, N, dtype=torch.float32)
    B.axonn_fp8_quantize(M, N, s["dy"], N, *dyq, *dyq_t, stream)
    B.axonn_gemm_fp8(B.EPI_BIAS, M, K, N, *dyq, s["w"], s["w_scale"], dx, K, stream=stream)
    B.axonn_gemm_fp8(B.EPI_ACC_F32, K, N, M, s["x_t"], s["x_t_scale"], *dyq_t, dw, N, stream=stream)
    return dx, dw


def run(state):
    return _library(state, state["case"]) if own else _plain(state, state["case"])


# --------------------------------------------------------------------------------------------------------------- exact
def _exact_codes(x):
    """The values that the 8-bit form of x ([R, C], blocks along C) stands for: every block is divided by the least power of
    two that brings its magnitudes down to 448, and rounded (ties to even) to 4 significant bits, not below steps of 2^-9."""
    R, C = x.shape
    v = torch.nn.functional.pad(x.double(), (0, -C % FP8_BLOCK)).view(R, -1, FP8_BLOCK)
    amax = v.abs().amax(dim=2, keepdim=True)
    e = torch.ceil(torch.log2(amax / 448.0)).nan_to_num(neginf=-127.0)
    e = torch.where(amax > 448.0 * torch.exp2(e), e + 1, torch.where(amax <= 448.0 * torch.exp2(e - 1), e - 1, e))
    scale = torch.exp2(e.clamp(-127, 127))
    u = v / scale
    _, ex = torch.frexp(u)
    step = torch.exp2((ex - 4).clamp(min=-9).double())
    return (torch.round(u / step) * step * scale).view(R, -1)


def _exact_stored(codes, scales):
    """Kept codes bit by bit: sign, 4 bits of exponent (bias 7), 3 of significand."""
    k = codes.long()
    ex, man = (k >> 3) & 15, (k & 7).double()
    mag = torch.where(ex == 0, man / 512.0, (1.0 + man / 8.0) * torch.exp2((ex - 7).double()))
    mag = torch.where(k >= 128, -mag, mag)
    per_block = torch.exp2(scales[:, :codes.shape[1] // FP8_BLOCK].double() - 127.0)
    return mag * per_block.repeat_interleave(FP8_BLOCK, dim=1)


def _exact_uniforms(T, h, seed, offset):
    """Half-words of the generator for every element, computed with 16-bit limbs on the host's words."""
    groups = (h + 7) // 8

    def split_product(a, m):
        """High and low word of the 64-bit product of 32-bit a and the constant m."""
        al, ah, ml, mh = a & 0xFFFF, a >> 16, m & 0xFFFF, m >> 16
        low, mid = al * ml, ah * ml + (al * mh)
        total = low + ((mid & 0xFFFF) << 16)
        return (ah * mh + (mid >> 16) + (total >> 32)) & 0xFFFFFFFF, total & 0xFFFFFFFF

    n = torch.arange(T * groups, device="cuda")
    a, b = n % groups, n // groups
    c, d = torch.full_like(n, offset % 2 ** 32), torch.full_like(n, offset // 2 ** 32)
    for r in range(10):
        key = ((seed % 2 ** 32) + r * 0x9E3779B9) % 2 ** 32, ((seed // 2 ** 32) + r * 0xBB67AE85) % 2 ** 32
        h0, l0 = split_product(a, 0xD2511F53)
        h1, l1 = split_product(c, 0xCD9E8D57)
        a, b, c, d = torch.bitwise_xor(torch.bitwise_xor(h1, b), key[0]), l1, torch.bitwise_xor(torch.bitwise_xor(h0, d), key[1]), l0
    u = torch.empty(T, groups, 8, dtype=torch.int32, device="cuda")
    for j, word in enumerate((a, b, c, d)):
        u[:, :, 2 * j] = (word % 65536).view(T, groups).int()
        u[:, :, 2 * j + 1] = (word // 65536).view(T, groups).int()
    return u.view(T, -1)[:, :h]


def _exact_qk(s, c):
    T, d, rot = c["T"], c["d"], c["rot"]
    pos = torch.arange(T, device="cuda").remainder(c["seq"]) if s["positions"] is None else s["positions"]
    turn = torch.polar(torch.ones(T, rot // 2, dtype=torch.float64, device="cuda"), torch.outer(pos.double(), s["inv_freq"]))
    idx = torch.arange(rot, device="cuda")
    first, second = (idx[0::2], idx[1::2]) if c["interleaved"] else (idx[:rot // 2], idx[rot // 2:])
    backward = c["kind"] == "qk_bwd"
    result = (s["dout"] if backward else s["qkv"]).double().view(T, -1, d)
    x_all = s["qkv"].view(T, -1, d)
    dgains = []
    for heads, gamma in ((range(c["heads"]), s["gamma_q"]), (range(c["heads"], c["heads"] + c["kv"]), s["gamma_k"])):
        dgain = torch.zeros(d, dtype=torch.float64, device="cuda")
        for j in heads:
            x, gam = x_all[:, j].double(), gamma.double()
            rms = torch.sqrt(x.square().sum(dim=1, keepdim=True) / d + EPS)
            z = result[:, j].clone() if backward else gam * x / rms
            pair = torch.complex(z[:, first], z[:, second]) * (turn.conj() if backward else turn)
            z[:, first], z[:, second] = pair.real, pair.imag
            if backward:
                dgain += (z * x / rms).sum(dim=0)
                w = z * gam
                z = w / rms - x * (w * x).sum(dim=1, keepdim=True) / (d * rms ** 3)
            result[:, j] = z
        dgains.append(dgain)
    result = result.reshape(T, -1)
    return (result, *dgains) if backward else result


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] == "embed_fwd":
        return torch.index_select(s["table"], 0, s["tokens"].long()).double() * s["scale"]
    if c["kind"] == "embed_bwd":
        ids, order = torch.sort(s["tokens"].long(), stable=True)
        rows, counts = torch.unique_consecutive(ids, return_counts=True)
        out = torch.zeros(c["vocab"], c["hidden"], dtype=torch.float64, device="cuda")
        terms = s["dout"][order]
        ends = torch.cumsum(counts, 0).tolist()
        for row, lo, hi in zip(rows.tolist(), [0] + ends, ends):
            out[row] = s["scale"] * terms[lo:hi].double().sum(dim=0)
        return out
    if c["kind"].startswith("qk"):
        return _exact_qk(s, c)
    if c["kind"].startswith("dropout"):
        thr = _keep_threshold(c["p"])
        kept = _exact_uniforms(c["T"], c["hidden"], s["seed"], s["offset"]) >= thr
        y = s["x"].double() * kept * (65536.0 / max(65536 - thr, 1))
        return y if s["res"] is None else y + s["res"].double()
    w = _exact_stored(s["w"], s["w_scale"])
    if c["kind"] == "fp8_fwd":
        z = _exact_codes(s["x"]) @ w.t().contiguous() + s["bias"].double()
        if c["epilogue"] == "gelu":
            phi = 0.5 * torch.erfc(-z / math.sqrt(2.0))
            return z * phi, phi + z * torch.exp(-z * z / 2.0) * (1.0 / math.sqrt(2.0 * math.pi))
        return z if s["res"] is None else z + s["res"].double()
    x_t = _exact_stored(s["x_t"], s["x_t_scale"])
    return (_exact_codes(s["dy"]) @ w.t().contiguous(),
            x_t @ _exact_codes(s["dy"].t().contiguous()).t().contiguous())
