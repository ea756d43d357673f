"""What the performance of the operators of a training step on packed sequences is measured on: causal attention inside sequences of
different lengths that lie one behind the other, with shared key / value heads, and the losses that such a step ends in.

A case is a plain dict.  `kind` says what one pass is:

  attn_fwd    attention of packed [Q | K | V] rows, its output and log-sum-exp
  attn_train  the same and its backward pass: the gradient of the packed rows as well
  policy      clipped policy loss with a KL term from logits: log-probabilities, losses, the logits' gradient
  prefer      preference loss of pairs of sequences from their tokens' log-probabilities: those, the losses, the logits' gradient
  distill     distillation from a teacher's top logits: the tokens' losses, their sum, the logits' gradient

`lens` are the sequences' lengths (their order in the pack comes from the seed); `pad` rows lie behind the last one.  `run` computes
the operators in plain torch where `own` is false, and calls the library's operators where it is true.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
TEMPERATURE = 2.0        # of the distillation
BETA, SMOOTHING = 0.1, 0.1                               # of the preference loss
KL_COEF = 0.04


# ------------------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # a layer's attention over a batch of documents of all lengths, 8 shared key / value heads: 8192 rows
        dict(name="attn_fwd_documents", kind="attn_fwd", elem="bf16", heads=32, kv=8, d=128, pad=0,
             lens="2048,1731,1500,1024,700,512,301,150,100,64,37,15,8,1,1"),
        # a few short prompts of a small model, where a call's latency counts; half precision
        dict(name="attn_fwd_few", kind="attn_fwd", elem="fp16", heads=16, kv=16, d=64, pad=0, lens="100,64,30,5,1"),
        # one long sequence, as the 8192-token stage has it, with 4 shared key / value heads
        dict(name="attn_train_long", kind="attn_train", elem="bf16", heads=16, kv=4, d=128, pad=0, lens="8192"),
        # the attention of a 12B-shape layer (40 heads of 128) in a step on conversations; the pack is not full
        dict(name="attn_train_pack", kind="attn_train", elem="bf16", heads=40, kv=40, d=128, pad=93,
             lens="1023,900,777,640,333,250,80"),
        # the heads of 188 of the paper's 12B model, eight sequences of about 512, one of them empty, half precision
        dict(name="attn_train_table1", kind="attn_train", elem="fp16", heads=24, kv=24, d=188, pad=0,
             lens="512,512,511,480,400,389,260,0"),
        # many short answers with 2 key / value heads for all query heads
        dict(name="attn_train_short", kind="attn_train", elem="bf16", heads=16, kv=2, d=64, pad=0,
             lens="90,77,64,61,50,48,40,33,32,31,30,27,25,22,20,18,17,16,15,12,11,10,9,8,7,6,5,4,3,2,1"),
        # the end of a policy step with a vocabulary of 51200; a quarter of the tokens are prompts and have no part
        dict(name="policy_51200", kind="policy", elem="bf16", T=4096, vocab=51200, masked=0.25),
        # a small model's, odd sizes, half precision
        dict(name="policy_small", kind="policy", elem="fp16", T=77, vocab=1003, masked=0.2),
        # eight pairs of answers with a vocabulary of 51200, prompts without a part
        dict(name="prefer_51200", kind="prefer", elem="bf16", vocab=51200, masked=0.3, pad=0,
             lens="400,390,300,256,256,222,200,180,128,120,100,77,64,33,20,12"),
        # two pairs of a small model, one answer empty, rows behind the last
        dict(name="prefer_small", kind="prefer", elem="fp16", vocab=2000, masked=0.1, pad=9, lens="30,17,5,0"),
        # a teacher's 64 top logits and the mass of all its others, vocabulary 51200
        dict(name="distill_51200", kind="distill", elem="bf16", T=4096, vocab=51200, top=64, tail=True, masked=0.1),
        # the 20 top logits alone, a vocabulary that fills no chunk, half precision
        dict(name="distill_odd", kind="distill", elem="fp16", T=333, vocab=32003, top=20, tail=False, masked=0.0),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_lens(rng, most, longest, n):
    lens, left = [], most
    for _ in range(n):
        size = 0 if rng.random() < 0.04 else min(left, _log_uniform(rng, 1, longest))
        lens.append(size)
        left -= size
    return sorted(lens, reverse=True)


def _draw_once(rng):
    kind = rng.choice(["attn_fwd", "attn_train", "attn_train", "policy", "prefer", "distill"])
    c = dict(kind=kind, elem=rng.choice(["bf16", "bf16", "fp16"]))
    if kind.startswith("attn"):
        kv = rng.choice([1, 2, 3, 4, 8, 8, 16])
        longest = _log_uniform(rng, 16, 8192)
        lens = _draw_lens(rng, 16384, longest, _log_uniform(rng, 1, 96))
        c.update(heads=kv * rng.choice([1, 1, 2, 4, 4, 8]), kv=kv, d=rng.choice([64, 64, 128, 128, 128, 80, 96, 188, 192, 4 * rng.randint(2, 48)]),
                 pad=rng.choice([0, 0, rng.randint(1, 200)]), lens=",".join(map(str, lens)))
        return c
    c.update(vocab=_log_uniform(rng, 100, 262144), masked=rng.choice([0.0, 0.1, 0.3, 0.6]))
    if kind == "prefer":
        lens = _draw_lens(rng, 8192, _log_uniform(rng, 4, 2048), 2 * _log_uniform(rng, 1, 32))
        c.update(lens=",".join(map(str, lens)), pad=rng.choice([0, 0, rng.randint(1, 100)]))
    else:
        c.update(T=_log_uniform(rng, 1, 8192))
    if kind == "distill":
        c.update(top=min(c["vocab"], _log_uniform(rng, 1, 256)), tail=rng.random() < 0.5)
    return c


def draw(rng):
    flops = max(work(c)["flops"] for c in listed())
    moved = max(work(c)["bytes"] for c in listed())
    while True:
        c = _draw_once(rng)
        lens = _lens(c)
        if c["kind"].startswith("attn") and (max(lens) < 8 or len(lens) * c["heads"] * max(lens) ** 2 > 1 << 31):
            continue         # sequences of one token have no gradient to compare; the plain form pads to the longest
        if c["kind"] == "prefer" and max(lens) < 1:
            continue
        w = work(c)
        if w["flops"] <= flops and w["bytes"] <= moved:
            return c


def _lens(c):
    return [int(x) for x in c["lens"].split(",")] if "lens" in c else []


def _rows(c):
    return c["T"] if "T" in c else sum(_lens(c)) + c["pad"]


def _masked(c):
    """Tokens that have no part in the loss."""
    used = _rows(c) - c.get("pad", 0)
    return min(int(round(c["masked"] * used)), used - 1) + c.get("pad", 0)


# -------------------------------------------------------------------------------------------------------------- work
def work(case):
    c = case
    if c["kind"].startswith("attn"):
        used = sum(_lens(c))
        pairs = sum(n * (n + 1) // 2 for n in _lens(c)) * c["heads"]              # (query, key) pairs that causality leaves
        qkv, o, lse = 2 * used * (c["heads"] + 2 * c["kv"]) * c["d"], 2 * used * c["heads"] * c["d"], 4 * used * c["heads"]
        if c["kind"] == "attn_fwd":
            return {"bytes": qkv + o + lse, "flops": 4 * pairs * c["d"]}
        return {"bytes": 2 * qkv + 2 * o + lse, "flops": 14 * pairs * c["d"]}       # dout is read, o written, dqkv written
    T, V, live = _rows(c), c["vocab"], _rows(c) - _masked(c)
    small = {"policy": 32 * T, "prefer": 24 * T, "distill": 8 * T + 8 * T * c.get("top", 0)}[c["kind"]]
    return {"bytes": 2 * live * V + 2 * T * V + small, "flops": 8 * live * V}


# ------------------------------------------------------------------------------------------------------------- state
def prepare(case, seed):
    c, dt = case, DTYPES[case["elem"]]
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rng = random.Random(seed)
    s = dict(case=c)

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=g, device="cuda") * std

    def uniform(*shape):
        return torch.rand(*shape, generator=g, device="cuda")

    T = _rows(c)
    if "lens" in c:
        lens = _lens(c)
        rng.shuffle(lens)
        ends = [0]
        for n in lens:
            ends.append(ends[-1] + n)
        s["offsets"] = torch.tensor(ends, dtype=torch.int32, device="cuda")
    if c["kind"].startswith("attn"):
        width = c["heads"] * c["d"]
        s["qkv"] = normal(T, width + 2 * c["kv"] * c["d"]).to(dt)
        # the step's buffers: rows behind the last sequence keep what they hold
        s["o"], s["lse"] = torch.zeros(T, width, dtype=dt, device="cuda"), torch.zeros(c["heads"], T, device="cuda")
        if c["kind"] == "attn_train":
            s["dout"], s["dqkv"] = normal(T, width).to(dt), torch.zeros_like(s["qkv"])
        return s

    V = c["vocab"]
    logits = torch.empty(T, V, dtype=dt, device="cuda").normal_(0.0, 1.5, generator=g)
    out_of = torch.zeros(T, dtype=torch.bool, device="cuda")                       # tokens without a part
    used = T - c.get("pad", 0)
    out_of[torch.randperm(used, generator=g, device="cuda")[:_masked(c) - c.get("pad", 0)]] = True
    out_of[used:] = True
    # loss scale of half precision: what a step there multiplies its gradients by
    s["loss_scale"] = 1024.0 if c["elem"] == "fp16" else 1.0
    live = T - _masked(c)
    if c["kind"] == "distill":
        K, rows = c["top"], torch.arange(T, device="cuda")[:, None]
        first = torch.randint(0, V, (T, 1), generator=g, device="cuda")
        step = torch.randint(1, V // K + 1, (T, 1), generator=g, device="cuda")
        ids = (first + step * torch.arange(K, device="cuda")) % V                  # distinct in a row
        top = 9.0 - 1.5 * torch.log(torch.arange(K, device="cuda") + 1.0) + normal(T, K, std=0.5)
        logits[rows, ids] = (0.8 * top + normal(T, K)).to(dt)                      # the student knows something already
        some = torch.arange(K, device="cuda") >= (uniform(T, 1) * 8 * K).ceil()    # a teacher that kept fewer for some tokens
        s["teacher"], s["ids"] = top, torch.where(some, -1, ids).int()
        s["teacher_lse"] = None
        if c["tail"]:
            mass = 0.7 + 0.29 * uniform(T)
            s["teacher_lse"] = torch.logsumexp(top / TEMPERATURE, dim=1) - torch.log(mass)
        s["weight"] = torch.where(out_of, 0.0, TEMPERATURE ** 2 / max(live, 1))
    else:
        targets = torch.randint(0, V, (T,), generator=g, device="cuda")
        at = (torch.arange(T, device="cuda"), targets)
        logits[at] = (8.0 + normal(T, std=2.0)).to(dt)                             # a model that mostly means what it says
        logp = logits[at].float() - torch.logsumexp(logits.float(), dim=1)
        s["targets"] = targets.int()
        s["ref_logp"] = logp + normal(T, std=0.2)
        if c["kind"] == "policy":
            # steps of 1/64 away from what the policy said when the tokens were drawn: no ratio lies at a limit of the clipping
            s["old_logp"] = logp - (torch.round(normal(T, std=12.0)) + 0.5) / 64.0
            s["advantage"] = normal(T)
            s["weight"] = torch.where(out_of, 0.0, 1.0 / max(live, 1))
        else:
            s["targets"][out_of] = -100
            s["scale"] = 2.0 / len(_lens(c))
    s["logits"], s["dlogits"] = logits, torch.empty_like(logits)
    return s


# --------------------------------------------------------------------------------------------------------- plain forms
def _softmax(z):
    """-> softmax, log-sum-exp of the last dimension."""
    m = z.amax(dim=-1, keepdim=True)
    e = torch.exp(z - m)
    total = e.sum(dim=-1, keepdim=True)
    return e / total, (m + torch.log(total)).squeeze(-1)


def _plain_attention(s, c):
    """All sequences padded to the longest: [sequence, key / value head, query head of it, position, ...]."""
    dt, T, d, kv, G = DTYPES[c["elem"]], _rows(c), c["d"], c["kv"], c["heads"] // c["kv"]
    L, off = max(_lens(c)), s["offsets"].long()
    pos, size = torch.arange(L, device="cuda"), (off[1:] - off[:-1])[:, None]
    rows = (off[:-1, None] + pos).clamp(max=T - 1)
    here = (pos < size)[:, None, None, :, None]

    def heads(x, n, per):
        return x[rows].float().view(len(rows), L, n, per, d).permute(0, 2, 3, 1, 4)

    # where every token lies in the padded form
    token = torch.arange(T, device="cuda")
    seq = (torch.searchsorted(off, token, right=True) - 1).clamp(max=len(rows) - 1)
    place, inside = (token - off[seq]).clamp(max=L - 1), token < off[-1]

    def packed(x):
        """[sequence, head, part, position, d] -> [T, ...], zeros behind the last sequence."""
        flat = x.permute(0, 3, 1, 2, 4).flatten(2)[seq, place]
        return torch.where(inside[:, None], flat, 0.0)

    w = c["heads"] * d
    q, k, v = heads(s["qkv"][:, :w], kv, G), heads(s["qkv"][:, w:w + kv * d], kv, 1), heads(s["qkv"][:, w + kv * d:], kv, 1)
    scale = d ** -0.5
    hidden = (pos[None, :] > pos[:, None]) | (pos[None, None, :] >= size[:, :, None])       # [sequence, query, key]
    hidden &= (pos > 0) | (size[:, :, None] > 0)            # an empty sequence keeps one key of nobody's, whose rows are dropped
    scores = ((q * scale) @ k.transpose(-1, -2)).masked_fill(hidden[:, None, None], float("-inf"))
    p, lse = _softmax(scores)
    o = p @ v
    lse = torch.where(inside[:, None], lse.permute(0, 3, 1, 2).flatten(2)[seq, place], 0.0).t().contiguous()
    if c["kind"] == "attn_fwd":
        return packed(o).to(dt), lse
    do = torch.where(here, heads(s["dout"], kv, G), 0.0)
    ds = p * (do @ v.transpose(-1, -2) - (do * o).sum(dim=-1, keepdim=True))
    dq = (ds @ k) * scale
    dk = (ds.transpose(-1, -2) @ (q * scale)).sum(dim=2, keepdim=True)
    dv = (p.transpose(-1, -2) @ do).sum(dim=2, keepdim=True)
    return packed(o).to(dt), lse, torch.cat((packed(dq), packed(dk), packed(dv)), dim=1).to(dt)


def _plain_logprobs(logits, targets, live):
    q, lse = _softmax(logits.float())
    at = torch.where(live, targets, 0).long()[:, None]
    return q, at, torch.where(live, logits.gather(1, at).squeeze(1).float() - lse, 0.0)


def _plain_gradient(q, at, dlogp, dt):
    """dlogp (onehot - softmax), rows without a gradient are zeros."""
    d = q * -dlogp[:, None]
    d.scatter_add_(1, at, dlogp[:, None])
    return torch.where(dlogp[:, None] != 0, d, 0.0).to(dt)


def _plain_policy(s, c):
    live = s["weight"] != 0
    q, at, logp = _plain_logprobs(s["logits"], s["targets"], live)
    A, ratio = s["advantage"], torch.exp(logp - s["old_logp"])
    clipped = ratio.clamp(0.8, 1.28)
    d = s["ref_logp"] - logp
    loss = -torch.minimum(ratio * A, clipped * A) + KL_COEF * (torch.expm1(d) - d)
    dlogp = torch.where(ratio * A <= clipped * A, -A * ratio, 0.0) - KL_COEF * torch.expm1(d)
    loss, dlogp = torch.where(live, loss, 0.0), torch.where(live, dlogp * s["weight"] * s["loss_scale"], 0.0)
    total = (loss.double() * s["weight"]).sum().float().view(1)
    return logp, loss, total, _plain_gradient(q, at, dlogp, DTYPES[c["elem"]])


def _plain_prefer(s, c):
    targets, off = s["targets"], s["offsets"].long()
    live = (targets >= 0) & (targets < c["vocab"])
    q, at, logp = _plain_logprobs(s["logits"], targets, live)
    # long sums: thousands of log-probabilities, and the difference of two of them
    sums = torch.cumsum(torch.where(live, logp.double() - s["ref_logp"], 0.0), 0)
    sums = torch.nn.functional.pad(sums, (1, 0))[off]
    per = (sums[1:] - sums[:-1]).view(-1, 2)
    m = BETA * (per[:, 0] - per[:, 1])

    def softplus(x):
        return torch.clamp(x, min=0) + torch.log1p(torch.exp(-x.abs()))

    loss = (1 - SMOOTHING) * softplus(-m) + SMOOTHING * softplus(m)
    dm = (SMOOTHING - 1) / (1 + torch.exp(m)) + SMOOTHING / (1 + torch.exp(-m))
    dseq = (s["scale"] * s["loss_scale"] * BETA * dm)[:, None] * torch.tensor([1.0, -1.0], device="cuda")
    token = torch.arange(len(targets), device="cuda")
    seq = (torch.searchsorted(off, token, right=True) - 1).clamp(max=len(off) - 2)
    dlogp = torch.where(live & (token < off[-1]), dseq.flatten()[seq], 0.0).float()
    return logp, loss.float(), (loss.sum() * s["scale"]).float().view(1), _plain_gradient(q, at, dlogp, DTYPES[c["elem"]])


def _plain_distill(s, c):
    t, V = TEMPERATURE, c["vocab"]
    q, lse = _softmax(s["logits"].float() / t)
    has = s["ids"] >= 0
    at = torch.where(has, s["ids"], 0).long()
    u = (s["teacher"] / t).masked_fill(~has, float("-inf"))
    logq = s["logits"].gather(1, at).float() / t - lse[:, None]
    any_ = has.any(dim=1)
    if c["tail"]:
        logp = u - s["teacher_lse"][:, None]
    else:
        logp = u - torch.where(any_, _softmax(torch.where(any_[:, None], u, 0.0))[1], 0.0)[:, None]
    p = torch.exp(logp)
    loss = torch.where(has, p * (logp - logq), 0.0).sum(dim=1)
    inside = torch.zeros(len(q), V + 1, dtype=torch.bool, device="cuda")
    inside.scatter_(1, torch.where(has, at, V), True)
    inside = inside[:, :V]
    if c["tail"]:
        rest = (1 - p.double().sum(dim=1)).clamp(min=0).float()
        q_rest = torch.where(inside, 0.0, q).sum(dim=1)
        loss = loss + torch.where(rest > 0, rest * (torch.log(rest) - torch.log(q_rest)), 0.0)
        share = torch.where(rest > 0, rest / q_rest, 0.0)
        dz = q * torch.where(inside, 1.0, (1.0 - share)[:, None])
    else:
        dz = q * any_[:, None]
    dz.scatter_add_(1, at, torch.where(has, -p, 0.0))
    live = s["weight"] != 0
    loss = torch.where(live, loss, 0.0)
    dz = torch.where(live[:, None], dz * (s["weight"] * (s["loss_scale"] / t))[:, None], 0.0)
    return loss, (loss.double() * s["weight"]).sum().float().view(1), dz.to(DTYPES[c["elem"]])


def _plain(s, c):
    if c["kind"].startswith("attn"):
        return _plain_attention(s, c)
    return {"policy": _plain_policy, "prefer": _plain_prefer, "distill": _plain_distill}[c["kind"]](s, c)


# ------------------------------------------------------------------------------------------------------- the operators
def _library(s, c):
    from paper_2110_13005_amd import binding as B
    B.select_elem(c["elem"])
    stream, T = torch.cuda.current_stream(), _rows(c)

    def floats(*shape):
        return torch.empty(*shape, device="cuda")

    if c["kind"].startswith("attn"):
        n, heads, kv, d = len(s["offsets"]) - 1, c["heads"], c["kv"], c["d"]
        ld, ld_o, scale = s["qkv"].shape[1], heads * d, d ** -0.5
        plan = torch.empty(B.axonn_attention_packed_plan_bytes(T, n), dtype=torch.uint8, device="cuda")
        B.axonn_attention_packed_plan(T, n, s["offsets"], plan, stream)
        B.axonn_attention_packed_fwd(T, n, heads, kv, d, scale, plan, s["qkv"], ld, s["o"], ld_o, s["lse"], stream)
        if c["kind"] == "attn_fwd":
            return s["o"], s["lse"]
        ws = torch.empty(B.axonn_attention_packed_bwd_workspace(T, n, heads, kv, d), dtype=torch.uint8, device="cuda")
        B.axonn_attention_packed_bwd(T, n, heads, kv, d, scale, plan, s["qkv"], ld, s["o"], ld_o, s["lse"], s["dout"], ld_o, s["dqkv"], ld,
                                     ws, stream)
        return s["o"], s["lse"], s["dqkv"]
    V = c["vocab"]
    if c["kind"] == "policy":
        logp, token_loss, loss = floats(T), floats(T), floats(1)
        B.axonn_policy_loss(T, V, s["logits"], V, s["targets"], s["old_logp"], s["ref_logp"], s["advantage"], s["weight"], 0.2, 0.28, KL_COEF,
                            s["loss_scale"], logp, token_loss, loss, s["dlogits"], V, stream)
        return logp, token_loss, loss, s["dlogits"]
    if c["kind"] == "prefer":
        n = (len(s["offsets"]) - 1) // 2
        logp, lse, dlogp, pair_loss, loss = floats(T), floats(T), floats(T), floats(n), floats(1)
        B.axonn_token_logprobs_fwd(T, V, s["logits"], V, s["targets"], logp, lse, stream)
        B.axonn_preference_loss(T, n, V, s["offsets"], s["targets"], logp, s["ref_logp"], BETA, SMOOTHING, s["scale"], s["loss_scale"],
                                pair_loss, loss, dlogp, stream)
        B.axonn_token_logprobs_bwd(T, V, s["logits"], V, s["targets"], lse, dlogp, s["dlogits"], V, stream)
        return logp, pair_loss, loss, s["dlogits"]
    token_loss, loss = floats(T), floats(1)
    B.axonn_distill_loss(T, V, c["top"], s["logits"], V, s["teacher"], s["ids"], c["top"], s["teacher_lse"], TEMPERATURE, s["weight"],
                         s["loss_scale"], token_loss, loss, s["dlogits"], V, stream)
    return token_loss, loss, s["dlogits"]


def run(state):
    return _library(state, state["case"]) if own else _plain(state, state["case"])


# --------------------------------------------------------------------------------------------------------------- exact
def _exact_attention(s, c):
    T, d, H, kv = _rows(c), c["d"], c["heads"], c["kv"]
    f64 = dict(dtype=torch.float64, device="cuda")
    o, lse, dqkv = torch.zeros(T, H * d, **f64), torch.zeros(H, T, **f64), torch.zeros(T, (H + 2 * kv) * d, **f64)
    ends = s["offsets"].tolist()
    for lo, hi in zip(ends, ends[1:]):
        n = hi - lo
        if n == 0:
            continue
        keep = torch.ones(n, n, dtype=torch.bool, device="cuda").tril()
        rows = s["qkv"][lo:hi].double()
        for h in range(H):
            j = H + h // (H // kv)
            cq, ck, cv = (slice(i * d, (i + 1) * d) for i in (h, j, j + kv))
            q, k, v = rows[:, cq].contiguous(), rows[:, ck].contiguous(), rows[:, cv].contiguous()
            a = torch.where(keep, q @ k.t().contiguous() / math.sqrt(d), -math.inf)
            lse[h, lo:hi] = torch.logsumexp(a, dim=1)
            a = torch.exp(a - lse[h, lo:hi, None])
            o[lo:hi, cq] = a @ v
            if c["kind"] == "attn_fwd":
                continue
            do = s["dout"][lo:hi, cq].double().contiguous()
            dqkv[lo:hi, cv] += a.t().contiguous() @ do
            g = do @ v.t().contiguous()
            g = a * (g - (a * g).sum(dim=1, keepdim=True)) / math.sqrt(d)
            dqkv[lo:hi, cq] = g @ k
            dqkv[lo:hi, ck] += g.t().contiguous() @ q
    return (o, lse) if c["kind"] == "attn_fwd" else (o, lse, dqkv)


def _exact_logits_gradient(z, logp_of, coefficient, at):
    """coefficient_t d logp_t / dz, row by row: softmax from the log-probabilities."""
    out = -coefficient[:, None] * torch.exp(logp_of)
    out[torch.arange(len(z), device="cuda"), at] += coefficient
    out[coefficient == 0] = 0.0
    return out


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"].startswith("attn"):
        return _exact_attention(s, c)
    z = s["logits"].double()
    T, V = z.shape
    if c["kind"] == "distill":
        loss, dz, weights = torch.zeros(T, dtype=torch.float64, device="cuda"), torch.zeros_like(z), s["weight"].double()
        logq = torch.log_softmax(z / TEMPERATURE, dim=1)
        u = s["teacher"].double() / TEMPERATURE
        u[s["ids"] < 0] = -math.inf
        some = (s["ids"] >= 0).any(dim=1)
        lse = torch.logsumexp(u, dim=1) if s["teacher_lse"] is None else s["teacher_lse"].double()
        full = torch.zeros(T, V + 1, dtype=torch.float64, device="cuda")           # the teacher's distribution over the vocabulary
        named = torch.zeros(T, V + 1, dtype=torch.bool, device="cuda")
        column = torch.where(s["ids"] < 0, V, s["ids"]).long()
        full.scatter_(1, column, torch.exp(u - lse[:, None]).nan_to_num(nan=0.0))
        named.scatter_(1, column, True)
        full, named = full[:, :V], named[:, :V]
        loss = torch.special.xlogy(full, full).sum(dim=1) - (full * logq).sum(dim=1)
        dz = torch.exp(logq) - full
        if s["teacher_lse"] is not None:
            P = (1.0 - full.sum(dim=1)).clamp(min=0.0)
            logQ = torch.logsumexp(torch.where(named, -math.inf, logq), dim=1)
            loss = loss + torch.where(P > 0, P * (torch.log(P) - logQ), 0.0)
            others = torch.exp(logq) - P[:, None] * torch.exp(logq - logQ[:, None])
            dz = torch.where(named, dz, others)
        part = some & (weights != 0)
        loss = torch.where(part, loss, 0.0)
        dz = torch.where(part[:, None], dz * (weights * s["loss_scale"] / TEMPERATURE)[:, None], 0.0)
        return loss, (loss * weights).sum().view(1), dz
    logp_of = z - torch.logsumexp(z, dim=1, keepdim=True)
    tokens, targets = torch.arange(T, device="cuda"), s["targets"].long()
    part = (targets >= 0) & (s["weight"] != 0 if c["kind"] == "policy" else True)
    at = torch.where(part, targets, 0)
    logp = torch.where(part, logp_of[tokens, at], 0.0)
    if c["kind"] == "policy":
        A, w, r = s["advantage"].double(), s["weight"].double(), torch.exp(logp - s["old_logp"].double())
        gain = torch.where(A >= 0, A * r.clamp(max=1.28), A * r.clamp(min=0.8))
        x = torch.exp(s["ref_logp"].double() - logp)
        loss = torch.where(part, KL_COEF * (x - torch.log(x) - 1.0) - gain, 0.0)
        moves = torch.where(A >= 0, r <= 1.28, r >= 0.8)
        slope = torch.where(part, w * s["loss_scale"] * (KL_COEF * (1.0 - x) - torch.where(moves, A * r, 0.0)), 0.0)
        return logp, loss, (loss * w).sum().view(1), _exact_logits_gradient(z, logp_of, slope, at)
    ends, pair_loss = s["offsets"].tolist(), []
    slope = torch.zeros(T, dtype=torch.float64, device="cuda")
    gain = torch.where(part, logp - s["ref_logp"].double(), 0.0)
    for i in range(0, len(ends) - 1, 2):
        a, b, e = ends[i:i + 3]
        m = BETA * (gain[a:b].sum() - gain[b:e].sum())
        pair_loss.append(-(1 - SMOOTHING) * torch.nn.functional.logsigmoid(m) - SMOOTHING * torch.nn.functional.logsigmoid(-m))
        dm = s["scale"] * s["loss_scale"] * BETA * (torch.sigmoid(m) - (1 - SMOOTHING))
        slope[a:b], slope[b:e] = dm, -dm
    pair_loss = torch.stack(pair_loss)
    return logp, pair_loss, (pair_loss.sum() * s["scale"]).view(1), _exact_logits_gradient(z, logp_of, torch.where(part, slope, 0.0), at)
