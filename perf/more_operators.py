"""Performance cases of two parts of an encoder-decoder layer: attention with a learned relative position bias, and the gated feed-forward block.

`listed()` names the cases, `draw(rng)` gives more of the same ranges, `prepare` makes what a program holds before the
call, `run` makes one pass (in plain torch operations, or with `own` through the framework's entry points), `work` says
what the pass cannot do without and `exact` gives the outputs in 64 bits.

Kinds of case
  rel_fwd    O = softmax(s Q K^T + bias[bucket(key position - query position)]) V over a padded micro-batch, or queries at the end of a cache
  rel_bwd    its gradient: dQ, dK, dV and that of the bias table; row sums of dO O are taken from O as it is stored, which the call is given
  glu_fwd    H = act(x Wg^T + bg) (x Wu^T + bu), with the two pre-activation tensors kept for the backward pass or not
  glu_bwd    dG, dU (from the kept tensors) and dx = dG Wg^T + dU Wu^T, weights [in, out]
  glu_wgrad  dWg = x^T dG, dWu = x^T dU and the biases' gradients

Values are N(0, 1) activations and gradients, weights N(0, 1 / in-features), biases of positions N(0, 1).
"""
import math

import torch

own = False
DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ACTS = ("gelu", "silu", "relu")


# ------------------------------------------------------------------------------------ the cases
def listed():
    return [
        # the encoder's own attention at the encoder-decoder stage's width: a micro-batch of medium inputs, 32 buckets up to distance 128
        dict(name="rel_fwd_encoder_64", kind="rel_fwd", dtype="bf16", seqs=31, q_max=523, k_max=523, heads=16, hd=64, causal=False, buckets=32, far=128, cache=False, shortest=0.7),
        dict(name="rel_bwd_encoder_64", kind="rel_bwd", dtype="bf16", seqs=31, q_max=523, k_max=523, heads=16, hd=64, causal=False, buckets=32, far=128, cache=False, shortest=0.7),
        # the longest micro-batch of the d = 2048 stage, causal, heads of 128
        dict(name="rel_fwd_causal_128", kind="rel_fwd", dtype="bf16", seqs=8, q_max=2048, k_max=2048, heads=16, hd=128, causal=True, buckets=32, far=128, cache=False, shortest=0.8),
        dict(name="rel_bwd_causal_128", kind="rel_bwd", dtype="bf16", seqs=8, q_max=2048, k_max=2048, heads=16, hd=128, causal=True, buckets=32, far=128, cache=False, shortest=0.8),
        # one token of each of 16 sequences on a cache of up to 1 019 tokens
        dict(name="rel_fwd_single_tokens", kind="rel_fwd", dtype="bf16", seqs=16, q_max=1, k_max=1019, heads=16, hd=64, causal=True, buckets=32, far=128, cache=True, shortest=0.3),
        # a short micro-batch of the small fp32 stage, gradient, where latency counts
        dict(name="rel_bwd_f32_64", kind="rel_bwd", dtype="f32", seqs=23, q_max=177, k_max=177, heads=4, hd=64, causal=True, buckets=32, far=128, cache=False, shortest=0.5),
        # the block of the encoder-decoder stage over a global batch of 65 536 input tokens, for training
        dict(name="glu_fwd_1024", kind="glu_fwd", dtype="bf16", rows=65629, d=1024, ff=2816, act="gelu", bias=False, keep=True, pad=0.01),
        dict(name="glu_bwd_1024", kind="glu_bwd", dtype="bf16", rows=65629, d=1024, ff=2816, act="gelu", bias=False, keep=True, pad=0.01),
        # one token of each of 16 sequences: the weights are what is read
        dict(name="glu_fwd_single_tokens", kind="glu_fwd", dtype="bf16", rows=16, d=1024, ff=2816, act="gelu", bias=False, keep=False, pad=0.0),
        # a short micro-batch of the target stream, SiLU with biases, nothing kept
        dict(name="glu_fwd_short", kind="glu_fwd", dtype="bf16", rows=957, d=1024, ff=2816, act="silu", bias=True, keep=False, pad=0.1),
        # a small fp32 stage
        dict(name="glu_fwd_f32_256", kind="glu_fwd", dtype="f32", rows=7684, d=256, ff=1024, act="gelu", bias=True, keep=True, pad=0.05),
        # weight gradients over the target stream of the global batch
        dict(name="glu_wgrad_1024", kind="glu_wgrad", dtype="bf16", rows=10485, d=1024, ff=2816, act="gelu", bias=True, keep=True, pad=0.0),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rel_fwd", "rel_fwd", "rel_bwd", "rel_bwd", "glu_fwd", "glu_fwd", "glu_bwd", "glu_wgrad"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind.startswith("glu"):
        d, ff = 64 * _spread(rng, 2, 32), 64 * _spread(rng, 3, 88)
        most = (1 << 37) if dtype == "bf16" else (1 << 33)
        return dict(kind=kind, dtype=dtype, rows=_spread(rng, 1 if kind != "glu_wgrad" else 8, min(65536, most // (d * ff))), d=d, ff=ff, act=rng.choice(ACTS), bias=rng.random() < 0.5,
                    keep=kind != "glu_fwd" or rng.random() < 0.5, pad=rng.choice([0.0, 0.1]) if kind != "glu_wgrad" else 0.0)
    hd = rng.choice([64, 128]) if dtype == "bf16" else rng.choice([32, 64, 96, 128])
    causal = rng.random() < 0.5
    cache = kind == "rel_fwd" and rng.random() < 0.4
    most = 512 if dtype == "f32" else 2048 if causal else 1024
    if cache:
        k_max, q_max = _spread(rng, 1, 8192 if dtype == "bf16" else 2048), rng.choice([1, 1, 2, 5, 33])
        q_max = min(q_max, k_max)
    else:
        k_max = _spread(rng, 1 if kind == "rel_fwd" else 8, most)    # (with a single key the gradients of the scores are nothing but rounding)
        q_max = k_max if causal else _spread(rng, 1, most)
    seqs = _spread(rng, 1, max(1, min(64, ((1 << 16) if cache else 4096 if dtype == "f32" else 12288) // max(q_max, k_max))))
    return dict(kind=kind, dtype=dtype, seqs=seqs, q_max=q_max, k_max=k_max, heads=rng.randint(1, 8 if dtype == "f32" else 16), hd=hd, causal=causal, buckets=rng.choice([8, 16, 32, 64]),
                far=rng.choice([40, 64, 128, 256]), cache=cache, shortest=rng.choice([0.1, 0.5, 1.0]))


def _lengths(case):
    """Ascending lengths of the micro-batch's sequences, as a plan orders them; the last is the longest.  On a cache every sequence has the same number of
    new tokens, as far as it is that long."""
    def spread(most, at):
        n = case["seqs"]
        lo = max(1, int(case["shortest"] * most))
        return [most if i == n - 1 else lo + (most - lo) * ((i * at) % n) // n for i in range(n)]
    kl = sorted(spread(case["k_max"], 1))
    if case["cache"]:
        return [min(case["q_max"], k) for k in kl], kl
    return (kl if case["causal"] else spread(case["q_max"], 7)), kl


def _pairs(case):
    """(visible pairs, query rows, key rows) of the micro-batch, from lengths that do not depend on the seed."""
    ql, kl = _lengths(case)
    first = [k - q if case["cache"] else 0 for q, k in zip(ql, kl)]
    if case["causal"]:
        n = sum(sum(min(f + i + 1, k) for i in range(q)) for q, k, f in zip(ql, kl, first))
    else:
        n = sum(q * k for q, k in zip(ql, kl))
    return n, sum(ql), sum(kl)


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["kind"].startswith("glu"):
        r, d, ff = case["rows"], case["d"], case["ff"]
        tensors = {"glu_fwd": r * d + r * ff * (3 if case["keep"] else 1), "glu_bwd": 5 * r * ff + r * d, "glu_wgrad": 2 * r * ff + r * d}[case["kind"]]
        return {"bytes": size * tensors + 2 * d * ff * (4 if case["kind"] == "glu_wgrad" else size), "flops": 4 * r * d * ff}
    n, qr, kr = _pairs(case)
    wide = case["heads"] * case["hd"]
    if case["kind"] == "rel_fwd":
        return {"bytes": (qr * 2 + kr * 2) * wide * size + 4 * qr * case["heads"], "flops": 4 * n * wide}
    return {"bytes": (qr * 4 + kr * 4) * wide * size + 4 * qr * case["heads"], "flops": 10 * n * wide}


# ------------------------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _normal(g, shape, dtype, scale=1.0):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).mul_(scale).to(dtype)


def prepare(case, seed):
    g, dt = _gen(seed), TYPES[case["dtype"]]
    return _prepare_glu(case, g, dt) if case["kind"].startswith("glu") else _prepare_rel(case, g, dt)


def _buckets(buckets, far, causal):
    """Bucket of each distance key - query from -far to far: half of them for the keys behind (all, where no key in front is seen), exact up to half of
    that, then by the distance's logarithm up to `far`, which the last one has.  Borders are compared in whole numbers."""
    half = buckets if causal else buckets // 2
    exact = half // 2
    def of(n):
        if n < exact:
            return n
        return max([exact] + [exact + t for t in range(1, half - exact) if n ** (half - exact) >= exact ** (half - exact - t) * far ** t])
    behind = [of(n) for n in range(far + 1)]
    front = [0 if causal else half + behind[n] for n in range(1, far + 1)]
    return behind[::-1] + front


def _prepare_rel(case, g, dt):
    n, H, hd = case["seqs"], case["heads"], case["hd"]
    ql, kl = _lengths(case)
    Lq, Lk = max(ql), max(kl)
    first = [k - q if case["cache"] else 0 for q, k in zip(ql, kl)]
    s = dict(case=case, ql=ql, kl=kl, Lq=Lq, Lk=Lk, first=first, scale=hd ** -0.5)
    at = lambda a: torch.tensor(a, device=DEV, dtype=torch.int32)  # noqa: E731
    s["q_row"], s["q_len"] = at([i * Lq for i in range(n)]), at(ql)
    s["k_row"], s["k_len"] = at([i * Lk for i in range(n)]), at(kl)
    s["q_pos"] = at(first) if case["cache"] else None
    s["bucket"] = at(_buckets(case["buckets"], case["far"], case["causal"]))
    s["bias"] = _normal(g, (case["buckets"], H), dt)
    w = H * hd
    if case["causal"] and not case["cache"]:   # self-attention: one packed tensor [rows, q | k | v]
        qkv = _normal(g, (n * Lq, 3 * w), dt)
        s["q"], s["k"], s["v"] = qkv[:, :w], qkv[:, w:2 * w], qkv[:, 2 * w:]
        grads = torch.zeros_like(qkv)
        s["dq"], s["dk"], s["dv"] = grads[:, :w], grads[:, w:2 * w], grads[:, 2 * w:]
    else:
        s["q"] = _normal(g, (n * Lq, w), dt)
        kv = _normal(g, (n * Lk, 2 * w), dt)
        s["k"], s["v"] = kv[:, :w], kv[:, w:]
        s["dq"], grads = torch.zeros_like(s["q"]), torch.zeros_like(kv)
        s["dk"], s["dv"] = grads[:, :w], grads[:, w:]
    s["o"] = torch.zeros((n * Lq, w), device=DEV, dtype=dt)
    s["lse"] = torch.zeros((H, n * Lq), device=DEV)
    if case["kind"] == "rel_bwd":
        s["d_o"] = _normal(g, (n * Lq, w), dt)
        s["o"], s["lse"] = _plain_rel_fwd(s)
        s["dbias"] = torch.zeros((case["buckets"], H), device=DEV)
    s["scratch"] = torch.zeros((1 << 26) + 2048 * H * (n * (Lq + Lk) // 64 + n), device=DEV, dtype=torch.uint8)
    return s


def _prepare_glu(case, g, dt):
    r, d, ff = case["rows"], case["d"], case["ff"]
    s = dict(case=case)
    s["valid"] = torch.where(torch.rand((r,), generator=g, device=DEV) < case["pad"], -1, 1).to(torch.int32) if case["pad"] else None
    s["workspace"] = torch.empty((1 << 25,), device=DEV)
    if case["kind"] == "glu_fwd":
        s["x"] = _normal(g, (r, d), dt)
        s["wg"], s["wu"] = _normal(g, (ff, d), dt, d ** -0.5), _normal(g, (ff, d), dt, d ** -0.5)          # [out, in]
        s["bg"], s["bu"] = (_normal(g, (ff,), dt, 0.1), _normal(g, (ff,), dt, 0.1)) if case["bias"] else (None, None)
        s["h"] = torch.empty((r, ff), device=DEV, dtype=dt)
        s["g"], s["u"] = (torch.empty_like(s["h"]), torch.empty_like(s["h"])) if case["keep"] else (None, None)
    elif case["kind"] == "glu_bwd":
        s["g"], s["u"], s["dh"] = (_normal(g, (r, ff), dt) for _ in range(3))
        s["wg"], s["wu"] = _normal(g, (d, ff), dt, d ** -0.5), _normal(g, (d, ff), dt, d ** -0.5)          # [in, out]
        s["dg"], s["du"] = torch.empty_like(s["g"]), torch.empty_like(s["g"])
        s["dx"] = torch.empty((r, d), device=DEV, dtype=dt)
    else:
        s["x"], s["dg"], s["du"] = _normal(g, (r, d), dt), _normal(g, (r, ff), dt), _normal(g, (r, ff), dt)
        s["dwg"], s["dwu"] = torch.zeros((d, ff), device=DEV), torch.zeros((d, ff), device=DEV)
        s["dbg"], s["dbu"] = (torch.zeros((ff,), device=DEV), torch.zeros((ff,), device=DEV)) if case["bias"] else (None, None)
    return s


# ------------------------------------------------------------------------------------ one pass
def run(state):
    kind = state["case"]["kind"]
    if kind == "rel_fwd":
        return _own_rel_fwd(state) if own else _plain_rel_fwd(state)
    if kind == "rel_bwd":
        return _own_rel_bwd(state) if own else _plain_rel_bwd(state)
    if kind == "glu_fwd":
        return _own_glu_fwd(state) if own else _plain_glu_fwd(state)
    if kind == "glu_bwd":
        return _own_glu_bwd(state) if own else _plain_glu_bwd(state)
    return _own_glu_wgrad(state) if own else _plain_glu_wgrad(state)


# the framework's calls
def _ds():
    from paper_2311_10418_amd import binding
    return binding


def _own_act(ds, c):
    return {"gelu": ds.DS_ACT_GELU, "silu": ds.DS_ACT_SILU, "relu": ds.DS_ACT_RELU}[c["act"]]


def _own_rel_fwd(s):
    c = s["case"]
    _ds().ds_rel_attention_fwd(s["q"], s["k"], s["v"], s["bias"], s["bucket"], s["o"], s["lse"], s["q_row"], s["q_len"], s["k_row"], s["k_len"], c["heads"], c["hd"], c["causal"],
                               s["Lq"], s["Lk"], s["scratch"], scale=s["scale"], q_pos=s["q_pos"])
    return [s["o"], s["lse"]]


def _own_rel_bwd(s):
    c = s["case"]
    _ds().ds_rel_attention_bwd(s["q"], s["k"], s["v"], s["bias"], s["bucket"], s["o"], s["d_o"], s["lse"], s["dq"], s["dk"], s["dv"], s["dbias"], s["q_row"], s["q_len"], s["k_row"],
                               s["k_len"], c["heads"], c["hd"], c["causal"], s["Lq"], s["Lk"], s["scratch"], scale=s["scale"], q_pos=s["q_pos"])
    return [s["dq"], s["dk"], s["dv"], s["dbias"]]


def _own_glu_fwd(s):
    ds = _ds()
    ds.ds_gated_mlp_fwd(s["x"], s["wg"], s["wu"], s["h"], bg=s["bg"], bu=s["bu"], g=s["g"], u=s["u"], act=_own_act(ds, s["case"]), row_valid=s["valid"], workspace=s["workspace"])
    return [t for t in (s["h"], s["g"], s["u"]) if t is not None]


def _own_glu_bwd(s):
    ds = _ds()
    ds.ds_gated_mlp_bwd(s["dh"], s["g"], s["u"], s["wg"], s["wu"], s["dg"], s["du"], s["dx"], act=_own_act(ds, s["case"]), row_valid=s["valid"], workspace=s["workspace"])
    return [s["dg"], s["du"], s["dx"]]


def _own_glu_wgrad(s):
    _ds().ds_gated_mlp_wgrad(s["x"], s["dg"], s["du"], s["dwg"], s["dwu"], dbg=s["dbg"], dbu=s["dbu"], workspace=s["workspace"])
    return [t for t in (s["dwg"], s["dwu"], s["dbg"], s["dbu"]) if t is not None]


# the plain forms: 32 bits, rounded once at the end (sums over all pairs of a bucket in 64)
def _plain_map(s):
    """Masked softmax [seqs, heads, Lq, Lk] with its inputs, the rows that exist, log-sum-exps and the table's place of each pair of a sequence."""
    c = s["case"]
    n, H, hd, Lq, Lk, far = c["seqs"], c["heads"], c["hd"], s["Lq"], s["Lk"], c["far"]
    q = s["q"].float().reshape(n, Lq, H, hd).transpose(1, 2)
    k = s["k"].float().reshape(n, Lk, H, hd).transpose(1, 2)
    v = s["v"].float().reshape(n, Lk, H, hd).transpose(1, 2)
    first = torch.zeros_like(s["q_len"]) if s["q_pos"] is None else s["q_pos"]
    i, j = torch.arange(Lq, device=DEV), torch.arange(Lk, device=DEV)
    at = first[:, None] + i[None]                                                 # positions of the queries
    rows = (i[None] < s["q_len"][:, None])[:, None, :, None]
    seen = (j[None] < s["k_len"][:, None])[:, None, None, :]
    apart = j[None, None] - at[:, :, None]                                        # [seqs, Lq, Lk]
    if c["causal"]:
        seen = seen & (apart <= 0)[:, None]
    if s["q_pos"] is None:
        apart = apart[:1]
    bucket = s["bucket"].long()[apart.clamp(-far, far) + far]
    score = torch.matmul(q, k.transpose(-1, -2)).mul_(s["scale"])
    score += s["bias"].float()[bucket].permute(0, 3, 1, 2)
    score.masked_fill_(~seen, float("-inf"))
    top = score.amax(-1, keepdim=True)
    p = score.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    lse = (top + total.log())[..., 0]
    return q, k, v, p.div_(total).masked_fill_(~rows, 0.0), torch.where(rows[..., 0], lse, torch.zeros((), device=DEV)), bucket


def _plain_back(t, like):
    """[seqs, heads, L, hd] -> stream rows."""
    return t.transpose(1, 2).reshape(t.shape[0] * t.shape[2], -1).to(like.dtype)


def _plain_rel_fwd(s):
    _, _, v, p, lse, _ = _plain_map(s)
    return [_plain_back(torch.matmul(p, v), s["q"]), lse.transpose(0, 1).reshape(s["case"]["heads"], -1).contiguous()]


def _plain_rel_bwd(s):
    c = s["case"]
    n, H, hd, Lq = c["seqs"], c["heads"], c["hd"], s["Lq"]
    q, k, v, p, _, bucket = _plain_map(s)
    rows = (torch.arange(Lq, device=DEV)[None] < s["q_len"][:, None])[:, None, :, None]
    heads = lambda t: torch.where(rows, t.float().reshape(n, Lq, H, hd).transpose(1, 2), torch.zeros((), device=DEV))  # noqa: E731
    d_o = heads(s["d_o"])
    dv = torch.matmul(p.transpose(-1, -2), d_o)
    ds = p.mul_(torch.matmul(d_o, v.transpose(-1, -2)).sub_((d_o * heads(s["o"])).sum(-1, keepdim=True)))
    one = torch.nn.functional.one_hot(bucket.reshape(-1), c["buckets"]).double()
    dbias = torch.matmul(ds.sum(0, dtype=torch.float64).reshape(H, -1), one).t().float().contiguous()
    ds *= s["scale"]
    return [_plain_back(torch.matmul(ds, k), s["q"]), _plain_back(torch.matmul(ds.transpose(-1, -2), q), s["q"]), _plain_back(dv, s["q"]), dbias]


_C, _A = math.sqrt(2.0 / math.pi), 0.044715


def _plain_act(z, act):
    """Activation and its derivative."""
    if act == "relu":
        return torch.clamp(z, min=0.0), (z > 0).to(z.dtype)
    if act == "silu":
        f = 1.0 / (1.0 + torch.exp(-z))
        return z * f, f * (1.0 + z * (1.0 - f))
    t = torch.tanh(_C * (z + _A * z * z * z))
    return 0.5 * z * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * _C * (1.0 + 3.0 * _A * z * z)


def _plain_rows(t, valid):
    return t if valid is None else torch.where(valid[:, None] >= 0, t, torch.zeros((), device=DEV, dtype=t.dtype))


def _plain_glu_fwd(s):
    dt = TYPES[s["case"]["dtype"]]
    x = _plain_rows(s["x"].float(), s["valid"])
    g, u = torch.matmul(x, s["wg"].float().t()), torch.matmul(x, s["wu"].float().t())
    if s["bg"] is not None:
        g, u = _plain_rows(g + s["bg"].float(), s["valid"]), _plain_rows(u + s["bu"].float(), s["valid"])
    h = (_plain_act(g, s["case"]["act"])[0] * u).to(dt)
    return [h, g.to(dt), u.to(dt)] if s["case"]["keep"] else [h]


def _plain_glu_bwd(s):
    dt = TYPES[s["case"]["dtype"]]
    f, df = _plain_act(s["g"].float(), s["case"]["act"])
    dh = _plain_rows(s["dh"].float(), s["valid"])
    dg, du = dh * s["u"].float() * df, dh * f
    dx = torch.matmul(dg, s["wg"].float().t()) + torch.matmul(du, s["wu"].float().t())
    return [dg.to(dt), du.to(dt), dx.to(dt)]


def _plain_glu_wgrad(s):
    xt, dg, du = s["x"].float().t(), s["dg"].float(), s["du"].float()
    out = [torch.matmul(xt, dg), torch.matmul(xt, du)]
    return out + [dg.sum(0), du.sum(0)] if s["dbg"] is not None else out


# ------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"].startswith("rel"):
        return _exact_rel(s)
    return _exact_glu(s)


def _exact_rel(s):
    """Every sequence alone."""
    c = s["case"]
    H, hd, far, back = c["heads"], c["hd"], c["far"], c["kind"] == "rel_bwd"
    wide = lambda t: torch.zeros(t.shape, device=DEV, dtype=torch.float64)  # noqa: E731
    o, lse, dq, dk, dv = wide(s["o"]), wide(s["lse"]), wide(s["q"]), wide(s["k"]), wide(s["v"])
    apart_sums = torch.zeros((H, 2 * far + 1), device=DEV, dtype=torch.float64)
    table = s["bias"].double()[s["bucket"].long()]                                # [distance, head]
    for n, (ql, kl) in enumerate(zip(s["ql"], s["kl"])):
        qs, ks = slice(n * s["Lq"], n * s["Lq"] + ql), slice(n * s["Lk"], n * s["Lk"] + kl)
        q, d_o, k, v = (t[at].double().view(-1, H, hd).transpose(0, 1) for t, at in ((s["q"], qs), (s.get("d_o", s["q"]), qs), (s["k"], ks), (s["v"], ks)))
        apart = torch.arange(kl, device=DEV).unsqueeze(0) - (torch.arange(ql, device=DEV) + s["first"][n]).unsqueeze(1)
        near = torch.clamp(apart, min=-far, max=far) + far
        score = torch.bmm(q, k.transpose(1, 2).contiguous()) * s["scale"] + table[near].permute(2, 0, 1)
        if c["causal"]:
            score = torch.where(apart > 0, torch.full((), float("-inf"), device=DEV, dtype=torch.float64), score)
        lse[:, qs] = torch.logsumexp(score, dim=-1)
        p = torch.softmax(score, dim=-1)
        o[qs] = torch.bmm(p, v.contiguous()).transpose(0, 1).reshape(ql, H * hd)
        if not back:
            continue
        delta = (d_o * s["o"][qs].double().view(ql, H, hd).transpose(0, 1)).sum(-1, keepdim=True)
        ds = p * (torch.bmm(d_o, v.transpose(1, 2).contiguous()) - delta)
        # row i of the flipped matrix moved i columns on: its columns are the diagonals, distances 1 - ql .. kl - 1
        moved = torch.nn.functional.pad(ds.flip(1), (0, ql)).reshape(H, -1)[:, :ql * (kl + ql - 1)].view(H, ql, kl + ql - 1).sum(1)
        apart_sums.index_add_(1, (torch.arange(1 - ql, kl, device=DEV) - s["first"][n]).clamp(-far, far) + far, moved)
        dq[qs] = s["scale"] * torch.bmm(ds, k.contiguous()).transpose(0, 1).reshape(ql, H * hd)
        dk[ks] = s["scale"] * torch.bmm(ds.transpose(1, 2).contiguous(), q.contiguous()).transpose(0, 1).reshape(kl, H * hd)
        dv[ks] = torch.bmm(p.transpose(1, 2).contiguous(), d_o.contiguous()).transpose(0, 1).reshape(kl, H * hd)
    if not back:
        return [o, lse]
    dbias = torch.zeros((c["buckets"], H), device=DEV, dtype=torch.float64).index_add_(0, s["bucket"].long(), apart_sums.t().contiguous())
    return [dq, dk, dv, dbias]


def _exact_glu(s):
    """The activation's derivative from an automatic one."""
    c = s["case"]
    act = {"relu": torch.relu, "silu": torch.nn.functional.silu, "gelu": lambda z: torch.nn.functional.gelu(z, approximate="tanh")}[c["act"]]
    if c["kind"] == "glu_wgrad":
        x, dg, du = s["x"].double(), s["dg"].double(), s["du"].double()
        out = [x.t().contiguous() @ dg, x.t().contiguous() @ du]
        return out + [dg.sum(0), du.sum(0)] if c["bias"] else out
    exists = torch.ones((c["rows"], 1), device=DEV, dtype=torch.float64) if s["valid"] is None else (s["valid"] >= 0).double().unsqueeze(1)
    wg, wu = s["wg"].double().t().contiguous(), s["wu"].double().t().contiguous()
    parts = []
    for at in torch.split(torch.arange(c["rows"], device=DEV), 16384):
        if c["kind"] == "glu_fwd":
            x = s["x"][at].double() * exists[at]
            g, u = x @ wg, x @ wu
            if c["bias"]:
                g, u = (g + s["bg"].double()) * exists[at], (u + s["bu"].double()) * exists[at]
            parts.append([act(g) * u] + ([g, u] if c["keep"] else []))
        else:
            g, u = s["g"][at].double().requires_grad_(), s["u"][at].double().requires_grad_()
            dg, du = torch.autograd.grad(act(g) * u, (g, u), s["dh"][at].double() * exists[at])
            parts.append([dg, du, dg @ wg + du @ wu])
    return [torch.cat(t) for t in zip(*parts)]
