"""Performance cases of the parts of a layer that stand beside the GEMM, attention and norm building blocks.

`listed()` names the cases, `draw(rng)` gives more of the same ranges, `prepare` makes what a program holds before the
call, `run` makes one pass (in plain torch operations, or with `own` through the framework's entry points), `work` says
what the pass cannot do without and `exact` gives the outputs in 64 bits.

Kinds of case
  resid_norm_fwd  the end of one block and the start of the next: y = a_r x + a_b gate N_post(h), u = N_pre(y)
  resid_norm_bwd  its gradient: inputs, row or column gate, all gains and biases
  rope            rotary positions of the query and key heads of a packed QKV tensor, or the inverse rotation of a gradient
  diff_fwd        differential attention, O = (softmax(Q1 K1^T) - lambda softmax(Q2 K2^T)) V, over a padded micro-batch
  diff_bwd        its gradient: dQ, dK, dV, dlambda

Values are N(0, 1) activations and gradients, gains and gates about 1, as the stage's workloads draw them.
"""
import math

import torch

own = False
DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
GATES = ("none", "col", "row")


# ------------------------------------------------------------------------------------ the cases
def listed():
    return [
        # the joint between two blocks of the d = 2048 decoder stage over a global batch of 65 536 tokens, column gate (layer scale)
        dict(name="resid_norm_fwd_2048", kind="resid_norm_fwd", dtype="bf16", rms=False, rows=65582, d=2048, gate="col", post=True, pre=True, pad=0.01),
        # the same of a small fp32 stage: one short micro-batch, where latency counts
        dict(name="resid_norm_fwd_256_f32", kind="resid_norm_fwd", dtype="f32", rms=True, rows=517, d=256, gate="none", post=True, pre=True, pad=0.1),
        # gradient at the encoder-decoder stage's width, no bias (RMSNorm), column gate, an odd number of rows
        dict(name="resid_norm_bwd_1024", kind="resid_norm_bwd", dtype="bf16", rms=True, rows=65629, d=1024, gate="col", post=True, pre=True, pad=0.05),
        # gradient of the largest workload's joint: 131 072 tokens, d = 4096, a gate per token and column
        dict(name="resid_norm_bwd_4096", kind="resid_norm_bwd", dtype="bf16", rms=False, rows=131072, d=4096, gate="row", post=True, pre=True, pad=0.0),
        # query and key heads of 65 536 tokens of the d = 2048 stage: two maps of 64 per head of 128, so 64 heads of 64
        dict(name="rope_2048", kind="rope", dtype="bf16", rows=65582, heads=64, hd=64, rot=64, interleaved=False, inverse=False, extra=2048, base=10000.0, far=2048, pad=0.01),
        # gradient in fp32, interleaved pairs, half of the head, positions of a long context with slowed frequencies
        dict(name="rope_far_f32_inverse", kind="rope", dtype="f32", rows=7685, heads=8, hd=128, rot=64, interleaved=True, inverse=True, extra=512, base=500000.0, far=1 << 20, pad=0.0),
        # one token of each of 64 sequences
        dict(name="rope_single_tokens", kind="rope", dtype="bf16", rows=64, heads=64, hd=64, rot=64, interleaved=False, inverse=False, extra=2048, base=10000.0, far=8192, pad=0.0),
        # the longest micro-batch of the d = 2048 stage: 8 sequences of up to 2048 tokens, causal, 16 heads of 128
        dict(name="diff_fwd_causal_128", kind="diff_fwd", dtype="bf16", seqs=8, q_max=2048, k_max=2048, heads=16, hd=128, causal=True, shortest=0.8),
        dict(name="diff_bwd_causal_128", kind="diff_bwd", dtype="bf16", seqs=8, q_max=2048, k_max=2048, heads=16, hd=128, causal=True, shortest=0.8),
        # cross-attention of the encoder-decoder stage: short targets over long inputs, heads of 64
        dict(name="diff_fwd_cross_64", kind="diff_fwd", dtype="bf16", seqs=16, q_max=33, k_max=1019, heads=16, hd=64, causal=False, shortest=0.3),
        # the encoder's own, gradient, unmasked
        dict(name="diff_bwd_full_64", kind="diff_bwd", dtype="bf16", seqs=31, q_max=523, k_max=523, heads=16, hd=64, causal=False, shortest=0.7),
        # a short micro-batch of the small fp32 stage, gradient
        dict(name="diff_bwd_f32_64", kind="diff_bwd", dtype="f32", seqs=23, q_max=177, k_max=177, heads=4, hd=64, causal=True, shortest=0.5),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["resid_norm_fwd", "resid_norm_bwd", "rope", "diff_fwd", "diff_bwd"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind.startswith("resid_norm"):
        d = 8 * _spread(rng, 8, 512)
        rows = _spread(rng, 1, (1 << 27) // d)
        return dict(kind=kind, dtype=dtype, rms=rng.random() < 0.5, rows=rows, d=d, gate=rng.choice(GATES), post=rng.random() < 0.8, pre=rng.random() < 0.9, pad=rng.choice([0.0, 0.1]))
    if kind == "rope":
        hd = rng.choice([32, 64, 96, 128])
        rot = rng.choice([hd, hd // 2, hd - 16])
        heads = rng.randint(1, 32)
        return dict(kind=kind, dtype=dtype, rows=_spread(rng, 1, (1 << 27) // (heads * hd)), heads=heads, hd=hd, rot=rot, interleaved=rng.random() < 0.5, inverse=rng.random() < 0.5,
                    extra=8 * rng.randint(0, 256), base=rng.choice([10000.0, 500000.0]), far=_spread(rng, 16, 1 << 20), pad=rng.choice([0.0, 0.1]))
    hd = rng.choice([64, 128]) if dtype == "bf16" else rng.choice([32, 64, 96, 128])
    causal = rng.random() < 0.5
    most = 512 if dtype == "f32" else 2048 if causal else 1024
    k_max = _spread(rng, 1 if kind == "diff_fwd" else 8, most)       # (with a single key the gradients of the scores are nothing but rounding)
    q_max = k_max if causal else _spread(rng, 1, most)
    heads = rng.randint(1, 8 if dtype == "f32" else 16)
    seqs = _spread(rng, 1, max(1, min(64, (4096 if dtype == "f32" else 12288) // max(q_max, k_max))))
    return dict(kind=kind, dtype=dtype, seqs=seqs, q_max=q_max, k_max=k_max, heads=heads, hd=hd, causal=causal, shortest=rng.choice([0.1, 0.5, 1.0]))


def _eps(case):
    return 1e-6 if case["rms"] else 1e-5


def _pairs(case):
    """(visible pairs, query rows, key rows) of the micro-batch, from lengths that do not depend on the seed."""
    ql, kl = _lengths(case)
    if case["causal"]:
        n = sum(sum(min(i + 1, k) for i in range(q)) for q, k in zip(ql, kl))
    else:
        n = sum(q * k for q, k in zip(ql, kl))
    return n, sum(ql), sum(kl)


def _lengths(case):
    """Ascending lengths of the micro-batch's sequences, as a plan orders them; the last is the longest."""
    def spread(most, at):
        n = case["seqs"]
        lo = max(1, int(case["shortest"] * most))
        return [most if i == n - 1 else lo + (most - lo) * ((i * at) % n) // n for i in range(n)]
    kl = sorted(spread(case["k_max"], 1))
    return (kl if case["causal"] else spread(case["q_max"], 7)), kl


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["kind"] in ("resid_norm_fwd", "resid_norm_bwd"):
        n, d = case["rows"] * case["d"], case["d"]
        vectors = (2 if case["rms"] else 4) + (1 if case["gate"] == "col" else 0)
        if case["kind"] == "resid_norm_fwd":
            tensors = 3 + case["pre"] + (case["gate"] == "row")
            return {"bytes": n * size * tensors + vectors * d * size, "flops": 20 * n}
        tensors = 4 + 2 * case["pre"] + 2 * (case["gate"] == "row") - (0 if case["post"] or case["gate"] != "none" else 1)
        return {"bytes": n * size * tensors + vectors * d * (size + 4), "flops": 40 * n}
    if case["kind"] == "rope":
        n = case["rows"] * case["heads"] * case["hd"]
        return {"bytes": 2 * n * size + 4 * case["rows"], "flops": 3 * n}
    n, qr, kr = _pairs(case)
    wide = case["heads"] * case["hd"]
    if case["kind"] == "diff_fwd":
        return {"bytes": (qr * 3 + kr * 2) * wide * size + 8 * qr * case["heads"], "flops": 4 * n * wide}
    return {"bytes": (qr * 5 + kr * 4) * wide * size + 8 * qr * case["heads"], "flops": 10 * n * wide}


# ------------------------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _normal(g, shape, dtype, scale=1.0, mean=0.0):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).mul_(scale).add_(mean).to(dtype)


def prepare(case, seed):
    g, dt = _gen(seed), TYPES[case["dtype"]]
    if case["kind"].startswith("resid_norm"):
        return _prepare_norm(case, g, dt)
    if case["kind"] == "rope":
        return _prepare_rope(case, g, dt)
    return _prepare_diff(case, g, dt)


def _prepare_norm(case, g, dt):
    rows, d = case["rows"], case["d"]
    s = dict(case=case, resid_scale=0.9, branch_scale=0.7)
    s["valid"] = torch.where(torch.rand((rows,), generator=g, device=DEV) < case["pad"], -1, 1).to(torch.int32)
    s["h"] = _normal(g, (rows, d), dt)
    s["post_g"] = _normal(g, (d,), dt, 0.1, 1.0) if case["post"] else None
    s["post_b"] = _normal(g, (d,), dt, 0.1) if case["post"] and not case["rms"] else None
    s["pre_g"] = _normal(g, (d,), dt, 0.1, 1.0) if case["pre"] else None
    s["pre_b"] = _normal(g, (d,), dt, 0.1) if case["pre"] and not case["rms"] else None
    s["gate"] = None if case["gate"] == "none" else _normal(g, (d,) if case["gate"] == "col" else (rows, d), dt, 0.3, 1.0)
    first = _normal(g, (rows, d), dt)
    if case["kind"] == "resid_norm_fwd":
        s["x"] = first
        s["stats"] = torch.zeros((4, rows), device=DEV)
        s["y"], s["u"] = torch.empty_like(first), (torch.empty_like(first) if case["pre"] else None)
        return s
    # the backward pass has the stream y, the statistics of both norms and the gradients of both outputs
    s["y"], s["dy"] = first, _normal(g, (rows, d), dt)
    s["du"] = _normal(g, (rows, d), dt) if case["pre"] else None
    hm, hr = _moments(case, s["h"])
    ym, yr = _moments(case, s["y"])
    s["stats"] = torch.stack([hm, hr, ym, yr]).contiguous()
    s["dx"], s["dh"] = torch.empty_like(first), torch.empty_like(first)
    s["dgate"] = {"none": None, "col": torch.zeros((d,), device=DEV), "row": torch.empty_like(first)}[case["gate"]]
    for k in ("post_g", "post_b", "pre_g", "pre_b"):
        s["d" + k] = None if s[k] is None else torch.zeros((d,), device=DEV)
    s["partial"] = torch.empty((1 << 24,), device=DEV)
    return s


def _moments(case, t):
    """Mean (0 for RMSNorm) and reciprocal deviation of every row, float32."""
    f = t.float()
    m = torch.zeros(t.shape[0], device=DEV) if case["rms"] else f.mean(1)
    return m, 1.0 / torch.sqrt(((f - m[:, None]) ** 2).mean(1) + _eps(case))


def _prepare_rope(case, g, dt):
    rows, heads, hd, rot = case["rows"], case["heads"], case["hd"], case["rot"]
    s = dict(case=case, amplitude=1.0 if case["far"] <= 8192 else 1.1)
    s["pos"] = torch.randint(0, case["far"], (rows,), generator=g, device=DEV, dtype=torch.int32)
    s["pos"] = torch.where(torch.rand((rows,), generator=g, device=DEV) < case["pad"], -1, s["pos"]).to(torch.int32)
    p = torch.arange(rot // 2, device=DEV, dtype=torch.float64)
    s["freq"] = case["base"] ** (-2.0 * p / rot)
    if case["far"] > 8192:                     # frequencies of far positions slowed by their wavelength's share of the known range
        w = torch.clamp((8192 * s["freq"] / (2 * math.pi) - 1.0) / 31.0, 0.0, 1.0)
        s["freq"] = s["freq"] * (w + (1.0 - w) / 8.0)
    wide = heads * hd + case["extra"]          # the value columns behind the query and key heads
    s["x"] = _normal(g, (rows, wide), dt)
    s["y"] = torch.zeros((rows, heads * hd), device=DEV, dtype=dt)
    return s


def _prepare_diff(case, g, dt):
    n, H, hd = case["seqs"], case["heads"], case["hd"]
    ql, kl = _lengths(case)
    Lq, Lk = max(ql), max(kl)
    s = dict(case=case, ql=ql, kl=kl, Lq=Lq, Lk=Lk)
    at = lambda a: torch.tensor(a, device=DEV, dtype=torch.int32)  # noqa: E731
    s["q_row"], s["q_len"] = at([i * Lq for i in range(n)]), at(ql)
    s["k_row"], s["k_len"] = at([i * Lk for i in range(n)]), at(kl)
    w = H * hd
    if case["causal"]:                         # self-attention: one packed tensor [rows, q | k | v]
        qkv = _normal(g, (n * Lq, 3 * w), dt)
        s["q"], s["k"], s["v"] = qkv[:, :w], qkv[:, w:2 * w], qkv[:, 2 * w:]
        grads = torch.zeros_like(qkv)
        s["dq"], s["dk"], s["dv"] = grads[:, :w], grads[:, w:2 * w], grads[:, 2 * w:]
    else:                                      # queries of one stream, packed keys and values of another
        s["q"] = _normal(g, (n * Lq, w), dt)
        kv = _normal(g, (n * Lk, 2 * w), dt)
        s["k"], s["v"] = kv[:, :w], kv[:, w:]
        s["dq"], grads = torch.zeros_like(s["q"]), torch.zeros_like(kv)
        s["dk"], s["dv"] = grads[:, :w], grads[:, w:]
    s["lam"] = torch.rand((H,), generator=g, device=DEV) * 0.6 + 0.2
    s["o"] = torch.zeros((n * Lq, w), device=DEV, dtype=dt)
    s["o2"] = torch.zeros((n * Lq, w), device=DEV, dtype=dt)
    s["lse"] = torch.zeros((2 * H, n * Lq), device=DEV)
    if case["kind"] == "diff_bwd":
        s["d_o"] = _normal(g, (n * Lq, w), dt)
        s["o"], s["o2"], s["lse"] = _plain_diff_fwd(s)
        s["dlam"] = torch.zeros((H,), device=DEV)
    s["scratch"] = torch.zeros((1 << 26) + 96 * H * n * (Lq + Lk), device=DEV, dtype=torch.uint8)
    return s


# ------------------------------------------------------------------------------------ one pass
def run(state):
    kind = state["case"]["kind"]
    if kind == "resid_norm_fwd":
        return _own_norm_fwd(state) if own else _plain_norm_fwd(state)
    if kind == "resid_norm_bwd":
        return _own_norm_bwd(state) if own else _plain_norm_bwd(state)
    if kind == "rope":
        return _own_rope(state) if own else _plain_rope(state)
    if kind == "diff_fwd":
        return _own_diff_fwd(state) if own else _plain_diff_fwd(state)
    return _own_diff_bwd(state) if own else _plain_diff_bwd(state)


# the framework's calls
def _ds():
    from paper_2311_10418_amd import binding
    return binding


def _own_norm_fwd(s):
    c = s["case"]
    _ds().ds_resid_norm_fwd(s["x"], s["h"], s["y"], s["stats"], post_g=s["post_g"], post_b=s["post_b"], gate=s["gate"], pre_g=s["pre_g"], pre_b=s["pre_b"], u=s["u"],
                            resid_scale=s["resid_scale"], branch_scale=s["branch_scale"], row_valid=s["valid"], rms=c["rms"])
    return [t for t in (s["y"], s["u"]) if t is not None]


def _own_norm_bwd(s):
    c = s["case"]
    _ds().ds_resid_norm_bwd(s["dy"], s["y"], s["h"], s["stats"], s["dx"], s["dh"], s["partial"], du=s["du"], post_g=s["post_g"], post_b=s["post_b"], gate=s["gate"], pre_g=s["pre_g"],
                            dgate=s["dgate"], dpost_g=s["dpost_g"], dpost_b=s["dpost_b"], dpre_g=s["dpre_g"], dpre_b=s["dpre_b"],
                            resid_scale=s["resid_scale"], branch_scale=s["branch_scale"], row_valid=s["valid"], rms=c["rms"])
    return [t for t in (s["dx"], s["dh"], s["dgate"], s["dpost_g"], s["dpost_b"], s["dpre_g"], s["dpre_b"]) if t is not None]


def _own_rope(s):
    c = s["case"]
    _ds().ds_rope(s["x"], s["y"], s["pos"], s["freq"], c["heads"], c["hd"], c["rot"], interleaved=c["interleaved"], inverse=c["inverse"], amplitude=s["amplitude"])
    return s["y"]


def _own_diff_fwd(s):
    c = s["case"]
    _ds().ds_diff_attention_fwd(s["q"], s["k"], s["v"], s["lam"], s["o"], s["lse"], s["q_row"], s["q_len"], s["k_row"], s["k_len"], c["heads"], c["hd"], c["causal"], s["Lq"], s["Lk"],
                                s["scratch"], o2=s["o2"])
    return [s["o"], s["o2"], s["lse"]]


def _own_diff_bwd(s):
    c = s["case"]
    _ds().ds_diff_attention_bwd(s["q"], s["k"], s["v"], s["lam"], s["o"], s["o2"], s["d_o"], s["lse"], s["dq"], s["dk"], s["dv"], s["dlam"], s["q_row"], s["q_len"], s["k_row"], s["k_len"],
                                c["heads"], c["hd"], c["causal"], s["Lq"], s["Lk"], s["scratch"])
    return [s["dq"], s["dk"], s["dv"], s["dlam"]]


# the plain forms: 32 bits (angles in 64), rounded once at the end.  A padding row is replaced by zeros first.
def _f(t, valid=None):
    f = t.float()
    return f if valid is None else torch.where(valid[:, None] >= 0, f, torch.zeros((), device=DEV))


def _plain_norm(f, gain, bias, mean, rstd):
    f = (f - mean[:, None]) * rstd[:, None] * gain.float()
    return f if bias is None else f + bias.float()


def _plain_norm_fwd(s):
    c, dt = s["case"], TYPES[s["case"]["dtype"]]
    valid = s["valid"]
    z = _f(s["h"], valid)
    if c["post"]:
        z = _plain_norm(z, s["post_g"], s["post_b"], *_moments(c, z))
    if s["gate"] is not None:
        z = z * s["gate"].float()
    y = _f((s["resid_scale"] * _f(s["x"], valid) + s["branch_scale"] * z).to(dt), valid)       # the stream, in its type
    if not c["pre"]:
        return [y.to(dt)]
    return [y.to(dt), _f(_plain_norm(y, s["pre_g"], s["pre_b"], *_moments(c, y)), valid).to(dt)]


def _plain_norm_back(a, hat, rstd, rms):
    """Gradient of the input of a norm from that of its normalised rows."""
    a_hat = (a * hat).mean(1, keepdim=True)
    return rstd[:, None] * (a - hat * a_hat if rms else a - a.mean(1, keepdim=True) - hat * a_hat)


def _plain_norm_bwd(s):
    c, dt = s["case"], TYPES[s["case"]["dtype"]]
    valid = s["valid"]
    hm, hr, ym, yr = s["stats"]
    dt_y, out = _f(s["dy"], valid), {}
    if c["pre"]:
        hat = _f((s["y"].float() - ym[:, None]) * yr[:, None], valid)
        du = _f(s["du"], valid)
        out["dpre_g"], out["dpre_b"] = (du * hat).sum(0), du.sum(0)
        dt_y = dt_y + _plain_norm_back(du * s["pre_g"].float(), hat, yr, c["rms"])
    dx = s["resid_scale"] * dt_y
    dz = s["branch_scale"] * dt_y
    z = hat_h = _f(s["h"], valid)
    if c["post"]:
        hat_h = _f((s["h"].float() - hm[:, None]) * hr[:, None], valid)
        z = hat_h * s["post_g"].float() + (0 if c["rms"] else s["post_b"].float())
    q = dz if s["gate"] is None else dz * s["gate"].float()
    if s["gate"] is not None:
        out["dgate"] = (dz * z).to(dt) if c["gate"] == "row" else (dz * z).sum(0)
    dh = q
    if c["post"]:
        out["dpost_g"], out["dpost_b"] = (q * hat_h).sum(0), q.sum(0)
        dh = _plain_norm_back(q * s["post_g"].float(), hat_h, hr, c["rms"])
    if c["rms"]:
        out.pop("dpost_b", None), out.pop("dpre_b", None)
    return [dx.to(dt), _f(dh, valid).to(dt)] + [out[k] for k in ("dgate", "dpost_g", "dpost_b", "dpre_g", "dpre_b") if k in out]


def _plain_rope(s):
    c = s["case"]
    rows, heads, hd, rot = c["rows"], c["heads"], c["hd"], c["rot"]
    angle = s["pos"].double()[:, None] * s["freq"]
    cos, sin = (s["amplitude"] * angle.cos()).float()[:, None], (s["amplitude"] * angle.sin()).float()[:, None]
    if c["inverse"]:
        sin = -sin
    x = s["x"][:, :heads * hd].float().reshape(rows, heads, hd)
    even = slice(0, rot, 2) if c["interleaved"] else slice(0, rot // 2)
    odd = slice(1, rot, 2) if c["interleaved"] else slice(rot // 2, rot)
    y = x.clone()
    y[:, :, even] = x[:, :, even] * cos - x[:, :, odd] * sin
    y[:, :, odd] = x[:, :, odd] * cos + x[:, :, even] * sin
    return torch.where(s["pos"][:, None] >= 0, y.reshape(rows, heads * hd), torch.zeros((), device=DEV)).to(s["x"].dtype)


def _plain_maps(s):
    """Scores and masked softmax of both maps, [2, seqs, heads, Lq, Lk], values [seqs, heads, Lk, hd], and the rows and keys that exist."""
    c = s["case"]
    n, H, hd, Lq, Lk = c["seqs"], c["heads"], c["hd"], s["Lq"], s["Lk"]
    q = s["q"].float().reshape(n, Lq, H, 2, hd // 2).permute(3, 0, 2, 1, 4)
    k = s["k"].float().reshape(n, Lk, H, 2, hd // 2).permute(3, 0, 2, 1, 4)
    v = s["v"].float().reshape(n, Lk, H, hd).permute(0, 2, 1, 3)
    i, j = torch.arange(Lq, device=DEV), torch.arange(Lk, device=DEV)
    rows = (i[None] < s["q_len"][:, None])[:, None, :, None]
    seen = (j[None] < s["k_len"][:, None])[:, None, None, :]
    if c["causal"]:
        seen = seen & (j[None, :] <= i[:, None])[None, None]
    score = (torch.matmul(q, k.transpose(-1, -2)) * (hd // 2) ** -0.5).masked_fill_(~seen, float("-inf"))
    top = score.amax(-1, keepdim=True)
    p = score.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    lse = (top + total.log())[..., 0]
    return q, k, v, p.div_(total).masked_fill_(~rows, 0.0), torch.where(rows[..., 0], lse, torch.zeros((), device=DEV))


def _plain_back(t, s, like):
    """[seqs, heads, L, hd] -> stream rows."""
    return t.permute(0, 2, 1, 3).reshape(t.shape[0] * t.shape[2], -1).to(like.dtype)


def _plain_diff_fwd(s):
    _, _, v, p, lse = _plain_maps(s)
    o1, o2 = torch.matmul(p, v)
    o = o1 - s["lam"][:, None, None] * o2
    n, H = s["case"]["seqs"], s["case"]["heads"]
    lse = lse.permute(2, 0, 1, 3).reshape(2 * H, n * s["Lq"]).contiguous()
    return [_plain_back(o, s, s["q"]), _plain_back(o2, s, s["q"]), lse]


def _plain_diff_bwd(s):
    c = s["case"]
    n, H, hd, Lq = c["seqs"], c["heads"], c["hd"], s["Lq"]
    q, k, v, p, _ = _plain_maps(s)
    lam = s["lam"][:, None, None]
    d_o = s["d_o"].float().reshape(n, Lq, H, hd).permute(0, 2, 1, 3)
    d_o = torch.where((torch.arange(Lq, device=DEV)[None] < s["q_len"][:, None])[:, None, :, None], d_o, torch.zeros((), device=DEV))
    dv = torch.matmul((p[0] - lam * p[1]).transpose(-1, -2), d_o)
    g = torch.matmul(d_o, v.transpose(-1, -2))
    delta = (p * g).sum(-1, keepdim=True)
    dlam = -delta[1, ..., 0].double().sum((0, 2)).float()
    ds = p.mul_(g - delta)
    ds[1] *= -lam
    ds *= (hd // 2) ** -0.5
    dq, dk = torch.matmul(ds, k), torch.matmul(ds.transpose(-1, -2), q)
    join = lambda t: _plain_back(t.permute(1, 2, 3, 0, 4).reshape(n, H, t.shape[3], hd), s, s["q"])  # noqa: E731
    return [join(dq), join(dk), _plain_back(dv, s, s["q"]), dlam]


# ------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "resid_norm_fwd":
        return _exact_norm_fwd(s)
    if case["kind"] == "resid_norm_bwd":
        return _exact_norm_bwd(s)
    if case["kind"] == "rope":
        return _exact_rope(s)
    return _exact_diff(s)


_STEP = 16384      # rows taken at a time, so that 64-bit copies of the largest tensors fit easily


def _exact_unit(t, rms):
    """(rows less their mean, over their deviation), deviation: LayerNorm or RMSNorm without gain."""
    if not rms:
        t = t - t.sum(-1, keepdim=True) / t.shape[-1]
    dev = (t.square().sum(-1, keepdim=True) / t.shape[-1] + (1e-6 if rms else 1e-5)).sqrt()
    return t / dev, dev


def _exact_norm_fwd(s):
    c, rms = s["case"], s["case"]["rms"]
    y_all, u_all = torch.zeros_like(s["x"], dtype=torch.float64), torch.zeros_like(s["x"], dtype=torch.float64)
    d64 = lambda t: None if t is None else t.double()  # noqa: E731
    pg, pb, ng, nb = d64(s["post_g"]), d64(s["post_b"]), d64(s["pre_g"]), d64(s["pre_b"])
    for r in range(0, c["rows"], _STEP):
        at = torch.nonzero(s["valid"][r:r + _STEP] >= 0)[:, 0] + r
        branch = s["h"][at].double()
        if c["post"]:
            branch = _exact_unit(branch, rms)[0] * pg
            if not rms:
                branch = branch + pb
        if c["gate"] != "none":
            branch = branch * (s["gate"].double() if c["gate"] == "col" else s["gate"][at].double())
        y = s["resid_scale"] * s["x"][at].double() + s["branch_scale"] * branch
        y_all[at] = y
        if c["pre"]:                           # of the stream as it is held
            u = _exact_unit(y.to(s["x"].dtype).double(), rms)[0] * ng
            u_all[at] = u if rms else u + nb
    return [y_all, u_all] if c["pre"] else [y_all]


def _exact_norm_bwd(s):
    c, rms, d = s["case"], s["case"]["rms"], s["case"]["d"]
    z64 = lambda: torch.zeros((d,), device=DEV, dtype=torch.float64)  # noqa: E731
    like = lambda: torch.zeros((c["rows"], d), device=DEV, dtype=torch.float64)  # noqa: E731
    dx, dh, dgate_row = like(), like(), (like() if c["gate"] == "row" else None)
    dgate, dpost_g, dpost_b, dpre_g, dpre_b = z64(), z64(), z64(), z64(), z64()

    def through(grad, unit, dev):
        """Gradient behind a norm's unit rows: less its parts along the unit row (and along ones)."""
        out = grad - unit * ((grad * unit).sum(-1, keepdim=True) / d)
        if not rms:
            out = out - grad.sum(-1, keepdim=True) / d
        return out / dev

    for r in range(0, c["rows"], _STEP):
        at = torch.nonzero(s["valid"][r:r + _STEP] >= 0)[:, 0] + r
        total = s["dy"][at].double()
        if c["pre"]:
            unit, dev = _exact_unit(s["y"][at].double(), rms)
            du = s["du"][at].double()
            dpre_g += (du * unit).sum(0)
            dpre_b += du.sum(0)
            total = total + through(du * s["pre_g"].double(), unit, dev)
        dx[at] = s["resid_scale"] * total
        total = s["branch_scale"] * total
        branch = s["h"][at].double()
        gate = 1.0 if c["gate"] == "none" else s["gate"].double() if c["gate"] == "col" else s["gate"][at].double()
        if c["post"]:
            unit, dev = _exact_unit(branch, rms)
            branch = unit * s["post_g"].double()
            if not rms:
                branch = branch + s["post_b"].double()
            dpost_g += (total * gate * unit).sum(0)
            dpost_b += (total * gate).sum(0)
            dh[at] = through(total * gate * s["post_g"].double(), unit, dev)
        else:
            dh[at] = total * gate
        if c["gate"] == "row":
            dgate_row[at] = total * branch
        dgate += (total * branch).sum(0)
    out = [dx, dh]
    if c["gate"] != "none":
        out.append(dgate_row if c["gate"] == "row" else dgate)
    if c["post"]:
        out += [dpost_g] if rms else [dpost_g, dpost_b]
    if c["pre"]:
        out += [dpre_g] if rms else [dpre_g, dpre_b]
    return out


def _exact_rope(s):
    """The pairs as complex numbers, turned."""
    c = s["case"]
    rows, heads, hd, rot = c["rows"], c["heads"], c["hd"], c["rot"]
    x = s["x"][:, :heads * hd].double().view(rows, heads, hd)
    turned = x[..., :rot].reshape(rows, heads, rot // 2, 2) if c["interleaved"] else x[..., :rot].reshape(rows, heads, 2, rot // 2).transpose(-1, -2)
    turned = torch.view_as_complex(turned.contiguous())
    angle = s["pos"].double().unsqueeze(-1) * s["freq"] * (-1.0 if c["inverse"] else 1.0)
    turned = torch.view_as_real(turned * torch.polar(torch.full_like(angle, s["amplitude"]), angle).unsqueeze(1))
    turned = turned.reshape(rows, heads, rot) if c["interleaved"] else turned.transpose(-1, -2).reshape(rows, heads, rot)
    y = torch.cat([turned, x[..., rot:]], dim=-1).reshape(rows, heads * hd)
    y[s["pos"] < 0] = 0.0
    return y


def _exact_diff(s):
    """Every sequence alone; the gradients by an automatic derivative of the definition."""
    c = s["case"]
    H, hd, back = c["heads"], c["hd"], c["kind"] == "diff_bwd"
    lam = s["lam"].double().requires_grad_(back)
    wide = lambda t: torch.zeros(t.shape, device=DEV, dtype=torch.float64)  # noqa: E731
    o, o2, lse = wide(s["o"]), wide(s["o2"]), wide(s["lse"])
    dq, dk, dv, dlam = wide(s["q"]), wide(s["k"]), wide(s["v"]), torch.zeros_like(lam, requires_grad=False)
    for i, (ql, kl) in enumerate(zip(s["ql"], s["kl"])):
        qs, ks = slice(i * s["Lq"], i * s["Lq"] + ql), slice(i * s["Lk"], i * s["Lk"] + kl)
        q, k, v = (t[at].double().requires_grad_(back) for t, at in ((s["q"], qs), (s["k"], ks), (s["v"], ks)))
        maps = []
        for half in range(2):
            qh, kh = (t.view(-1, H, 2, hd // 2)[:, :, half].transpose(0, 1) for t in (q, k))
            score = qh @ kh.transpose(1, 2) / math.sqrt(hd // 2)
            if c["causal"]:
                score = score + torch.full((ql, kl), float("-inf"), device=DEV, dtype=torch.float64).triu(1)
            maps.append(torch.softmax(score, dim=-1))
            lse[half::2, qs] = torch.logsumexp(score, dim=-1).detach()
        vh = v.view(-1, H, hd).transpose(0, 1)
        second = maps[1] @ vh
        out = maps[0] @ vh - lam[:, None, None] * second
        o[qs] = out.detach().transpose(0, 1).reshape(ql, H * hd)
        o2[qs] = second.detach().transpose(0, 1).reshape(ql, H * hd)
        if back:
            grads = torch.autograd.grad(out, (q, k, v, lam), s["d_o"][qs].double().view(ql, H, hd).transpose(0, 1))
            dq[qs], dk[ks], dv[ks] = grads[:3]
            dlam += grads[3]
    return [dq, dk, dv, dlam] if back else [o, o2, lse]
