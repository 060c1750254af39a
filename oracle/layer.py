"""Plain float64 numpy of the layer parts beside GEMM, attention and norms: the joint between two blocks (norms on both sides,
gate, residual scale), rotary positions, differential attention; forward and backward, written from the formulas."""
import math

import numpy as np

LN_EPS, RMS_EPS = 1e-5, 1e-6


def moments(t, rms):
    """Mean (0 for RMSNorm) and reciprocal deviation of every row."""
    m = np.zeros(t.shape[0]) if rms else t.mean(axis=1)
    return m, 1.0 / np.sqrt(((t - m[:, None]) ** 2).mean(axis=1) + (RMS_EPS if rms else LN_EPS))


def _norm(t, g, b, rms):
    m, r = moments(t, rms)
    out = (t - m[:, None]) * r[:, None] * g
    return out if rms else out + b


def resid_norm_y(x, h, post, gate, a_r, a_b, rms):
    """post: None or (gain, bias)."""
    z = h if post is None else _norm(h, post[0], post[1], rms)
    return a_r * x + a_b * (z if gate is None else gate * z)


def resid_norm_u(y, pre, rms):
    return _norm(y, pre[0], pre[1], rms)


def _norm_back(c, hat, r, rms):
    out = c - hat * (c * hat).mean(axis=1, keepdims=True)
    return r[:, None] * (out if rms else out - c.mean(axis=1, keepdims=True))


def resid_norm_back(dy, du, y, h, post, gate, pre, a_r, a_b, rms, stats):
    """stats [4, rows] -> dict of gradients.  dy may be None."""
    out = {}
    dt = np.zeros_like(h) if dy is None else dy.copy()
    if pre is not None:
        hat = (y - stats[2][:, None]) * stats[3][:, None]
        out["dpre_g"], out["dpre_b"] = (du * hat).sum(axis=0), du.sum(axis=0)
        dt = dt + _norm_back(du * pre[0], hat, stats[3], rms)
    out["dx"] = a_r * dt
    z = hat = h
    if post is not None:
        hat = (h - stats[0][:, None]) * stats[1][:, None]
        z = hat * post[0] + (0 if rms else post[1])
    if gate is not None:
        out["dgate"] = a_b * dt * z if gate.ndim == 2 else (a_b * dt * z).sum(axis=0)
    q = a_b * dt if gate is None else a_b * gate * dt
    out["dh"] = q
    if post is not None:
        out["dpost_g"], out["dpost_b"] = (q * hat).sum(axis=0), q.sum(axis=0)
        out["dh"] = _norm_back(q * post[0], hat, stats[1], rms)
    return out


def rope(x, pos, freq, n_heads, head_dim, rot, interleaved, inverse, amplitude):
    """x [rows, n_heads * head_dim] -> the same, turned; rows with a negative position as they are."""
    y = x.astype(np.float64).copy()
    for r, t in enumerate(pos):
        if t < 0:
            continue
        for p in range(rot // 2):
            a = float(t) * float(freq[p]) * (-1.0 if inverse else 1.0)
            c, s = amplitude * math.cos(a), amplitude * math.sin(a)
            for h in range(n_heads):
                i = h * head_dim + (2 * p if interleaved else p)
                j = i + (1 if interleaved else rot // 2)
                y[r, i], y[r, j] = x[r, i] * c - x[r, j] * s, x[r, j] * c + x[r, i] * s
    return y


def _heads(t, h):
    """[l, h * hd] -> [h, l, hd]"""
    return t.reshape(t.shape[0], h, -1).transpose(1, 0, 2)


def _flat(t):
    return t.transpose(1, 0, 2).reshape(t.shape[1], -1)


def _scores(q, k, causal):
    """One map of one head: scaled scores with -inf where hidden; a query of position i sees the keys up to i."""
    s = q @ k.T / math.sqrt(q.shape[1])
    if causal:
        s = np.where(np.arange(k.shape[0])[None] > np.arange(q.shape[0])[:, None], -np.inf, s)
    return s


def _log_sum(s):
    top = s.max(axis=1)
    return top + np.log(np.exp(s - top[:, None]).sum(axis=1))


def diff_attention(q, k, v, lam, n_heads, causal):
    """One sequence: q [lq, n_heads * hd], k, v [lk, ...] -> o, o2, lse [2 n_heads, lq], size (what o is a difference of), terms (what a score is a sum of)."""
    o, o2, lse, size, size2, terms = [], [], [], [], [], 0.0
    for h, (qh, kh, vh) in enumerate(zip(_heads(q, n_heads), _heads(k, n_heads), _heads(v, n_heads))):
        half = qh.shape[1] // 2
        p = []
        for m in range(2):
            qm, km = qh[:, m * half:(m + 1) * half], kh[:, m * half:(m + 1) * half]
            s = _scores(qm, km, causal)
            lse.append(_log_sum(s))
            p.append(np.exp(s - lse[-1][:, None]))
            terms = max(terms, float((np.abs(qm) @ np.abs(km).T).max()) / math.sqrt(half))
        o2.append(p[1] @ vh)
        o.append(p[0] @ vh - lam[h] * o2[-1])
        size2.append(p[1] @ np.abs(vh))
        size.append(p[0] @ np.abs(vh) + abs(lam[h]) * size2[-1])
    join = lambda t: _flat(np.stack(t))  # noqa: E731
    return join(o), join(o2), np.stack(lse), join(size), join(size2), terms


def diff_attention_back(q, k, v, lam, o, o2, d_o, lse, n_heads, causal):
    """Gradients of one sequence from what the forward pass left -> dict; "size_*" hold the same sums over absolute values, "part_dv" that of
    both maps' probabilities one by one."""
    names = ("dq", "dk", "dv", "dlam", "size_dq", "size_dk", "size_dv", "part_dv", "part_dq", "part_dk", "size_dlam")
    out = {n: [] for n in names}
    for h in range(n_heads):
        qh, kh, vh, oh, o2h, dh = (_heads(t, n_heads)[h] for t in (q, k, v, o, o2, d_o))
        half = qh.shape[1] // 2
        g = dh @ vh.T
        g_size = np.abs(dh) @ np.abs(vh).T
        d2 = (dh * o2h).sum(axis=1, keepdims=True)
        d1 = (dh * oh).sum(axis=1, keepdims=True) + lam[h] * d2
        d_size = (np.abs(dh) * (np.abs(oh) + 2 * abs(lam[h]) * np.abs(o2h))).sum(axis=1, keepdims=True)
        p = [np.exp(_scores(qh[:, m * half:(m + 1) * half], kh[:, m * half:(m + 1) * half], causal) - lse[2 * h + m][:, None]) for m in range(2)]
        ds = [p[0] * (g - d1), -lam[h] * p[1] * (g - d2)]
        part = [p[0] * (g_size + d_size), abs(lam[h]) * p[1] * (g_size + d_size)]
        c = 1 / math.sqrt(half)
        q_of = lambda m: qh[:, m * half:(m + 1) * half]  # noqa: E731
        k_of = lambda m: kh[:, m * half:(m + 1) * half]  # noqa: E731
        out["dq"].append(np.concatenate([c * ds[m] @ k_of(m) for m in range(2)], axis=1))
        out["dk"].append(np.concatenate([c * ds[m].T @ q_of(m) for m in range(2)], axis=1))
        out["size_dq"].append(np.concatenate([c * np.abs(ds[m]) @ np.abs(k_of(m)) for m in range(2)], axis=1))
        out["size_dk"].append(np.concatenate([c * np.abs(ds[m]).T @ np.abs(q_of(m)) for m in range(2)], axis=1))
        out["part_dq"].append(np.concatenate([c * part[m] @ np.abs(k_of(m)) for m in range(2)], axis=1))
        out["part_dk"].append(np.concatenate([c * part[m].T @ np.abs(q_of(m)) for m in range(2)], axis=1))
        both = p[0] - lam[h] * p[1]
        out["dv"].append(both.T @ dh)
        out["size_dv"].append(np.abs(both).T @ np.abs(dh))
        out["part_dv"].append((p[0] + abs(lam[h]) * p[1]).T @ np.abs(dh))
        out["dlam"].append(-(p[1] * g).sum())
        out["size_dlam"].append((p[1] * g_size).sum())
    return {n: np.array(t) if "dlam" in n else _flat(np.stack(t)) for n, t in out.items()}


# ---------------------------------------------------------------- attention with a relative position bias
def rel_buckets(n_buckets, max_distance, bidirectional):
    """Bucket of each distance -max_distance .. max_distance; borders of the logarithmic ones compared in whole numbers."""
    half = n_buckets // 2 if bidirectional else n_buckets
    exact = half // 2
    m = half - exact

    def of(n):
        if n < exact:
            return n
        return exact + max([t for t in range(m) if n ** m * exact ** t >= exact ** m * max_distance ** t])

    side = [of(n) for n in range(max_distance + 1)]
    return np.array(side[::-1] + [half + b if bidirectional else 0 for b in side[1:]])


def _rel_scores(q, k, bias, bucket, n_heads, causal, pos, scale):
    """Per head: scores, the sum of the sizes of their products, the table's place of each pair."""
    lq, lk, reach = q.shape[0], k.shape[0], len(bucket) // 2
    apart = np.arange(lk)[None, :] - (pos + np.arange(lq))[:, None]
    of = np.clip(bucket, 0, bias.shape[0] - 1)[np.clip(apart, -reach, reach) + reach]
    hd = q.shape[1] // n_heads
    for h in range(n_heads):
        c = slice(h * hd, (h + 1) * hd)
        s = scale * (q[:, c] @ k[:, c].T) + bias[of, h]
        if causal:
            s = np.where(apart > 0, -np.inf, s)
        yield h, c, s, scale * (np.abs(q[:, c]) @ np.abs(k[:, c]).T), of


def _rel_probs(s):
    """(softmax with rows of nothing as zeros, log-sum-exp)."""
    with np.errstate(divide="ignore", invalid="ignore"):
        top = np.where(np.isneginf(s.max(axis=1, initial=-np.inf)), 0.0, s.max(axis=1, initial=-np.inf))
        e = np.exp(s - top[:, None])
        total = e.sum(axis=1)
        return np.where(total[:, None] > 0, e / np.where(total > 0, total, 1.0)[:, None], 0.0), top + np.log(total)


def rel_attention(q, k, v, bias, bucket, n_heads, causal, pos=0, scale=1.0):
    """-> o, lse [heads, lq], size of o, largest sum of sizes of a score's products [heads, lq]."""
    o, size = np.zeros(q.shape), np.zeros(q.shape)
    lse, terms = np.zeros((n_heads, q.shape[0])), np.zeros((n_heads, q.shape[0]))
    for h, c, s, t, _ in _rel_scores(q, k, bias, bucket, n_heads, causal, pos, scale):
        p, lse[h] = _rel_probs(s)
        o[:, c], size[:, c] = p @ v[:, c], p @ np.abs(v[:, c])
        terms[h] = np.where(np.isneginf(s), 0.0, t).max(axis=1, initial=0.0)
    return o, lse, size, terms


def rel_attention_back(q, k, v, bias, bucket, o, d_o, n_heads, causal, pos=0, scale=1.0):
    """Gradients with D from o as given; "<name>_part": the same with everything that dS is a difference of counted by its absolute value."""
    out = {n: np.zeros(t.shape) for n, t in (("dq", q), ("dk", k), ("dv", v), ("dbias", bias))}
    out.update({n + "_part": np.zeros(t.shape) for n, t in list(out.items())})
    for h, c, s, _, of in _rel_scores(q, k, bias, bucket, n_heads, causal, pos, scale):
        p = _rel_probs(s)[0]
        d = (d_o[:, c] * o[:, c]).sum(axis=1, keepdims=True)
        ds = p * (d_o[:, c] @ v[:, c].T - d)
        part = p * (np.abs(d_o[:, c]) @ np.abs(v[:, c]).T + (np.abs(d_o[:, c]) * np.abs(o[:, c])).sum(axis=1, keepdims=True))
        for end, w, f in (("", ds, lambda t: t), ("_part", part, np.abs)):
            out["dq" + end][:, c], out["dk" + end][:, c] = scale * w @ f(k[:, c]), scale * w.T @ f(q[:, c])
            out["dbias" + end][:, h] = np.bincount(of.ravel(), w.ravel(), bias.shape[0])
        out["dv"][:, c], out["dv_part"][:, c] = p.T @ d_o[:, c], p.T @ np.abs(d_o[:, c])
    return out


# ---------------------------------------------------------------- the gated feed-forward block
def act(z, kind):
    """Activation and its derivative: "gelu" (tanh form), "silu", "relu"."""
    if kind == "relu":
        return np.maximum(z, 0.0), (z > 0) * 1.0
    if kind == "silu":
        s = 0.5 * (1.0 + np.tanh(0.5 * z))
        return z * s, s + z * s * (1.0 - s)
    c, a = math.sqrt(2.0 / math.pi), 0.044715
    t = np.tanh(c * (z + a * z ** 3))
    return 0.5 * z * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * c * (1.0 + 3.0 * a * z * z)


def gated_mlp(x, wg, wu, bg, bu, kind):
    """Weights [in, out] -> h, g, u."""
    g, u = x @ wg + bg, x @ wu + bu
    return act(g, kind)[0] * u, g, u


def gated_mlp_back(dh, g, u, kind):
    """-> dg, du."""
    f, df = act(g, kind)
    return dh * u * df, dh * f
