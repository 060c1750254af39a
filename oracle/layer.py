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
