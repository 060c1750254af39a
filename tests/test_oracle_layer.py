"""Pins of oracle/layer.py: gradients against central differences, turns against their closed forms."""
import numpy as np
import pytest

from oracle import layer


@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("gate_kind", ["none", "col", "row"])
@pytest.mark.parametrize("with_post,with_pre", [(True, True), (False, True), (True, False)])
def test_resid_norm_gradients_against_differences(rms, gate_kind, with_post, with_pre):
    rng = np.random.default_rng(3)
    rows, d, a_r, a_b = 3, 8, 0.9, 0.7
    v = {k: rng.standard_normal((rows, d)) for k in ("x", "h", "dy", "du")}
    for k in ("post_g", "post_b", "pre_g", "pre_b"):
        v[k] = rng.standard_normal(d)
    v["gate"] = rng.standard_normal(d if gate_kind == "col" else (rows, d))

    def parts(v):
        return ((v["post_g"], v["post_b"]) if with_post else None, None if gate_kind == "none" else v["gate"],
                (v["pre_g"], v["pre_b"]) if with_pre else None)

    def loss(v):
        post, gate, pre = parts(v)
        y = layer.resid_norm_y(v["x"], v["h"], post, gate, a_r, a_b, rms)
        out = (y * v["dy"]).sum()
        return out + (layer.resid_norm_u(y, pre, rms) * v["du"]).sum() if with_pre else out

    post, gate, pre = parts(v)
    y = layer.resid_norm_y(v["x"], v["h"], post, gate, a_r, a_b, rms)
    stats = np.stack([*layer.moments(v["h"], rms), *layer.moments(y, rms)])
    g = layer.resid_norm_back(v["dy"], v["du"], y, v["h"], post, gate, pre, a_r, a_b, rms, stats)
    for key in ["x", "h"] + (["gate"] if gate is not None else []) + (["post_g"] + ([] if rms else ["post_b"]) if with_post else []) + \
            (["pre_g"] + ([] if rms else ["pre_b"]) if with_pre else []):
        got = g["d" + key]
        for at in np.ndindex(v[key].shape):
            hi, lo = dict(v), dict(v)
            hi[key], lo[key] = v[key].copy(), v[key].copy()
            hi[key][at] += 1e-6
            lo[key][at] -= 1e-6
            assert abs((loss(hi) - loss(lo)) / 2e-6 - got[at]) <= 1e-7 * (1 + abs(got[at])) * 10, key


def test_rope_closed_forms():
    rng = np.random.default_rng(4)
    x = rng.standard_normal((3, 2 * 6))
    freq = np.array([np.pi / 2, np.pi / 4])
    y = layer.rope(x, [1, -1, 0], freq, 2, 6, 4, True, False, 1.0)
    assert np.array_equal(y[1:], x[1:])                               # no position; no turn
    assert np.allclose(y[0, [0, 1]], [-x[0, 1], x[0, 0]])             # a quarter
    assert np.allclose(y[0, [8, 9]], [(x[0, 8] - x[0, 9]) / np.sqrt(2), (x[0, 8] + x[0, 9]) / np.sqrt(2)])
    assert np.array_equal(y[0, [4, 5, 10, 11]], x[0, [4, 5, 10, 11]])  # columns beyond
    z = layer.rope(x, [1, -1, 0], freq, 2, 6, 4, False, False, 1.0)
    assert np.allclose(z[0, [0, 2]], [-x[0, 2], x[0, 0]])
    for inter in (True, False):
        there = layer.rope(x, [5, 7, 100], freq, 2, 6, 4, inter, False, 2.0)
        assert np.allclose(layer.rope(there, [5, 7, 100], freq, 2, 6, 4, inter, True, 0.5), x)


@pytest.mark.parametrize("causal", [False, True])
def test_differential_attention_gradients_against_differences(causal):
    rng = np.random.default_rng(5)
    H, hd, lq, lk = 2, 4, 5, 5 if causal else 3
    v = {"q": rng.standard_normal((lq, H * hd)), "k": rng.standard_normal((lk, H * hd)), "v": rng.standard_normal((lk, H * hd)), "lam": rng.standard_normal(H)}
    d_o = rng.standard_normal((lq, H * hd))

    def forward(v):
        return layer.diff_attention(v["q"], v["k"], v["v"], v["lam"], H, causal)

    o, o2, lse = forward(v)[:3]
    g = layer.diff_attention_back(v["q"], v["k"], v["v"], v["lam"], o, o2, d_o, lse, H, causal)
    for key in v:
        for at in np.ndindex(v[key].shape):
            hi, lo = dict(v), dict(v)
            hi[key], lo[key] = v[key].copy(), v[key].copy()
            hi[key][at] += 1e-6
            lo[key][at] -= 1e-6
            slope = ((forward(hi)[0] - forward(lo)[0]) * d_o).sum() / 2e-6
            assert abs(slope - g["d" + key][at]) <= 1e-6 * (1 + abs(slope)), key


def test_differential_attention_closed_forms():
    rng = np.random.default_rng(6)
    H, hd, l = 2, 8, 4
    q, k, v = (rng.standard_normal((l, H * hd)) for _ in range(3))
    lam = np.array([0.3, -0.5])
    o, o2, lse = layer.diff_attention(q[:1], k[:1], v[:1], lam, H, True)[:3]          # one key: every probability is 1
    assert np.allclose(o, v[:1] * np.repeat(1 - lam, hd)) and np.allclose(o2, v[:1])
    o, o2, lse = layer.diff_attention(np.zeros_like(q), k, v, lam, H, False)[:3]      # uniform scores
    assert np.allclose(o, np.tile(v.mean(axis=0) * np.repeat(1 - lam, hd), (l, 1))) and np.allclose(lse, np.log(l))
    same = np.concatenate([np.concatenate([t[:, :hd // 2]] * 2, axis=1) for t in (q, k)], axis=0)      # both maps alike, lambda = 1: nothing is left
    o = layer.diff_attention(same[:l], same[l:], v[:, :hd], np.ones(1), 1, True)[0]
    assert np.allclose(o, 0)


@pytest.mark.parametrize("causal,pos", [(False, 0), (True, 0), (True, 2), (False, -3)])
def test_relative_bias_gradients_against_differences(causal, pos):
    rng = np.random.default_rng(7)
    H, hd, lq, lk, scale = 2, 4, 4, 5, 0.7
    v = {"q": rng.standard_normal((lq, H * hd)), "k": rng.standard_normal((lk, H * hd)), "v": rng.standard_normal((lk, H * hd)), "bias": rng.standard_normal((6, H))}
    bucket = np.array([0, 1, 1, 2, 3, 5, 4])
    d_o = rng.standard_normal((lq, H * hd))

    def forward(v):
        return layer.rel_attention(v["q"], v["k"], v["v"], v["bias"], bucket, H, causal, pos, scale)[0]

    g = layer.rel_attention_back(v["q"], v["k"], v["v"], v["bias"], bucket, forward(v), d_o, H, causal, pos, scale)
    for key in v:
        for at in np.ndindex(v[key].shape):
            hi, lo = dict(v), dict(v)
            hi[key], lo[key] = v[key].copy(), v[key].copy()
            hi[key][at] += 1e-6
            lo[key][at] -= 1e-6
            slope = ((forward(hi) - forward(lo)) * d_o).sum() / 2e-6
            assert abs(slope - g["d" + key][at]) <= 1e-6 * (1 + abs(slope)), key


def test_relative_bias_closed_forms():
    rng = np.random.default_rng(8)
    k, v = rng.standard_normal((4, 8)), rng.standard_normal((4, 8))
    bucket = layer.rel_buckets(4, 2, True)
    assert list(bucket) == [1, 1, 0, 3, 3]
    bias = np.log(np.array([[1.0], [2.0], [4.0], [8.0]]))           # zero queries: probabilities go by the buckets alone
    o, lse = layer.rel_attention(np.zeros((2, 8)), k, v, bias, bucket, 1, False)[:2]
    w = np.array([[1, 8, 8, 8], [2, 1, 8, 8.0]])
    assert np.allclose(o, (w / w.sum(axis=1, keepdims=True)) @ v) and np.allclose(lse, np.log(w.sum(axis=1)))
    o, lse = layer.rel_attention(np.zeros((2, 8)), k, v, bias, bucket, 1, True, pos=-1)[:2]      # the first row sees nothing, the second the first key
    assert np.all(o[0] == 0) and lse[0, 0] == -np.inf and np.allclose(o[1], v[0])
    half = 16                                                       # 32 buckets up to 128: 0..7 alone, 8..15 by the logarithm in steps of sqrt(sqrt(2))
    b = layer.rel_buckets(32, 128, True)[:129][::-1]
    assert list(b[:9]) == list(range(8)) + [8] and b[16] == 10 and b[32] == 12 and b[64] == 14 and b[128] == half - 1 and b[11] == 8 and b[12] == 9


@pytest.mark.parametrize("kind", ["gelu", "silu", "relu"])
def test_gated_mlp_gradients_against_differences(kind):
    rng = np.random.default_rng(9)
    v = {"x": rng.standard_normal((3, 4)), "wg": rng.standard_normal((4, 5)), "wu": rng.standard_normal((4, 5)), "bg": rng.standard_normal(5), "bu": rng.standard_normal(5)}
    dh = rng.standard_normal((3, 5))

    def forward(v):
        return layer.gated_mlp(v["x"], v["wg"], v["wu"], v["bg"], v["bu"], kind)

    _, g, u = forward(v)
    dg, du = layer.gated_mlp_back(dh, g, u, kind)
    grads = {"x": dg @ v["wg"].T + du @ v["wu"].T, "wg": v["x"].T @ dg, "wu": v["x"].T @ du, "bg": dg.sum(axis=0), "bu": du.sum(axis=0)}
    for key in v:
        for at in np.ndindex(v[key].shape):
            hi, lo = dict(v), dict(v)
            hi[key], lo[key] = v[key].copy(), v[key].copy()
            hi[key][at] += 1e-6
            lo[key][at] -= 1e-6
            slope = ((forward(hi)[0] - forward(lo)[0]) * dh).sum() / 2e-6
            assert abs(slope - grads[key][at]) <= 1e-6 * (1 + abs(slope)), key


def test_activations():
    z = np.array([-30.0, -1.0, 0.0, 1.0, 30.0])
    assert np.allclose(layer.act(z, "silu")[0], z / (1 + np.exp(-z))) and np.allclose(layer.act(z, "relu")[0], [0, 0, 0, 1, 30])
    assert np.allclose(layer.act(z, "gelu")[0], [0, -0.15880801, 0, 0.84119199, 30])
