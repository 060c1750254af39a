"""ds_resid_norm_fwd / ds_resid_norm_bwd against oracle/layer.py.

Tolerances, elementwise: half a step of the output's type, relative (2^-8 for bf16, 2^-24 for fp32), plus the arithmetic in fp32.  A sum of n
terms taken in a tree over lanes and wavefronts (8 in a lane, 6 levels, 8 wavefronts) or row by row is off by at most
(its depth) x 2^-24 x the sum of the terms' sizes, and some ten operations follow: K = 64 units of 2^-24 of `size`, the result computed
from absolute values (so that what cancels counts in full), cover row sums; column sums add the rows a work-group takes one after the
other (at most 8 x 4 here, 64 work-groups' sums in line at most, 6 levels): 128 units in all."""
import numpy as np
import pytest
import torch

from oracle import layer
from paper_2311_10418_amd import binding as ds
from paper_2311_10418_amd import workload as wl
from helpers import DEV, to_dev, to_np

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
HALF = {BF: 2.0 ** -8, F32: 2.0 ** -24}
UNIT = 2.0 ** -24


def _rnd(rng, shape, dt, scale=1.0, mean=0.0):
    a = (rng.standard_normal(shape) * scale + mean).astype(np.float32)
    return (wl.to_bf16_grid(a) if dt == BF else a).astype(np.float64)


def _near(got, ref, size, half, units, tag):
    dev = np.abs(got - ref)
    lim = half * np.abs(ref) + units * UNIT * size
    assert np.all(np.isfinite(got)), tag
    assert np.all(dev <= lim), (tag, float((dev / np.maximum(lim, 1e-300)).max()))


def _sizes(t, m, r, g, b, rms):
    """Size of a norm's terms: what (t - m) r g + b is a difference of."""
    top = np.abs(t).max(axis=1, keepdims=True)
    return (np.abs(t) + (0 if rms else top)) * r[:, None] * np.abs(g) + (0 if rms else np.abs(b))


class Case:
    def __init__(self, seed, dt, rms, rows, d, gate_kind, with_post, with_pre, pad=0.0, mean=0.0):
        rng = np.random.default_rng(seed)
        self.dt, self.rms, self.rows, self.d = dt, rms, rows, d
        self.a_r, self.a_b = float(np.float32(0.9)), float(np.float32(-1.3))
        self.x, self.h = _rnd(rng, (rows, d), dt), _rnd(rng, (rows, d), dt, 1.0, mean)
        self.dy, self.du = _rnd(rng, (rows, d), dt), _rnd(rng, (rows, d), dt)
        self.post = (_rnd(rng, (d,), dt, 0.3, 1.0), None if rms else _rnd(rng, (d,), dt)) if with_post else None
        self.pre = (_rnd(rng, (d,), dt, 0.3, 1.0), None if rms else _rnd(rng, (d,), dt)) if with_pre else None
        self.gate = None if gate_kind == "none" else _rnd(rng, (d,) if gate_kind == "col" else (rows, d), dt, 0.5, 1.0)
        self.valid = np.where(rng.random(rows) < pad, -1, rng.integers(0, 9, rows)).astype(np.int32) if pad else None
        self.ok = np.ones(rows, bool) if self.valid is None else self.valid >= 0

    def dev(self, a):
        return None if a is None else to_dev(a, self.dt)

    def tensors(self, fill=float("nan")):
        """Device inputs; rows that are padding hold `fill`."""
        def rows(a):
            a = a.copy()
            a[~self.ok] = fill
            return self.dev(a)
        t = {k: rows(getattr(self, k)) for k in ("x", "h", "dy", "du")}
        t["gate"] = None if self.gate is None else rows(self.gate) if self.gate.ndim == 2 else self.dev(self.gate)
        for name, p in (("post", self.post), ("pre", self.pre)):
            t[name + "_g"], t[name + "_b"] = (None, None) if p is None else (self.dev(p[0]), self.dev(p[1]))
        t["row_valid"] = None if self.valid is None else torch.from_numpy(self.valid).to(DEV)
        return t

    def forward(self, t, **out):
        y = out.get("y", torch.full((self.rows, self.d), 7.0, dtype=self.dt, device=DEV))
        u = out.get("u", torch.full((self.rows, self.d), 7.0, dtype=self.dt, device=DEV)) if self.pre else None
        stats = torch.full((4, self.rows), 7.0, device=DEV)
        ds.ds_resid_norm_fwd(t["x"], t["h"], y, stats, post_g=t["post_g"], post_b=t["post_b"], gate=t["gate"], pre_g=t["pre_g"], pre_b=t["pre_b"], u=u,
                             resid_scale=self.a_r, branch_scale=self.a_b, row_valid=t["row_valid"], rms=self.rms)
        return y, u, stats

    def check_forward(self, y, u, stats):
        y, ok = to_np(y), self.ok
        assert np.all(y[~ok] == 0)
        gate = None if self.gate is None else self.gate[ok] if self.gate.ndim == 2 else self.gate
        x, h = self.x[ok], self.h[ok]
        ref = layer.resid_norm_y(x, h, self.post, gate, self.a_r, self.a_b, self.rms)
        m, r = layer.moments(h, self.rms)
        z = np.abs(h) if self.post is None else _sizes(h, m, r, self.post[0], self.post[1], self.rms)
        size = np.abs(self.a_r * x) + np.abs(self.a_b) * (z if gate is None else np.abs(gate) * z)
        _near(y[ok], ref, size, HALF[self.dt], 64, "y")
        if self.post is not None:
            s = to_np(stats)[:, ok]
            assert np.all(np.abs(s[0] - m) <= 64 * UNIT * np.abs(h).max(axis=1)) and np.all(np.abs(s[1] / r - 1) <= 64 * UNIT * (1 + np.abs(m) * r))
        if self.pre is not None:                       # of the stream as it came out
            u = to_np(u)
            assert np.all(u[~ok] == 0)
            m, r = layer.moments(y[ok], self.rms)
            _near(u[ok], layer.resid_norm_u(y[ok], self.pre, self.rms), _sizes(y[ok], m, r, self.pre[0], self.pre[1], self.rms), HALF[self.dt], 64, "u")

    def backward(self, t, y, stats, with_dy=True, accumulate=False, start=5.0, **out):
        f = lambda: torch.full((self.d,), start, device=DEV)  # noqa: E731
        full = lambda: torch.full((self.rows, self.d), 7.0, dtype=self.dt, device=DEV)  # noqa: E731
        o = {"dx": out.get("dx", None), "dh": out.get("dh", None)}
        for k in o:
            o[k] = full() if o[k] is None else o[k]
        o["dgate"] = None if self.gate is None else full() if self.gate.ndim == 2 else f()
        for name, p in (("post", self.post), ("pre", self.pre)):
            o["d%s_g" % name], o["d%s_b" % name] = (None, None) if p is None else (f(), None if self.rms else f())
        partial = torch.full((int(ds.ds_resid_norm_bwd_scratch_floats(self.rows, self.d)),), float("nan"), device=DEV)
        ds.ds_resid_norm_bwd(t["dy"] if with_dy else None, y, t["h"], stats, o["dx"], o["dh"], partial, du=t["du"] if self.pre else None, post_g=t["post_g"],
                             post_b=t["post_b"], gate=t["gate"], pre_g=t["pre_g"], dgate=o["dgate"], dpost_g=o["dpost_g"], dpost_b=o["dpost_b"],
                             dpre_g=o["dpre_g"], dpre_b=o["dpre_b"], resid_scale=self.a_r, branch_scale=self.a_b, row_valid=t["row_valid"], rms=self.rms,
                             accumulate=accumulate)
        return o

    def check_backward(self, o, y, stats, with_dy=True, base=0.0):
        ok = self.ok
        y, s = to_np(y)[ok], to_np(stats)[:, ok]
        gate = None if self.gate is None else self.gate[ok] if self.gate.ndim == 2 else self.gate
        dy, du, h = self.dy[ok] if with_dy else None, self.du[ok], self.h[ok]
        ref = layer.resid_norm_back(dy, du, y, h, self.post, gate, self.pre, self.a_r, self.a_b, self.rms, s)
        # sizes: the same with every term counted by its absolute value
        A = np.abs

        def back_size(c, hat, r):
            out = A(c) + A(hat) * (A(c) * A(hat)).mean(axis=1, keepdims=True) + (0 if self.rms else A(c).mean(axis=1, keepdims=True))
            return r[:, None] * out

        def hat_size(v, m, r):
            return (A(v) + A(m)[:, None]) * r[:, None]

        dt = np.zeros_like(h) if dy is None else A(dy)
        size = {}
        if self.pre is not None:
            hat = hat_size(y, s[2], s[3])
            dt = dt + back_size(du * self.pre[0], hat, s[3])
            size["dpre_g"], size["dpre_b"] = (A(du) * hat).sum(0), A(du).sum(0)
        size["dx"] = A(self.a_r) * dt
        z = hat = A(h)
        if self.post is not None:
            hat = hat_size(h, s[0], s[1])
            z = hat * A(self.post[0]) + (0 if self.rms else A(self.post[1]))
        q = A(self.a_b) * dt * (1 if gate is None else A(gate))
        size["dh"] = q if self.post is None else back_size(q * self.post[0], hat, s[1])
        if gate is not None:
            size["dgate"] = A(self.a_b) * dt * z if gate.ndim == 2 else (A(self.a_b) * dt * z).sum(0)
        if self.post is not None:
            size["dpost_g"], size["dpost_b"] = (q * hat).sum(0), q.sum(0)
        for k, got in o.items():
            if got is None:
                continue
            got = to_np(got)
            if got.ndim == 2:
                assert np.all(got[~ok] == 0), k
                _near(got[ok], ref[k], size[k], HALF[self.dt], 64, k)
            else:
                _near(got, ref[k] + base, size[k] + A(base), 0.0, 128, k)


SIZES = [(1, 8), (5, 64), (3, 520), (9, 1024), (37, 1032), (130, 2048), (67, 2168), (11, 4096), (3, 3000), (517, 256)]


@pytest.mark.parametrize("dt", [F32, BF])
@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("rows,d", SIZES)
def test_both_directions(dt, rms, rows, d):
    for k, (gate, post, pre) in enumerate([("col", True, True), ("row", True, True), ("none", True, True), ("row", False, True), ("col", False, False), ("none", False, True)]):
        c = Case(rows * 7 + k, dt, rms, rows, d, gate, post, pre, pad=0.2 if k % 2 else 0.0, mean=3.0 if k == 2 else 0.0)
        t = c.tensors()
        y, u, stats = c.forward(t)
        torch.cuda.synchronize()
        c.check_forward(y, u, stats)
        o = c.backward(t, y, stats)
        torch.cuda.synchronize()
        c.check_backward(o, y, stats)


@pytest.mark.parametrize("dt", [F32, BF])
def test_every_row_padding_and_no_gradient_of_the_stream(dt):
    c = Case(1, dt, False, 6, 72, "col", True, True, pad=1.1)
    t = c.tensors()
    y, u, stats = c.forward(t)
    o = c.backward(t, y, stats, start=0.0)
    torch.cuda.synchronize()
    for v in [y, u] + list(o.values()):
        assert float(v.float().abs().max()) == 0.0
    c = Case(2, dt, True, 300, 136, "row", True, True)
    t = c.tensors()
    y, u, stats = c.forward(t)
    o = c.backward(t, y, stats, with_dy=False, accumulate=True)
    torch.cuda.synchronize()
    c.check_backward(o, y, stats, with_dy=False, base=5.0)


@pytest.mark.parametrize("rms", [False, True])
def test_in_place(rms):
    """y = x, u = h, then dx = dy, dh = du: what came out of tensors of their own, to the bit."""
    c = Case(3, BF, rms, 1500, 1024, "col", True, True, pad=0.1)
    t = c.tensors(fill=0.5)
    y, u, stats = c.forward(t)
    o = c.backward(t, y, stats)
    x2, h2 = t["x"].clone(), t["h"].clone()
    y2, u2, stats2 = c.forward(dict(t, x=x2, h=h2), y=x2, u=h2)
    dy2, du2 = t["dy"].clone(), t["du"].clone()
    o2 = c.backward(dict(t, dy=dy2, du=du2), y, stats, dx=dy2, dh=du2)
    h3 = t["h"].clone()
    o3 = c.backward(dict(t, h=h3), y, stats, dh=h3)
    torch.cuda.synchronize()
    assert torch.equal(y, y2) and torch.equal(u, u2) and torch.equal(stats, stats2)
    for k in o:
        if o[k] is not None:
            assert torch.equal(o[k], o2[k]) and torch.equal(o[k], o3[k]), k


def test_values_far_from_zero_and_rows_without_spread():
    """A mean 1000 times the deviation costs the digits that it must, and no more; constant rows are 0 before the bias."""
    c = Case(4, F32, False, 40, 1032, "none", True, True, mean=1000.0)
    c.h[5] = 123.0
    t = c.tensors()
    y, u, stats = c.forward(t)
    torch.cuda.synchronize()
    c.check_forward(y, u, stats)


def test_twice_the_same_and_in_a_graph():
    c = Case(5, BF, False, 3001, 512, "col", True, True, pad=0.1)
    t = c.tensors()
    y, u, stats = c.forward(t)
    o = c.backward(t, y, stats)
    y2, u2, stats2 = torch.zeros_like(y), torch.zeros_like(u), torch.zeros_like(stats)
    o2 = {k: torch.zeros_like(v) for k, v in o.items()}
    partial = torch.zeros((int(ds.ds_resid_norm_bwd_scratch_floats(c.rows, c.d)),), device=DEV)

    def call():
        ds.ds_resid_norm_fwd(t["x"], t["h"], y2, stats2, post_g=t["post_g"], post_b=t["post_b"], gate=t["gate"], pre_g=t["pre_g"], pre_b=t["pre_b"], u=u2,
                             resid_scale=c.a_r, branch_scale=c.a_b, row_valid=t["row_valid"])
        ds.ds_resid_norm_bwd(t["dy"], y2, t["h"], stats2, o2["dx"], o2["dh"], partial, du=t["du"], post_g=t["post_g"], post_b=t["post_b"], gate=t["gate"],
                             pre_g=t["pre_g"], dgate=o2["dgate"], dpost_g=o2["dpost_g"], dpost_b=o2["dpost_b"], dpre_g=o2["dpre_g"], dpre_b=o2["dpre_b"],
                             resid_scale=c.a_r, branch_scale=c.a_b, row_valid=t["row_valid"])

    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        for v in [y2, u2, stats2, partial] + list(o2.values()):
            v.fill_(3.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, y2) and torch.equal(u, u2) and torch.equal(stats, stats2)
        for k in o:
            assert torch.equal(o[k], o2[k]), k


def test_directional_derivative():
    """fp32 gradients against central differences of the forward definition in 64 bits."""
    c = Case(6, F32, False, 12, 136, "row", True, True)
    t = c.tensors()
    y64 = layer.resid_norm_y(c.x, c.h, c.post, c.gate, c.a_r, c.a_b, False)
    stats = to_dev(np.stack([*layer.moments(c.h, False), *layer.moments(y64, False)]), F32)
    o = {k: to_np(v) for k, v in c.backward(t, to_dev(y64, F32), stats, start=0.0).items()}
    rng = np.random.default_rng(7)
    keys = {"x": "dx", "h": "dh", "gate": "dgate"}

    def loss(v):
        y = layer.resid_norm_y(v["x"], v["h"], c.post, v["gate"], c.a_r, c.a_b, False)
        return (y * c.dy).sum() + (layer.resid_norm_u(y, c.pre, False) * c.du).sum()

    at = {"x": c.x, "h": c.h, "gate": c.gate}
    for k, g in keys.items():
        v = rng.standard_normal(at[k].shape)
        v /= np.linalg.norm(v)
        e = 1e-5
        slope = (loss(dict(at, **{k: at[k] + e * v})) - loss(dict(at, **{k: at[k] - e * v}))) / (2 * e)
        # 64 units of each product's size, and the differences' own error (e^2, rounding / e)
        assert abs(slope - (o[g] * v).sum()) <= 64 * UNIT * 50 * (np.abs(o[g]) * np.abs(v)).sum() + 1e-7, k


def test_tensors_that_do_not_fit_are_refused():
    c = Case(8, BF, False, 16, 64, "col", True, True)
    t = c.tensors()
    y, u, stats = c.forward(t)
    for bad in (dict(x=t["x"][:8]), dict(h=t["h"].float()), dict(post_g=t["post_g"].float()), dict(gate=t["gate"][:32]), dict(row_valid=torch.zeros(3, dtype=torch.int32, device=DEV))):
        with pytest.raises(ValueError):
            c.forward(dict(t, **bad))
    with pytest.raises(ValueError):
        c.forward(dict(t, x=t["x"].t().contiguous().t()))
    with pytest.raises(ValueError):
        ds.ds_resid_norm_bwd(t["dy"], y, t["h"], stats, torch.empty_like(y), torch.empty_like(y), torch.zeros(8, device=DEV), du=t["du"], pre_g=t["pre_g"])
