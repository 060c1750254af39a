"""ds_gated_mlp_fwd / _bwd / _wgrad against oracle/layer.py.

Tolerances, elementwise (`size`: a sum of products with every product counted by its absolute value; U = 2^-24; roundings to the type count half a step, 2^-8
in bf16 and U in fp32):
  a sum of n products in fp32, in any order: n U size; the bias one addition more.
  H = act(G) U of the unrounded sums: |act'| <= 1.2 times the error of G, |act(G)| <= |G| times that of U, and the activation itself: one exponential whose argument is
  off by at most 4 U of its size, which is below 30 where it matters (beyond, the logistic term is 0 or 1 to 2^-24), one reciprocal, five operations: 2^-17 |G|.
  dG, dU: the same for act' and act, (1 + |G|) 2^-17 of |dH U| and |dH|.
  dx: a sum of 2 d_ff products of dG and dU as stored.  dW: rows products (split sums: the same additions in another order).  db: rows additions.
  Half-steps of subnormal results: 2^-133 in bf16."""
import numpy as np
import pytest
import torch

from oracle import layer
from paper_2311_10418_amd import binding as ds
from paper_2311_10418_amd import workload as wl
from helpers import DEV, to_dev, to_np

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
U = 2.0 ** -24
ACT = {"gelu": ds.DS_ACT_GELU, "silu": ds.DS_ACT_SILU, "relu": ds.DS_ACT_RELU}


def _rnd(rng, shape, dt, scale=1.0):
    a = (rng.standard_normal(shape) * scale).astype(np.float32)
    return (wl.to_bf16_grid(a) if dt == BF else a).astype(np.float64)


def _near(got, ref, lim, tag):
    assert np.all(np.isfinite(got)), tag
    dev = np.abs(got - ref)
    lim = lim + 2.0 ** -130
    assert np.all(dev <= lim), (tag, float((dev / lim).max()), np.unravel_index(np.argmax(dev / lim), dev.shape))


class Block:
    """Rows that do not count hold NaN; every output is three rows longer than the call knows, which stay as they were."""

    def __init__(self, dt, rows, d, ff, act, bias=False, keep=True, pad=0.0, seed=1, floats=1 << 24):
        rng = np.random.default_rng([seed, rows, d, ff])
        self.dt, self.rows, self.d, self.ff, self.act = dt, rows, d, ff, act
        self.off = rng.random(rows) < pad
        self.x = _rnd(rng, (rows, d), dt)
        self.wg, self.wu = _rnd(rng, (d, ff), dt, d ** -0.5), _rnd(rng, (d, ff), dt, d ** -0.5)
        self.bg, self.bu = (_rnd(rng, (ff,), dt), _rnd(rng, (ff,), dt)) if bias else (np.zeros(ff), np.zeros(ff))
        self.dh = _rnd(rng, (rows, ff), dt)
        self.valid = torch.tensor(np.where(self.off, -1, 5).astype(np.int32), device=DEV) if pad else None
        put = lambda a: to_dev(a, dt).contiguous()  # noqa: E731
        nan = lambda a: put(np.where(self.off[:, None], np.nan, a))  # noqa: E731
        self.tx, self.tdh = nan(self.x), nan(self.dh)
        self.w_out, self.w_in = (put(self.wg.T), put(self.wu.T)), (put(self.wg), put(self.wu))
        self.tb = (put(self.bg), put(self.bu)) if bias else (None, None)
        self.bias, self.keep = bias, keep
        self.whole = {n: torch.full((rows + 3, c), 9.0, device=DEV, dtype=dt) for n, c in (("h", ff), ("g", ff), ("u", ff), ("dg", ff), ("du", ff), ("dx", d))}
        self.t = {n: w[:rows] for n, w in self.whole.items()}
        self.ws = torch.full((floats,), float("nan"), device=DEV) if floats else None

    def forward(self, generic=False):
        ds.ds_gated_mlp_fwd(self.tx, *self.w_out, self.t["h"], bg=self.tb[0], bu=self.tb[1], g=self.t["g"] if self.keep else None, u=self.t["u"] if self.keep else None, act=ACT[self.act],
                            row_valid=self.valid, workspace=self.ws, force_generic=generic)

    def backward(self, generic=False):
        ds.ds_gated_mlp_bwd(self.tdh, self.t["g"], self.t["u"], *self.w_in, self.t["dg"], self.t["du"], self.t["dx"], act=ACT[self.act], row_valid=self.valid, workspace=self.ws,
                            force_generic=generic)

    def check_forward(self):
        half = 2.0 ** -8 if self.dt == BF else U
        on = ~self.off
        h, g, u = layer.gated_mlp(self.x[on], self.wg, self.wu, self.bg, self.bu, self.act)
        eg = (self.d + 4) * U * (np.abs(self.x[on]) @ np.abs(self.wg) + np.abs(self.bg))
        eu = (self.d + 4) * U * (np.abs(self.x[on]) @ np.abs(self.wu) + np.abs(self.bu))
        lim = np.abs(u) * (1.2 * eg + 2.0 ** -17 * np.abs(g)) + np.abs(g) * eu + 2 * eg * eu
        refs = [("h", h, half * np.abs(h) + (1 + half) * lim)] + ([("g", g, half * np.abs(g) + 2 * eg), ("u", u, half * np.abs(u) + 2 * eu)] if self.keep else [])
        for n, ref, lim in refs:
            got = to_np(self.whole[n])
            assert np.all(got[self.rows:] == 9.0) and np.all(got[:self.rows][self.off] == 0), n
            _near(got[:self.rows][on], ref, lim, n)

    def check_backward(self):
        half = 2.0 ** -8 if self.dt == BF else U
        on = ~self.off
        g, u, dg, du, dx = (to_np(self.whole[n])[:self.rows][on] for n in ("g", "u", "dg", "du", "dx"))
        for n in ("dg", "du", "dx"):
            got = to_np(self.whole[n])
            assert np.all(got[self.rows:] == 9.0) and np.all(got[:self.rows][self.off] == 0), n
        rg, ru = layer.gated_mlp_back(self.dh[on], g, u, self.act)
        _near(dg, rg, half * np.abs(rg) + 2.0 ** -17 * (1 + np.abs(g)) * np.abs(self.dh[on] * u), "dg")
        _near(du, ru, half * np.abs(ru) + 2.0 ** -17 * (1 + np.abs(g)) * np.abs(self.dh[on]), "du")
        ref = dg @ self.wg.T + du @ self.wu.T
        _near(dx, ref, half * np.abs(ref) + 2 * self.ff * U * (np.abs(dg) @ np.abs(self.wg.T) + np.abs(du) @ np.abs(self.wu.T)), "dx")

    def run(self, generic=False):
        self.forward(generic)
        if self.keep:
            self.backward(generic)
        torch.cuda.synchronize()
        self.check_forward()
        if self.keep:
            self.check_backward()


SHAPES = [(1, 8, 8), (1, 64, 128), (2, 72, 24), (15, 200, 136), (16, 256, 512), (17, 40, 64), (33, 1024, 200), (64, 128, 320), (65, 64, 64), (127, 136, 72), (129, 320, 192), (200, 512, 704), (257, 96, 1000),
          (300, 64, 256), (513, 256, 256), (700, 1032, 264)]


@pytest.mark.parametrize("generic", [False, True])
@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_both_directions(shape, dt, generic):
    act = ("gelu", "silu", "relu")[shape[0] % 3]
    Block(dt, *shape, act, bias=shape[0] % 2 == 0, pad=0.2 if shape[0] > 4 else 0.0).run(generic)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("act", ["gelu", "silu", "relu"])
@pytest.mark.parametrize("rows", [3, 20, 40, 150, 600])
def test_activations(rows, act, dt):
    Block(dt, rows, 128, 256, act, bias=True, pad=0.1).run()
    Block(dt, rows, 128, 192, act, keep=False, floats=0).run()


# rows enough for the large tiles: several rounds over the compute units, a part of one, ragged columns, ragged rows, no workspace
@pytest.mark.parametrize("rows,d,ff,floats", [(2000, 256, 1088, 1 << 24), (1025, 512, 448, 1 << 24), (1537, 1024, 512, 1 << 24), (5000, 256, 2816, 0), (9000, 128, 832, 1 << 24), (4099, 768, 640, 1 << 20)])
@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_large(rows, d, ff, floats, act):
    b = Block(BF, rows, d, ff, act, bias=act == "silu", keep=True, pad=0.05, floats=floats)
    b.run()


@pytest.mark.parametrize("dt", [BF, F32])
def test_extremes(dt):
    """Pre-activations from far below to far above 0, and exactly 0."""
    for act in ACT:
        b = Block(dt, 40, 64, 64, act, bias=True)
        b.x[:20] *= 64
        b.x[20:24] = 0
        b.bg[:8] = 0
        b.tx, b.tb = to_dev(b.x, dt), (to_dev(b.bg, dt), b.tb[1])
        b.run()
        big = torch.tensor([3e38, -3e38, 100.0, -100.0, 0.0, -0.0, 1e-30, -1e-30], device=DEV, dtype=dt)[None].contiguous()
        one, dg, du, dx = torch.ones_like(big), torch.empty_like(big), torch.empty_like(big), torch.empty_like(big)
        eye = torch.eye(8, device=DEV, dtype=dt)
        ds.ds_gated_mlp_bwd(one, big, one, eye, torch.zeros_like(eye), dg, du, dx, act=ACT[act])
        assert torch.isfinite(dg).all() and torch.equal(dx, dg)
        f, df = layer.act(np.clip(to_np(big), -200, 200), act)
        assert np.allclose(to_np(dg), df, rtol=2.0 ** -7, atol=1e-30) and np.allclose(to_np(du)[:, 2:], f[:, 2:], rtol=2.0 ** -7, atol=1e-37)


@pytest.mark.parametrize("dt", [BF, F32])
def test_gradients_in_the_place_of_what_was_kept(dt):
    a, b = (Block(dt, 300, 128, 256, "gelu", pad=0.1) for _ in range(2))
    for t in (a, b):
        t.forward()
    a.backward()
    b.t["dg"], b.t["du"] = b.t["g"], b.t["u"]
    b.backward()
    assert torch.equal(a.t["dg"], b.t["g"]) and torch.equal(a.t["du"], b.t["u"]) and torch.equal(a.t["dx"], b.t["dx"])


WGRADS = [(1, 8, 8, 1 << 17), (5, 64, 136, 0), (64, 256, 512, 1 << 24), (129, 320, 192, 1 << 24), (1000, 256, 256, 1 << 24), (2000, 128, 704, 1 << 24), (777, 200, 264, 0), (3001, 64, 64, 1 << 24), (4100, 512, 768, 1 << 24),
          (600, 72, 1000, 1 << 18)]


@pytest.mark.parametrize("generic", [False, True])
@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("rows,d,ff,floats", WGRADS)
def test_weight_gradients(rows, d, ff, floats, dt, generic):
    rng = np.random.default_rng([7, rows, d, ff])
    x, dg, du = _rnd(rng, (rows, d), dt), _rnd(rng, (rows, ff), dt), _rnd(rng, (rows, ff), dt)
    ws = torch.full((floats,), float("nan"), device=DEV) if floats else None
    for accumulate in (False, True):
        out = [torch.full((d, ff), 3.0, device=DEV) for _ in range(2)] + ([torch.full((ff,), 3.0, device=DEV) for _ in range(2)] if floats else [None, None])
        ds.ds_gated_mlp_wgrad(to_dev(x, dt), to_dev(dg, dt), to_dev(du, dt), out[0], out[1], dbg=out[2], dbu=out[3], accumulate=accumulate, workspace=ws, force_generic=generic)
        add = 3.0 if accumulate else 0.0
        for i, dy in enumerate((dg, du)):
            size = np.abs(x).T @ np.abs(dy)
            _near(to_np(out[i]), x.T @ dy + add, (rows + 2) * U * (size + add), "dw")
            if floats:
                _near(to_np(out[2 + i]), dy.sum(axis=0) + add, (rows + 2) * U * (np.abs(dy).sum(axis=0) + add), "db")


def test_no_bias_gradients_without_room():
    t = torch.zeros((8, 64), device=DEV)
    with pytest.raises(ds.DsError):
        ds.ds_gated_mlp_wgrad(t, t, t, torch.zeros((64, 64), device=DEV), torch.zeros((64, 64), device=DEV), dbg=torch.zeros(64, device=DEV), dbu=torch.zeros(64, device=DEV))


@pytest.mark.parametrize("dt,rows,d,ff", [(BF, 16, 256, 512), (BF, 300, 320, 192), (BF, 3000, 256, 1024), (F32, 300, 128, 256)])
def test_same_bits_again_on_another_stream_and_in_a_graph(dt, rows, d, ff):
    b = Block(dt, rows, d, ff, "gelu", bias=True, pad=0.0)
    out = [torch.zeros((d, ff), device=DEV), torch.zeros((d, ff), device=DEV), torch.zeros(ff, device=DEV), torch.zeros(ff, device=DEV)]

    def all_three():
        b.forward()
        b.backward()
        ds.ds_gated_mlp_wgrad(b.tx, b.t["dg"], b.t["du"], out[0], out[1], dbg=out[2], dbu=out[3], workspace=b.ws)

    everything = lambda: list(b.whole.values()) + out  # noqa: E731
    all_three()
    torch.cuda.synchronize()
    first = [t.clone() for t in everything()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        all_three()
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(first, everything()))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        all_three()
    for _ in range(4):
        for t in list(b.t.values()) + out:
            t.fill_(4.0)
        b.ws.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(first, everything()))
        (b.whole["h"].float().sum() + 1).item()


def test_refused_tensors():
    b = Block(BF, 10, 64, 128, "gelu")
    wg, wu = b.w_out
    h = b.t["h"]
    for bad in (dict(x=b.tx.float()), dict(wg=wg.t()), dict(wu=wu[:, :32]), dict(h=h[:9]), dict(x=b.tx.cpu()), dict(wg=wg.float()), dict(h=h.float())):
        a = dict(dict(x=b.tx, wg=wg, wu=wu, h=h), **bad)
        with pytest.raises(ValueError):
            ds.ds_gated_mlp_fwd(a["x"], a["wg"], a["wu"], a["h"])
    with pytest.raises(ValueError):
        ds.ds_gated_mlp_fwd(b.tx, wg, wu, h, row_valid=torch.zeros(9, dtype=torch.int32, device=DEV))
    with pytest.raises(ds.DsError):
        ds.ds_gated_mlp_fwd(b.tx, wg, wu, h, g=b.t["g"])
