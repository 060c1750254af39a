"""A layer of an encoder-decoder model as its parts make it: RMSNorm, QKV product, attention with a relative position bias, output product with residual, RMSNorm, gated feed-forward
block, second product with residual; forward and backward on a padded layout, against the same formulas in float64 with automatic differentiation; captured into a graph; token by
token on a cache.

Tolerances (normwise, and elementwise in the terms of helpers.check).  On the way to a result lie at most 9 roundings of tensors forward (u, qkv, P, o, x1, its norm, g / u, h, y) and 9
backward; a norm's gradient is a difference that is not small here (at least a third of what it is made of).  The roundings are independent: sqrt(18) x 3 x 2^-8 in bf16 < 5.0e-2.  In
fp32 a product of K <= 768 terms errs by at most sqrt(768) x 2^-24 of its terms, whose sum of squares is what the result is made of: sqrt(18) x 3 x 27.8 x 2^-24 < 2.2e-5."""
import numpy as np
import pytest
import torch

from paper_2311_10418_amd import binding as ds
from paper_2311_10418_amd import workload as wl
from helpers import DEV, check, to_np

pytestmark = pytest.mark.gpu

BF, F32, F64 = torch.bfloat16, torch.float32, torch.float64
TOL = {BF: 5.0e-2, F32: 2.2e-5}
PARAMS = ("ln1", "wqkv", "bias", "wo", "ln2", "wg", "wu", "w2")
BUCKETS, FAR = 16, 50


def _norm64(t, g):
    return t * torch.rsqrt((t * t).mean(-1, keepdim=True) + 1e-6) * g


def layer64(x, p, heads, causal, bucket):
    l, d = x.shape
    q, k, v = ((_norm64(x, p["ln1"]) @ p["wqkv"])[:, i * d:(i + 1) * d].reshape(l, heads, -1).transpose(0, 1) for i in range(3))
    apart = torch.arange(l)[None] - torch.arange(l)[:, None]
    s = q @ k.transpose(1, 2) / (d // heads) ** 0.5 + p["bias"][bucket[apart.clamp(-FAR, FAR) + FAR]].permute(2, 0, 1)
    if causal:
        s = s.masked_fill(apart > 0, -torch.inf)
    x1 = x + (torch.softmax(s, -1) @ v).transpose(0, 1).reshape(l, d) @ p["wo"]
    u = _norm64(x1, p["ln2"])
    return x1 + (torch.nn.functional.gelu(u @ p["wg"], approximate="tanh") * (u @ p["wu"])) @ p["w2"]


class Layer:
    """On the rows of a layout, all buffers made here: forward() and backward() only call the library."""

    def __init__(self, lay, p, x, dy, heads, causal, dt):
        self.n, self.d = x.shape
        self.ff, self.heads, self.hd, self.causal = p["w2"].shape[0], heads, self.d // heads, causal
        n, d, ff = self.n, self.d, self.ff
        dev = lambda a: a.to(dt).to(DEV).contiguous()  # noqa: E731
        ints = lambda a: torch.as_tensor(np.asarray(a, dtype=np.int32), device=DEV)  # noqa: E731
        self.x, self.dy = dev(x), dev(dy)
        self.p = {k: dev(v) for k, v in p.items()}
        self.t = {k: dev(p[k].t()) for k in ("wqkv", "wo", "wg", "wu", "w2")}              # [out, in], as forward products read them
        self.valid = ints(ds.ds_layout_positions(lay))
        self.tables = [ints(a) for a in (lay.seq_row, lay.seq_len)] * 2
        self.longest = int(max(lay.seq_len))
        self.bucket = ints(ds.ds_rel_buckets(BUCKETS, FAR, not causal))
        new = lambda *s, t=dt: torch.zeros(s, dtype=t, device=DEV)  # noqa: E731
        f = lambda *s: new(*s, t=F32)  # noqa: E731
        self.u0, self.qkv, self.o, self.x1, self.u1, self.h, self.g, self.u, self.y = new(n, d), new(n, 3 * d), new(n, d), new(n, d), new(n, d), new(n, ff), new(n, ff), new(n, ff), new(n, d)
        self.st0, self.st1, self.lse = f(2, n), f(2, n), f(heads, n)
        self.dh, self.dg, self.du, self.du1, self.dx1, self.do, self.dqkv, self.du0, self.dx = (new(n, c) for c in (ff, ff, ff, d, d, d, 3 * d, d, d))
        self.grads = {k: f(*v.shape) for k, v in self.p.items()}
        self.scratch = new(int(ds.ds_rel_attention_scratch_bytes(heads, self.hd, FAR, n, n, len(lay.seq_len))), t=torch.uint8)
        self.ws = f(int(ds.ds_gated_mlp_workspace_floats(n, d, ff)))
        self.partial = f(int(ds.ds_norm_bwd_scratch_floats(n, d)))

    def parts(self, t):
        return [t[:, i * self.d:(i + 1) * self.d] for i in range(3)]

    def shape(self):
        return (*self.tables, self.heads, self.hd, self.causal, self.longest, self.longest, self.scratch)

    def forward(self):
        p, t, n, d, ff = self.p, self.t, self.n, self.d, self.ff
        ds.ds_norm_fwd(self.x, p["ln1"], None, self.u0, self.st0, rms=True)
        ds.ds_gemm(self.u0, t["wqkv"], self.qkv, n, 3 * d, d, trans_b=True)
        ds.ds_rel_attention_fwd(*self.parts(self.qkv), p["bias"], self.bucket, self.o, self.lse, *self.shape())
        ds.ds_gemm(self.o, t["wo"], self.x1, n, d, d, trans_b=True, epilogue=ds.DS_EPI_RESID, R=self.x, row_valid=self.valid)
        ds.ds_norm_fwd(self.x1, p["ln2"], None, self.u1, self.st1, rms=True)
        ds.ds_gated_mlp_fwd(self.u1, t["wg"], t["wu"], self.h, g=self.g, u=self.u, row_valid=self.valid, workspace=self.ws)
        ds.ds_gemm(self.h, t["w2"], self.y, n, d, ff, trans_b=True, epilogue=ds.DS_EPI_RESID, R=self.x1, row_valid=self.valid)

    def backward(self):
        p, g, n, d, ff = self.p, self.grads, self.n, self.d, self.ff
        wgrad = lambda a, b, out, m, c: ds.ds_gemm(a, b, out, m, c, n, trans_a=True, epilogue=ds.DS_EPI_ACC32)  # noqa: E731
        ds.ds_gemm(self.dy, p["w2"], self.dh, n, ff, d, trans_b=True)
        wgrad(self.h, self.dy, g["w2"], ff, d)
        ds.ds_gated_mlp_bwd(self.dh, self.g, self.u, p["wg"], p["wu"], self.dg, self.du, self.du1, row_valid=self.valid, workspace=self.ws)
        ds.ds_gated_mlp_wgrad(self.u1, self.dg, self.du, g["wg"], g["wu"], workspace=self.ws)
        ds.ds_norm_bwd(self.du1, self.x1, p["ln2"], self.st1, self.dy, self.dx1, g["ln2"], None, self.partial, rms=True)
        ds.ds_gemm(self.dx1, p["wo"], self.do, n, d, d, trans_b=True)
        wgrad(self.o, self.dx1, g["wo"], d, d)
        ds.ds_rel_attention_bwd(*self.parts(self.qkv), p["bias"], self.bucket, self.o, self.do, self.lse, *self.parts(self.dqkv), g["bias"], *self.shape())
        wgrad(self.u0, self.dqkv, g["wqkv"], d, 3 * d)
        ds.ds_gemm(self.dqkv, p["wqkv"], self.du0, n, d, 3 * d, trans_b=True)
        ds.ds_norm_bwd(self.du0, self.x, p["ln1"], self.st0, self.dx1, self.dx, g["ln1"], None, self.partial, rms=True)


def _problem(seed, lens, cuts, heads, hd, ff, dt):
    rng = np.random.default_rng(seed)
    lay, d = ds.ds_layout_from_cuts(lens, cuts), heads * hd

    def rnd(*shape, scale=1.0, mean=0.0):
        a = (mean + scale * rng.standard_normal(shape)).astype(np.float32)
        return torch.from_numpy((wl.to_bf16_grid(a) if dt == BF else a).astype(np.float64))

    p = dict(ln1=rnd(d, scale=0.1, mean=1.0), wqkv=rnd(d, 3 * d, scale=d ** -0.5), bias=rnd(BUCKETS, heads), wo=rnd(d, d, scale=d ** -0.5), ln2=rnd(d, scale=0.1, mean=1.0),
             wg=rnd(d, ff, scale=d ** -0.5), wu=rnd(d, ff, scale=d ** -0.5), w2=rnd(ff, d, scale=ff ** -0.5))
    on = torch.from_numpy(ds.ds_layout_positions(lay) >= 0)[:, None]
    return lay, p, rnd(lay.total_rows, d) * on, rnd(lay.total_rows, d) * on


def _exact(lay, p, x, dy, heads, causal):
    p = {k: v.clone().requires_grad_(True) for k, v in p.items()}
    x = x.clone().requires_grad_(True)
    bucket = torch.from_numpy(ds.ds_rel_buckets(BUCKETS, FAR, not causal)).long()
    y, loss = torch.zeros_like(x), 0.0
    for r, n in zip(lay.seq_row, lay.seq_len):
        ys = layer64(x[r:r + n], p, heads, causal, bucket)
        loss = loss + (ys * dy[r:r + n]).sum()
        y[r:r + n] = ys
    grads = torch.autograd.grad(loss, [x] + [p[k] for k in PARAMS])
    return y.detach(), grads[0], dict(zip(PARAMS, grads[1:]))


# lengths (padded to the longest of their micro-batch), micro-batch cuts, heads, head size, d_ff
SHAPES = [([130, 3, 77, 1], [0, 2, 4], 4, 64, 704), ([65, 129], [0, 2], 2, 128, 512), ([19, 40, 300], [0, 1, 3], 3, 32, 136)]


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dt", [F32, BF])
@pytest.mark.parametrize("lens,cuts,heads,hd,ff", SHAPES)
def test_layer(dt, lens, cuts, heads, hd, ff, causal):
    lay, p, x, dy = _problem(sum(lens), lens, cuts, heads, hd, ff, dt)
    y, dx, grads = _exact(lay, p, x, dy, heads, causal)
    a = Layer(lay, p, x, dy, heads, causal, dt)
    a.forward()
    a.backward()
    torch.cuda.synchronize()
    for name, got, ref in (("y", a.y, y), ("dx", a.dx, dx)):
        for r, n in zip(lay.seq_row, lay.seq_len):
            check(to_np(got)[r:r + n], ref[r:r + n].numpy(), TOL[dt], "%s rows %d" % (name, r))
    off = torch.from_numpy(ds.ds_layout_positions(lay) < 0).to(DEV)
    assert not a.y[off].any() and not a.dx[off].any()
    for name in PARAMS:
        check(to_np(a.grads[name]), grads[name].numpy(), TOL[dt], "d" + name)


@pytest.mark.parametrize("dt", [F32, BF])
def test_layer_in_a_graph(dt):
    lay, p, x, dy = _problem(3, [130, 3, 77, 1], [0, 2, 4], 4, 64, 704, dt)
    a = Layer(lay, p, x, dy, 4, True, dt)
    a.forward()
    a.backward()
    torch.cuda.synchronize()
    results = lambda: [a.y, a.dx, *a.grads.values()]  # noqa: E731
    first = [t.clone() for t in results()]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        a.forward()
        a.backward()
    for _ in range(4):
        for t in results():
            t.fill_(7.0)
        a.ws.fill_(float("nan"))
        a.scratch.fill_(255)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(s, t) for s, t in zip(first, results()))
        (a.y.float().sum() + 1).item()


def test_two_layers_at_once_on_two_streams():
    """Each with a scratch and a workspace of its own."""
    made = []
    for seed in (4, 5):
        prob = _problem(seed, [200, 90, 300], [0, 3], 4, 128, 512, BF)
        a = Layer(*prob, 4, False, BF)
        a.forward()
        a.backward()
        torch.cuda.synchronize()
        made.append((a, [t.clone() for t in (a.y, a.dx, *a.grads.values())], torch.cuda.Stream()))
    for _ in range(5):
        for a, _, st in made:
            st.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(st):
                a.forward()
                a.backward()
        torch.cuda.synchronize()
        for a, first, _ in made:
            assert all(torch.equal(s, t) for s, t in zip(first, (a.y, a.dx, *a.grads.values())))


@pytest.mark.parametrize("dt", [F32, BF])
@pytest.mark.parametrize("hd", [64, 96])
def test_token_by_token(hd, dt):
    """A causal layer over whole sequences, and the same one token at a time on a cache of keys and values."""
    lens, heads, ff = [150, 150, 150], 4, 264
    lay, p, x, dy = _problem(9, lens, [0, 3], heads, hd, ff, dt)
    y = _exact(lay, p, x, dy, heads, True)[0]
    a = Layer(lay, p, x, dy, heads, True, dt)
    n, d, L = len(lens), heads * hd, 160
    at = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    new = lambda r, c: torch.zeros((r, c), dtype=dt, device=DEV)  # noqa: E731
    cache, q_row, one, k_row = new(n * L, 2 * d), at([0, 1, 2]), at([1] * n), at([i * L for i in range(n)])
    lse, out, qkv = torch.zeros((heads, n), device=DEV), new(n, d), new(n, 3 * d)
    st, u, o, x1, h = torch.zeros((2, n), device=DEV), new(n, d), new(n, d), new(n, d), new(n, ff)
    scratch = torch.zeros(int(ds.ds_rel_attention_scratch_bytes(heads, hd, FAR, n, n * L, n)), dtype=torch.uint8, device=DEV)
    for i in range(lens[0]):
        rows = [int(r) + i for r in lay.seq_row]
        xi = a.x[rows].contiguous()
        ds.ds_norm_fwd(xi, a.p["ln1"], None, u, st, rms=True)
        ds.ds_gemm(u, a.t["wqkv"], qkv, n, 3 * d, d, trans_b=True)
        cache.view(n, L, 2 * d)[:, i] = qkv[:, d:]
        ds.ds_rel_attention_fwd(qkv[:, :d], cache[:, :d], cache[:, d:], a.p["bias"], a.bucket, o, lse, q_row, one, k_row, at([i + 1] * n), heads, hd, True, 1, i + 1, scratch,
                                q_pos=at([i] * n))
        ds.ds_gemm(o, a.t["wo"], x1, n, d, d, trans_b=True, epilogue=ds.DS_EPI_RESID, R=xi)
        ds.ds_norm_fwd(x1, a.p["ln2"], None, u, st, rms=True)
        ds.ds_gated_mlp_fwd(u, a.t["wg"], a.t["wu"], h)
        ds.ds_gemm(h, a.t["w2"], out, n, d, ff, trans_b=True, epilogue=ds.DS_EPI_RESID, R=x1)
        check(to_np(out), y[rows].numpy(), TOL[dt], "token %d" % i)
