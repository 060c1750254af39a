"""ds_rel_attention_fwd / ds_rel_attention_bwd against oracle/layer.py, one sequence at a time.

Tolerances, elementwise, in the terms of the formulas (`size`: the result with every product counted by its absolute value).  Roundings count half a
step: 2^-8 in bf16, U = 2^-24 in fp32.
  scores in fp32: a sum of hd <= 128 products is off by at most 128 U of its terms (`terms`, times the scale); bias, maximum and log-sum-exp are added in two more
  operations, and all of it is the argument of an exponential, so that it is the relative error of a probability; with the exponential and the sum of up to
  2 048 of them (in lanes and tiles), E = U (128 terms + 8 (|bias| + |lse|) + 256).
  general kernels: o: 2 E size; gradients: dP and D are sums of hd <= 128 products more, 2 E + 256 U of `part` (what dS is a difference of).
  matrix-core kernels (bf16): probabilities and dS are rounded to bf16 before they are multiplied: 2^-8 size more; log-sum-exp and D reach the dK / dV kernel
  as two bf16 values, 2^-16 of their size: 2^-16 x (2 + |lse|) of `part`.
  dbias is summed from dS in fp32 in every kernel: up to 2 048 sums of each kind in a row (lanes, blocks, slots): 2 048 U of `part` more.
  What is below 2^-126 counts as 0 in fp32, at worst in every factor of a term: with |dP - D| <= 2^9, |q|, |k|, |dO| <= 2^5 and at most 2^9 rows a sum loses
  less than 2^-126 x 2^9 x 2^5 x 2^9 = 2^-103 (TINY) by it.
  Each result is rounded once to its type."""
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
TINY = 2.0 ** -103


def _rnd(rng, shape, dt, scale=1.0):
    a = (rng.standard_normal(shape) * scale).astype(np.float32)
    return (wl.to_bf16_grid(a) if dt == BF else a).astype(np.float64)


class Case:
    """Sequences with gaps between them; the rows of no sequence hold NaN (inputs) and 9 (outputs)."""

    def __init__(self, seed, dt, heads, hd, ql, kl, causal, pos=None, buckets=32, reach=128, table=None, pad_cols=0, scale=None, gap=3, bias=None):
        rng = np.random.default_rng(seed)
        self.dt, self.heads, self.hd, self.causal, self.ql, self.kl = dt, heads, hd, causal, ql, kl
        self.scale = float(np.float32(hd ** -0.5 if scale is None else scale))
        w = heads * hd
        rows = lambda ls: (np.cumsum([2] + [l + gap for l in ls[:-1]]), 2 + sum(ls) + gap * len(ls))  # noqa: E731
        (self.q_row, self.Tq), (self.k_row, self.Tk) = rows(ql), rows(kl)
        self.q, self.k, self.v = _rnd(rng, (self.Tq, w), dt), _rnd(rng, (self.Tk, w), dt), _rnd(rng, (self.Tk, w), dt)
        self.d_o = _rnd(rng, (self.Tq, w), dt)
        self.bias = _rnd(rng, (buckets, heads), dt) if bias is None else bias
        self.bucket = ds.ds_rel_buckets(buckets, reach, not causal) if table is None else np.asarray(table)
        self.pos = [0] * len(ql) if pos is None else list(pos)
        self.pad = pad_cols
        ints = lambda a: torch.tensor(np.asarray(a, dtype=np.int32), device=DEV)  # noqa: E731
        self.tables = [ints(a) for a in (self.q_row, ql, self.k_row, kl)]
        self.q_pos = None if pos is None else ints(pos)
        self.tbias, self.tbucket = to_dev(self.bias, dt).contiguous(), ints(self.bucket)
        self.scratch = torch.full((int(ds.ds_rel_attention_scratch_bytes(heads, hd, len(self.bucket) // 2, self.Tq, self.Tk, len(ql))),), 255, dtype=torch.uint8, device=DEV)
        self.q_on, self.k_on = np.zeros(self.Tq, bool), np.zeros(self.Tk, bool)
        for r, l in zip(self.q_row, ql):
            self.q_on[r:r + l] = True
        for r, l in zip(self.k_row, kl):
            self.k_on[r:r + l] = True

    def place(self, a, on, fill):
        """A device tensor with `pad` more columns than it shows."""
        t = torch.full((a.shape[0], a.shape[1] + self.pad), fill, dtype=self.dt, device=DEV)
        b = a.copy()
        b[~on] = fill
        t[:, self.pad:] = to_dev(b, self.dt)
        return t[:, self.pad:]

    def tensors(self):
        self.tq, self.tk, self.tv = self.place(self.q, self.q_on, np.nan), self.place(self.k, self.k_on, np.nan), self.place(self.v, self.k_on, np.nan)
        self.tdo = self.place(self.d_o, self.q_on, np.nan)
        nine = lambda t: self.place(np.full(t.shape, 9.0), np.ones(t.shape[0], bool), 9.0)  # noqa: E731
        self.o, self.dq, self.dk, self.dv = nine(self.tq), nine(self.tq), nine(self.tk), nine(self.tv)
        self.lse = torch.full((self.heads, self.Tq), 9.0, device=DEV)
        self.dbias = torch.full(self.bias.shape, 5.0, device=DEV)
        return self

    def args(self):
        return (*self.tables, self.heads, self.hd, self.causal, max(max(self.ql), 1), max(max(self.kl), 1), self.scratch)

    def forward(self, generic=False, stream=None):
        ds.ds_rel_attention_fwd(self.tq, self.tk, self.tv, self.tbias, self.tbucket, self.o, self.lse, *self.args(), scale=self.scale, q_pos=self.q_pos, force_generic=generic, stream=stream)

    def backward(self, generic=False, accumulate=False, stream=None):
        ds.ds_rel_attention_bwd(self.tq, self.tk, self.tv, self.tbias, self.tbucket, self.o, self.tdo, self.lse, self.dq, self.dk, self.dv, self.dbias, *self.args(), scale=self.scale,
                                q_pos=self.q_pos, accumulate=accumulate, force_generic=generic, stream=stream)

    def check(self, generic, accumulate=False, back=True):
        half = 2.0 ** -8 if self.dt == BF else U
        core = self.dt == BF and not generic               # may have gone through bf16 products
        more = 2.0 ** -8 if core else 0.0
        o, lse = to_np(self.o), to_np(self.lse)
        dq, dk, dv = to_np(self.dq), to_np(self.dk), to_np(self.dv)
        for t, on in ((o, self.q_on), (lse.T, self.q_on)) + (((dq, self.q_on), (dk, self.k_on), (dv, self.k_on)) if back else ()):
            assert np.all(t[~on] == 9.0), "rows of no sequence"
        dbias, dbias_lim = np.zeros(self.bias.shape), np.zeros(self.bias.shape)
        biggest = np.abs(self.bias[np.isfinite(self.bias)]).max()

        def near(got, ref, lim, tag):
            assert np.all(np.isfinite(got)), tag
            dev = np.abs(got - ref)
            lim = lim + TINY
            assert np.all(dev <= lim), (tag, float((dev / lim).max()))

        for s, (qr, l, kr, n) in enumerate(zip(self.q_row, self.ql, self.k_row, self.kl)):
            qs, ks = slice(qr, qr + l), slice(kr, kr + n)
            q, k, v, d_o = self.q[qs], self.k[ks], self.v[ks], self.d_o[qs]
            ro, rl, size, terms = layer.rel_attention(q, k, v, self.bias, self.bucket, self.heads, self.causal, self.pos[s], self.scale)
            none = np.isneginf(rl)
            assert np.array_equal(np.isneginf(lse[:, qs]), none), "rows that see nothing"
            E = U * (128 * terms + 8 * (biggest + np.abs(np.where(none, 0.0, rl))) + 256)
            near(np.where(none, 0.0, lse[:, qs]), np.where(none, 0.0, rl), E, "lse")
            wide = lambda t: np.repeat(t.T, self.hd, axis=1)  # noqa: E731
            near(o[qs], ro, half * np.abs(ro) + (2 * wide(E) + more) * size, "o")
            assert np.all(o[qs][wide(none)] == 0)
            if not back:
                continue
            ref = layer.rel_attention_back(q, k, v, self.bias, self.bucket, to_np(self.o)[qs], d_o, self.heads, self.causal, self.pos[s], self.scale)
            Em = E.max(initial=0.0)
            rel = 2 * Em + 256 * U
            stat = 2.0 ** -16 * (2 + np.abs(np.where(none, 0.0, rl)).max(initial=0.0)) if core else 0.0
            near(dq[qs], ref["dq"], half * np.abs(ref["dq"]) + (rel + more) * ref["dq_part"], "dq")
            near(dk[ks], ref["dk"], half * np.abs(ref["dk"]) + (rel + more + stat) * ref["dk_part"], "dk")
            near(dv[ks], ref["dv"], half * np.abs(ref["dv"]) + (rel + more + stat) * ref["dv_part"], "dv")
            dbias += ref["dbias"]
            dbias_lim += (rel + 2048 * U) * ref["dbias_part"]
        if back:
            near(to_np(self.dbias), dbias + (5.0 if accumulate else 0.0), dbias_lim + 8 * U * (5.0 + np.abs(dbias)), "dbias")

    def run(self, generic, accumulate=False, back=True):
        self.tensors()
        self.forward(generic)
        if back:
            self.backward(generic, accumulate)
        torch.cuda.synchronize()
        self.check(generic, accumulate, back)


SHAPES = [  # heads, head size, query lengths, key lengths, causal
    (1, 64, [1], [1], True), (2, 64, [5, 64, 1], [5, 64, 1], True), (3, 64, [130, 0, 33], [130, 4, 33], True), (2, 64, [257, 200], [257, 200], False),
    (2, 128, [65, 300], [65, 300], True), (1, 128, [40, 1, 129], [300, 17, 64], False), (2, 64, [31], [0], False), (2, 64, [333, 100], [100, 333], False),
    (1, 128, [400], [400], True), (2, 128, [200, 64, 63], [222, 64, 65], False), (1, 64, [500], [500], False), (16, 64, [20, 31], [20, 31], True)]


@pytest.mark.parametrize("generic", [False, True])
@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)).replace(" ", ""))
def test_both_directions(shape, dt, generic):
    Case(11, dt, *shape).run(generic)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("hd", [8, 24, 32, 40, 72, 96, 120])
def test_other_head_sizes(hd, dt):
    Case(12, dt, 2, hd, [77, 130], [77, 130], True).run(False)
    Case(13, dt, 2, hd, [20, 70], [90, 140], False, pad_cols=1).run(False, accumulate=True)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("pad", [1, 4, 8])
def test_strides_and_alignment(pad, hd, dt):
    Case(14, dt, 2, hd, [100, 3], [100, 3], True, pad_cols=pad).run(False)


@pytest.mark.parametrize("generic", [False, True])
@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("reach,buckets", [(1, 3), (5, 11), (40, 16), (200, 32), (1024, 1024)])
def test_any_table(reach, buckets, hd, dt, generic):
    """Tables in no order, entries outside of the buckets (clamped), every reach."""
    rng = np.random.default_rng(reach)
    table = rng.integers(0, buckets, 2 * reach + 1)
    table[rng.integers(0, 2 * reach + 1)] = -7
    table[rng.integers(0, 2 * reach + 1)] = buckets + 100
    Case(15, dt, 2, hd, [150, 300], [290, 170], False, buckets=buckets, table=table).run(generic)
    Case(16, dt, 1, hd, [280], [280], True, buckets=buckets, table=table).run(generic, accumulate=True)


@pytest.mark.parametrize("generic", [False, True])
@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_positions(causal, hd, dt, generic):
    """Queries in the middle, at the end and far behind the end of their keys, and in front of them: rows that see nothing under a mask."""
    ql, kl = [70, 130, 5, 64, 200], [300, 130, 90, 100, 150]
    Case(17, dt, 2, hd, ql, kl, causal, pos=[100, -60, 85, 5000, -130]).run(generic)
    Case(18, dt, 1, hd, [3, 3, 4], [200, 7, 9], causal, pos=[2 ** 31 - 1, -2 ** 31, -2]).run(generic)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("ql,kl", [([1], [1]), ([1], [128]), ([1], [4100]), ([1, 1, 1], [129, 1, 1000]), ([1] * 16, list(range(100, 1700, 100))), ([2, 5, 1], [700, 300, 1]), ([8, 7], [513, 512]),
                                   ([33, 16], [900, 257]), ([64], [2000]), ([0, 1], [5, 0]), ([4, 3, 0, 2], [300, 3, 7, 65]), ([1], [0]), ([2], [5000])])
def test_tokens_on_a_cache(ql, kl, hd, dt):
    """The last tokens of sequences whose keys lie in a cache (shared out over work-groups where there are few)."""
    for heads in (1, 16):
        for causal in (True, False):
            Case(19, dt, heads, hd, ql, kl, causal, pos=[k - q for q, k in zip(ql, kl)]).run(False, back=heads == 1 and max(kl) < 1500)


@pytest.mark.parametrize("generic", [False, True])
@pytest.mark.parametrize("dt", [BF, F32])
def test_biases_that_hide(dt, generic):
    """Biases of -inf: buckets that nothing is seen through, up to whole rows; what they hide has no gradient."""
    rng = np.random.default_rng(3)
    bias = _rnd(rng, (4, 2), dt)
    bias[1, 0] = bias[2, 1] = -np.inf
    table = [0, 1, 1, 2, 2, 3, 1]                       # head 0 sees no key 1, 2 or 3 and more behind or in front, as the table says
    for causal in (False, True):
        c = Case(20, dt, 2, 64, [100, 70], [100, 160], causal, buckets=4, table=table, bias=bias)
        c.run(generic)
    low = torch.finfo(dt).min                           # the type's lowest value hides as well
    bias = _rnd(rng, (4, 2), dt)
    bias[2] = low
    c = Case(26, dt, 2, 64, [100], [130], False, buckets=4, table=table, bias=bias).tensors()
    c.bias = np.where(bias == low, -np.inf, bias)
    c.forward(generic)
    c.backward(generic)
    c.check(generic)
    bias = np.full((1, 1), -np.inf)
    c = Case(21, dt, 1, 64, [70], [90], False, buckets=1, table=[0, 0, 0], bias=np.where(np.isinf(bias), -np.inf, 0.0)).tensors()
    c.bias = bias
    c.forward(generic)
    c.backward(generic)
    on = torch.tensor(c.q_on, device=DEV)
    assert torch.all(torch.isneginf(c.lse[:, on])) and torch.all(c.o[on] == 0) and torch.all(c.dq[on] == 0)
    assert torch.all(c.dk[torch.tensor(c.k_on, device=DEV)] == 0) and torch.all(c.dv[torch.tensor(c.k_on, device=DEV)] == 0) and torch.all(c.dbias == 0)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("hd", [64, 128])
def test_scales(hd, dt):
    """No scaling (queries that bring their own), large and small ones; biases much larger than the scores."""
    rng = np.random.default_rng(4)
    for scale, size in ((1.0, 1.0), (0.001, 1.0), (0.1, 30.0)):
        Case(22, dt, 2, hd, [150, 33], [150, 33], True, scale=scale, bias=_rnd(rng, (32, 2), dt, size)).run(False)


@pytest.mark.parametrize("dt", [BF, F32])
def test_values_that_are_not_finite(dt):
    """General kernels: what a causal mask hides does not matter, whatever it is.  Wavefronts that share a tile of 64 keys with a row that is not finite sum theirs
    in another order: each order is off by at most 2 E (of a size of about 1) with E = U (128 terms + 256) and terms < 7 here, 2^-12 in fp32 for both; in bf16 two roundings of
    2^-8 besides."""
    for bad in (np.inf, np.nan):
        c = Case(23, dt, 2, 64, [150], [150], True)
        r = c.k_row[0]
        ref = Case(23, dt, 2, 64, [150], [150], True).tensors()
        ref.forward(True)
        c.k[r + 140, :] = bad
        c.v[r + 100, 3] = bad
        c.tensors()
        c.forward(True)
        q = c.q_row[0]
        half = 2.0 ** -6.9 if dt == BF else 2.0 ** -12
        assert torch.equal(c.o[q:q + 64], ref.o[q:q + 64]) and torch.equal(c.lse[:, q:q + 140], ref.lse[:, q:q + 140])
        assert torch.allclose(c.o[q + 64:q + 100].float(), ref.o[q + 64:q + 100].float(), rtol=half, atol=half)
        seen = c.o[q + 100:q + 150, 3]
        assert not torch.isfinite(seen).any()
        cols = [i for i in range(128) if i != 3]
        assert torch.allclose(c.o[q + 100:q + 140][:, cols].float(), ref.o[q + 100:q + 140][:, cols].float(), rtol=half, atol=half)
        # backward: a gradient and a query that are not finite, seen by the keys up to their own
        c = Case(23, dt, 2, 64, [150], [150], True)
        ref.backward(True)
        c.d_o[q + 60, 7] = bad
        c.tensors()
        c.forward(True)
        c.backward(True)
        k = c.k_row[0]
        assert torch.allclose(c.dv[k + 61:k + 150].float(), ref.dv[k + 61:k + 150].float(), rtol=half, atol=half * 8)
        assert torch.allclose(c.dk[k + 61:k + 150].float(), ref.dk[k + 61:k + 150].float(), rtol=half, atol=half * 8)
        assert not torch.isfinite(c.dv[k:k + 61, 7]).any()
        others = torch.tensor([i for i in range(150) if i != 60], device=DEV) + q
        assert torch.allclose(c.dq[others].float(), ref.dq[others].float(), rtol=half, atol=half * 8)
        assert not torch.isfinite(c.dbias[:, 0]).all()


@pytest.mark.parametrize("dt,hd", [(BF, 64), (BF, 128), (F32, 64)])
def test_same_bits_again_on_another_stream_and_in_a_graph(dt, hd):
    c = Case(24, dt, 4, hd, [300, 129, 7], [300, 129, 7], True).tensors()
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    names = ("o", "lse", "dq", "dk", "dv", "dbias")
    first = {n: getattr(c, n).clone() for n in names}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.forward()
        c.backward()
    side.synchronize()
    assert all(torch.equal(first[n], getattr(c, n)) for n in names)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.forward()
        c.backward()
    for _ in range(4):
        for n in names:
            getattr(c, n).fill_(3.0)
        c.scratch.fill_(255)
        g.replay()
        torch.cuda.synchronize()
        on = {"o": c.q_on, "dq": c.q_on, "dk": c.k_on, "dv": c.k_on}
        for n in names:
            rows = torch.tensor(on[n], device=DEV) if n in on else slice(None)
            if n == "lse":
                assert torch.equal(first[n][:, torch.tensor(c.q_on, device=DEV)], c.lse[:, torch.tensor(c.q_on, device=DEV)])
            else:
                assert torch.equal(first[n][rows], getattr(c, n)[rows]), n
        (c.o.float().sum() + 1).item()


def test_refused_tensors():
    c = Case(25, BF, 2, 64, [10], [10], True).tensors()
    with pytest.raises(ValueError):
        ds.ds_rel_attention_fwd(c.tq, c.tk, c.tv, c.tbias.float(), c.tbucket, c.o, c.lse, *c.args())
    with pytest.raises(ValueError):
        ds.ds_rel_attention_fwd(c.tq, c.tk, c.tv, c.tbias, c.tbucket[:-1], c.o, c.lse, *c.args())
    with pytest.raises(ValueError):
        ds.ds_rel_attention_fwd(c.tq, c.tk, c.tv, c.tbias[:, :1], c.tbucket, c.o, c.lse, *c.args())
    with pytest.raises(ValueError):
        ds.ds_rel_attention_fwd(c.tq.cpu(), c.tk, c.tv, c.tbias, c.tbucket, c.o, c.lse, *c.args())
    with pytest.raises(ValueError):
        ds.ds_rel_attention_bwd(c.tq, c.tk, c.tv, c.tbias, c.tbucket, c.o, c.tdo, c.lse, c.dq, c.dk, c.dv, c.dbias.to(BF), *c.args())
    with pytest.raises(ds.DsError):
        ds.ds_rel_attention_fwd(c.tq, c.tk, c.tv, c.tbias, c.tbucket, c.o, c.lse, *c.args()[:-1], c.scratch[:1000])
