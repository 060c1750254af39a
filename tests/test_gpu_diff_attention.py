"""ds_diff_attention_fwd / ds_diff_attention_bwd against oracle/layer.py, one sequence at a time.

Tolerances, elementwise, in the terms of the formulas (`size`: the result with every product counted by its absolute value).  Roundings count half a
step: 2^-8 in bf16.
  scores in fp32: a sum of hd / 2 <= 64 products is off by at most 64 x 2^-24 x its terms (`terms`, times the scale), which is the relative error of a
  probability; with the exponential, its argument and the sum of up to 2 048 of them (in lanes and tiles) E = 2^-24 (64 terms + 128).
  general kernels: o: 2 E size; gradients: dP and D are sums of hd <= 128 products more, 2 E + 256 x 2^-24 of `part` (what dS is a difference of).
  matrix-core kernels (bf16): the probabilities, their difference, and dS are rounded to bf16 before they are multiplied: 2^-8 size more; log-sum-exp and D reach
  the dK / dV kernel as two bf16 values, 2^-16 of their size: 2^-16 x (1 + |lse|) of `part`.
  What is below 2^-126 counts as 0 in fp32, at worst in every factor of a term: with |G - D| <= 2^9, |q|, |k|, |dO| <= 2^5 and at most 2^9 rows a sum loses
  less than 2^-126 x 2^9 x 2^5 x 2^9 = 2^-103 (TINY) by it.
  Each result is rounded once to its type.  dlambda is fp32 in every kernel."""
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

    def __init__(self, seed, dt, heads, hd, ql, kl, causal, pad_cols=0, scale=1.0, gap=3):
        rng = np.random.default_rng(seed)
        self.dt, self.heads, self.hd, self.causal, self.ql, self.kl = dt, heads, hd, causal, ql, kl
        w = heads * hd
        rows = lambda ls: (np.cumsum([2] + [l + gap for l in ls[:-1]]), 2 + sum(ls) + gap * len(ls))  # noqa: E731
        (self.q_row, self.Tq), (self.k_row, self.Tk) = rows(ql), rows(kl)
        self.q = _rnd(rng, (self.Tq, w), dt, scale)
        self.k, self.v = _rnd(rng, (self.Tk, w), dt, scale), _rnd(rng, (self.Tk, w), dt)
        self.d_o = _rnd(rng, (self.Tq, w), dt)
        self.lam = rng.uniform(-0.2, 0.9, heads).astype(np.float32).astype(np.float64)
        self.pad = pad_cols
        table = lambda a: torch.tensor(np.asarray(a, dtype=np.int32), device=DEV)  # noqa: E731
        self.tables = [table(a) for a in (self.q_row, ql, self.k_row, kl)]
        self.dlam_in = to_dev(self.lam, F32)
        self.scratch = torch.full((int(ds.ds_diff_attention_scratch_bytes(heads, self.Tq, self.Tk, len(ql))),), 255, dtype=torch.uint8, device=DEV)
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
        self.o, self.o2, self.dq, self.dk, self.dv = nine(self.tq), nine(self.tq), nine(self.tq), nine(self.tk), nine(self.tv)
        self.lse = torch.full((2 * self.heads, self.Tq), 9.0, device=DEV)
        self.dlam = torch.full((self.heads,), 5.0, device=DEV)

    def args(self):
        return (*self.tables, self.heads, self.hd, self.causal, max(max(self.ql), 1), max(max(self.kl), 1), self.scratch)

    def forward(self, generic=False, keep=True, stream=None):
        ds.ds_diff_attention_fwd(self.tq, self.tk, self.tv, self.dlam_in, self.o, self.lse, *self.args(), o2=self.o2 if keep else None, force_generic=generic, stream=stream)

    def backward(self, generic=False, accumulate=False, stream=None):
        ds.ds_diff_attention_bwd(self.tq, self.tk, self.tv, self.dlam_in, self.o, self.o2, self.tdo, self.lse, self.dq, self.dk, self.dv, self.dlam, *self.args(),
                                 accumulate=accumulate, force_generic=generic, stream=stream)

    def check(self, generic, accumulate=False):
        half = 2.0 ** -8 if self.dt == BF else 2.0 ** -24
        core = self.dt == BF and not generic               # may have gone through bf16 products
        o, o2, lse = to_np(self.o), to_np(self.o2), to_np(self.lse)
        dq, dk, dv = to_np(self.dq), to_np(self.dk), to_np(self.dv)
        for t, on in ((o, self.q_on), (o2, self.q_on), (dq, self.q_on), (dk, self.k_on), (dv, self.k_on), (lse.T, self.q_on)):
            assert np.all(t[~on] == 9.0), "rows of no sequence"
        dlam, dlam_size = np.zeros(self.heads), np.zeros(self.heads)

        def near(got, ref, lim, tag):
            assert np.all(np.isfinite(got)), tag
            dev = np.abs(got - ref)
            lim = lim + TINY
            assert np.all(dev <= lim), (tag, float((dev / lim).max()))

        for s, (qr, l, kr, n) in enumerate(zip(self.q_row, self.ql, self.k_row, self.kl)):
            qs, ks = slice(qr, qr + l), slice(kr, kr + n)
            if n == 0 or l == 0:
                assert np.all(o[qs] == 0) and np.all(o2[qs] == 0) and np.all(dq[qs] == 0) and np.all(dk[ks] == 0) and np.all(dv[ks] == 0)
                continue
            q, k, v, d_o = self.q[qs], self.k[ks], self.v[ks], self.d_o[qs]
            ro, ro2, rl, size, size2, terms = layer.diff_attention(q, k, v, self.lam, self.heads, self.causal)
            E = U * (64 * terms + 128)
            more = 2.0 ** -8 if core else 0.0
            near(lse[:, qs], rl, E + 8 * U * np.abs(rl), "lse")
            near(o2[qs], ro2, half * np.abs(ro2) + (2 * E + more) * size2, "o2")
            near(o[qs], ro, half * np.abs(ro) + (2 * E + more) * size, "o")
            g = layer.diff_attention_back(q, k, v, self.lam, o[qs], o2[qs], d_o, lse[:, qs], self.heads, self.causal)
            F = 2 * E + 256 * U
            near(dq[qs], g["dq"], half * np.abs(g["dq"]) + more * g["size_dq"] + F * g["part_dq"], "dq")
            if core:
                F += 2.0 ** -16 * (1 + np.abs(rl).max())
            near(dk[ks], g["dk"], half * np.abs(g["dk"]) + more * g["size_dk"] + F * g["part_dk"], "dk")
            near(dv[ks], g["dv"], half * np.abs(g["dv"]) + more * g["size_dv"] + F * g["part_dv"], "dv")
            dlam += g["dlam"]
            dlam_size += (2 * E + 256 * U) * g["size_dlam"]
        near(to_np(self.dlam), dlam + (5.0 if accumulate else 0.0), dlam_size + 8 * U * (5 + np.abs(dlam)), "dlam")

    def run(self, generic, accumulate=False):
        self.tensors()
        self.forward(generic)
        self.backward(generic, accumulate)
        torch.cuda.synchronize()
        self.check(generic, accumulate)


LENGTHS = [[1], [5, 64, 1, 17], [130, 63, 129], [300]]
KINDS = [(F32, False), (BF, True), (BF, False)]


@pytest.mark.parametrize("dt,generic", KINDS)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("hd", [16, 32, 48, 64, 80, 96, 128])
def test_own_sequences(dt, generic, causal, hd):
    for i, lens in enumerate(LENGTHS):
        Case(hd + i, dt, 3 if i % 2 else 8, hd, lens, lens, causal).run(generic, accumulate=i % 2 == 1)


@pytest.mark.parametrize("dt,generic", KINDS)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("hd", [64, 112, 128])
def test_other_sequences_and_none(dt, generic, causal, hd):
    """Queries and keys of different lengths, sequences without queries or without keys, single queries over many keys and many over one."""
    Case(hd, dt, 2, hd, [1, 40, 0, 7, 200, 3, 65], [257, 1, 9, 0, 33, 400, 64], causal).run(generic, accumulate=True)


@pytest.mark.parametrize("dt,generic", KINDS)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("hd", [64, 128])
def test_short_queries(dt, generic, causal, hd):
    """At most 32 or 64 queries (a work-group then shares the keys out): fewer steps of 32 keys than wavefronts, many, one key, no query or none."""
    for q in ([1, 32, 0, 17, 5, 31, 9], [64, 33, 0, 1, 40, 64, 63]):
        Case(hd + q[0], dt, 2, hd, q, [700, 1, 40, 0, 97, 64, 129], causal).run(generic)
        Case(hd + q[0], dt, 8, hd, q[:1], [33], causal).run(generic)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("hd", [64, 128])
def test_very_short_sequences(causal, hd):
    """At most 16 tokens: bf16 calls that need not round what they multiply, few or many of them."""
    Case(hd, BF, 2, hd, [16, 1, 9, 0, 12], [16, 3, 9, 5, 0], causal).run(False)
    Case(hd + 1, BF, 16, hd, [16, 7] * 9, [16, 7] * 9, causal).run(False, accumulate=True)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("hd", [64, 128])
def test_sequences_of_one_block(causal, hd):
    """At most 128 tokens on either side, which need no work list: without queries, without keys, of different lengths; few and many of them."""
    Case(hd, BF, 2, hd, [100, 1, 0, 64, 128, 20], [120, 0, 33, 1, 128, 90], causal).run(False)
    Case(hd + 1, BF, 1, hd, [0, 33, 0], [40, 0, 7], causal).run(False)
    Case(hd + 2, BF, 8, hd, [40, 0, 17, 128] * 10, [33, 5, 0, 100] * 10, causal).run(False, accumulate=True)


@pytest.mark.parametrize("dt,generic", KINDS)
@pytest.mark.parametrize("hd", [16, 64, 96, 128])
def test_few_queries_over_long_keys(dt, generic, hd):
    """Single tokens and short runs over keys that several work-groups share: shares that end inside a tile, sequences with fewer keys than shares or none."""
    Case(hd, dt, 4, hd, [1], [5000], False).run(generic)
    Case(hd + 1, dt, 2, hd, [1, 1, 0, 1, 1, 1], [2049, 1, 700, 0, 64, 1300], False).run(generic)
    Case(hd + 2, dt, 3, hd, [64, 33, 2], [900, 513, 3], False, pad_cols=8).run(generic)
    Case(hd + 3, dt, 1, hd, [17], [1900], False, scale=6.0).run(generic)


@pytest.mark.parametrize("dt,generic", KINDS)
def test_single_tokens_in_a_graph(dt, generic):
    c = Case(8, dt, 4, 128, [1, 1, 1], [1500, 33, 700], False)
    c.tensors()
    c.forward(generic, keep=False)
    torch.cuda.synchronize()
    want = [c.o.clone(), c.lse.clone()]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.forward(generic, keep=False)
    for _ in range(3):
        c.o[:] = 9.0
        c.lse.fill_(9.0)
        c.scratch.fill_(200)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.o, want[0]) and torch.equal(c.lse, want[1])


@pytest.mark.parametrize("dt,generic", KINDS)
@pytest.mark.parametrize("hd,pad", [(64, 8), (64, 4), (64, 1), (128, 3), (128, 64), (16, 2)])
def test_columns_of_wider_tensors(dt, generic, hd, pad):
    """Row strides and first columns that allow accesses of 16, 8, or only 2 or 4 bytes."""
    Case(pad, dt, 2, hd, [70, 9], [70, 9], True, pad_cols=pad).run(generic)


@pytest.mark.parametrize("dt,generic", KINDS)
def test_many_sequences(dt, generic):
    rng = np.random.default_rng(1)
    lens = [int(x) for x in rng.integers(1, 40, 150)]
    Case(2, dt, 2, 64, lens, lens, True).run(generic)


@pytest.mark.parametrize("dt,generic", KINDS)
@pytest.mark.parametrize("causal", [False, True])
def test_scores_far_apart(dt, generic, causal):
    """Scores in the hundreds: a row's probability on one key, maxima that move from tile to tile."""
    Case(3, dt, 2, 64, [200], [200], causal, scale=6.0).run(generic)


@pytest.mark.parametrize("dt,generic", KINDS)
def test_without_second_output_and_the_same_again(dt, generic):
    c = Case(4, dt, 4, 128, [150, 33, 260], [150, 33, 260], True)
    c.tensors()
    c.forward(generic)
    c.backward(generic)
    first = [t.clone() for t in (c.o, c.lse, c.dq, c.dk, c.dv, c.dlam)]
    c.o.fill_(9.0)
    c.lse.fill_(9.0)
    c.scratch.fill_(77)
    c.forward(generic, keep=False)
    c.backward(generic)
    torch.cuda.synchronize()
    for a, b in zip(first, (c.o, c.lse, c.dq, c.dk, c.dv, c.dlam)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dt,generic", KINDS)
def test_in_a_graph(dt, generic):
    c = Case(5, dt, 2, 64, [90, 128, 5], [90, 128, 5], True)
    c.run(generic)
    outs = (c.o, c.o2, c.lse, c.dq, c.dk, c.dv, c.dlam)
    want = [t.clone() for t in outs]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        c.forward(generic)
        c.backward(generic)
    for _ in range(3):
        for t in outs:
            t[:] = 9.0
        c.scratch.fill_(200)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, outs):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dt,generic", KINDS)
def test_gradients_against_differences(dt, generic):
    """A step along a direction, in 64 bits, against the products of the gradients with it.  What bounds the gradients' own error (see above) bounds
    the product's; the differences add e^2 and rounding / e."""
    c = Case(6, dt, 2, 64, [37], [37], True)
    c.run(generic)
    rng = np.random.default_rng(9)
    qs = slice(int(c.q_row[0]), int(c.q_row[0]) + 37)
    at = {"q": c.q[qs], "k": c.k[qs], "v": c.v[qs], "lam": c.lam}
    got = {"q": to_np(c.dq)[qs], "k": to_np(c.dk)[qs], "v": to_np(c.dv)[qs], "lam": to_np(c.dlam)}
    loss = lambda a: (layer.diff_attention(a["q"], a["k"], a["v"], a["lam"], 2, True)[0] * c.d_o[qs]).sum()  # noqa: E731
    o, o2, lse, _, _, terms = layer.diff_attention(at["q"], at["k"], at["v"], at["lam"], 2, True)
    g = layer.diff_attention_back(at["q"], at["k"], at["v"], at["lam"], o, o2, c.d_o[qs], lse, 2, True)
    E = U * (64 * terms + 128)
    half = 2.0 ** -8 if dt == BF else 2.0 ** -24
    for k in at:
        v = rng.standard_normal(at[k].shape)
        slope = (loss(dict(at, **{k: at[k] + 1e-6 * v})) - loss(dict(at, **{k: at[k] - 1e-6 * v}))) / 2e-6
        if k == "lam":
            lim = (2 * E + 256 * U) * (g["size_dlam"] * np.abs(v)).sum()
        else:
            # outputs, o and o2 in D (part holds |dO| |O|), probabilities and dS rounded; all signs alike
            lim = ((3 * half + 2 * E + 256 * U + 2.0 ** -12 * (dt == BF)) * g["part_d" + k] * np.abs(v)).sum()
        assert abs(slope - (got[k] * v).sum()) <= lim + 1e-6 * (1 + abs(slope)), k


def test_tensors_that_do_not_fit_are_refused():
    c = Case(7, BF, 2, 64, [9], [9], True)
    c.tensors()
    with pytest.raises(ValueError):
        ds.ds_diff_attention_fwd(c.tq, c.tk, c.tv.float(), c.dlam_in, c.o, c.lse, *c.args())
    with pytest.raises(ValueError):
        ds.ds_diff_attention_fwd(c.tq, c.tk, c.tv, c.dlam_in, c.o, c.lse[:2], *c.args())
    with pytest.raises(ValueError):
        ds.ds_diff_attention_fwd(c.tq, c.tk, c.tv, c.dlam_in, c.o, c.lse, *c.args()[:-1], c.scratch[:64])
    with pytest.raises(ValueError):
        ds.ds_diff_attention_fwd(c.tq, c.tk[:, :64], c.tv, c.dlam_in, c.o, c.lse, *c.args())
    with pytest.raises(ValueError):
        ds.ds_diff_attention_fwd(c.tq, c.tk, c.tv, c.dlam_in, c.o, c.lse, *c.args(), o2=torch.zeros((c.Tq, 200), dtype=BF, device=DEV))
