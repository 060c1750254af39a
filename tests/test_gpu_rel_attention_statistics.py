"""How exactly log-sum-exps reach the gradients of keys and values in the bf16 matrix-core kernels of attention with a relative position bias, with many queries to a key.

All scores are their bias, 4224 (queries of 2^-40): every query of n = 300 keys has the same log-sum-exp L = 4224 + ln 300 and probabilities of 1 / 300, and with gradients dO > 0 all terms of
dV (and, as v_j is a_j in all features, of dK) have one sign, so that nothing averages an error of L out.  L / scale = 8 L as two bf16 values would be off by 0.12, a probability by 1.5 %.

What the kernels may be off by, relative to a probability (U = 2^-24): the maximum is the bias's own entry of the table in both passes, so that its rounding is none of a difference; the
log-sum-exp is the sum of it and a logarithm (U), times ln 2 (U and U of the constant), 8 L is exact, and times scale log2 e (U of the constant) it is subtracted in one rounding: 5 U L, and 256 U for the
exponentials and their sum: E.  P is rounded to bf16 (2^-8), dS as well (2^-8 of dS); dP and D are sums of hd <= 128 products (128 U of their sizes).  Results are rounded once (2^-8)."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2311_10418_amd import binding
from paper_2311_10418_amd import workload as wl
from helpers import to_np
from test_gpu_rel_attention import BF, TINY, U, Case

pytestmark = pytest.mark.gpu

N, BIAS, SCALE = 300, 4224.0, 0.125


def _bf16(x):
    return float(wl.to_bf16_grid(np.array([x], np.float32))[0])


def test_what_two_parts_would_do():
    v = float(np.float32((BIAS + np.log(N)) / SCALE))
    two = _bf16(v) + _bf16(v - _bf16(v))
    assert SCALE * abs(two - v) > 0.014 and _bf16(BIAS) == BIAS


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("ql,listed,shared", [([160, 200, 133], False, False), ([900], False, True), ([5] * 40 + [700], True, False), ([1], False, False)], ids=["no_list", "shared", "list", "one"])
def test_gradients_of_keys_and_values(ql, listed, shared, hd):
    heads, n = 2, len(ql)
    rng = np.random.default_rng(hd)
    c = Case(51, BF, heads, hd, ql, [N] * n, False, buckets=1, table=[0, 0, 0], bias=np.full((1, heads), BIAS), scale=SCALE)
    grid = lambda a: wl.to_bf16_grid(a.astype(np.float32)).astype(np.float64)  # noqa: E731
    c.q, c.d_o = grid(1 + rng.random(c.q.shape)) * 2.0 ** -40, grid(1 + rng.random(c.d_o.shape))
    c.v = np.repeat(grid((1 + rng.random((c.Tk, heads))) * rng.choice([-1.0, 1.0], (c.Tk, heads))), hd, axis=1)
    out = (ctypes.c_int32 * 8)()
    binding.lib().ds_rel_attention_choice(1, n, heads, hd, max(ql), N, c.Tq, c.Tk, 1, 0, out)
    assert out[0] == 0 and (out[2] == 0) == listed and (out[7] > 1) == shared
    c.tensors()
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    o, dk, dv = to_np(c.o), to_np(c.dk), to_np(c.dv)
    E = (5 * (BIAS + np.log(N)) + 256) * U
    for s in range(n):
        qs, ks = slice(c.q_row[s], c.q_row[s] + ql[s]), slice(c.k_row[s], c.k_row[s] + N)
        for h in range(heads):
            f = slice(h * hd, (h + 1) * hd)
            d_o, v, q, p = c.d_o[qs, f], c.v[ks, f], c.q[qs, f], 1.0 / N
            d = (d_o * o[qs, f]).sum(axis=1, keepdims=True)
            ds = p * (d_o @ v.T - d)
            ref = p * np.broadcast_to(d_o.sum(axis=0), (N, hd))
            assert np.all(np.abs(dv[ks, f] - ref) <= (2.0 ** -8 + 2.0 ** -8 + E + 512 * U) * ref)
            terms = p * (np.abs(d_o) @ np.abs(v).T + np.abs(d_o * o[qs, f]).sum(axis=1, keepdims=True))
            ref = SCALE * ds.T @ q
            lim = 2.0 ** -8 * np.abs(ref) + SCALE * ((2.0 ** -8 + E + 512 * U) * np.abs(ds) + 128 * U * terms).T @ q
            assert np.all(np.abs(dk[ks, f] - ref) <= lim + TINY)
