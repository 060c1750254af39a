"""The gated feed-forward block's gradients for tensors beyond 2^31 elements and for more rows than a grid of 64 has.  All rows but the last 700 are zeros, so that the oracle stays small; tolerances
as in test_gpu_gated_mlp.py (zeros add nothing to a sum: 700 products, and one addition for each of at most 128 shares)."""
import numpy as np
import pytest
import torch

from oracle import layer
from paper_2311_10418_amd import binding as ds
from helpers import DEV, to_np
from test_gpu_gated_mlp import BF, F32, U

pytestmark = pytest.mark.gpu

LAST = 700


def _far(g, rows, cols, dt, scale=1.0):
    t = torch.zeros((rows, cols), dtype=dt, device=DEV)
    t[-LAST:] = (torch.randn((LAST, cols), generator=g, device=DEV) * scale).to(dt)
    return t


@pytest.mark.parametrize("dt,rows,d,ff", [(F32, (1 << 31) // 1024 + 300, 256, 1024), (F32, 65535 * 64 + 70, 64, 64), (BF, (1 << 31) // 1032 + 300, 200, 1032)])
def test_backward(dt, rows, d, ff):
    """dG, dU in place of G and U, and dx.  The second case has more rows than the fp32 kernel of bf16 parts takes."""
    if dt == F32:
        assert ds.lib().ds_gated_mlp_f32_columns(rows, d, ff) == (128 if d == 256 else -1)
    gen = torch.Generator(device=DEV).manual_seed(3)
    g, dh = _far(gen, rows, ff, dt), _far(gen, rows, ff, dt)
    u = torch.ones_like(g)
    w = [(torch.randn((d, ff), generator=gen, device=DEV) * d ** -0.5).to(dt) for _ in range(2)]
    dx = torch.empty((rows, d), dtype=dt, device=DEV)
    ga, da = to_np(g[-LAST:]), to_np(dh[-LAST:])
    ds.ds_gated_mlp_bwd(dh, g, u, *w, g, u, dx, act=ds.DS_ACT_SILU, workspace=torch.empty(1 << 24, device=DEV))
    half = 2.0 ** -8 if dt == BF else U
    for got, want in zip((g, u), layer.gated_mlp_back(da, ga, np.ones_like(ga), "silu")):
        assert np.all(np.abs(to_np(got[-LAST:]) - want) <= half * np.abs(want) + 2.0 ** -17 * (1 + np.abs(ga)) * np.abs(da)) and not got[:-LAST].any()
    dg, du, wg, wu = to_np(g[-LAST:]), to_np(u[-LAST:]), to_np(w[0]).T, to_np(w[1]).T
    ref, size = dg @ wg + du @ wu, np.abs(dg) @ np.abs(wg) + np.abs(du) @ np.abs(wu)
    assert np.all(np.abs(to_np(dx[-LAST:]) - ref) <= half * np.abs(ref) + 2 * ff * U * size) and not dx[:-LAST].any()


@pytest.mark.parametrize("dt,rows,d,ff", [(BF, (1 << 31) // 1024 + 300, 256, 1024), (F32, (1 << 31) // 1024 + 300, 256, 1024), (BF, (1 << 31) // 1032 + 300, 200, 1032)])
def test_gradients_of_the_parameters(dt, rows, d, ff):
    gen = torch.Generator(device=DEV).manual_seed(4)
    x, dg, du = (_far(gen, rows, c, dt) for c in (d, ff, ff))
    out = [torch.full(s, 3.0, device=DEV) for s in ((d, ff), (d, ff), (ff,), (ff,))]
    ds.ds_gated_mlp_wgrad(x, dg, du, *out, workspace=torch.full((1 << 24,), float("nan"), device=DEV))
    xa = to_np(x[-LAST:])
    for dw, db, dy in ((out[0], out[2], to_np(dg[-LAST:])), (out[1], out[3], to_np(du[-LAST:]))):
        assert np.all(np.abs(to_np(dw) - xa.T @ dy) <= (LAST + 130) * U * (np.abs(xa).T @ np.abs(dy)))
        assert np.all(np.abs(to_np(db) - dy.sum(axis=0)) <= (LAST + 130) * U * np.abs(dy).sum(axis=0))
