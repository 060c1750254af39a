"""The gated block's dx in fp32 as bf16 parts of each value: tiles 64 and 128 columns wide, whose loop runs through (dG, Wg) and then through (dU, Wu), the repetition of a tile with fp32
products, and the two products that few tiles are made of instead.  Inputs and tolerances as in test_gpu_gated_mlp.py.  Every case states which of them it takes (ds_gated_mlp_f32_columns)."""
import numpy as np
import pytest
import torch

from oracle import layer
from paper_2311_10418_amd import binding as ds
from helpers import DEV, to_dev, to_np
from test_gpu_gated_mlp import ACT, F32, U, Block, _near, _rnd

pytestmark = pytest.mark.gpu


def columns(rows, d, ff):
    return ds.lib().ds_gated_mlp_f32_columns(rows, d, ff)


# rows, d, d_ff (multiples of the K tile of 32 and not, shorter than one, of one and of two); columns of a tile
SHAPES = [((3700, 256, 512), 64), ((3521, 264, 520), 64), ((2200, 448, 136), 64), ((3521, 1024, 40), 64), ((14337, 64, 8), 64), ((7684, 256, 1024), 64), ((8200, 512, 520), 128), ((8205, 512, 72), 128),
          ((5500, 744, 96), 128), ((32768, 128, 32), 128), ((957, 256, 1024), 0), ((128, 1024, 264), 0)]


@pytest.mark.parametrize("shape,want", SHAPES, ids=lambda s: "x".join(map(str, s)) if isinstance(s, tuple) else str(s))
def test_both_pairs_of_operands(shape, want):
    """Rows that do not count hold NaN in x and dh; ragged last tiles of rows and columns."""
    assert columns(*shape) == want
    for act, floats in (("silu", 1 << 24), ("gelu", 0)):
        b = Block(F32, *shape, act, pad=0.1 if act == "silu" else 0.0, floats=floats)
        b.run()


@pytest.mark.parametrize("shape,want", [((3700, 256, 72), 64), ((8205, 512, 40), 128), ((200, 256, 72), 0)], ids=lambda s: "x".join(map(str, s)) if isinstance(s, tuple) else str(s))
def test_tiles_that_are_repeated(shape, want):
    """Values whose three bf16 parts do not hold all their bits (of 2^-122: the third part would lie below every bf16 value), and an infinity: their tiles are taken again with fp32
    products, over both pairs of operands.  Weights of 2^60 bring small gradients back to where each bit counts: without their last parts they would be off by 2^-9 of their size, where
    2 d_ff U allows 2^-17."""
    assert columns(*shape) == want
    rows, d, ff = shape
    rng = np.random.default_rng(rows)
    one = lambda s: (1 + rng.random(s)).astype(np.float32).astype(np.float64)  # noqa: E731
    g, u = one((rows, ff)), one((rows, ff)) * rng.choice([-1.0, 1.0], (rows, ff))
    dh = _rnd(rng, (rows, ff), F32)
    small = np.zeros(rows, bool)
    small[[0, 70, 131, rows - 1]] = True
    dh[small] = one((small.sum(), ff)) * 2.0 ** -122
    w = [_rnd(rng, (d, ff), F32) * 2.0 ** 60 for _ in range(2)]
    for bad in (None, np.inf):
        if bad:
            dh[133, 5] = bad
        t = [to_dev(a, F32) for a in (dh, g, u, *w)]
        dg, du = torch.empty_like(t[0]), torch.empty_like(t[0])
        dx = torch.full((rows + 1, d), 9.0, device=DEV)
        ds.ds_gated_mlp_bwd(*t, dg, du, dx[:rows], act=ACT["relu"], workspace=torch.full((1 << 22,), float("nan"), device=DEV))
        torch.cuda.synchronize()
        got_dg, got_du, got = to_np(dg), to_np(du), to_np(dx)
        assert np.all(got[rows] == 9.0)
        on = np.ones(rows, bool)
        on[133] = bad is None
        rg, ru = layer.gated_mlp_back(dh[on], g[on], u[on], "relu")
        _near(got_dg[on], rg, 3 * U * np.abs(rg), "dg")
        _near(got_du[on], ru, 3 * U * np.abs(ru), "du")
        ref = got_dg[on] @ w[0].T + got_du[on] @ w[1].T
        size = np.abs(got_dg[on]) @ np.abs(w[0].T) + np.abs(got_du[on]) @ np.abs(w[1].T)
        assert np.abs(ref[small[on]]).max() < 2.0 ** -50
        _near(got[:rows][on], ref, U * np.abs(ref) + 2 * ff * U * size, "dx")
        assert bad is None or not np.isfinite(got[133]).any()
