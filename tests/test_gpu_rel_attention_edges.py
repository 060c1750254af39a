"""Attention with a relative position bias at scales near the ends of their range.  Tolerances as in test_gpu_rel_attention.py."""
import numpy as np
import pytest
import torch

from paper_2311_10418_amd import workload as wl
from helpers import to_np
from test_gpu_rel_attention import Case

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def _signed(rng, shape, dt, power):
    """Values between 2^power and 2^(power + 1) of either sign, so that none of them is subnormal."""
    a = ((1 + rng.random(shape)) * rng.choice([-1.0, 1.0], shape)).astype(np.float32)
    return (wl.to_bf16_grid(a) if dt == BF else a).astype(np.float64) * 2.0 ** power


@pytest.mark.parametrize("generic", [False, True])
@pytest.mark.parametrize("dt,hd", [(F32, 64), (F32, 32), (F32, 128), (BF, 96), (BF, 64)])
def test_queries_times_scale_beyond_the_largest_float(dt, hd, generic):
    """Single tokens on a cache (one of them with its keys shared out): scale * q overflows, scale * (q . k) does not."""
    rng = np.random.default_rng(hd)
    for kl in ([40, 300], [5000]):
        c = Case(41, dt, 2, hd, [1] * len(kl), kl, True, pos=[k - 1 for k in kl], scale=2.0 ** 110)
        c.q, c.k = _signed(rng, c.q.shape, dt, 17), _signed(rng, c.k.shape, dt, -124)
        assert np.abs(c.q).max() * c.scale * 1.4426 > 3.5e38
        c.run(generic, back=False)


@pytest.mark.parametrize("generic", [False, True])
@pytest.mark.parametrize("dt,hd", [(F32, 64), (BF, 64), (BF, 128), (F32, 40)])
def test_largest_scale(dt, hd, generic):
    """2.3e38, with queries of 0: every score is its bias."""
    for ql, kl in (([1, 1], [40, 300]), ([70, 3], [90, 200])):
        c = Case(42, dt, 2, hd, ql, kl, False, scale=2.3e38)
        c.q[:] = 0
        c.tensors()
        c.forward(generic)
        torch.cuda.synchronize()
        c.scale = 1.0                                   # (for the check: 0 times anything)
        c.check(generic, back=False)
        assert np.isfinite(to_np(c.lse)).all()
