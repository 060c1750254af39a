"""Attention with a relative position bias at scales near the ends of their range, and how far values that are not finite reach.  Tolerances as in test_gpu_rel_attention.py."""
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


# queries at any position see blocks of 64 (32) keys that begin at a multiple of 64 (32): where positions are not a multiple of 32 a block that the last of 32 queries sees
# lies 31 tokens further in front of the first of them
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
@pytest.mark.parametrize("pos", [0, 64, 1, 45, 31])
@pytest.mark.parametrize("length", [300, 1100])
@pytest.mark.parametrize("hd", [64, 128])
def test_how_far_hidden_values_that_are_not_finite_reach(hd, length, pos, bad):
    """bf16 matrix-core kernels under a causal mask: rows further off than the header says keep their bits, in o, dq, dk and dv."""
    front, back = (63, 31) if pos % 32 == 0 else (94, 62)
    ref = Case(43, BF, 2, hd, [length], [length + pos], True, pos=[pos] if pos else None).tensors()
    ref.forward()
    ref.backward()
    q0, k0 = ref.q_row[0], ref.k_row[0]
    at = torch.arange(length, device="cuda") + pos          # positions of the queries
    keys = torch.arange(length + pos, device="cuda")
    farthest = {"o": 0, "dq": 0, "dk": 0, "dv": 0}

    def differ(name, got, want, off):
        """The largest distance of a row that differs; off: distance of each row, positive where the value is hidden from it."""
        rows = (got != want).any(dim=1) & (off > 0)
        far = int(off[rows].max()) if bool(rows.any()) else 0
        farthest[name] = max(farthest[name], far)

    for t in sorted({127, 128, 159, 191, 200, 223, 255, length + pos - 1, length // 2 + pos}):
        c = Case(43, BF, 2, hd, [length], [length + pos], True, pos=[pos] if pos else None)
        c.k[k0 + t] = c.v[k0 + t] = bad
        c.tensors()
        c.forward()
        differ("o", c.o[q0:q0 + length], ref.o[q0:q0 + length], t - at)
        c.o, c.lse = ref.o, ref.lse
        c.backward()
        differ("dq", c.dq[q0:q0 + length], ref.dq[q0:q0 + length], t - at)
        i = min(t, length - 1)
        c = Case(43, BF, 2, hd, [length], [length + pos], True, pos=[pos] if pos else None)
        c.q[q0 + i] = c.d_o[q0 + i] = bad
        c.tensors()
        c.o, c.lse = ref.o, ref.lse
        c.backward()
        for n in ("dk", "dv"):
            differ(n, getattr(c, n)[k0:k0 + length + pos], getattr(ref, n)[k0:k0 + length + pos], keys - (pos + i))
    assert farthest["o"] <= front and max(farthest["dq"], farthest["dk"], farthest["dv"]) <= back


@pytest.mark.parametrize("dt,hd,generic", [(BF, 64, False), (BF, 128, False), (BF, 64, True), (F32, 64, False), (F32, 32, False)])
def test_row_strides_that_put_tensors_beyond_2_31_elements(dt, hd, generic):
    """Column ranges of tensors with 2^20 columns more: the last of 2 100 rows begin behind 2^31 elements."""
    c = Case(44, dt, 2, hd, [1200, 900], [1000, 1200], False, pad_cols=1 << 20)
    assert min(c.Tq, c.Tk) > 2048 + 50
    c.run(generic)
    torch.cuda.synchronize()
    c = Case(45, dt, 2, hd, [1, 1], [1000, 1100], True, pos=[999, 1099], pad_cols=1 << 20)
    c.run(generic, back=False)
