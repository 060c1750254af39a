"""ds_rope against oracle/layer.py.

Tolerance, elementwise: half a step of the output's type relative to the value, and 2^-21 of amplitude x (|x0| + |x1|): cosine and sine are
within 2^-23 of their own values' scale (the series end below 2^-27, a handful of fp32 roundings), two products, one sum.  An angle is a
product in 64 bits: at |angle| <= 2^21 off by 2^-31."""
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


def _rnd(rng, shape, dt):
    a = rng.standard_normal(shape).astype(np.float32)
    return (wl.to_bf16_grid(a) if dt == BF else a).astype(np.float64)


def _check(got, x, pos, freq, heads, hd, rot, inter, inverse, amp, dt, before):
    ref = layer.rope(x, pos, freq, heads, hd, rot, inter, inverse, amp)
    size = np.abs(x).reshape(len(pos), heads, hd).copy()
    turned = np.zeros_like(size)
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if inter else (slice(0, rot // 2), slice(rot // 2, rot))
    turned[:, :, a] = turned[:, :, b] = amp * (size[:, :, a] + size[:, :, b])
    turned = turned.reshape(x.shape)
    on = np.asarray(pos) >= 0
    assert np.all(np.abs(got - ref)[on] <= (HALF[dt] * np.abs(ref) + 2.0 ** -21 * turned)[on])
    same = (turned == 0) & on[:, None] & (np.arange(x.shape[1]) % hd >= rot)[None]
    assert np.array_equal(got[same], x[same])                         # columns beyond the turned ones: as they are
    assert np.array_equal(got[~on], before[~on])                      # rows without a position: not touched


# rows, heads, head_dim, rot, columns behind the heads, columns in front (an offset that breaks the alignment where odd)
SHAPES = [(1, 1, 64, 64, 0, 0), (37, 3, 64, 64, 64, 0), (64, 5, 128, 64, 8, 8), (19, 2, 96, 80, 0, 0), (33, 4, 32, 16, 16, 0), (7, 3, 64, 62, 0, 0), (9, 2, 10, 6, 3, 1),
          (5, 33, 64, 64, 0, 0), (21, 2, 64, 32, 1, 0), (6, 1, 2, 2, 0, 0)]


@pytest.mark.parametrize("dt", [F32, BF])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("rows,heads,hd,rot,behind,front", SHAPES)
def test_turns(dt, inter, rows, heads, hd, rot, behind, front):
    rng = np.random.default_rng(rows + heads)
    width = heads * hd
    wide = _rnd(rng, (rows, front + width + behind), dt)
    pos = rng.integers(0, 1 << 20, rows).astype(np.int32)
    pos[rng.random(rows) < 0.2] = -1
    pos[0] = 0
    freq = ds.ds_rope_freqs(rot, 10000.0) if rot > 2 else np.array([0.7])
    dpos, dfreq = torch.from_numpy(pos).to(DEV), torch.from_numpy(freq).to(DEV)
    x = wide[:, front:front + width]
    for inverse, amp in ((False, 1.0), (True, float(np.float32(1.3)))):
        src = to_dev(wide, dt)
        dst = torch.full((rows + 2, width + behind), 9.0, dtype=dt, device=DEV)
        ds.ds_rope(src[:, front:], dst, dpos, dfreq, heads, hd, rot, interleaved=inter, inverse=inverse, amplitude=amp)
        torch.cuda.synchronize()
        got = to_np(dst)
        _check(got[:rows, :width], x, pos, freq, heads, hd, rot, inter, inverse, amp, dt, np.full_like(x, 9.0))
        assert np.all(got[rows:] == 9.0) and np.all(got[:, width:] == 9.0)
        assert np.array_equal(to_np(src), wide)
        ds.ds_rope(src[:, front:], src[:, front:], dpos, dfreq, heads, hd, rot, interleaved=inter, inverse=inverse, amplitude=amp)      # in place
        torch.cuda.synchronize()
        both = to_np(src)
        assert np.array_equal(both[:, :front], wide[:, :front]) and np.array_equal(both[:, front + width:], wide[:, front + width:])
        _check(both[:, front:front + width], x, pos, freq, heads, hd, rot, inter, inverse, amp, dt, x)
        on = pos >= 0
        assert np.array_equal(both[on, front:front + width], got[:rows, :width][on])


def test_far_positions_and_every_quarter():
    """Angles up to 2^31 radians: 2^-22 of a turn by the 64-bit product there, 2^-21 of the size with it; and turns next to the borders of the quarters."""
    pos = np.array([0, 1, 2, 3, 4, 5, 6, 7, 1 << 20, (1 << 28) + 1, 0x7fffffff, 12345677], dtype=np.int32)
    freq = np.array([1.0, np.pi / 4, np.pi / 2, np.pi / 2 + 1e-9, 1e-6, 0.5, 0.0, 3.0])
    x = np.ones((len(pos), 16))
    dst = torch.zeros((len(pos), 16), device=DEV)
    ds.ds_rope(to_dev(x, F32), dst, torch.from_numpy(pos).to(DEV), torch.from_numpy(freq).to(DEV), 1, 16, 16)
    torch.cuda.synchronize()
    got = to_np(dst)
    angle = pos[:, None].astype(np.float64) * freq
    assert np.abs(got[:, :8] - (np.cos(angle) - np.sin(angle))).max() <= 2.0 ** -20
    assert np.abs(got[:, 8:] - (np.cos(angle) + np.sin(angle))).max() <= 2.0 ** -20


def test_scores_depend_on_distance_only():
    """The dot product of a turned query and a turned key is that of their distance."""
    rng = np.random.default_rng(2)
    q, k = rng.standard_normal(64), rng.standard_normal(64)
    freq = torch.from_numpy(ds.ds_rope_freqs(64)).to(DEV)
    x = to_dev(np.tile(np.concatenate([q, k]), (3, 1)), F32)
    out = []
    for tq, tk in ((5, 0), (1005, 1000), (500005, 500000)):
        y = torch.empty_like(x)
        pos = torch.tensor([tq, tk, 0], dtype=torch.int32, device=DEV)
        ds.ds_rope(x, y, pos, freq, 2, 64, 64)
        y = to_np(y)
        out.append(y[0, :64] @ y[1, 64:])
    size = np.abs(q) @ np.abs(k) * 4
    assert max(out) - min(out) <= 2.0 ** -19 * size


def test_positions_of_a_layout_and_another_stream():
    lay = ds.ds_layout_from_cuts([5, 2, 9], [0, 2, 3])
    pos = ds.ds_layout_positions(lay)
    rng = np.random.default_rng(3)
    x = _rnd(rng, (lay.total_rows, 128), BF)
    freq = ds.ds_rope_freqs(64)
    src, dst = to_dev(x, BF), torch.zeros((lay.total_rows, 128), dtype=BF, device=DEV)
    dpos, dfreq = torch.from_numpy(pos).to(DEV), torch.from_numpy(freq).to(DEV)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    ds.ds_rope(src, dst, dpos, dfreq, 2, 64, 64, stream=side.cuda_stream)
    side.synchronize()
    _check(to_np(dst), x, pos, freq, 2, 64, 64, False, False, 1.0, BF, np.zeros_like(x))


def test_tensors_that_do_not_fit_are_refused():
    x = torch.zeros((4, 128), dtype=BF, device=DEV)
    pos, freq = torch.zeros(4, dtype=torch.int32, device=DEV), torch.zeros(32, dtype=torch.float64, device=DEV)
    for bad in (dict(x=x[:3]), dict(y=x[:, :64]), dict(x=x.float()), dict(pos=pos.long()), dict(freq=freq[:31]), dict(freq=freq.float()), dict(y=x.t())):
        with pytest.raises(ValueError):
            a = dict(dict(x=x, y=x.clone(), pos=pos, freq=freq), **bad)
            ds.ds_rope(a["x"], a["y"], a["pos"], a["freq"], 2, 64, 64)
