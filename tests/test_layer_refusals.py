"""What the entry points of the layer parts refuse before anything is launched, and their host functions (no GPU needed)."""
import ctypes as C
import math

import numpy as np
import pytest

from paper_2311_10418_amd import binding as ds

P = 4096        # stands for an aligned address; a call that is refused does not look behind it
BAD = ds.DS_EINVAL


def _fwd(**kw):
    a = dict(dtype=1, rms=0, rows=0, d=64, x=P, h=P, row_valid=None, post_g=P, post_b=P, gate_kind=0, gate=None, resid_scale=C.c_float(1),
             branch_scale=C.c_float(1), pre_g=P, pre_b=P, y=P, u=P, stats=P, stream=None)
    a.update(kw)
    vp = ("x", "h", "row_valid", "post_g", "post_b", "gate", "pre_g", "pre_b", "y", "u", "stats", "stream")
    return ds.lib().ds_resid_norm_fwd(*[C.c_void_p(v) if k in vp else v for k, v in a.items()])


def test_resid_norm_forward():
    assert _fwd() == ds.DS_OK                                   # no rows: nothing to do
    assert _fwd(rms=1, post_b=None, pre_b=None) == ds.DS_OK
    assert _fwd(post_g=None, post_b=None, pre_g=None, pre_b=None, u=None) == ds.DS_OK
    for kw in (dict(dtype=2), dict(rms=2), dict(rows=-1), dict(d=0), dict(d=60), dict(d=4104), dict(x=None), dict(h=None), dict(y=None), dict(stats=None),
               dict(post_b=None), dict(pre_b=None), dict(u=None), dict(gate=P), dict(gate_kind=1), dict(gate_kind=3, gate=P), dict(x=P + 8), dict(h=P + 2),
               dict(y=P + 8), dict(u=P + 8), dict(post_g=P + 4), dict(pre_g=P + 4), dict(pre_b=P + 8), dict(post_b=P + 8), dict(gate_kind=2, gate=P + 8)):
        assert _fwd(**kw) == BAD, kw


def _bwd(**kw):
    a = dict(dtype=1, rms=0, rows=4, d=64, dy=P, du=P, y=P, h=P, row_valid=None, post_g=P, post_b=P, gate_kind=1, gate=P, resid_scale=C.c_float(1),
             branch_scale=C.c_float(1), pre_g=P, stats=P, dx=P, dh=P, dgate=P, dpost_g=P, dpost_b=P, dpre_g=P, dpre_b=P, partial=P, accumulate=0, stream=None)
    a.update(kw)
    other = ("dtype", "rms", "rows", "d", "gate_kind", "resid_scale", "branch_scale", "accumulate")
    return ds.lib().ds_resid_norm_bwd(*[v if k in other else C.c_void_p(v) for k, v in a.items()])


def test_resid_norm_backward():
    for kw in (dict(rows=0), dict(d=4), dict(dtype=-1), dict(rms=-1), dict(accumulate=2), dict(dy=None, pre_g=None), dict(du=None), dict(y=None), dict(h=None),
               dict(stats=None), dict(dx=None), dict(dh=None), dict(dgate=None), dict(dpost_g=None), dict(dpost_b=None), dict(dpre_g=None), dict(dpre_b=None),
               dict(partial=None), dict(partial=P + 4), dict(gate=None), dict(dy=P + 8), dict(du=P + 8), dict(dx=P + 2), dict(dh=P + 8), dict(dgate=P + 8)):
        assert _bwd(**kw) == BAD, kw
    assert ds.ds_resid_norm_bwd_scratch_floats(0, 64) == 0 and ds.ds_resid_norm_bwd_scratch_floats(5, 0) == 0
    for rows in (1, 100, 1 << 20):
        for d in (8, 512, 2056, 4096):
            assert 4 * d <= ds.ds_resid_norm_bwd_scratch_floats(rows, d) <= 1 << 24


def _rope(**kw):
    a = dict(dtype=1, rows=0, n_heads=2, head_dim=64, rot_dim=64, interleaved=0, inverse=0, pos=P, freq=P, amplitude=C.c_float(1), x=P, ldx=C.c_int64(128),
             y=P, ldy=C.c_int64(128), stream=None)
    a.update(kw)
    return ds.lib().ds_rope(*[C.c_void_p(v) if k in ("pos", "freq", "x", "y", "stream") else v for k, v in a.items()])


def test_rope():
    assert _rope() == ds.DS_OK
    for kw in (dict(dtype=7), dict(rows=-1), dict(n_heads=0), dict(head_dim=0), dict(rot_dim=0), dict(rot_dim=3), dict(rot_dim=66), dict(interleaved=2),
               dict(inverse=-1), dict(pos=None), dict(freq=None), dict(x=None), dict(y=None), dict(ldx=C.c_int64(127)), dict(ldy=C.c_int64(127)),
               dict(ldy=C.c_int64(256)), dict(x=P + 1), dict(y=P + 1), dict(pos=P + 2), dict(freq=P + 4), dict(n_heads=1 << 30, head_dim=1 << 30)):
        assert _rope(**kw) == BAD, kw


def test_rope_freqs():
    plain = ds.ds_rope_freqs(8, 10000.0)
    assert np.allclose(plain, [1.0, 0.1, 0.01, 0.001], rtol=1e-15)
    assert np.allclose(ds.ds_rope_freqs(8, 10000.0, ds.DS_ROPE_LINEAR, factor=4.0), plain / 4, rtol=1e-15)
    slowed = ds.ds_rope_freqs(8, 10000.0, ds.DS_ROPE_BASE, factor=4.0)
    assert slowed[0] == 1.0 and math.isclose(slowed[3], plain[3] / 4, rel_tol=1e-12)
    turns = 1000.0 * plain / (2 * math.pi)                       # 159, 15.9, 1.59, 0.159
    bands = ds.ds_rope_freqs(8, 10000.0, ds.DS_ROPE_BANDS, factor=4.0, context=1000.0, low_turns=1.0, high_turns=32.0)
    w = np.clip((turns - 1) / 31, 0, 1)
    assert np.allclose(bands, plain * (w + (1 - w) / 4), rtol=1e-14)
    assert bands[0] == plain[0] and math.isclose(bands[3], plain[3] / 4, rel_tol=1e-14)
    for args in ((0,), (3,), (8, 0.0), (8, float("nan")), (8, 10000.0, 4), (8, 10000.0, 1, 0.0), (2, 10000.0, 2, 2.0), (8, 10000.0, 3, 2.0, 0.0),
                 (8, 10000.0, 3, 2.0, 100.0, 5.0, 5.0)):
        with pytest.raises(ds.DsError):
            ds.ds_rope_freqs(*args)


def test_layout_positions():
    lay = ds.ds_layout_from_cuts([3, 1, 4], [0, 2, 3])
    pos = ds.ds_layout_positions(lay)
    assert pos.tolist() == [0, 1, 2, 0, -1, -1, 0, 1, 2, 3]
    with pytest.raises(ds.DsError) as e:
        ds.ds_layout_positions(lay, which=1)
    assert e.value.code == ds.DS_ELAYOUT
    two = ds.ds_layout_from_cuts([2, 3], [0, 2], lengths_tgt=[2, 1])
    assert ds.ds_layout_positions(two, which=1).tolist() == [0, 1, 0, -1]
    packed = ds.ds_layout_packed([3, 2, 4], 5, 1)
    pos = ds.ds_layout_positions(packed)
    for row, n in zip(packed.seq_row, packed.seq_len):
        assert pos[row:row + n].tolist() == list(range(n))
    assert (pos >= 0).sum() == 9
    assert ds.lib().ds_layout_positions(None, 0, C.c_void_p(P)) == BAD and ds.lib().ds_layout_positions(lay.handle, 2, C.c_void_p(P)) == BAD


def test_the_binding_refuses_tensors_that_are_not_on_the_gpu():
    import torch
    t = torch.zeros((4, 64))
    with pytest.raises(ValueError):
        ds.ds_resid_norm_fwd(t, t, t.clone(), torch.zeros((4, 4)))
    with pytest.raises(ValueError):
        ds.ds_rope(t, t, torch.zeros(4, dtype=torch.int32), torch.zeros(32, dtype=torch.float64), 1, 64, 64)


def _diff(back, **kw):
    a = dict(dtype=1, n_seq=2, n_heads=2, head_dim=64, mask=1, q_row=P, q_len=P, k_row=P, k_len=P, max_q_len=8, max_k_len=8, q=P, ldq=128, k=P, ldk=128, v=P,
             ldv=128, lam=P, o=P, o2=P)
    if back:
        a.update(d_o=P)
    a.update(ldo=128, lse=P)
    if back:
        a.update(dq=P, dk=P, dv=P, dlam=P, accumulate=0)
    a.update(q_total_rows=16, k_total_rows=16, scratch=P, scratch_bytes=0, force_generic=0, stream=None)
    a.update(kw)                                                # (no scratch bytes: refused whatever else is right)
    ints = ("dtype", "n_seq", "n_heads", "head_dim", "mask", "max_q_len", "max_k_len", "ldq", "ldk", "ldv", "ldo", "accumulate", "q_total_rows", "k_total_rows", "force_generic")
    f = ds.lib().ds_diff_attention_bwd if back else ds.lib().ds_diff_attention_fwd
    return f(*[v if k in ints else C.c_int64(v) if k == "scratch_bytes" else C.c_void_p(v) for k, v in a.items()])


@pytest.mark.parametrize("back", [False, True])
def test_differential_attention(back):
    need = ds.ds_diff_attention_scratch_bytes(2, 16, 16, 2)
    assert need > 0 and ds.ds_diff_attention_scratch_bytes(0, 16, 16, 2) == 0 and ds.ds_diff_attention_scratch_bytes(2, 16, 0, 2) == 0
    assert _diff(back, scratch_bytes=need - 1) == BAD and _diff(back, scratch_bytes=-1) == BAD
    bad = [dict(dtype=3), dict(n_seq=0), dict(n_heads=0), dict(head_dim=0), dict(head_dim=72), dict(head_dim=144), dict(mask=2), dict(q_row=None), dict(q_len=None),
           dict(k_row=None), dict(k_len=None), dict(max_q_len=0), dict(max_k_len=0), dict(q=None), dict(k=None), dict(v=None), dict(ldq=127), dict(ldk=127),
           dict(ldv=127), dict(ldo=127), dict(lam=None), dict(o=None), dict(lse=None), dict(q_total_rows=0), dict(k_total_rows=0), dict(scratch=None),
           dict(scratch=P + 8), dict(q=P + 1), dict(k=P + 1), dict(v=P + 1), dict(o=P + 1), dict(o2=P + 1), dict(n_seq=70000), dict(n_heads=70000, head_dim=16, ldq=1 << 21, ldk=1 << 21, ldv=1 << 21, ldo=1 << 21)]
    if back:
        bad += [dict(o2=None), dict(d_o=None), dict(dq=None), dict(dk=None), dict(dv=None), dict(dlam=None), dict(accumulate=2), dict(dq=P + 1), dict(d_o=P + 1)]
    for kw in bad:
        assert _diff(back, **dict(dict(scratch_bytes=1 << 40), **kw)) == BAD, kw


@pytest.mark.parametrize("back", [False, True])
def test_differential_attention_of_too_long_sequences(back):
    """The fp32 kernels, in bf16 too: more than 2^28 tokens of a sequence, queries or keys."""
    n = (1 << 28) + 1
    small = dict(scratch_bytes=1 << 60, n_seq=1, n_heads=1, head_dim=16, ldq=16, ldk=16, ldv=16, ldo=16)
    for kw in (dict(max_q_len=n, q_total_rows=n), dict(max_k_len=n, k_total_rows=n), dict(max_q_len=0x7fffffff, q_total_rows=0x7fffffff, dtype=0)):
        assert _diff(back, **dict(small, **kw)) == BAD, kw
