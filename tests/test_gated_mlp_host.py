"""The gated feed-forward block: what its entry points refuse before anything is launched (no GPU needed)."""
import pytest

from paper_2311_10418_amd import binding as ds

P = 4096        # stands for an aligned address; a call that is refused does not look behind it
BAD = ds.DS_EINVAL


def _fwd(**kw):
    a = dict(dtype=1, act=0, rows=0, d=64, d_ff=128, x=P, wg=P, wu=P, bg=None, bu=None, row_valid=None, h=P, g=None, u=None, workspace=None, floats=0, generic=0, stream=None)
    a.update(kw)
    return ds.lib().ds_gated_mlp_fwd(*a.values())


def _bwd(**kw):
    a = dict(dtype=1, act=0, rows=0, d=64, d_ff=128, dh=P, g=P, u=P, wg=P, wu=P, row_valid=None, dg=P, du=P, dx=P, workspace=None, floats=0, generic=0, stream=None)
    a.update(kw)
    return ds.lib().ds_gated_mlp_bwd(*a.values())


def _wgrad(**kw):
    a = dict(dtype=1, rows=4, d=64, d_ff=128, x=P, dg=P, du=P, dwg=P, dwu=P, dbg=None, dbu=None, accumulate=0, workspace=None, floats=0, generic=0, stream=None)
    a.update(kw)
    return ds.lib().ds_gated_mlp_wgrad(*a.values())


SIZES = [dict(dtype=2), dict(dtype=-1), dict(rows=-1), dict(rows=2 ** 31 - 1), dict(d=0), dict(d=-8), dict(d=60), dict(d=65544), dict(d_ff=0), dict(d_ff=100), dict(d_ff=65544), dict(floats=-1), dict(floats=4),
         dict(workspace=P + 4, floats=4), dict(rows=2 ** 30, d_ff=65536)]


@pytest.mark.parametrize("call,needed,others", [(_fwd, ("x", "wg", "wu", "h"), ("bg", "bu", "g", "u")), (_bwd, ("dh", "g", "u", "wg", "wu", "dg", "du", "dx"), ()),
                                                (_wgrad, ("x", "dg", "du", "dwg", "dwu"), ("dbg", "dbu"))])
def test_refusals(call, needed, others):
    for kw in SIZES + [{n: None, "rows": 4} for n in needed] + [{n: P + 8} for n in needed + others] + ([] if call is _wgrad else [dict(act=3), dict(act=-1)]):
        assert call(**kw) == BAD, kw


def test_pairs_and_nothing_to_do():
    assert _fwd() == _bwd() == ds.DS_OK                         # no rows
    assert _fwd(x=None, h=None) == _bwd(dh=None, g=None, u=None, dg=None, du=None, dx=None) == ds.DS_OK
    assert _fwd(g=P) == BAD and _fwd(u=P) == BAD
    assert _wgrad(rows=0) == BAD and _wgrad(accumulate=2) == BAD and _wgrad(dbg=P) == BAD and _wgrad(dbu=P) == BAD
    assert _wgrad(dbg=P, dbu=P) == BAD and _wgrad(dbg=P, dbu=P, workspace=P, floats=128 * 128 - 1) == BAD


def test_workspace():
    f = ds.ds_gated_mlp_workspace_floats
    assert f(0, 64, 64) == f(4, 0, 64) == f(4, 64, 0) == 0
    assert f(1, 8, 8) == f(65536, 1024, 2816) == 1 << 24 and f(1, 8, 65536) >= 128 * 65536
