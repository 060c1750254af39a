"""The gated feed-forward block's 256 x 256 tiles against oracle/layer.py: whole tiles, tiles whose contraction is cut up, persistent work-groups, with room for all of that and without.
Every case states how its tiles are divided (ds_gated_mlp_division), so that none of them quietly goes to other kernels.  Inputs and tolerances as in test_gpu_gated_mlp.py: rows that do not
count hold NaN, a workspace is NaN throughout before the first call.  Pieces of a contraction are the same additions in another order, which the tolerances allow."""
import ctypes

import pytest
import torch

from paper_2311_10418_amd import binding as ds
from test_gpu_gated_mlp import BF, Block

pytestmark = pytest.mark.gpu


def division(rows, d, ff, dx, floats):
    """(whether a call takes these tiles, whole tiles, tiles cut up, pieces of each, persistent work-groups)"""
    out = (ctypes.c_int32 * 5)()
    ds.lib().ds_gated_mlp_division(rows, d, ff, int(dx), ctypes.c_int64(floats), out)
    return tuple(out)


FORWARD = [((4099, 512, 1408), (187, 0, 1, 0)), ((2500, 2048, 64), (0, 10, 8, 0)), ((33001, 1024, 448), (512, 4, 4, 1)), ((16400, 256, 1024), (520, 0, 1, 1))]


@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("shape,want", FORWARD, ids=lambda s: "x".join(map(str, s)))
def test_forward(shape, want, bias):
    """Ragged rows, d_ff that is and is not a multiple of 128, biases or none, G and U kept or not, rows that do not count."""
    assert division(*shape, False, 1 << 24) == (1, *want)
    b = Block(BF, *shape, "gelu" if bias else "silu", bias=bias, keep=not bias, pad=0.05)
    b.forward()
    torch.cuda.synchronize()
    b.check_forward()


def test_forward_keeps_and_adds_biases():
    """Tiles cut up, with everything at once; then without row_valid."""
    assert division(33001, 1024, 448, False, 1 << 24) == (1, 512, 4, 4, 1)
    for pad in (0.03, 0.0):
        b = Block(BF, 33001, 1024, 448, "gelu", bias=True, pad=pad)
        b.forward()
        torch.cuda.synchronize()
        b.check_forward()


DX = [((8205, 1024, 832), (132, 0, 1, 0)), ((16400, 1024, 832), (256, 4, 6, 0)), ((33001, 1024, 448), (512, 4, 3, 1)), ((16400, 2048, 128), (520, 0, 1, 1))]


@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("shape,want", DX, ids=lambda s: "x".join(map(str, s)))
def test_backward(shape, want, act):
    assert division(*shape, True, 1 << 24) == (1, *want)
    b = Block(BF, *shape, act, pad=0.05 if act == "gelu" else 0.0)
    b.forward()
    b.backward()
    torch.cuda.synchronize()
    b.check_backward()


@pytest.mark.parametrize("floats,forward,dx", [(0, None, (516, 0, 1, 0)), (16, None, (516, 0, 1, 0)), (20, None, (516, 0, 1, 1)), (70000, None, (516, 0, 1, 1)), (600000, (512, 4, 2, 1), (512, 4, 2, 1)),
                                               (1 << 20, (512, 4, 3, 1), (512, 4, 3, 1)), (1 << 21, (512, 4, 4, 1), (512, 4, 3, 1))])
def test_any_workspace(floats, forward, dx):
    """No room, room for the counters of persistent work-groups alone, for some pieces of the last tiles, for all."""
    shape = (33001, 1024, 448)
    assert division(*shape, True, floats) == (1, *dx) and division(*shape, False, floats) == ((1, *forward) if forward else (0, 516, 0, 1, dx[3]))
    b = Block(BF, *shape, "relu", pad=0.05, floats=floats)
    b.run()


@pytest.mark.parametrize("floats,want", [(0, (520, 0, 1, 0)), (16, (520, 0, 1, 0)), (20, (520, 0, 1, 1)), (1 << 24, (520, 0, 1, 1))])
def test_any_workspace_forward(floats, want):
    """The same of a forward pass whose tiles are whole: persistent from 20 floats on."""
    assert division(16400, 256, 1024, False, floats) == (1, *want)
    b = Block(BF, 16400, 256, 1024, "silu", bias=True, pad=0.05, floats=floats)
    b.forward()
    torch.cuda.synchronize()
    b.check_forward()


def test_the_end_of_a_workspace():
    """What lies behind the floats that a call is given stays as it was: counters are the last 16 of them."""
    for floats in (20, 21, 300000, 600001):
        b = Block(BF, 33001, 1024, 448, "gelu", floats=floats + 64)
        whole, b.ws = b.ws, b.ws[:floats]
        whole.fill_(7.0)
        b.forward()
        b.backward()
        torch.cuda.synchronize()
        assert bool((whole[floats:] == 7.0).all())
        b.check_backward()


def test_two_calls_at_once():
    """Two persistent calls, forward and backward, with a workspace each, on two streams and replayed from two graphs: every pass gives the bits of the first, which are checked."""
    made = []
    for seed in (1, 2):
        assert division(33001, 1024, 448, False, 1 << 24)[4] == division(33001, 1024, 448, True, 1 << 24)[4] == 1
        b = Block(BF, 33001, 1024, 448, "gelu", seed=seed, pad=0.05)
        b.run()
        first = {n: t.clone() for n, t in b.t.items()}
        g, st = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        with torch.cuda.graph(g):
            b.forward()
            b.backward()
        made.append((b, first, g, st))
    for _ in range(3):
        for b, _, g, st in made:
            for t in b.t.values():
                t.fill_(5.0)
            st.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        for b, first, _, _ in made:
            assert all(torch.equal(first[n], b.t[n]) for n in first)
