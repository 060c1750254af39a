"""Differential attention on both sides of the borders between its kernels, each test with what it means to run; tolerances as in test_gpu_diff_attention.py."""
import numpy as np
import pytest
import torch

from helpers import diff_choice
from test_gpu_diff_attention import Case

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def _run(dt, heads, hd, ql, kl, causal, forward, backward, generic=False, accumulate=False):
    c = Case(hd + sum(ql) + sum(kl), dt, heads, hd, ql, kl, causal)
    for back, want in ((False, forward), (True, backward)):
        got = diff_choice(dt == BF, len(ql), heads, hd, causal, max(ql), max(kl), c.Tq, c.Tk, back, generic)
        assert {k: got[k] for k in want} == want, (back, got)
    c.run(generic, accumulate)


SHARE = {1: dict(general=0, sharing=1, splits=1), 2: dict(general=0, sharing=2), 4: dict(general=0, sharing=4)}


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("q,k,ks", [(32, 320, 1), (32, 321, 4), (33, 320, 1), (33, 321, 2), (64, 700, 2), (65, 700, 1), (1, 320, 1), (1, 321, 4)])
def test_wavefronts_that_share_keys(hd, q, k, ks):
    _run(BF, 3, hd, [q, min(q, 3), 1], [k, 5, k - 1], False, SHARE[ks], dict(general=0, sharing=ks))


@pytest.mark.parametrize("hd,n,ks", [(64, 16, 4), (64, 17, 1), (128, 8, 4), (128, 9, 1)])
def test_as_many_sequences_as_share_keys(hd, n, ks):
    rng = np.random.default_rng(n)
    ql, kl = [7] + [int(x) for x in rng.integers(1, 8, n - 1)], [400] + [int(x) for x in rng.integers(1, 401, n - 1)]
    _run(BF, 16, hd, ql, kl, False, SHARE[ks], dict(general=0, sharing=ks))


@pytest.mark.parametrize("hd,k,splits", [(64, 320, 1), (64, 321, 3), (64, 1024, 8), (64, 2048, 16), (128, 321, 3), (128, 2048, 16)])
def test_work_groups_that_share_keys(hd, k, splits):
    """The rows of the query tensor are at most 64 for each sequence here (a larger tensor is not shared over work-groups)."""
    _run(BF, 16, hd, [2], [k], False, dict(general=0, sharing=1 if k == 320 else 4, splits=splits), dict(general=0))


@pytest.mark.parametrize("dt", [F32, BF])
@pytest.mark.parametrize("hd,k,splits", [(64, 128, 1), (64, 129, 3), (48, 1000, 16), (112, 129, 3), (96, 5000, 64)])
def test_work_groups_that_share_keys_in_fp32(dt, hd, k, splits):
    _run(dt, 2, hd, [3], [k], False, dict(general=1, splits=splits), dict(general=1), generic=True)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("hd,n,length,direct", [(64, 17, 128, 1), (64, 17, 129, 0), (128, 16, 128, 1), (128, 17, 128, 0), (128, 16, 129, 0), (64, 130, 128, 0), (64, 130, 120, 1)])
def test_with_and_without_a_list(causal, hd, n, length, direct):
    """16 heads; sequences without queries or without keys among them."""
    rng = np.random.default_rng(n + length)
    lens = [length] + [int(x) for x in rng.integers(0, 30, n - 1)]
    _run(BF, 16, hd, lens, [length] + lens[2:] + [0], causal, dict(general=0, direct=direct, sharing=1), dict(general=0, direct=direct))


@pytest.mark.parametrize("n", [16, 17])
@pytest.mark.parametrize("hd", [64, 128])
def test_sixteen_tokens_and_one_more(hd, n):
    _run(BF, 2, hd, [n, 3, 16], [n, 3, 16], True, dict(general=0), dict(general=0))


@pytest.mark.parametrize("hd,n,length,cols", [(64, 32, 255, 32), (64, 32, 256, 64), (96, 16, 100, 32), (16, 130, 60, 64), (112, 2, 50, 64)])
def test_columns_of_the_fp32_backward_kernels(hd, n, length, cols):
    rng = np.random.default_rng(n + length)
    lens = [length] + [int(x) for x in rng.integers(1, 40, n - 1)]
    _run(F32, 4, hd, lens, lens, True, dict(general=1), dict(general=1, dq_columns=cols, dkv_columns=cols))


@pytest.mark.parametrize("causal", [False, True])
def test_many_items_for_each_persistent_work_group(causal):
    """Heads of 128: work-groups of the dK/dV kernel draw three blocks of keys and more (over 4 x 256 pairs of block and head): blocks of many steps, whose ring of
    four stages wraps, of one, and without any (no queries; keys beyond the last query of a causal sequence) in one order and another."""
    rng = np.random.default_rng(12)
    ql, kl = [], []
    for i in range(52):
        ql.append([0, 1, int(rng.integers(300, 420)), int(rng.integers(2, 70)), int(rng.integers(130, 300))][i % 5])
        kl.append([int(rng.integers(1, 300)), int(rng.integers(130, 400)), int(rng.integers(1, 200)), int(rng.integers(150, 300)), 0 if i % 3 else 130][i % 5])
    assert 16 * sum((k + 127) // 128 for k in kl) > 4 * 256
    _run(BF, 16, 128, ql, kl, causal, dict(general=0, direct=0), dict(general=0, direct=0))


@pytest.mark.parametrize("dt,hd,direct", [(BF, 64, 0), (BF, 128, 0), (BF, 64, 1), (BF, 128, 1), (F32, 64, 0)])
@pytest.mark.parametrize("causal", [False, True])
def test_lists_and_draws_in_a_graph(dt, hd, direct, causal):
    """Both directions captured with a scratch that holds anything before each replay: lists, counters of the persistent kernel and statistics are the call's own."""
    lens = [40, 0, 128, 33] * 4 if direct else [150, 0, 129, 300, 64, 17] * 5
    heads = 8
    c = Case(3, dt, heads, hd, lens, lens[::-1], causal)
    got = diff_choice(dt == BF, len(lens), heads, hd, causal, max(lens), max(lens), c.Tq, c.Tk, True)
    assert (got["general"], got["direct"]) == (int(dt == F32), direct)
    c.run(False)
    outs = (c.o, c.o2, c.lse, c.dq, c.dk, c.dv, c.dlam)
    want = [t.clone() for t in outs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.forward()
        c.backward()
    for i in range(4):
        for t in outs:
            t[:] = 9.0
        c.scratch.fill_(50 * i)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, outs):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dt,generic", [(F32, False), (BF, True), (BF, False)])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("bound", [0, 50, 200, 5000])
def test_no_tokens_at_all_and_bounds_that_are_too_large(dt, generic, causal, hd, bound):
    """Sequences without queries, without keys, without either; upper bounds of the lengths above the lengths and above the rows."""
    for ql, kl in (([0, 0, 0], [5, 0, 70]), ([5, 70, 0], [0, 0, 0]), ([0], [0]), ([3, 40, 130, 0], [200, 7, 1, 9])):
        c = Case(hd + bound, dt, 2, hd, ql, kl, causal)
        tables = c.args()
        c.args = lambda: (*tables[:-3], max(tables[-3], bound), max(tables[-2], bound), tables[-1])
        c.run(generic, accumulate=True)
        lse = c.lse.cpu()
        for r, n, k in zip(c.q_row, ql, kl):
            assert k or bool((lse[:, r:r + n] == -float("inf")).all())
