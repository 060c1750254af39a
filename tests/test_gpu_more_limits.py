"""Attention with a relative position bias and the gated feed-forward block at their limits: tensors beyond 2^31 elements, many items for persistent work-groups, long tails of
sequences, lengths of zero throughout, workspaces of any size.  Tolerances as in test_gpu_rel_attention.py and test_gpu_gated_mlp.py."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import layer
from paper_2311_10418_amd import binding as ds
from helpers import DEV, to_dev, to_np
from test_gpu_gated_mlp import Block, _rnd
from test_gpu_rel_attention import Case

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
U = 2.0 ** -24


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_long_tail(causal, hd):
    """One long sequence among many short ones: work goes by a list, and at head size 128 persistent work-groups draw several items."""
    lens = [1 + (7 * i) % 40 for i in range(60)] + [900]
    Case(31, BF, 6 if hd == 128 else 2, hd, lens, lens, causal).run(False)


@pytest.mark.parametrize("hd", [64, 128])
def test_sequences_of_all_lengths_without_a_list(hd):
    """Blocks behind the ends of sequences, of queries and of keys."""
    for ql, kl, causal in (([400, 300, 390, 385, 257, 300], [300, 400, 390, 1, 390, 385], False), ([300, 257, 384, 290], [300, 257, 384, 290], True)):
        c = Case(32, BF, 2, hd, ql, kl, causal, gap=0)
        for backward in (0, 1):
            out = (ctypes.c_int32 * 8)()
            ds.lib().ds_rel_attention_choice(1, len(ql), 2, hd, max(ql), max(kl), c.Tq, c.Tk, backward, 0, out)
            assert out[2] > 0
        c.run(False, accumulate=causal)


# query lengths, key lengths, causal, positions
SHARED = [([700], [700], False, None), ([1500], [1500], True, None), ([1100, 3, 0, 700], [900, 1100, 50, 0], False, None), ([1030, 1100], [1030, 1100], True, None), ([520], [2000], True, [1480]),
          ([60], [1300], False, [-700]), ([1300], [70], True, [-300]), ([2000, 1, 30, 2, 15], [2000, 1, 30, 2, 15], True, None), ([900], [1], False, None), ([1], [900], True, [899])]


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("case", SHARED, ids=lambda c: "-".join(map(str, c)).replace(" ", ""))
def test_work_groups_share_blocks(case, hd):
    """Backward with few blocks of rows: long ones, ends of sequences and positions that fall into any share, shares without anything."""
    ql, kl, causal, pos = case
    c = Case(36, BF, 1, hd, ql, kl, causal, pos=pos)
    out = (ctypes.c_int32 * 8)()
    ds.lib().ds_rel_attention_choice(1, len(ql), 1, hd, max(ql), max(kl), c.Tq, c.Tk, 1 + 2 * causal, 0, out)
    assert out[7] > 1
    c.run(False, accumulate=causal)
    first = [t.clone() for t in (c.dq, c.dk, c.dv)]
    for t in (c.dq, c.dk, c.dv):
        t.fill_(9.0)
    c.scratch.fill_(255)
    c.backward()
    torch.cuda.synchronize()
    for s, t in zip(first, (c.dq, c.dk, c.dv)):
        assert torch.equal(s, t)


@pytest.mark.parametrize("hd", [64, 128])
def test_large_log_sum_exps(hd):
    """Scores of about 3008 by their bias: an error of 2^-17 of that would be one of 2 % of every probability.  One query to a sequence, so that nothing averages it out; the only
    roundings are those of P to bf16, of the results, and of fp32 scores of this size (E)."""
    n, heads = 24, 2
    c = Case(35, BF, heads, hd, [1] * n, [9 + i for i in range(n)], False, buckets=1, table=[0, 0, 0], bias=np.full((1, heads), 3008.0)).tensors()
    c.d_o = np.abs(c.d_o)
    c.tdo = c.place(c.d_o, c.q_on, np.nan)
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    dv = to_np(c.dv)
    for s in range(n):
        qs, ks = slice(c.q_row[s], c.q_row[s] + 1), slice(c.k_row[s], c.k_row[s] + c.kl[s])
        terms = layer.rel_attention(c.q[qs], c.k[ks], c.v[ks], c.bias, c.bucket, heads, False, 0, c.scale)[3]
        ref = layer.rel_attention_back(c.q[qs], c.k[ks], c.v[ks], c.bias, c.bucket, to_np(c.o)[qs], c.d_o[qs], heads, False, 0, c.scale)
        E = U * (128 * terms.max() + 8 * 2 * 3010.0 + 256)
        assert np.all(np.abs(dv[ks] - ref["dv"]) <= 2.0 ** -8 * np.abs(ref["dv"]) + (2.0 ** -8 + 2 * E + 256 * U) * ref["dv_part"])


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("hd", [64, 128])
def test_no_tokens_at_all(hd, dt):
    for ql, kl in (([0, 0], [0, 0]), ([0, 0], [5, 200]), ([7, 150], [0, 0])):
        for causal in (False, True):
            c = Case(34, dt, 2, hd, ql, kl, causal)
            c.run(False)
            assert np.all(to_np(c.dbias) == 0)


@pytest.mark.parametrize("dt,hd", [(BF, 64), (BF, 128), (F32, 64), (BF, 96)])
def test_keys_behind_2_31_elements(dt, hd):
    """A cache of more than 2^31 elements, single queries over sequences at its end."""
    heads, wide, n = 2, 4096, 3
    rows = (1 << 31) // wide + 2048
    cache = torch.zeros((rows, wide), dtype=dt, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(1)
    kl = [300, 1, 77]
    k_row = [rows - 1000, rows - 600, rows - 77]
    k, v = cache[:, wide - 2 * heads * hd:wide - heads * hd], cache[:, wide - heads * hd:]
    for r, l in zip(k_row, kl):
        cache[r:r + l, wide - 2 * heads * hd:] = torch.randn((l, 2 * heads * hd), generator=g, device=DEV).to(dt)
    q = torch.randn((n, heads * hd), generator=g, device=DEV).to(dt)
    bias = torch.randn((32, heads), generator=g, device=DEV).to(dt)
    bucket = ds.ds_rel_buckets(32, 128, False)
    at = lambda a: torch.tensor(np.asarray(a, dtype=np.int32), device=DEV)  # noqa: E731
    o, lse = torch.zeros_like(q), torch.zeros((heads, n), device=DEV)
    scratch = torch.zeros(int(ds.ds_rel_attention_scratch_bytes(heads, hd, 128, n, rows, n)), dtype=torch.uint8, device=DEV)
    for generic in (False, True):
        o.zero_()
        ds.ds_rel_attention_fwd(q, k, v, bias, at(bucket), o, lse, at([0, 1, 2]), at([1, 1, 1]), at(k_row), at(kl), heads, hd, True, 1, 300, scratch, q_pos=at([l - 1 for l in kl]),
                                force_generic=generic)
        for i, (r, l) in enumerate(zip(k_row, kl)):
            ro, rl, size, terms = layer.rel_attention(to_np(q)[i:i + 1], to_np(k[r:r + l]), to_np(v[r:r + l]), to_np(bias), bucket, heads, True, l - 1, float(np.float32(hd ** -0.5)))
            E = U * (128 * terms + 8 * (5 + np.abs(rl)) + 256)
            half = 2.0 ** -8 if dt == BF else U
            lim = half * np.abs(ro) + (2 * np.repeat(E.T, hd, axis=1) + (2.0 ** -8 if dt == BF else 0.0)) * size
            assert np.all(np.abs(to_np(o)[i:i + 1] - ro) <= lim) and np.all(np.abs(to_np(lse)[:, i:i + 1] - rl) <= E)


@pytest.mark.parametrize("dt,rows", [(BF, (1 << 31) // 1024 + 300), (F32, (1 << 31) // 1024 + 300)])
def test_gated_block_behind_2_31_elements(dt, rows):
    d, ff = 256, 1024
    g = torch.Generator(device=DEV).manual_seed(2)
    make = lambda *s, scale=1.0: (torch.randn(s, generator=g, device=DEV) * scale).to(dt)  # noqa: E731
    x = torch.zeros((rows, d), dtype=dt, device=DEV)
    x[-700:] = make(700, d)
    wg, wu = make(ff, d, scale=d ** -0.5), make(ff, d, scale=d ** -0.5)
    h = torch.empty((rows, ff), dtype=dt, device=DEV)
    ws = torch.empty(1 << 24, device=DEV)
    ds.ds_gated_mlp_fwd(x, wg, wu, h, act=ds.DS_ACT_SILU, workspace=ws)
    xa, wga, wua = to_np(x[-700:]), to_np(wg).T, to_np(wu).T
    ref, rg, ru = layer.gated_mlp(xa, wga, wua, 0.0, 0.0, "silu")
    eg, eu = ((d + 4) * U * (np.abs(xa) @ np.abs(w)) for w in (wga, wua))
    half = 2.0 ** -8 if dt == BF else U
    lim = half * np.abs(ref) + (1 + half) * (np.abs(ru) * (1.2 * eg + 2.0 ** -17 * np.abs(rg)) + np.abs(rg) * eu + 2 * eg * eu)
    assert np.all(np.abs(to_np(h[-700:]) - ref) <= lim) and not h[:-700].any()
    # backward in place: dG, dU over the memory of G and U
    u = torch.ones_like(h)
    h[:-700] = 0
    ga, ua = to_np(h[-700:]), np.ones((700, ff))
    dx = torch.empty_like(x)
    w1, w2 = wg.t().contiguous(), wu.t().contiguous()
    dh = torch.zeros_like(h) if dt == BF else None
    if dh is not None:
        dh[-700:] = make(700, ff)
        da = to_np(dh[-700:])
        ds.ds_gated_mlp_bwd(dh, h, u, w1, w2, h, u, dx, act=ds.DS_ACT_SILU, workspace=ws)
        dg, du = layer.gated_mlp_back(da, ga, ua, "silu")
        for got, want in ((h, dg), (u, du)):
            assert np.all(np.abs(to_np(got[-700:]) - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -17 * (1 + np.abs(ga)) * np.abs(da)) and not got[:-700].any()
        assert not dx[:-700].any()
        got = (to_np(h[-700:]), to_np(u[-700:]))
        ref = got[0] @ to_np(w1).T + got[1] @ to_np(w2).T
        size = np.abs(got[0]) @ np.abs(to_np(w1).T) + np.abs(got[1]) @ np.abs(to_np(w2).T)
        assert np.all(np.abs(to_np(dx[-700:]) - ref) <= 2.0 ** -8 * np.abs(ref) + 2 * ff * U * size)


@pytest.mark.parametrize("dt", [BF, F32])
def test_gated_block_without_rows(dt):
    x, h, w = torch.zeros((0, 64), dtype=dt, device=DEV), torch.zeros((0, 128), dtype=dt, device=DEV), torch.ones((128, 64), dtype=dt, device=DEV)
    ds.ds_gated_mlp_fwd(x, w, w, h)
    ds.ds_gated_mlp_bwd(h, h, h, w.t().contiguous(), w.t().contiguous(), h, h, x)


@pytest.mark.parametrize("floats", [0, 4, 16, 20, 1000, 70000, 1 << 20])
def test_gated_block_with_any_workspace(floats):
    """Large tiles with and without room for their counters and for partial sums."""
    Block(BF, 3000, 256, 1024, "gelu", bias=True, pad=0.1, floats=floats).run()
    Block(BF, 20000, 256, 512, "relu", pad=0.1, floats=floats).run()
    Block(F32, 300, 200, 520, "silu", bias=True, floats=floats).run()


@pytest.mark.parametrize("rows,d,ff,floats", [(64 * 70, 128, 192, 1 << 24), (64 * 70, 128, 192, 5 * 2 * 128 * 192 + 7), (3000, 1000, 72, 1 << 24), (1000, 72, 1000, 1 << 20), (65, 128, 192, 1 << 20),
                                               (1, 200, 8, 1 << 20), (20000, 136, 328, 1 << 24)])
def test_shares_of_weight_gradients(rows, d, ff, floats):
    """Rows of the tiles' weight gradients shared out, from one share to dozens; rounding: rows additions in fp32, in any order, and one more where they are added to what is there."""
    rng = np.random.default_rng([6, rows, d, ff])
    x, dg, du = (_rnd(rng, (rows, c), BF) for c in (d, ff, ff))
    out = [torch.full((d, ff), 3.0, device=DEV) for _ in range(2)]
    ws = torch.full((floats,), float("nan"), device=DEV)
    for accumulate in (False, True):
        before = [to_np(t) for t in out]
        ds.ds_gated_mlp_wgrad(to_dev(x, BF), to_dev(dg, BF), to_dev(du, BF), *out, accumulate=accumulate, workspace=ws)
        for got, dy, was in zip(out, (dg, du), before):
            ref = x.T @ dy + (was if accumulate else 0.0)
            assert np.all(np.abs(to_np(got) - ref) <= U * (rows * (np.abs(x).T @ np.abs(dy)) + np.abs(ref)) + 2.0 ** -130)


def test_persistent_tiles_of_two_calls_at_once():
    """Calls with a workspace each, on two streams, of two captured graphs: their tile counters are not shared."""
    made = []
    for seed in (1, 2):
        b = Block(BF, 40000, 256, 1024, "gelu", seed=seed)
        b.forward()
        b.backward()
        torch.cuda.synchronize()
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
