"""The layer parts at the ends of their ranges: sums that overflow, scores far below zero, statistics of many digits, values that are not finite."""
import numpy as np
import pytest
import torch

from paper_2311_10418_amd import binding as ds
from helpers import DEV, diff_choice

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)  # noqa: E731


# ------------------------------------------------------------------------------------ the joint of two blocks
@pytest.mark.parametrize("dt", [F32, BF])
@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("d", [64, 1024, 2048, 4096])
def test_rows_whose_sum_of_squares_overflows(dt, rms, d):
    """A norm of such a row is its bias, as in ds_norm_fwd: the reciprocal deviation is 0.  Exactly so: with post_g . 0 + post_b for z, y = 0 x + 1 z is the bias."""
    rows = 5
    g = torch.Generator(device=DEV).manual_seed(d)
    rnd = lambda *s: torch.randn(s, generator=g, device=DEV).to(dt)  # noqa: E731
    large, plain = rnd(rows, d), rnd(rows, d)
    large[1] *= 1e25
    large[3] *= 3e18 if d == 4096 else 1e30
    gain, bias = rnd(d), None if rms else rnd(d)
    ref, st = torch.empty_like(large), torch.zeros((2, rows), device=DEV)
    ds.ds_norm_fwd(large, gain, bias, ref, st, rms=rms)
    new = lambda: torch.full((rows, d), 7.0, dtype=dt, device=DEV)  # noqa: E731
    y, u, y2, stats, stats2 = new(), new(), new(), torch.zeros((4, rows), device=DEV), torch.zeros((4, rows), device=DEV)
    ds.ds_resid_norm_fwd(large, plain, y, stats, pre_g=gain, pre_b=bias, u=u, resid_scale=1.0, branch_scale=0.0, rms=rms)       # the norm before the next block
    ds.ds_resid_norm_fwd(plain, large, y2, stats2, post_g=gain, post_b=bias, resid_scale=0.0, branch_scale=1.0, rms=rms)        # the norm behind a block
    f32 = lambda: torch.zeros(d, device=DEV)  # noqa: E731
    dx, dh, dgate, sums = new(), new(), None, [f32() for _ in range(4)]
    partial = torch.zeros(int(ds.ds_resid_norm_bwd_scratch_floats(rows, d)), device=DEV)
    ds.ds_resid_norm_bwd(plain, y, plain, stats, dx, dh, partial, du=plain, pre_g=gain, dpre_g=sums[0], dpre_b=None if rms else sums[1], rms=rms)
    dx2, dh2 = new(), new()
    ds.ds_resid_norm_bwd(plain, y2, large, stats2, dx2, dh2, partial, post_g=gain, post_b=bias, dpost_g=sums[2], dpost_b=None if rms else sums[3], rms=rms)
    torch.cuda.synchronize()
    none = torch.zeros(d, device=DEV, dtype=dt) if rms else bias
    for r in (1, 3):
        assert torch.equal(ref[r], none) and torch.equal(u[r], none) and torch.equal(y2[r], none)
        assert stats[3, r] == 0 and stats2[1, r] == 0
        assert torch.equal(dx[r], plain[r]) and not dh2[r].any()                     # nothing goes through the norm
    for t in (y, u, y2, dx, dh, dx2, dh2, *sums):
        assert torch.isfinite(t).all()


# ------------------------------------------------------------------------------------ differential attention
def _run(q, k, v, d_o, lam, ql, kl, heads, hd, causal, generic=False, q_row=None, k_row=None, back=True):
    """Sequences one behind the other (or at the rows given) -> o, o2, lse, dq, dk, dv, dlam."""
    q_row = np.cumsum([0] + list(ql[:-1])).tolist() if q_row is None else q_row
    k_row = np.cumsum([0] + list(kl[:-1])).tolist() if k_row is None else k_row
    o, o2, dq, dk, dv = (torch.zeros_like(t) for t in (q, q, q, k, v))
    lse, dlam = torch.zeros((2 * heads, q.shape[0]), device=DEV), torch.zeros(heads, device=DEV)
    scratch = torch.zeros(int(ds.ds_diff_attention_scratch_bytes(heads, q.shape[0], k.shape[0], len(ql))), dtype=torch.uint8, device=DEV)
    rest = (i32(q_row), i32(ql), i32(k_row), i32(kl), heads, hd, causal, max(ql), max(kl), scratch)
    ds.ds_diff_attention_fwd(q, k, v, lam, o, lse, *rest, o2=o2, force_generic=generic)
    if back:
        ds.ds_diff_attention_bwd(q, k, v, lam, o, o2, d_o, lse, dq, dk, dv, dlam, *rest, force_generic=generic)
    torch.cuda.synchronize()
    return o, o2, lse, dq, dk, dv, dlam


@pytest.mark.parametrize("dt,generic", [(F32, False), (BF, True), (BF, False)])
@pytest.mark.parametrize("ql,kl,causal", [(5, 64, False), (1, 512, False), (33, 1024, False), (40, 1024, False), (200, 128, False), (150, 150, True)])
@pytest.mark.parametrize("hd", [64, 128])
def test_scores_far_below_zero(dt, generic, ql, kl, causal, hd):
    """Every score -2^108 (before the scale, a power of two, so that products with it round nothing): all visible probabilities alike, and their sums and values,
    small whole numbers, exact up to the rounding of results (half a step, and one of O2's in O) and of the reciprocal of the number of keys (2^-23)."""
    g = torch.Generator(device=DEV).manual_seed(ql)
    heads = 2
    exp = 5 if hd == 64 else 6                          # a map has 2^exp features
    q, k = torch.full((ql, heads * hd), 2.0 ** (54 - exp), dtype=dt, device=DEV), torch.full((kl, heads * hd), -2.0 ** 54, dtype=dt, device=DEV)
    v = torch.randint(-8, 9, (kl, heads * hd), generator=g, device=DEV).to(dt)
    lam = torch.tensor([0.5, 0.25], device=DEV)
    o, o2, lse = _run(q, k, v, None, lam, [ql], [kl], heads, hd, causal, generic, back=False)[:3]
    seen = torch.arange(1, ql + 1, device=DEV).clamp(max=kl) if causal else torch.full((ql,), kl, device=DEV)
    mean = v.double().cumsum(0)[seen - 1] / seen[:, None]
    half = 2.0 ** -8 if dt == BF else 2.0 ** -24
    most = (half + 2.0 ** -21) * mean.abs()
    assert ((o2.double() - mean).abs() <= most).all()
    assert ((o.double() - mean * (1 - lam.double().repeat_interleave(hd))).abs() <= most).all()
    assert torch.isfinite(lse).all()


@pytest.mark.parametrize("generic", [False, True])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("ql,kl", [(48, 64), (33, 256)])
def test_statistics_keep_all_their_digits(generic, hd, ql, kl):
    """Keys and values all alike, lambda = -1: every probability is 1 / kl, a power of two, their sum twice that, and dP - D is 0.  The log-sum-exps (up to 2^11, the
    second map's negative) and D (whole numbers of up to 21 bits) are what backward subtracts.  Eight roundings of 2^-24 in a log-sum-exp on its way are 2^-10 of a
    probability, below half a step of bf16 (2^-9 downwards), so that rounding takes them away: dV is exact (within 2^-10 in the kernels that do not
    round probabilities) and dK zero.  With 2^-17 of a log-sum-exp a probability would be up to 2^-6 off."""
    rng = np.random.default_rng(hd + ql)
    m = hd // 2
    at = lambda a: torch.from_numpy(np.asarray(a, dtype=np.float32)).to(DEV).to(BF)  # noqa: E731
    q = rng.integers(1, 128, (ql, hd)).astype(np.float64)
    k = rng.integers(1, 128, (1, hd)) * 2.0 ** 10 / (q[:, :m].sum(1).max() * 64 / np.sqrt(m))
    k = np.repeat(2.0 ** np.round(np.log2(k)) * np.where(np.arange(hd) < m, 1.0, -1.0), kl, 0)      # scores: whole numbers times powers of two, exact in fp32
    top = np.abs(np.stack([q[:, :m] @ k[0, :m], q[:, m:] @ k[0, m:]])).max() / np.sqrt(m)
    assert 2 ** 9 < top < 2 ** 11
    v = np.repeat(rng.integers(65, 128, (1, hd)), kl, 0)
    lam = torch.tensor([-1.0], device=DEV)
    for d_o in (64.0 * np.eye(ql, hd), rng.integers(65, 128, (ql, hd)) * rng.choice([-1, 1], (ql, hd))):     # one probability in every value of dV; D of many digits
        o, o2, lse, dq, dk, dv, dlam = _run(at(q), at(k), at(v), at(d_o), lam, [ql], [kl], 1, hd, False, generic)
        assert torch.equal(o2, at(v[:1]).expand(ql, hd)) and torch.equal(o, at(2 * v[:1]).expand(ql, hd))
        assert not dq.any() and not dk.any()
        want = at(d_o.sum(0, keepdims=True) * 2 / kl).expand(kl, hd)
        if generic:
            size = torch.from_numpy(np.abs(d_o).sum(0) * 2 / kl).to(DEV)
            assert ((dv.double() - want.double()).abs() <= 2.0 ** -7 * want.double().abs() + 2.0 ** -9 * size).all()
        else:
            assert torch.equal(dv, want)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("hd", [64, 128])
def test_gradients_of_a_sequence_do_not_depend_on_the_others(causal, hd):
    """Short bf16 sequences alone, as the first of many, and beside longer ones: the same bits."""
    heads = 8
    short = [16, 1, 9, 12]
    rng = np.random.default_rng(hd)
    lens = {"alone": short, "many": short + [5, 16] * 40, "beside one more token": short + [17], "beside long ones": short + [200, 130]}
    n = sum(max(lens.values(), key=sum))
    t = [torch.from_numpy(rng.standard_normal((n, heads * hd)).astype(np.float32)).to(DEV).to(BF) for _ in range(4)]
    lam = torch.linspace(0.1, 0.8, heads, device=DEV)
    out = {name: _run(*[x[:sum(l)].clone() for x in t], lam, l, l, heads, hd, causal) for name, l in lens.items()}
    m = sum(short)
    for name, r in out.items():
        for a, b in zip(out["alone"], r):
            if a.shape[0] == m:
                assert torch.equal(a, b[:m]), name
        assert torch.equal(out["alone"][2], r[2][:, :m]), name


def _alike(a, b, exact, tag):
    """The rows of `exact` to the bit.  The others may have been summed in another order: half a step of the type on either side, and what fp32 sums of these sizes
    (scores of up to 2^3 of terms, 2^7 terms in dP - D, 16 times as large as their sum) are off by at most, 2^-9 of the largest value."""
    half = 2.0 ** -8 if a.dtype == BF else 2.0 ** -24
    assert torch.equal(a[exact], b[exact]), tag
    if a.numel():
        assert ((a.double() - b.double()).abs() <= 2 * half * a.double().abs() + 2.0 ** -9 * a.double().abs().max()).all(), tag


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("dt,generic", [(F32, False), (BF, True), (BF, False)])
@pytest.mark.parametrize("heads,n,at", [(2, 300, 140), (2, 90, 67), (16, 700, 0), (16, 700, 700 - 1), (2, 40, 17)])
@pytest.mark.parametrize("hd", [16, 48, 64, 80, 128])
def test_values_that_are_not_finite_stay_where_they_are_seen(bad, dt, generic, heads, n, at, hd):
    """Causal: a key or value row does not touch earlier queries (in the bf16 matrix-core kernels: earlier ones than those within 31 tokens), a query's row
    not the gradients of later keys."""
    reach = 31 if dt == BF and not generic and hd in (64, 128) else 0
    rng = np.random.default_rng(n + hd)
    t = [torch.from_numpy(rng.standard_normal((n, heads * hd)).astype(np.float32)).to(DEV).to(dt) for _ in range(4)]
    lam = torch.linspace(0.1, 0.8, heads, device=DEV)
    clean = _run(*t, lam, [n], [n], heads, hd, True, generic)
    for i in (1, 2):                                    # a key, a value
        s = [x.clone() for x in t]
        s[i][at] = bad
        r = _run(*s, lam, [n], [n], heads, hd, True, generic)
        upto = max(0, at - reach)
        for name, a, b in (("o", clean[0], r[0]), ("o2", clean[1], r[1]), ("dq", clean[3], r[3])):
            _alike(a[:upto], b[:upto], slice(0, upto if reach else at // 64 * 64), (name, i))
        assert torch.equal(clean[2][:, :at], r[2][:, :at]), i
        if i == 2:
            assert not torch.isfinite(r[0][at:]).any()
    for i in (0, 3):                                    # a query, a gradient
        s = [x.clone() for x in t]
        s[i][at] = bad
        r = _run(*s, lam, [n], [n], heads, hd, True, generic)
        first = at + 1 + reach
        for name, a, b in (("dk", clean[4], r[4]), ("dv", clean[5], r[5])):
            _alike(a[first:], b[first:], slice(0 if reach else (at // 64 + 1) * 64 - first, None), (name, i))
        assert not torch.isfinite(r[4 if i == 0 else 5][:at + 1]).all(dim=1).any(), i


@pytest.mark.parametrize("dt,generic", [(F32, False), (BF, True), (BF, False)])
@pytest.mark.parametrize("hd", [16, 64, 128])
def test_products_with_hidden_rows_may_overflow(dt, generic, hd):
    """Causal: a value row and a gradient row of 2^100 each, finite, whose product is not; the value row's query and those behind it have gradients of 0, so that
    nothing sees both.  Earlier queries' gradients and later keys' are what they are without."""
    heads, n, at = 2, 80, 37
    rng = np.random.default_rng(hd)
    t = [torch.from_numpy(rng.standard_normal((n, heads * hd)).astype(np.float32)).to(DEV).to(dt) for _ in range(4)]
    t[3][at:] = 0
    lam = torch.linspace(0.1, 0.8, heads, device=DEV)
    t[3][at - 2] = 2.0 ** 100
    clean = _run(*t, lam, [n], [n], heads, hd, True, generic)
    assert all(torch.isfinite(x).all() for x in clean)
    s = [x.clone() for x in t]
    s[2][at] = 2.0 ** 100
    r = _run(*s, lam, [n], [n], heads, hd, True, generic)
    for name, a, b in (("o", clean[0][:at], r[0][:at]), ("dq", clean[3][:at], r[3][:at]), ("dk", clean[4][at + 1:], r[4][at + 1:]), ("dv", clean[5], r[5])):
        _alike(a, b, slice(0, 0), name)
    assert torch.isfinite(r[6]).all()


def test_more_work_groups_than_a_launch_of_the_matrix_core_kernels_has():
    """64 000 single tokens, 261 heads: one key, so that O2 = V, O = (1 - lambda) V = V / 2 and dV = dO / 2, exactly; dP - D and with it dQ and dK are what two sums of 64
    products in different orders differ by, 128 x 2^-24 of at most 2^10."""
    n, heads, hd = 64000, 261, 64
    assert diff_choice(True, n, heads, hd, True, 1, 1)["general"] and not diff_choice(True, n, heads - 1, hd, True, 1, 1)["general"]
    g = torch.Generator(device=DEV).manual_seed(2)
    q, k, v, d_o = (torch.randn((n, heads * hd), generator=g, device=DEV, dtype=BF) for _ in range(4))
    lam = torch.full((heads,), 0.5, device=DEV)
    o, o2, lse, dq, dk, dv, dlam = _run(q, k, v, d_o, lam, [1] * n, [1] * n, heads, hd, True)
    assert torch.equal(o2, v) and torch.equal(o, v / 2) and torch.equal(dv, d_o / 2)
    assert float(dq.abs().max()) <= 2.0 ** -7 and float(dk.abs().max()) <= 2.0 ** -7
    assert torch.isfinite(dlam).all()


# ------------------------------------------------------------------------------------ rotary positions
def test_rows_of_more_threads_than_a_launch_has():
    """Single pairs of more rows than fit into 2^32 threads: the rows around the border and the last ones get what they get alone, all others are left alone."""
    rows, hd = (1 << 32) // 3 + 1000, 6
    freq = torch.from_numpy(ds.ds_rope_freqs(hd)).to(DEV)
    x = torch.zeros((rows, hd), dtype=BF, device=DEV)
    pos = torch.full((rows,), -1, dtype=torch.int32, device=DEV)
    border = ((1 << 32) - 256) // 3
    at = torch.tensor([0, 1, border - 1, border, border + 1, rows - 2, rows - 1], device=DEV)
    g = torch.Generator(device=DEV).manual_seed(1)
    x[at] = torch.randn((len(at), hd), generator=g, device=DEV).to(BF)
    x[border + 2] = 5.0
    pos[at] = torch.arange(3, 3 + len(at), dtype=torch.int32, device=DEV)
    one = x[at].contiguous()
    before = one.clone()
    ds.ds_rope(x, x, pos, freq, 1, hd, hd)
    ds.ds_rope(one, one, pos[at].contiguous(), freq, 1, hd, hd)
    torch.cuda.synchronize()
    assert torch.equal(x[at], one) and not torch.equal(one, before)
    assert (x[border + 2] == 5.0).all() and not x[2:border - 1:9973].any() and not x[border + 3:rows - 2:9973].any()


# ------------------------------------------------------------------------------------ numbers of more than 32 bits
def test_strides_rows_and_lengths_beyond_32_bits_are_refused():
    """(Taken modulo 2^32 each of these would be a call on other rows.)"""
    heads, hd, ld = 2, 64, (1 << 32) + 256
    w = heads * hd
    far = torch.empty(ld + w, dtype=BF, device=DEV).as_strided((2, w), (ld, 1))      # two rows 2^32 + 256 elements apart
    near = [torch.zeros((2, w), dtype=BF, device=DEV) for _ in range(5)]
    lam, lse = torch.zeros(heads, device=DEV), torch.zeros((2 * heads, 2), device=DEV)
    scratch = torch.zeros(int(ds.ds_diff_attention_scratch_bytes(heads, 2, 2, 1)), dtype=torch.uint8, device=DEV)
    rest = (i32([0]), i32([2]), i32([0]), i32([2]), heads, hd, True)

    def forward(q=near[0], k=near[1], v=near[2], o=near[3], longest=2):
        ds.ds_diff_attention_fwd(q, k, v, lam, o, lse, *rest, longest, longest, scratch)

    forward()
    for kw in (dict(q=far), dict(k=far), dict(v=far), dict(o=far), dict(longest=(1 << 32) + 2)):
        with pytest.raises(ValueError):
            forward(**kw)
    with pytest.raises(ValueError):
        ds.ds_diff_attention_bwd(*near[:3], lam, far, far, far, lse, *near[:3], lam, *rest, 2, 2, scratch)
    x = torch.empty(((1 << 32) + 2, 8), dtype=BF, device=DEV)
    with pytest.raises(ValueError):
        ds.ds_resid_norm_fwd(x, x, x, torch.empty(1, device=DEV).expand(4, (1 << 32) + 2))
    with pytest.raises(ValueError):
        ds.ds_resid_norm_bwd(x, x, x, lse, x, x, lam)
    with pytest.raises(ValueError):
        ds.ds_rope(x, x, torch.empty(1, dtype=torch.int32, device=DEV).expand((1 << 32) + 2), torch.zeros(4, dtype=torch.float64, device=DEV), 1, 8, 8)
    torch.cuda.synchronize()
