"""Which kernels a call of attention with a relative position bias and of the gated feed-forward block goes to, on the host: both sides of the borders of the rules."""
import ctypes

import pytest

from paper_2311_10418_amd import binding as ds

REL = ("general", "splits", "direct", "few", "direct_k", "dq_columns", "dkv_columns", "shares")


def rel(bf16=True, n_seq=16, heads=16, hd=64, max_q=100, max_k=100, q_rows=None, k_rows=None, backward=False, generic=False, causal=False):
    out = (ctypes.c_int32 * len(REL))()
    ds.lib().ds_rel_attention_choice(int(bf16), n_seq, heads, hd, max_q, max_k, q_rows or n_seq * max_q, k_rows or n_seq * max_k, int(backward) + 2 * int(causal), int(generic), out)
    return dict(zip(REL, out))


def glu(rows, d, ff, dx=False, floats=1 << 24):
    out = (ctypes.c_int32 * 2)()
    ds.lib().ds_gated_mlp_choice(rows, d, ff, int(dx), ctypes.c_int64(floats), out)
    return bool(out[0]), out[1]


def test_matrix_cores():
    for hd in range(8, 129, 8):
        for backward in (False, True):
            assert rel(hd=hd, backward=backward)["general"] == (hd not in (64, 128))
            assert rel(bf16=False, hd=hd, backward=backward)["general"] == rel(hd=hd, generic=True, backward=backward)["general"] == 1


def test_single_tokens():
    assert rel(bf16=False, max_q=1, max_k=1000)["few"] == 1 and rel(bf16=False, max_q=2, max_k=1000)["few"] == 0
    assert rel(max_q=1, max_k=1000)["few"] == 0 and rel(hd=96, max_q=1, max_k=1000)["few"] == 1
    assert rel(bf16=False, max_q=1, max_k=1000, generic=True)["few"] == rel(bf16=False, max_q=1, max_k=1000, backward=True)["few"] == 0
    # its shares: four work-groups to a compute unit, of 2048 / lanes keys at least (16 lanes hold a row of 64 floats)
    assert rel(bf16=False, max_q=1, max_k=128)["splits"] == 1 and rel(bf16=False, max_q=1, max_k=129)["splits"] == 2
    assert rel(bf16=False, max_q=1, max_k=10000)["splits"] == 4 and rel(bf16=False, n_seq=1, max_q=1, max_k=100000)["splits"] == 64 and rel(bf16=False, n_seq=65, max_q=1, max_k=10000)["splits"] == 1


def test_work_groups_share_keys():
    assert rel(max_q=8, max_k=128)["splits"] == 1 and rel(max_q=8, max_k=129)["splits"] == 2
    assert rel(max_q=64, max_k=4000)["splits"] == 2 and rel(max_q=8, max_k=4000, q_rows=16 * 64 + 1)["splits"] == 1
    assert rel(n_seq=17, max_q=8, max_k=4000)["splits"] == 1 and rel(n_seq=9, hd=128, max_q=8, max_k=4000)["splits"] == 1 and rel(n_seq=8, hd=128, max_q=8, max_k=4000)["splits"] == 2
    assert rel(bf16=False, max_q=8, max_k=4000)["splits"] == 3 and rel(n_seq=1, heads=1, max_q=8, max_k=10000)["splits"] == 64 and rel(n_seq=1, heads=1, max_q=8, max_k=300)["splits"] == 5
    assert rel(max_q=8, max_k=4000, backward=True)["splits"] == 1


def test_scratch_holds_the_shares():
    for bf16 in (False, True):
        for hd in (32, 64, 96, 128):
            for n_seq in (1, 3, 16, 40):
                for max_q in (1, 5, 64, 65, 1000):
                    for max_k in (1, 200, 5000):
                        c = rel(bf16, n_seq, 4, hd, max_q, max_k)
                        need = 4 * n_seq * max_q * c["splits"] * (hd + 4) * 4 if c["splits"] > 1 else 0
                        assert ds.ds_rel_attention_scratch_bytes(4, hd, 128, n_seq * max_q, n_seq * max_k, n_seq) >= need


def test_no_list():
    assert rel(max_q=128, max_k=128)["direct"] == 1 and rel(max_q=128, max_k=128, backward=True)["direct_k"] == 1
    assert rel(n_seq=31, max_q=523, max_k=523)["direct"] == 5 and rel(n_seq=31, max_q=523, max_k=523, backward=True)["direct_k"] == 5
    # 8 sequences that may have 5 blocks each: the list of so many rows is 4/5 of that, or shorter
    assert rel(n_seq=8, max_q=600, max_k=600, q_rows=128 * 24)["direct"] == 5 and rel(n_seq=8, max_q=600, max_k=600, q_rows=128 * 24 - 1)["direct"] == 0
    assert rel(n_seq=8, max_q=600, max_k=600, k_rows=128 * 24 - 1, backward=True)["direct"] == 0
    # never more blocks than slots
    for n_seq in (1, 2, 5, 100):
        for max_q in (1, 100, 129, 1000, 9000):
            for q_rows in (max_q, n_seq * max_q // 2 + max_q, n_seq * max_q, n_seq * max_q + 7):
                c = rel(n_seq=n_seq, max_q=max_q, max_k=max_q, q_rows=q_rows, k_rows=q_rows, backward=True)
                assert c["direct"] * n_seq <= q_rows // 64 + n_seq and c["direct_k"] * n_seq <= q_rows // 64 + n_seq


def test_work_groups_share_blocks():
    def shares(n_seq, length, heads, hd, **more):
        return rel(n_seq=n_seq, heads=heads, hd=hd, max_q=length, max_k=length, backward=True, **more)["shares"]

    assert shares(1, 1565, 4, 128) > 1 and shares(1, 511, 4, 64) == 1 and shares(1, 512, 4, 64) == 2 and shares(4, 600, 9, 128) == 1 and shares(31, 523, 16, 64) == 1
    assert shares(1, 1565, 4, 128, bf16=False) == shares(1, 1565, 4, 128, generic=True) == shares(1, 1565, 4, 96) == 1
    assert shares(1, 1565, 4, 128, causal=True) > 1 and shares(3, 1193, 5, 128, causal=True) == 2 and shares(2, 1181, 16, 64, causal=True) == 1
    assert rel(n_seq=1, heads=4, max_q=1565, max_k=1565)["shares"] == 1                     # forward: shares of keys
    assert rel(n_seq=1, heads=4, hd=128, max_q=1565, max_k=1565, causal=True)["splits"] > 1 and rel(n_seq=1, heads=4, hd=128, max_q=1565, max_k=511)["splits"] == 1
    assert rel(n_seq=4, heads=9, hd=128, max_q=600, max_k=600)["splits"] == 1 and rel(n_seq=1, heads=4, max_q=1565, max_k=1565, bf16=False)["splits"] == 1
    for n_seq in (1, 2, 7):
        for length in (100, 600, 3000, 20000):
            for heads in (1, 3, 16):
                for hd in (64, 128):
                    s = max(shares(n_seq, length, heads, hd), shares(n_seq, length, heads, hd, causal=True))
                    assert 1 <= s <= 8 and (s == 1 or s * (n_seq * length // 128 + n_seq) * heads <= 3 * 256 and length >= 256 * s and 12 * s * n_seq * length * heads * hd <= 56 << 20)
                    rows = n_seq * length
                    assert ds.ds_rel_attention_scratch_bytes(heads, hd, 128, rows, rows, n_seq) >= 4 * 3 * s * rows * heads * hd * (s > 1)


def test_general_columns():
    assert rel(bf16=False, n_seq=23, heads=4, max_q=177, max_k=177)["dq_columns"] == 32 and rel(bf16=False, n_seq=43, heads=4, max_q=177, max_k=177)["dq_columns"] == 64
    assert rel(bf16=False, hd=104, n_seq=1, heads=1, max_q=177, max_k=177)["dkv_columns"] == 64


def test_gated_block_tiles():
    assert glu(957, 1024, 2816) == (False, 1) and glu(65629, 1024, 2816) == (True, 1) and glu(65629, 1024, 2816, dx=True)[0]
    assert glu(65629, 1000, 2816) == (False, 1) and glu(65629, 1024, 2824) == (False, 1)                        # sizes that the large tiles do not take
    assert glu(65629, 1024 + 64, 2816)[0] and not glu(65629, 1024 + 64, 2816, dx=True)[0]
    big, splits = glu(957, 1024, 2816, dx=True)
    assert not big and splits > 1 and glu(957, 1024, 2816, dx=True, floats=0)[1] == 1
    for rows in (65, 300, 957, 3000):
        for floats in (0, 1 << 18, 1 << 24):
            big, splits = glu(rows, 512, 1408, dx=True, floats=floats)
            assert splits == 1 or splits * rows * 512 <= floats


def test_shares_of_weight_gradients():
    def shares(rows, d, ff, floats=1 << 24):
        return glu(rows, d, ff, 2, floats)[1]

    assert shares(1418, 1856, 960) == 1 and shares(64, 8, 8) == 1 and shares(20000, 1000, 1000) > 1 and shares(65536, 128, 192) > 32
    for rows in (1, 65, 1000, 65536):
        for d, ff in ((128, 192), (8, 8), (1000, 1000), (512, 4416), (65536, 65536)):
            for floats in (0, 1 << 16, 1 << 24, 1 << 40):
                s = shares(rows, d, ff, floats)
                assert 1 <= s <= 128 and (s == 1 or 2 * s * d * ff <= floats and s <= (rows + 63) // 64)
