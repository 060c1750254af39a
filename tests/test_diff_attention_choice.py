"""Which kernels a call of differential attention goes to, on the host: both sides of every border of the rules."""
import pytest

from paper_2311_10418_amd import binding as ds
from helpers import diff_choice


def _sides(key, low, high, **kw):
    """diff_choice's `key` with the one argument that the dict names, at a value and one further."""
    (name, at), = kw.pop("at").items()
    a, b = diff_choice(**{**kw, name: at})[key], diff_choice(**{**kw, name: at + 1})[key]
    assert (a, b) == (low, high), (key, name, at, a, b)


def test_bf16_heads_of_64_and_128_take_the_matrix_cores():
    for hd in range(16, 129, 16):
        for backward in (False, True):
            a = dict(n_seq=3, heads=2, hd=hd, causal=True, max_q=50, max_k=50, backward=backward)
            assert diff_choice(True, **a)["general"] == (hd not in (64, 128))
            assert diff_choice(False, **a)["general"] == diff_choice(True, generic=True, **a)["general"] == 1
            for n_seq, n in ((1, 1), (1, 16), (1, 17), (1000, 16), (1000, 5)):       # neither the number of sequences nor their length matters
                assert diff_choice(True, **dict(a, n_seq=n_seq, max_q=n, max_k=n))["general"] == (hd not in (64, 128))


def test_no_list_for_sequences_of_one_block():
    few = dict(bf16=True, n_seq=16, heads=16, hd=128, causal=True, max_q=128, max_k=128)
    for backward in (False, True):
        assert diff_choice(**few, backward=backward)["direct"] == 1
        _sides("direct", 1, 0, at=dict(n_seq=16), **{k: v for k, v in few.items() if k != "n_seq"}, backward=backward)
        _sides("direct", 1, 0, at=dict(max_q=128), **{k: v for k, v in few.items() if k != "max_q"}, backward=backward)
    long_keys = dict(few, max_k=129)
    assert diff_choice(**long_keys)["direct"] == 1 and diff_choice(**long_keys, backward=True)["direct"] == 0
    short = dict(bf16=True, n_seq=256, heads=16, hd=64, causal=True, max_q=64, max_k=64)               # 4 096 items of 64 rows: 2^18
    assert diff_choice(**short)["direct"] == 1
    _sides("direct", 1, 0, at=dict(max_q=64), **{k: v for k, v in short.items() if k != "max_q"})
    _sides("direct", 1, 0, at=dict(max_k=128), **{k: v for k, v in short.items() if k != "max_k"})
    assert diff_choice(**dict(short, hd=128))["direct"] == 0


def test_short_queries_share_their_keys():
    one = dict(bf16=True, n_seq=16, heads=16, hd=64, causal=False, max_q=32, max_k=1000)
    _sides("sharing", 4, 2, at=dict(max_q=32), **{k: v for k, v in one.items() if k != "max_q"})
    _sides("sharing", 2, 1, at=dict(max_q=64), **{k: v for k, v in one.items() if k != "max_q"})
    _sides("sharing", 1, 4, at=dict(max_k=320), **{k: v for k, v in one.items() if k != "max_k"})
    _sides("sharing", 4, 1, at=dict(n_seq=16), **{k: v for k, v in one.items() if k != "n_seq"})
    _sides("sharing", 4, 1, at=dict(n_seq=8), **dict({k: v for k, v in one.items() if k != "n_seq"}, hd=128))
    assert diff_choice(**dict(one, causal=True))["sharing"] == 1


def test_work_groups_share_keys_forward():
    bf = dict(bf16=True, n_seq=1, heads=16, hd=64, causal=False, max_q=1, max_k=512)
    assert [diff_choice(**dict(bf, max_k=k))["splits"] for k in (320, 321, 512, 1024, 4096, 32768)] == [1, 3, 4, 8, 16, 32]
    assert [diff_choice(**dict(bf, hd=128, max_k=k))["splits"] for k in (320, 321, 512, 4096, 32768)] == [1, 3, 4, 16, 16]
    assert [diff_choice(**dict(bf, n_seq=n, max_k=4096))["splits"] for n in (2, 8, 15, 16)] == [8, 4, 2, 2]      # from 1 024 keys each on two for a compute unit
    assert [diff_choice(**dict(bf, n_seq=16, hd=64, max_k=k))["splits"] for k in (1024, 1025)] == [1, 2]
    f32 = dict(bf, bf16=False)
    assert [diff_choice(**dict(f32, max_k=k))["splits"] for k in (128, 129, 512, 4096)] == [1, 3, 8, 32]
    assert diff_choice(**dict(f32, heads=1, max_k=1 << 20))["splits"] == 64                                   # a lane of the joining wavefront each
    for a in (bf, f32):
        a = dict(a, max_k=4096)
        _sides("splits", diff_choice(**a)["splits"], 1, at=dict(max_q=64), **{k: v for k, v in a.items() if k != "max_q"})
        assert diff_choice(**a, q_rows=65)["splits"] == 1       # rows of the query tensor beyond 64 for each sequence: see the header
        assert diff_choice(**dict(a, causal=True))["splits"] == 1 and diff_choice(**a, backward=True)["splits"] == 1


def test_the_scratch_holds_the_shares():
    """Whatever a call is: maxima, sums and outputs of every share, for each row and head, behind the lists (at least 256 bytes)."""
    for bf16 in (False, True):
        for hd in (16, 64, 96, 128):
            for heads in (1, 3, 16):
                for n_seq in (1, 7, 16):
                    for q in (1, 33, 64):
                        for k in (100, 129, 321, 1025, 9999, 1 << 18):
                            c = diff_choice(bf16, n_seq, heads, hd, False, q, k)
                            need = heads * n_seq * q * (c["splits"] * (2 * hd + 4) * 4 if c["splits"] > 1 else 0)
                            assert ds.ds_diff_attention_scratch_bytes(heads, n_seq * q, n_seq * k, n_seq) >= 256 + need


@pytest.mark.parametrize("which,length", [("dq_columns", "max_q"), ("dkv_columns", "max_k")])
def test_columns_of_the_fp32_backward_kernels(which, length):
    a = dict(bf16=False, n_seq=32, heads=4, hd=64, causal=True, max_q=100, max_k=100, backward=True)
    for hd in (16, 64, 96):
        _sides(which, 32, 64, at={length: 255}, **{k: v for k, v in dict(a, hd=hd).items() if k != length})      # 128 pairs of 4 blocks: two for a compute unit
    assert diff_choice(**dict(a, hd=112))[which] == 64


def test_grids_stay_below_two_to_the_32_threads():
    """16 777 215 work-groups of 256 threads: beyond, bf16 calls take the general kernels, whose grids have heads and sequences on axes of their own."""
    a = dict(bf16=True, n_seq=64000, hd=64, causal=True, max_q=1, max_k=1)
    for backward in (False, True):
        _sides("general", 0, 1, at=dict(heads=260), **a, backward=backward)          # (500 + 64 000 + 8) x 260
        assert diff_choice(True, 1, 16, 64, False, 1, (1 << 31) - 1, 1, (1 << 31) - 1, backward)["general"] == 1
        assert diff_choice(True, 1, 16, 64, False, 1, 1 << 26, 1, 1 << 26, backward)["general"] == 0
