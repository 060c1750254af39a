"""How the 256 x 256 tiles of the gated feed-forward block are divided, on the host: what tests/test_gpu_gated_mlp_tiles.py counts on."""
import ctypes

import pytest

from paper_2311_10418_amd import binding as ds


def division(rows, d, ff, dx, floats):
    out = (ctypes.c_int32 * 5)()
    ds.lib().ds_gated_mlp_division(rows, d, ff, int(dx), ctypes.c_int64(floats), out)
    return tuple(out)


@pytest.mark.parametrize("dx", [False, True])
def test_pieces_fit_the_workspace(dx):
    for rows in (1, 300, 2500, 8205, 33001, 65629):
        for d, ff in ((256, 1024), (1024, 448), (2048, 64), (1024, 2816)):
            for floats in (0, 4, 16, 17, 20, 65536, 65552, 600000, 1 << 20, 1 << 24, (1 << 24) + 16):
                _, whole, cut, pieces, persistent = division(rows, d, ff, dx, floats)
                tiles = (rows + 255) // 256 * (d // 256 if dx else (ff + 127) // 128)
                assert whole + cut == tiles and (cut > 0) == (pieces > 1)
                assert cut * pieces * 65536 + 16 <= floats or not cut
                assert not persistent or floats > 19 and whole >= 512


def test_divisions_that_are_tested():
    assert division(65629, 1024, 2816, False, 1 << 24) == (1, 5632, 22, 4, 1) and division(65629, 1024, 2816, True, 1 << 24) == (1, 1024, 4, 22, 1)
    assert division(33001, 1024, 448, False, 1 << 24) == (1, 512, 4, 4, 1) and division(33001, 1024, 448, True, 1 << 24) == (1, 512, 4, 3, 1)
