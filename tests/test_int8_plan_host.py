"""The tiles that moe_expert_ffn_plan names on an 8-bit handle: the persistent loop's are 256 features wide, however
tiles of the other kernels would be cut at that size."""
import ctypes as C

import pytest

from test_abi_host import L  # noqa: F401
from test_int8_host import INT8

GROUPED = 2


def _plan(L, N, E, d, f):  # noqa: F811
    from paper_2402_07033_amd import binding
    p = binding.FfnPlan()
    assert L.moe_expert_ffn_plan(N, E, d, f, INT8, GROUPED, C.byref(p)) == 0 and p.path == GROUPED
    return p.up_tile_rows, p.up_tile_features, p.down_tile_rows, p.down_tile_features


@pytest.mark.parametrize("E,d,f,N,rows", [
    (8, 4096, 14336, 8192, 256), (8, 4096, 14336, 8448, 256), (8, 4096, 14336, 4608, 256), (8, 4096, 14336, 2320, 256),
    (16, 4096, 6400, 2200, 192), (16, 4096, 6400, 2600, 192), (8, 4096, 14336, 1400, 192), (64, 2048, 1408, 24576, 256)])
def test_plans_of_the_persistent_loop(L, E, d, f, N, rows):  # noqa: F811
    assert _plan(L, N, E, d, f) == (rows, 256, rows, 256)


@pytest.mark.parametrize("E,d,f", [(8, 4096, 14336), (16, 4096, 6400), (64, 2048, 1408), (1, 512, 384), (5, 2304, 1152)])
def test_whole_tiles_of_both_projections_are_the_persistent_loop(L, E, d, f):  # noqa: F811
    """(These shapes it serves; it runs where the tiles of both projections would have 256 rows.)"""
    seen = set()
    for N in list(range(40 * E, 700 * E, max(1, 13 * E // 2))) + list(range(20000, 60000, 777)):
        up, uf, down, df = _plan(L, N, E, d, f)
        if up == down and up in (256, 192):
            assert (uf, df) == (256, 256), N
            seen.add(up)
    assert 256 in seen


def test_other_tiles_keep_their_features(L):  # noqa: F811
    assert _plan(L, 2048, 1, 14272, 64)[2:] == (256, 224)   # f that the persistent loop does not serve
    assert _plan(L, 40 * 8, 8, 4096, 14336) == (128, 128, 128, 128)
    assert _plan(L, 60, 1, 64, 64) == (32, 128, 32, 128)
