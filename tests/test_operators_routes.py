"""Which rows of drafted trees are split over workgroups, as the workspace
queries tell: one rule on units and chunks, for all of its range."""
import ctypes

import pytest

from paper_2511_00576_amd import _lib


def workspace(units, chunks, d=64, T=16):
    """fp32 cache of `units` (sequence, kv head) pairs of 16 columns whose longest
    row has `chunks` chunks of 32 keys: one of summaries, one drafted, the window's."""
    W, C = 32 * (chunks - 3), 32
    c = _lib.EvaRCacheStruct(B=units, H=1, H_kv=1, d=d, W=W, C=C, dtype=_lib.EVA_F32, window=0, R=W + 32, S_max=64,
                             max_tok=W + 700, n_tok=0x50000, arrive=0x60000, k_ring=0x10000, vt_ring=0x20000,
                             k_sum=0x30000, vt_sum=0x40000)
    return _lib.load().eva_rtree_workspace_bytes(ctypes.byref(c), T)


@pytest.mark.parametrize("units", [1, 8, 24, 33, 40, 48, 60, 72, 80])
def test_fp32_rows_of_few_units_are_split_from_nine_chunks(units):
    assert all(workspace(units, n) == 0 for n in range(5, 9))
    assert all(workspace(units, n) > 0 for n in range(9, 21))


@pytest.mark.parametrize("units,most", [(81, 12), (96, 12), (128, 12), (129, 20), (160, 20), (240, 20)])
def test_fp32_rows_of_more_units(units, most):
    assert all(workspace(units, n) == 0 for n in range(5, most + 1))
    assert workspace(units, most + 1) > 0
