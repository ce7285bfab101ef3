"""sfb_adapter_get_plan (host arithmetic; no GPU)."""
import ctypes

import pytest

import paper_1409_5705_b200 as S


def config(n, rows, cols, adapters, rank):
    up = lambda d: (d + 7) // 8 * 8
    return S.sfb_adapter_config(rows, cols, up(cols), up(rows), up(cols), adapters, rank, n, 0)


def test_arguments():
    cfg, o = config(50, 100, 64, 3, 8), [ctypes.c_int32(7) for _ in range(4)]
    refs = [ctypes.byref(x) for x in o]
    L = S.lib()
    assert L.sfb_adapter_get_plan(ctypes.byref(cfg), 50, 0, *refs) == 0 and [x.value for x in o] == [0, 0, 0, 0]
    assert L.sfb_adapter_get_plan(ctypes.byref(cfg), 0, 1, *refs) == 0 and o[3].value == 0
    assert L.sfb_adapter_get_plan(ctypes.byref(cfg), 51, 0, *refs) == -3 and L.sfb_adapter_get_plan(ctypes.byref(cfg), -1, 0, *refs) == -1
    assert L.sfb_adapter_get_plan(None, 1, 0, *refs) == -1
    for k in range(4):
        assert L.sfb_adapter_get_plan(ctypes.byref(cfg), 1, 0, *(None if j == k else r for j, r in enumerate(refs))) == -1
    with pytest.raises(S.SfbError):
        S.sfb_adapter_get_plan(config(50, 100, 64, 3, 200), 1)


@pytest.mark.parametrize("n,rows,cols,adapters,rank,backward,want", [
    (1, 10_000, 5_000, 16, 16, False, (0, 0, 0, 0)),    # a few products: fp32 FMAs
    (16, 130, 25_000, 5, 128, False, (1, 14, 0, 0)),    # 391 k-blocks over 29 parts of five chunks
    (4_100, 72, 7_000, 3, 16, False, (1, 14, 0, 0)),    # 110 over eight
    (7_000, 72, 64, 1, 20, True, (1, 2, 0, 14)),        # 110 of the samples over eight shares
    (1_024, 1_000, 9_000, 64, 8, True, (0, 0, 1, 16)),
])
def test_ways(n, rows, cols, adapters, rank, backward, want):
    assert S.sfb_adapter_get_plan(config(n, rows, cols, adapters, rank), n, backward) == want
