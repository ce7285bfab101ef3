"""Sizes at the ends of what the adapters' handles allow, on the host (no GPU)."""
import os
import subprocess
import sys

import pytest

import paper_1409_5705_b200 as S

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("rows,cols,ldw,ldu,adapters,rank", [(64, 64, 0, 0, 2, 4), (1, 1, 8, 8, 1, 1), (10_000, 20_000, 0, 0, 65_536, 128), (1 << 26, 64, 0, 0, 1, 1)])
def test_no_room_for_samples(rows, cols, ldw, ldu, adapters, rank):
    """A handle of max_samples = 0, whose calls are of no samples.  In a process of its own: a division by zero would end this one."""
    code = ("import paper_1409_5705_b200 as S\n"
            f"sizes = [S.sfb_adapter_workspace_bytes(S.sfb_adapter_config({rows}, {cols}, {ldw}, {ldu}, {ldw}, {adapters}, {rank}, m, 0)) for m in (0, 1)]\n"
            "assert 0 < sizes[0] <= sizes[1], sizes\n")
    done = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, (done.returncode, done.stderr[-500:])


@pytest.mark.parametrize("rows,cols,adapters,rank", [(1000, 20_000, 64, 8), (10_000, 5_000, 8, 64), (100, 64, 300, 128)])
def test_room_grows_with_the_samples(rows, cols, adapters, rank):
    """Workspace for more samples holds that of fewer ones."""
    before = 0
    for m in (1, 16, 17, 64, 65, 128, 129, 1000, 5000, 40_000, 1 << 20):
        got = S.sfb_adapter_workspace_bytes(S.sfb_adapter_config(rows, cols, 0, (rows + 7) // 8 * 8, 0, adapters, rank, m, 0))
        assert got >= before, m
        before = got
