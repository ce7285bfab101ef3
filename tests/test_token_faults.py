"""What once went wrong around lookup, dropout and sampling, as far as it shows without a GPU."""
import ctypes
import os
import re

import pytest

import paper_1409_5705_b200 as S

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1409_5705_b200", "csrc")


@pytest.mark.parametrize("name", ["sfb_elem.cuh", "sfb_embed.cu", "sfb_sample.cu"])
def test_kernels_that_start_early_read_coherently(name):
    """A kernel that is there before the one ahead of it has ended may not load through the path for data that nobody writes while it runs: what that
    holds may be older than its wait, and the compiler may move such a load above it."""
    code = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
    assert not re.search(r"__ldg\s*\(|ld\.global(\.\w+)*\.nc", code)


def closed_dropout():
    """As ``Dropout.close`` leaves one; the library never sees it."""
    drop = S.Dropout.__new__(S.Dropout)
    drop._h = ctypes.c_void_p()
    drop.close()
    return drop


def test_a_closed_dropout_is_not_none():
    """A handle that is gone may not be taken for no dropout at all."""
    plan = S.Embedding.__new__(S.Embedding)
    assert plan._drop(None) is None
    for bad in (closed_dropout(), 0.1, S.Embedding):
        with pytest.raises(ValueError):
            plan._drop(bad)


@pytest.mark.parametrize("max_ids,dim,code", [(65_472, 1 << 24, 0), (65_473, 1 << 24, -3), (1 << 26, 16_376, 0), (1 << 26, 16_377, -3), (0, 1 << 24, 0), (1 << 26, 1, 0)])
def test_what_a_lookup_of_that_size_would_refuse_is_refused_before(max_ids, dim, code):
    """ceil(max_ids / 64) * ceil(dim / 8) up to 2^31 - 257, as include/sfb.h has it: a handle that there is takes every call of up to max_ids."""
    cfg, n = S.sfb_embed_config(100, dim, 0, 0, 1, 1.0, max_ids, None), ctypes.c_size_t(0)
    assert S.lib().sfb_embed_workspace_bytes(ctypes.byref(cfg), ctypes.byref(n)) == code
    h = ctypes.c_void_p(1)
    assert code == 0 or (S.lib().sfb_embed_init(ctypes.byref(cfg), 1024, 1024, 1 << 62, ctypes.byref(h)) == code and not h.value)
