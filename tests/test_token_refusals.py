"""What the lookup, the dropout and the sampling refuse, before anything is launched (no GPU)."""
import ctypes

import pytest
import torch

import paper_1409_5705_b200 as S


def embed(**k):
    d = dict(tokens=100, dim=20, ldt=0, table_dtype=0, out_dtype=1, scale=1.0, max_ids=50, stream=0)
    d.update(k)
    return S.sfb_embed_config(*(d[n] for n, _ in S.sfb_embed_config._fields_))


@pytest.mark.parametrize("change,code", [
    (dict(tokens=0), -1), (dict(dim=-1), -1), (dict(ldt=-1), -1), (dict(table_dtype=3), -1), (dict(out_dtype=-1), -1), (dict(max_ids=-1), -1),
    (dict(scale=float("nan")), -1), (dict(scale=float("inf")), -1), (dict(ldt=19), -3), (dict(tokens=(1 << 30) + 1), -3), (dict(dim=(1 << 24) + 1), -3),
    (dict(max_ids=(1 << 26) + 1), -3),
])
def test_embed_configs(change, code):
    n = ctypes.c_size_t(0)
    assert S.lib().sfb_embed_workspace_bytes(ctypes.byref(embed(**change)), ctypes.byref(n)) == code


def test_embed_arguments():
    L, n, h, cfg = S.lib(), ctypes.c_size_t(0), ctypes.c_void_p(1), embed()
    assert L.sfb_embed_workspace_bytes(None, ctypes.byref(n)) == -1 and L.sfb_embed_workspace_bytes(ctypes.byref(cfg), None) == -1
    assert L.sfb_embed_workspace_bytes(ctypes.byref(cfg), ctypes.byref(n)) == 0 and n.value >= 4 * 50 * 4
    init = lambda table, ws, nbytes, out=ctypes.byref(h): L.sfb_embed_init(ctypes.byref(cfg), table, ws, nbytes, out)
    assert init(None, 1024, n.value) == -1 and not h.value and init(16, None, n.value) == -1 and init(16, 1024, n.value, None) == -1
    assert init(18, 1024, n.value) == -2 and init(16, 512, n.value) == -2 and init(16, 1024, n.value - 1) == -4
    assert L.sfb_embed_forward(None, 0, None, None, 0, None, 0) == -1
    assert L.sfb_embed_backward(None, 0, None, None, 0, None, 0, 1.0, 0, None, 0) == -1
    assert L.sfb_embed_get_status(None, None) == -1 and L.sfb_embed_destroy(None) == -1 and L.sfb_embed_last_cuda_error(None) == 0


def test_dropout_arguments():
    L, h = S.lib(), ctypes.c_void_p(1)
    for p in (-0.1, 1.1, float("nan")):
        assert L.sfb_dropout_init(p, 16, None, ctypes.byref(h)) == -1 and not h.value
    assert L.sfb_dropout_init(0.5, None, None, ctypes.byref(h)) == -1 and L.sfb_dropout_init(0.5, 16, None, None) == -1
    assert L.sfb_dropout_init(0.5, 12, None, ctypes.byref(h)) == -2
    assert L.sfb_dropout_apply(None, 0, 0, 1, 0, None, 0, None, 0, None, 0) == -1
    assert L.sfb_dropout_destroy(None) == -1 and L.sfb_dropout_last_cuda_error(None) == 0


@pytest.mark.parametrize("classes,most,dtype,code", [(0, 1, 0, -1), (5, -1, 0, -1), (5, 1, 3, -1), ((1 << 30) + 1, 1, 0, -3), (5, (1 << 27) + 1, 0, -3)])
def test_sampler_configs(classes, most, dtype, code):
    h = ctypes.c_void_p(1)
    assert S.lib().sfb_sampler_init(ctypes.byref(S.sfb_sampler_config(classes, most, dtype, None)), ctypes.byref(h)) == code and not h.value


def test_sampler_arguments():
    L = S.lib()
    assert L.sfb_sampler_init(None, ctypes.byref(ctypes.c_void_p())) == -1
    assert L.sfb_sampler_init(ctypes.byref(S.sfb_sampler_config(5, 1, 0, None)), None) == -1
    assert L.sfb_sample(None, 1, 16, 5, 16, None, None, None, None, 16, None, None) == -1
    assert L.sfb_sampler_destroy(None) == -1 and L.sfb_sampler_last_cuda_error(None) == 0


def test_struct_layouts_match_the_header():
    import os
    import subprocess
    import tempfile
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    prog = '#include <stdio.h>\n#include "sfb.h"\nint main(){printf("%zu %zu", sizeof(sfb_embed_config), sizeof(sfb_sampler_config));return 0;}\n'
    with tempfile.TemporaryDirectory() as d:
        c, exe = os.path.join(d, "t.c"), os.path.join(d, "t")
        open(c, "w").write(prog)
        subprocess.check_call(["gcc", "-I" + os.path.join(root, "include"), c, "-o", exe])
        assert list(map(int, subprocess.check_output([exe]).split())) == [ctypes.sizeof(S.sfb_embed_config), ctypes.sizeof(S.sfb_sampler_config)]


def test_tensors_that_are_not_on_the_gpu():
    with pytest.raises(ValueError):
        S.Embedding(torch.zeros(4, 8), 3)
    with pytest.raises(ValueError):
        S.Dropout(0.1, torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError):
        S.Dropout(0.1, torch.zeros(2))
