"""What the adapters and the clipping refuse, before anything is launched (no GPU)."""
import ctypes

import pytest
import torch

import paper_1409_5705_b200 as S


def config(**k):
    d = dict(rows=100, cols=64, ldw=0, ldu=104, ldv=0, adapters=3, rank=8, max_samples=50, stream=0)
    d.update(k)
    return S.sfb_adapter_config(*(d[n] for n, _ in S.sfb_adapter_config._fields_))


@pytest.mark.parametrize("change,code", [
    (dict(rows=0), -1), (dict(cols=-4), -1), (dict(adapters=0), -1), (dict(rank=0), -1), (dict(max_samples=-1), -1), (dict(ldu=-8), -1),
    (dict(ldu=0), -3),                                  # 100 rows without a pitch: not a multiple of 8
    (dict(ldu=96), -3), (dict(ldw=68), -3), (dict(ldv=60), -3), (dict(rank=129), -3), (dict(adapters=65537), -3),
    (dict(max_samples=1 << 23), -3), (dict(rows=1 << 27, ldu=1 << 27), -3),
])
def test_adapter_configs(change, code):
    n = ctypes.c_size_t(0)
    assert S.lib().sfb_adapter_workspace_bytes(ctypes.byref(config(**change)), ctypes.byref(n)) == code


def test_adapter_arguments():
    L, n, h = S.lib(), ctypes.c_size_t(0), ctypes.c_void_p(1)
    cfg = config()
    assert L.sfb_adapter_workspace_bytes(None, ctypes.byref(n)) == -1 and L.sfb_adapter_workspace_bytes(ctypes.byref(cfg), None) == -1
    assert L.sfb_adapter_workspace_bytes(ctypes.byref(cfg), ctypes.byref(n)) == 0 and n.value >= 50 * 8 * 4 * 2
    for args in ((None, 16, 16, 16, 1024), (16, None, 16, 16, 1024), (16, 16, None, 16, 1024), (16, 16, 16, None, 1024), (16, 16, 16, 16, None)):
        assert L.sfb_adapter_init(ctypes.byref(cfg), *args, n.value, ctypes.byref(h)) == -1 and not h.value
    for args in ((8, 16, 16, 16, 1024), (16, 8, 16, 16, 1024), (16, 16, 8, 16, 1024), (16, 16, 16, 2, 1024), (16, 16, 16, 16, 512)):
        assert L.sfb_adapter_init(ctypes.byref(cfg), *args, n.value, ctypes.byref(h)) == -2
    assert L.sfb_adapter_init(ctypes.byref(cfg), 16, 16, 16, 16, 1024, n.value - 1, ctypes.byref(h)) == -4
    assert L.sfb_adapter_init(ctypes.byref(cfg), 16, 16, 16, 16, 1024, n.value, None) == -1
    assert L.sfb_adapter_forward(None, 0, None, 0, None, None, 0, None) == -1
    assert L.sfb_adapter_backward(None, 0, None, 0, None, 0, None, None, None, 0, None, None) == -1
    assert L.sfb_adapter_get_status(None, None) == -1 and L.sfb_adapter_destroy(None) == -1 and L.sfb_adapter_last_cuda_error(None) == 0


def clip_init(src, dst, counts, types, workspace=1 << 12, nbytes=None):
    L, m, h = S.lib(), len(counts), ctypes.c_void_p(1)
    c, t = (ctypes.c_int64 * m)(*counts), (ctypes.c_int32 * m)(*types)
    n = ctypes.c_size_t(0)
    rc = L.sfb_clip_workspace_bytes(m, c, t, ctypes.byref(n))
    if rc:
        return rc
    s = (ctypes.c_void_p * m)(*src)
    d = (ctypes.c_void_p * m)(*dst) if dst else None
    return L.sfb_clip_init(m, s, d, c, t, workspace, n.value if nbytes is None else nbytes, None, ctypes.byref(h))


def test_clip_arguments():
    L = S.lib()
    assert clip_init([4096], None, [-1], [0]) == -3 and clip_init([4096], None, [10], [3]) == -1
    assert clip_init([None], None, [10], [0]) == -1 and clip_init([4098], None, [10], [0]) == -2 and clip_init([4097], None, [10], [1]) == -2
    assert clip_init([4096], [8194], [10], [0]) == -2 and clip_init([4096], None, [10], [0], workspace=None) == -1
    assert clip_init([4096], None, [10], [0], workspace=4104) == -2 and clip_init([4096], None, [10], [0], nbytes=64) == -4
    assert L.sfb_clip_workspace_bytes(1, None, None, ctypes.byref(ctypes.c_size_t())) == -1 and L.sfb_clip_workspace_bytes(0, None, None, None) == -1
    assert L.sfb_clip_gradients(None, 1.0, None) == -1 and L.sfb_clip_sum(None, None) == -1 and L.sfb_clip_scale(None, 1.0, None, None) == -1
    assert L.sfb_clip_destroy(None) == -1 and L.sfb_clip_last_cuda_error(None) == 0


def test_tensors_that_are_not_on_the_gpu():
    W, U, V, s = torch.zeros(8, 16), torch.zeros(2, 4, 8), torch.zeros(2, 4, 16), torch.ones(2)
    with pytest.raises(ValueError):
        S.Adapters(W, U, V, s, 4)
    with pytest.raises(ValueError):
        S.Adapters(W.bfloat16(), U.bfloat16(), V.bfloat16(), s, 4)
    with pytest.raises(ValueError):
        S.Adapters(W, U, U, s, 4)
    for bad in ([], [torch.zeros(4)], [torch.zeros(4, dtype=torch.float64)]):
        with pytest.raises(ValueError):
            S.GradientClip(bad)


def test_overlaps_are_refused_before_the_device_is_asked():
    # (where there is no device a list that is in order ends at the device query)
    inside = [([4096, 4096], None), ([4096, 4120], None), ([4096, 8192], [16384, 16400]), ([4096, 8192], [8192, 16384]), ([4096], [4112])]
    for src, dst in inside:
        assert clip_init(src, dst, [10] * len(src), [0] * len(src)) == -1
