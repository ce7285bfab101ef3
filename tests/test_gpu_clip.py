"""Global gradient norm and clipping on the GPU against 64 bits.

Bounds: a sum of squares is off by 8 * 2^-24 at most (groups of eight in fp32, all positive) and less in fp64, its root by half of that,
2^-22, and result[0] by its own rounding, 2^-24; so the factor, and a product g * coef is rounded once more to fp32 (2^-24) and once
to its type (eps / 2; fp16 below its normal numbers 2^-25).
"""
import math

import pytest
import torch

import paper_1409_5705_b200 as S

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TINY = {F32: 2.0 ** -149, BF16: 2.0 ** -133, F16: 2.0 ** -25}
NORM = 2.0 ** -22 + 2.0 ** -24


def tensors(sizes, types, std=1.0, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.empty(n, device="cuda").normal_(0.0, std, generator=gen).to(types[i % len(types)]) for i, n in enumerate(sizes)]


def norm_of(ts):
    return math.sqrt(sum(t.double().square().sum().item() for t in ts))


def check(ts, outs, limit, result):
    norm = norm_of(ts)
    coef = limit / norm if norm > limit else 1.0
    n, c = result.tolist()
    assert abs(n - norm) <= NORM * norm and abs(c - coef) <= (NORM + 2.0 ** -24) * coef
    for t, o in zip(ts, outs):
        want = t.double() * coef
        tol = want.abs() * (torch.finfo(t.dtype).eps / 2 + 2 * NORM) + TINY[t.dtype]
        assert ((o.double() - want).abs() <= tol).all()


LISTS = [
    ([1], [F32]), ([1], [F16]), ([3, 5, 7], [BF16]), ([0, 1, 0, 8], [F32, BF16]),
    ([4095, 4096, 4097], [F32]), ([8191, 8192, 8193, 16385], [BF16, F16]), ([100_003, 17, 65_536, 1], [F32, BF16, F16]),
    ([1_000_001] * 7, [F32, F16, BF16]), ([13] * 3000, [F32, BF16]), ([20_000_003], [BF16]),
]


@pytest.mark.parametrize("sizes,types", LISTS, ids=lambda v: f"{len(v)}x{v[0]}" if isinstance(v[0], int) else "".join(str(t)[6] for t in v))
@pytest.mark.parametrize("share", [0.3, 2.0])
@pytest.mark.parametrize("place", ["apart", "inside"])
def test_against_64_bits(sizes, types, share, place):
    ts = tensors(sizes, types, seed=len(sizes))
    limit = share * norm_of(ts)
    result = torch.full((3,), 9.0, device="cuda")
    src = [t.clone() for t in ts]
    outs = [torch.full_like(t, 5.0) for t in ts] if place == "apart" else None
    plan = S.GradientClip(src, outs)
    plan.sfb_clip_gradients(limit, result)
    torch.cuda.synchronize()
    check(ts, outs if outs is not None else src, limit, result[:2])
    assert result[2] == 9.0
    if place == "apart":
        assert all(torch.equal(a, b) for a, b in zip(src, ts))
    if share > 1:
        assert result[1] == 1.0 and all(torch.equal(a, b) for a, b in zip(outs or src, ts))


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("shift", [(1, 0), (0, 1), (3, 2), (5, 5)])
def test_offsets_within_a_buffer(dtype, shift):
    """Tensors at any entry of a flattened buffer; what lies around them stays."""
    n, (a, b) = 70_001, shift
    buf, to = tensors([n + 16], [dtype])[0], torch.full((n + 16,), 3.0, dtype=dtype, device="cuda")
    result = torch.zeros(2, device="cuda")
    plan = S.GradientClip([buf[a : a + n]], [to[b : b + n]])
    plan.sfb_clip_gradients(1.0, result)
    torch.cuda.synchronize()
    check([buf[a : a + n]], [to[b : b + n]], 1.0, result)
    assert (to[:b] == 3).all() and (to[b + n :] == 3).all()


@pytest.mark.parametrize("std", [1e-30, 1e-20, 1e18, 1e25])
def test_squares_beyond_fp32(std):
    ts = tensors([5000, 3001], [F32, BF16], std=std)
    result, limit = torch.zeros(2, device="cuda"), 0.5 * norm_of(ts)
    outs = [torch.zeros_like(t) for t in ts]
    S.GradientClip(ts, outs).sfb_clip_gradients(limit, result)
    torch.cuda.synchronize()
    check(ts, outs, limit, result)


@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("place", ["apart", "inside"])
def test_a_norm_that_is_not_finite_scales_nothing(value, place):
    ts = tensors([1000, 9000, 33], [F32, F16, BF16])
    ts[1][4567] = value
    src, outs = [t.clone() for t in ts], [torch.zeros_like(t) for t in ts] if place == "apart" else None
    result = torch.ones(2, device="cuda")
    S.GradientClip(src, outs).sfb_clip_gradients(1.0, result)
    torch.cuda.synchronize()
    assert not math.isfinite(result[0]) and result[1] == 0
    for t, o in zip(ts, outs or src):
        assert torch.equal(t.view(torch.int16 if t.element_size() == 2 else torch.int32), o.view(torch.int16 if o.element_size() == 2 else torch.int32))


def test_zero_norm_and_zero_limit():
    z, result = [torch.zeros(100, device="cuda")], torch.ones(2, device="cuda")
    S.GradientClip(z).sfb_clip_gradients(1.0, result)
    assert result.tolist() == [0.0, 1.0]
    t = tensors([77], [F32])
    S.GradientClip(t).sfb_clip_gradients(0.0, result)
    assert result[1] == 0 and (t[0] == 0).all()


def test_two_halves_are_the_whole():
    """sfb_clip_sum over two lists, added by the caller, then sfb_clip_scale of both: as one list over ranks."""
    ts = tensors([5001, 300_000, 12], [F32, BF16, F16], seed=3)
    limit = 0.25 * norm_of(ts)
    plans = [S.GradientClip([ts[0].clone()]), S.GradientClip([t.clone() for t in ts[1:]])]
    sums, result = torch.zeros(2, dtype=torch.float64, device="cuda"), torch.zeros(2, device="cuda")
    for k, p in enumerate(plans):
        p.sfb_clip_sum(sums[k : k + 1])
    total = sums.sum().reshape(1)
    for p in plans:
        p.sfb_clip_scale(limit, total, result)
        torch.cuda.synchronize()
        assert abs(result[0].item() - norm_of(ts)) <= NORM * norm_of(ts)
    check(ts, plans[0].grads + plans[1].grads, limit, result)


def test_captured_replayed_and_the_same_bits():
    s = torch.cuda.Stream()
    ts = tensors([100_000, 3, 70_000], [F32, BF16, F16], seed=4)
    outs, result = [torch.zeros_like(t) for t in ts], torch.zeros(2, device="cuda")
    torch.cuda.synchronize()
    plan = S.GradientClip(ts, outs, stream=s)
    plan.sfb_clip_gradients(1.0, result)
    g = plan.capture(lambda: plan.sfb_clip_gradients(1.0, result))
    for t, u in zip(ts, tensors([100_000, 3, 70_000], [F32, BF16, F16], std=3.0, seed=5)):
        t.copy_(u)
    torch.cuda.synchronize()
    got = []
    for _ in range(2):
        with torch.cuda.stream(s):
            g.replay()
        torch.cuda.synchronize()
        got.append([result.clone()] + [o.clone() for o in outs])
    check(ts, outs, 1.0, result)
    assert all(torch.equal(a, b) for a, b in zip(*got))
