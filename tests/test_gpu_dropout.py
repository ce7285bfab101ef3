"""Dropout on the GPU against 64 bits: which entries are kept is exact; a kept one is off by the rounding of the factor (2^-24), of the product or
the sum in fp32 (2^-24) and to its type (eps / 2)."""
import pytest
import torch

import paper_1409_5705_b200 as S
from _tokens import mask

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TINY = {F32: 2.0 ** -149, BF16: 2.0 ** -133, F16: 2.0 ** -25}
ULP = 2.0 ** -24


def matrix(n, cols, dtype, seed, pitch=0, offset=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    pitch = pitch or cols
    flat = torch.empty(n * pitch + offset, device="cuda").normal_(0.0, 1.0, generator=gen).to(dtype)
    return flat[offset:].view(n, pitch)[:, :cols]


def check(X, R, Y, m):
    part = X.double() * m
    part = torch.where(m == 0, 0.0, part)
    want = part if R is None else part + R.double()
    tol = want.abs() * (torch.finfo(X.dtype).eps / 2 + ULP) + part.abs() * ULP * 2 + TINY[X.dtype]
    assert ((Y.double() - want).abs() <= tol).all()


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("n,cols", [(1, 1), (1, 8), (3, 7), (17, 65), (128, 256), (1000, 999), (5, 70_001), (2049, 1024)])
@pytest.mark.parametrize("p,residual", [(0.1, False), (0.5, True), (0.0, True), (1.0, True), (1.0, False), (1e-9, False)])
def test_against_64_bits(n, cols, dtype, p, residual):
    X, R = matrix(n, cols, dtype, 1), matrix(n, cols, dtype, 2) if residual else None
    rng, Y = torch.tensor([n * 77, -cols], device="cuda"), torch.full((n, cols), 9.0, dtype=dtype, device="cuda")
    S.Dropout(p, rng).sfb_dropout_apply(X, Y, R, call=5)
    check(X, R, Y, mask(rng, 5, n, cols, p).cuda())


@pytest.mark.parametrize("pitch,offset", [(104, 0), (101, 0), (100, 3), (112, 8)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_pitches_and_places(pitch, offset, dtype):
    n, cols, rng = 333, 100, torch.tensor([1, 2], device="cuda")
    m = mask(rng, 0, n, cols, 0.3).cuda()
    X, R, Y = matrix(n, cols, dtype, 1, pitch, offset), matrix(n, cols, dtype, 2), matrix(n, cols, dtype, 3, 107, 1)
    whole = Y._base.clone()
    S.Dropout(0.3, rng).sfb_dropout_apply(X, Y, R)
    check(X, R, Y, m)
    around = torch.ones_like(whole, dtype=torch.bool)
    around[1:].view(n, 107)[:, :cols] = False
    assert torch.equal(Y._base[around], whole[around])
    # in place of x, and of r
    for place in (X, R):
        x, r = X.clone(), R.clone()
        S.Dropout(0.3, rng).sfb_dropout_apply(X, place, R)
        check(x, r, place, m)


def test_dropped_entries_are_zero_whatever_they_are():
    rng, n, cols = torch.tensor([9, 9], device="cuda"), 64, 80
    m = mask(rng, 0, n, cols, 0.4).cuda()
    X = torch.where(m == 0, float("nan"), 1.0).to(BF16)
    X[m == 0] = torch.where(torch.arange(int((m == 0).sum()), device="cuda") % 2 == 0, float("inf"), float("nan")).to(BF16)
    Y = torch.empty_like(X)
    S.Dropout(0.4, rng).sfb_dropout_apply(X, Y)
    assert torch.isfinite(Y).all() and torch.equal(Y == 0, m == 0)


def test_the_backward_pass_is_the_same_call():
    """Linear in x: the mask of dy is the mask of x; another call or offset is another mask."""
    rng, n, cols = torch.tensor([4, 2 ** 40], device="cuda"), 100, 333
    drop, ones = S.Dropout(0.2, rng), torch.ones(100, 333, device="cuda")
    a, b, c = (torch.empty_like(ones) for _ in range(3))
    drop.sfb_dropout_apply(ones, a, call=1)
    drop.sfb_dropout_apply(ones, b, call=1)
    drop.sfb_dropout_apply(ones, c, call=2)
    assert torch.equal(a, b) and not torch.equal(a, c)
    rng[1] += 1
    drop.sfb_dropout_apply(ones, b, call=1)
    assert torch.equal(b, c)
    assert torch.equal(a.double(), mask(torch.tensor([4, 2 ** 40]), 1, n, cols, 0.2).float().double().cuda())


def test_captured_on_another_stream():
    s = torch.cuda.Stream()
    rng, X, R = torch.tensor([11, 0], device="cuda"), matrix(500, 200, BF16, 1), matrix(500, 200, BF16, 2)
    Y = torch.empty_like(X)
    torch.cuda.synchronize()
    drop = S.Dropout(0.1, rng, stream=s)
    drop.sfb_dropout_apply(X, Y, R)
    g = drop.capture(lambda: drop.sfb_dropout_apply(X, Y, R))
    for step in range(3):
        rng[1] += 1
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            g.replay()
        torch.cuda.synchronize()
        check(X, R, Y, mask(rng, 0, 500, 200, 0.1).cuda())
