"""Lookup and its gradient on the GPU against 64 bits.

Bounds.  Lookup: the factor is rounded twice (the dropout's share of it, its product with the scale), the product once, to fp32, and
once to the result's type: 3 * 2^-24 and eps / 2 of the value.  Gradient: c terms, added in some order, are off by c * 2^-24 of the sum
of their magnitudes at most; the factor is rounded three times, the product (with what it is added to) once: (c + 4) * 2^-24 of the
magnitudes, and 2^-24 of what was there before.  Below its normal numbers a type is off by half its smallest step.
"""
import pytest
import torch

import paper_1409_5705_b200 as S
from _tokens import mask

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TINY = {F32: 2.0 ** -149, BF16: 2.0 ** -133, F16: 2.0 ** -25}
ULP = 2.0 ** -24


def ids_of(n, tokens, kind, seed):
    gen = torch.Generator().manual_seed(seed)
    if kind == "uniform":
        return torch.randint(-1, tokens, (n,), generator=gen, dtype=torch.int32)
    if kind == "one":
        return torch.full((n,), tokens // 2, dtype=torch.int32)
    if kind == "none":
        return torch.full((n,), -1, dtype=torch.int32)
    if kind == "skew":                      # half of them one token, the rest falling off; the last one too
        i = (torch.rand(n, generator=gen).double() ** 6 * tokens).int()
        i[torch.rand(n, generator=gen) < 0.4] = tokens - 1
        return i
    return torch.sort(torch.randint(0, tokens, (n,), generator=gen, dtype=torch.int32)).values       # "runs"


def matrix(n, cols, dtype, seed, pitch=0, offset=0, std=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    pitch = pitch or cols
    flat = torch.empty(n * pitch + offset, device="cuda").normal_(0.0, std, generator=gen).to(dtype)
    return flat[offset:].view(n, pitch)[:, :cols]


def gradient_of(ids, dX, tokens, factor, m=1.0):
    """The sums, the sums of magnitudes and the counts, in fp64."""
    named = ids >= 0
    part = (dX.double() * m)[named] * factor
    at = ids[named].long()
    z = torch.zeros((tokens, dX.shape[1]), dtype=torch.float64, device=dX.device)
    return z.index_add(0, at, part), z.index_add(0, at, part.abs()), torch.bincount(at, minlength=tokens).double()[:, None]


SHAPES = [(1, 1, 1, "uniform"), (1, 5, 8, "one"), (7, 100, 33, "uniform"), (64, 3, 256, "skew"), (300, 1000, 77, "none"), (1024, 50, 100, "one"),
          (1025, 5000, 24, "uniform"), (4099, 333, 129, "skew"), (9000, 70_000, 40, "uniform"), (20_000, 1 << 20, 16, "skew"), (70_001, 2000, 9, "skew"),
          (70_000, 300_000, 8, "runs"), (200_003, 40, 4, "skew")]


@pytest.mark.parametrize("table_dtype,out_dtype", [(F32, BF16), (BF16, BF16), (F16, F32), (BF16, F16), (F32, F32)])
@pytest.mark.parametrize("n,tokens,dim,kind", SHAPES)
@pytest.mark.parametrize("p", [0.0, 0.2])
def test_lookup(n, tokens, dim, kind, table_dtype, out_dtype, p):
    table, ids = matrix(tokens, dim, table_dtype, 1, pitch=(dim + 7) // 8 * 8 if n % 2 else 0), ids_of(n, tokens, kind, 2).cuda()
    rng = torch.tensor([n, -tokens], device="cuda")
    X = torch.full((n + 1, dim), 7.0, dtype=out_dtype, device="cuda")
    plan, drop = S.Embedding(table, n, out_dtype, scale=1.7), S.Dropout(p, rng) if p else None
    plan.sfb_embed_forward(ids, X[:n], drop, 3)
    m = mask(rng, 3, n, dim, p).cuda() if p else 1.0
    want = table.double()[ids.long().clamp(min=0)] * (ids >= 0)[:, None] * float(torch.tensor(1.7)) * m
    assert ((X[:n].double() - want).abs() <= want.abs() * (torch.finfo(out_dtype).eps / 2 + 3 * ULP) + TINY[out_dtype]).all()
    assert (X[n] == 7).all() and plan.sfb_embed_get_status() == 0


def check_gradient(n, tokens, dim, kind, dtype, p, add, pitch=0, offset=0, out_pitch=0, out_offset=0, alpha=-0.3):
    ids, dX = ids_of(n, tokens, kind, 3).cuda(), matrix(n, dim, dtype, 4, pitch, offset)
    before = matrix(tokens, dim, F32, 5, out_pitch, out_offset)
    dE, rng = before.clone() if not (out_pitch or out_offset) else before, torch.tensor([-n, tokens], device="cuda")
    old, whole = before.clone(), dE._base.clone() if dE._base is not None else None
    plan, drop = S.Embedding(torch.zeros((tokens, dim), dtype=dtype, device="cuda"), n, scale=2.5), S.Dropout(p, rng) if p else None
    plan.sfb_embed_backward(ids, dX, dE, drop, 9, alpha=alpha, add=add)
    sums, most, counts = gradient_of(ids, dX, tokens, 2.5 * float(torch.tensor(alpha)), mask(rng, 9, n, dim, p).cuda() if p else 1.0)
    want = sums + old.double() if add else sums
    tol = (counts + 4) * ULP * most + (ULP * want.abs() if add else 0.0) + TINY[F32]
    assert ((dE.double() - want).abs() <= tol).all()
    if add:
        assert torch.equal(dE[counts[:, 0] == 0], old[counts[:, 0] == 0])
    if whole is not None:                   # what lies around the matrix stays
        rows = torch.ones_like(whole, dtype=torch.bool)
        rows[out_offset:].view(tokens, -1)[:, :dim] = False
        assert torch.equal(dE._base[rows], whole[rows])
    assert plan.sfb_embed_get_status() == 0
    return dE


@pytest.mark.parametrize("dtype", [BF16, F32, F16])
@pytest.mark.parametrize("n,tokens,dim,kind", SHAPES)
@pytest.mark.parametrize("p,add", [(0.0, False), (0.0, True), (0.3, False), (0.3, True)])
def test_gradient(n, tokens, dim, kind, dtype, p, add):
    check_gradient(n, tokens, dim, kind, dtype, p, add)


@pytest.mark.parametrize("dim,pitch,offset,out_pitch,out_offset", [(40, 41, 0, 40, 1), (40, 48, 8, 44, 4), (33, 40, 1, 33, 3), (8, 8, 1, 9, 0), (1, 1, 0, 3, 2)])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("add", [False, True])
def test_strides_and_offsets(dim, pitch, offset, out_pitch, out_offset, dtype, add):
    check_gradient(3000, 700, dim, "skew", dtype, 0.1, add, pitch, offset, out_pitch, out_offset)
    table, ids = matrix(700, dim, dtype, 6, pitch, offset), ids_of(3000, 700, "uniform", 7).cuda()
    X = matrix(3000, dim, dtype, 8, out_pitch, out_offset)
    whole = X._base.clone()
    S.Embedding(table, 3000).sfb_embed_forward(ids, X)
    assert torch.equal(X, torch.where((ids >= 0)[:, None], table[ids.long().clamp(min=0)], 0.0).to(dtype))
    rows = torch.ones_like(whole, dtype=torch.bool)
    rows[out_offset:].view(3000, -1)[:, :dim] = False
    assert torch.equal(X._base[rows], whole[rows])


def test_ids_out_of_range_and_calls_of_any_size():
    table = matrix(50, 20, F32, 0)
    plan, dE = S.Embedding(table, 40), torch.zeros(50, 20, device="cuda")
    ids = torch.tensor([3, 50, -2, 49, 2 ** 31 - 1, -2 ** 31, -1, 3], dtype=torch.int32, device="cuda")
    X = torch.ones(8, 20, device="cuda")
    plan.sfb_embed_forward(ids, X)
    assert plan.sfb_embed_get_status() == S.STATUS_INDEX_RANGE and plan.sfb_embed_get_status() == 0
    good = torch.tensor([0, 3, 7], device="cuda")
    assert torch.equal(X[good], table[ids[good].long()]) and (X[[1, 2, 4, 5, 6]] == 0).all()
    dX = torch.ones(8, 20, device="cuda")
    plan.sfb_embed_backward(ids, dX, dE)
    assert plan.sfb_embed_get_status() == S.STATUS_INDEX_RANGE
    assert dE.sum() == 60 and (dE[3] == 2).all() and (dE[49] == 1).all()
    dE.fill_(5.0)                            # no samples: zeros, or nothing
    plan.sfb_embed_backward(ids[:0], dX[:0], dE, add=True)
    assert (dE == 5).all()
    plan.sfb_embed_backward(ids[:0], dX[:0], dE)
    assert (dE == 0).all()
    plan.sfb_embed_forward(ids[:0], X[:0])
    with pytest.raises(S.SfbError):
        plan.sfb_embed_forward(torch.zeros(41, dtype=torch.int32, device="cuda"), torch.zeros(41, 20, device="cuda"))


def test_values_that_are_not_finite_stay_with_their_token():
    n, tokens, dim = 5000, 60, 48
    ids, dX = ids_of(n, tokens, "skew", 1).cuda(), matrix(n, dim, BF16, 2)
    plan, dE, clean = S.Embedding(torch.zeros(tokens, dim, dtype=BF16, device="cuda"), n), *(torch.zeros(tokens, dim, device="cuda") for _ in "ab")
    plan.sfb_embed_backward(ids, dX, clean)
    hit = int(ids[17])
    dX[17, 5], dX[17, 6] = float("nan"), float("inf")
    plan.sfb_embed_backward(ids, dX, dE)
    assert torch.isnan(dE[hit, 5]) and torch.isinf(dE[hit, 6])
    dE[hit, 5], dE[hit, 6] = clean[hit, 5], clean[hit, 6]
    assert torch.equal(dE, clean)
    # a dropped entry is gone, whatever it is
    rng = torch.tensor([1, 2], device="cuda")
    m = mask(rng, 0, n, dim, 0.5).cuda()
    dX = torch.where(m == 0, float("nan"), 1.0).to(BF16)
    plan.sfb_embed_backward(ids, dX, dE, S.Dropout(0.5, rng))
    assert torch.isfinite(dE).all()


def test_same_bits_from_call_to_call_and_between_dropout_forms():
    n, tokens, dim = 66_000, 900, 100
    ids, dX = ids_of(n, tokens, "skew", 1).cuda(), matrix(n, dim, BF16, 2)
    plan, a, b = S.Embedding(torch.zeros(tokens, dim, dtype=BF16, device="cuda"), n), *(torch.zeros(tokens, dim, device="cuda") for _ in "ab")
    plan.sfb_embed_backward(ids, dX, a)
    for _ in range(5):
        plan.sfb_embed_backward(ids[:777], dX[:777], b)
        plan.sfb_embed_backward(ids, dX, b)
        assert torch.equal(a, b)


def test_gradient_against_differences():
    """f(E) = sum of C * X(E): f is linear, so differences are its gradient but for rounding: X in fp32 is off by 3 * 2^-24, f by that of the
    sum of magnitudes; a step of 1 divides by 2."""
    n, tokens, dim = 50, 11, 13
    ids, C, rng = ids_of(n, tokens, "uniform", 1).cuda(), matrix(n, dim, F32, 2), torch.tensor([3, 4], device="cuda")
    table, X, dE = matrix(tokens, dim, F32, 3), torch.zeros(n, dim, device="cuda"), torch.zeros(tokens, dim, device="cuda")
    plan, drop = S.Embedding(table, n, scale=1.5), S.Dropout(0.25, rng)
    plan.sfb_embed_backward(ids, C, dE, drop)

    def f(t, j, by):
        table[t, j] += by
        plan.sfb_embed_forward(ids, X, drop)
        table[t, j] -= by
        v = X.double() * C.double()
        return v.sum().item(), v.abs().sum().item()

    for t, j in ((0, 0), (5, 7), (10, 12), (3, 4)):
        old = table[t, j].item()
        table[t, j] = 0.0                   # (so that adding and taking off 1 is exact)
        (up, a), (down, b) = f(t, j, 1.0), f(t, j, -1.0)
        table[t, j] = old
        assert abs((up - down) / 2 - dE[t, j].item()) <= 4 * ULP * (a + b)


def test_captured_replayed_on_other_ids_and_masks():
    s = torch.cuda.Stream()
    n, tokens, dim = 3000, 400, 64
    ids, dX, rng = ids_of(n, tokens, "skew", 1).cuda(), matrix(n, dim, BF16, 2), torch.tensor([7, 1], device="cuda")
    table, X, dE = matrix(tokens, dim, F32, 3), torch.zeros(n, dim, dtype=BF16, device="cuda"), torch.zeros(tokens, dim, device="cuda")
    torch.cuda.synchronize()
    plan, drop = S.Embedding(table, n, BF16, stream=s), S.Dropout(0.1, rng, stream=s)

    def calls():
        plan.sfb_embed_forward(ids, X, drop, 1)
        plan.sfb_embed_backward(ids, dX, dE, drop, 1)

    calls()
    g = plan.capture(calls)
    for step in range(3):
        ids.copy_(ids_of(n, tokens, "uniform", 10 + step))
        rng[1] += 1
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            g.replay()
        torch.cuda.synchronize()
        m = mask(rng, 1, n, dim, 0.1).cuda()
        want = table.double()[ids.long().clamp(min=0)] * (ids >= 0)[:, None] * m
        assert ((X.double() - want).abs() <= want.abs() * (2.0 ** -8 + 3 * ULP)).all()
        sums, most, counts = gradient_of(ids, dX, tokens, 1.0, m)
        assert ((dE.double() - sums).abs() <= (counts + 4) * ULP * most).all()
