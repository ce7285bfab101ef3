"""What once went wrong around lookup, dropout and sampling, on the GPU.  Bounds: those of the operators' own tests."""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

import paper_1409_5705_b200 as S
from test_gpu_adapters import Case

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def test_draws_right_behind_the_product_that_made_the_logits():
    """Without top-k and top-p, a CTA a row: draws from logits that the launch before writes, and not from the ones that stood there."""
    n, classes = 300, 8_200
    c = Case(n, classes, 64, 3, 4, "mixed", seed=2)
    Y, u, samples = torch.zeros(n, classes, dtype=BF16, device="cuda"), torch.rand(n, device="cuda"), [torch.randn(n, 64, device="cuda").bfloat16() * 4 for _ in range(8)]
    plan, ids, logp = S.Sampler(classes, BF16, n), torch.zeros(8, n, dtype=torch.int32, device="cuda"), torch.zeros(8, n, device="cuda")
    torch.cuda.synchronize()
    for i, X in enumerate(samples):
        c.plan.sfb_adapter_forward(X, c.ids, Y)
        plan.sfb_sample(Y, u, ids[i], logp=logp[i])
    torch.cuda.synchronize()
    got, logs = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(n, device="cuda")
    for i, X in enumerate(samples):
        c.plan.sfb_adapter_forward(X, c.ids, Y)
        torch.cuda.synchronize()
        plan.sfb_sample(Y, u, got, logp=logs)
        torch.cuda.synchronize()
        assert torch.equal(got, ids[i]) and torch.equal(logs, logp[i])


def drawn(z, u=0.5, **settings):
    """(class, log-probability, kept) of one row, and the settings as they come to the GPU."""
    dev = {k: torch.tensor([v], dtype=torch.int32 if k == "top_k" else F32, device="cuda") for k, v in settings.items()}
    ids, kept, logp = torch.full((1,), -7, dtype=torch.int32, device="cuda"), torch.full((1,), -7, dtype=torch.int32, device="cuda"), torch.zeros(1, device="cuda")
    S.Sampler(z.numel(), z.dtype, 1).sfb_sample(z[None].cuda(), torch.tensor([u], device="cuda"), ids, logp=logp, kept=kept, **dev)
    return (int(ids), float(logp), int(kept)), {k: v.item() for k, v in dev.items()}


def long_sample(z, u, top_k=0, top_p=1.0, min_p=0.0, temperature=1.0):
    """The formulas for one row without holes, in 80-bit numbers: a running sum of millions of equal weights is off by half a unit of its last place
    for each, 64-bit ones by more than a weight."""
    order = np.lexsort((np.arange(z.size), -z))
    s = z[order].astype(np.longdouble)
    w = np.exp((s - s[0]) / temperature)
    n = min(z.size, top_k) if top_k > 0 else z.size
    if top_p < 1:
        upto = np.cumsum(w[:n])
        n = 1 + int(np.searchsorted(upto, top_p * upto[-1], side="left"))
    n = int(np.count_nonzero(w[:n] >= min_p))
    by_place = np.argsort(order[:n])
    kept, w = order[:n][by_place], w[:n][by_place]
    upto = np.cumsum(w)
    i = int(np.searchsorted(upto, u * upto[-1], side="right"))
    return int(kept[i]), float(np.log(w[i] / upto[-1])), n


def agree(z, u=0.5, **settings):
    got, settings = drawn(z, u, **settings)
    want = long_sample(z.double().numpy(), u, **settings)
    assert (got[0], got[2]) == (want[0], want[2]) and abs(got[1] - want[1]) <= 2.0 ** -24 * abs(want[1]) + 1e-12, (got, want)


@pytest.mark.parametrize("dtype", [F32, BF16, torch.float16])
@pytest.mark.parametrize("classes", [325_000, 5_000_001])
@pytest.mark.parametrize("p,cut", [(0.9999, 0), (0.99999, 0), (0.99999, 100), (0.999999, 17)])
def test_nuclei_that_end_among_many_small_equals(classes, dtype, p, cut):
    """One large logit and two values of small ones, some hundred thousand or million times each: what one of their weights is off by, all are.  (By
    the formula top-p's end lies 0.01 of a small one's weight or more from an edge; the sums' roundings, 1e-16 each, are 1e-7 of it.)"""
    z = torch.full((classes,), 1.0)
    z[1::2], z[7] = 0.9921875, 21.5
    for u in (0.5, 1.0 - 2.0 ** -24):
        agree(z.to(dtype), u, top_p=p, **({"top_k": classes - cut} if cut else {}))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tail", [-31.25, -31.75])
def test_nuclei_that_end_among_millions_of_tiny_ones(dtype, tail):
    """One logit and 4 million small ones, w = e^-31 of it each: together 1.1e-7, of which top-p leaves 2^-24 out.  With N small ones the nucleus has
    1 + ceil((p (1 + N w) - 1) / w).  Sums are off by 2^-53 for each addition to the largest weight: a thread of 16 CTAs has 512 of the row's logits, and 33
    more sums and products follow."""
    n, w, p = (1 << 22) - 1, Fraction(math.exp(tail)), 1 - Fraction(1, 1 << 24)
    want = 1 + math.ceil((p * (1 + n * w) - 1) / w)
    z = torch.full((n + 1,), tail)
    z[5] = 0.0
    (at, logp, kept), _ = drawn(z.to(dtype), top_p=float(p))
    assert at == 5 and abs(kept - want) <= 545 * 2.0 ** -53 / w + 1 and 1 << 18 < want < n - (1 << 18)
    assert abs(logp + math.log1p((kept - 1) * w)) <= 2.0 ** -24 * 2e-7 + 1e-12


@pytest.mark.parametrize("dtype,edge", [(BF16, (-23.75, -23.875))])
@pytest.mark.parametrize("units,past", [(26.3, -0.006), (26.3, 0.006), (26.7, -0.006), (26.7, 0.006)])
def test_nuclei_that_end_beside_the_bin_that_rounded_sums_point_to(dtype, edge, units, past):
    """Some 400,000 weights, and more in the next bin behind them: in units of 2^-39 of the largest weight one of them is `units`, 26 or 27 as a whole number,
    a per cent off; top-p ends `past` of their sum behind or before their last one, on the other side than sums of whole numbers have it in two cases."""
    classes, first = 5_000_000, 384_616
    temperature = float(np.float32(-edge[0] / math.log(2.0 ** 39 / units)))
    z = torch.full((classes,), edge[1])
    z[::13], z[5] = edge[0], 0.0
    w = [math.exp(e / temperature) for e in edge]
    total = 1 + first * w[0] + (classes - first - 1) * w[1]
    agree(z.to(dtype), top_p=float(np.float32((1 + first * w[0] * (1 + past)) / total)), temperature=temperature)


@pytest.mark.parametrize("dtype", [F32, BF16, torch.float16])
@pytest.mark.parametrize("classes", [1000, 200_001])
@pytest.mark.parametrize("settings", [dict(), dict(top_k=20), dict(top_k=900), dict(top_p=0.5), dict(temperature=0.5), dict(temperature=2.0, top_p=0.9)], ids=str)
def test_min_p_far_below_the_largest_weight(dtype, classes, settings):
    """Classes are kept where their weights are min-p or more, however small both are: down to fp32's least number."""
    z = torch.full((classes,), -50.0)
    z[::3], z[1::7], z[5] = -60.0, -103.0, 0.0
    for min_p in (2.0 ** -149, 1e-44, 1e-38, 1e-25, 1e-21):
        for u in (0.25, 1.0 - 2.0 ** -24):
            agree(z.to(dtype), u, min_p=min_p, **settings)


def test_a_closed_dropout_before_a_lookup_and_before_a_gradient():
    E, ids = torch.randn(10, 16, device="cuda"), torch.arange(4, dtype=torch.int32, device="cuda")
    X, dE = torch.full((4, 16), 7.0, device="cuda"), torch.full((10, 16), 7.0, device="cuda")
    plan, drop = S.Embedding(E, 4), S.Dropout(0.5, torch.zeros(2, dtype=torch.int64, device="cuda"))
    drop.close()
    for call in (lambda: plan.sfb_embed_forward(ids, X, drop), lambda: plan.sfb_embed_backward(ids, X, dE, drop)):
        with pytest.raises(ValueError):
            call()
    assert (X == 7).all() and (dE == 7).all()


def test_factors_that_are_no_number():
    """scale and alpha are finite, their product is not: zeros of dX would become NaN."""
    E, ids = torch.ones(10, 16, device="cuda"), torch.arange(4, dtype=torch.int32, device="cuda")
    X, dE, rng = torch.zeros(4, 16, device="cuda"), torch.full((10, 16), 7.0, device="cuda"), torch.zeros(2, dtype=torch.int64, device="cuda")
    plan = S.Embedding(E, 4, scale=1e35)
    for call in (lambda: plan.sfb_embed_backward(ids, X, dE, alpha=1e5), lambda: plan.sfb_embed_backward(ids, X, dE, alpha=-1e5, add=True),
                 lambda: plan.sfb_embed_forward(ids, X, S.Dropout(0.9999, rng))):
        with pytest.raises(S.SfbError):
            call()
    assert (X == 0).all() and (dE == 7).all()
    plan.sfb_embed_backward(ids, X, dE, S.Dropout(1.0, rng), alpha=1.0)
    assert (dE == 0).all()
