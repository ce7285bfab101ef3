"""The ways that calls of the adapters take, each by a case that provably takes it (sfb_adapter_get_plan, asserted, so that a later change of the
rules cannot empty one), entry by entry against the formulas in 64 bits.  Bounds: those of test_gpu_adapters."""
import itertools

import pytest
import torch

import paper_1409_5705_b200 as S
from test_gpu_adapters import Case, check

pytestmark = pytest.mark.gpu
FMAS, TENSOR = 0, 1
DRAIN = 12                                              # k-blocks that a sum stays in the tensor cores for, at most


def plan(c, backward=False):
    return dict(zip(("factors", "factor_blocks", "in_order", "share_blocks"), S.sfb_adapter_get_plan(c.plan.cfg, c.n, backward)))


# up to 64 samples whose products with the factors are on the tensor cores: tiles of 16, 32 and 64 columns, one to several turns of a sum
FEW_FORWARD = [(64, 200, 6_400, 9, 128, "mixed"), (16, 130, 25_000, 5, 128, "mixed"), (24, 130, 17_000, 5, 128, "every"), (40, 72, 30_001, 40, 48, "every"),
               (1, 50, 400_000, 1, 128, "one")]
FEW_BACKWARD = [(64, 20_001, 130, 9, 128, "mixed"), (16, 25_000, 130, 5, 128, "mixed"), (24, 17_000, 130, 5, 128, "every"), (1, 400_000, 50, 1, 128, "one")]
# samples in the order of their adapters, their products with the factors in fp32 FMAs
ORDERED_FMAS = [((1_024, 1_000, 9_000, 64, 8, "mixed"), True), ((1_024, 9_000, 1_000, 64, 8, "mixed"), False)]


def ident(v):
    return "-".join(map(str, v)) if isinstance(v, tuple) else str(v)


@pytest.mark.parametrize("size,backward", [(s, False) for s in FEW_FORWARD] + [(s, True) for s in FEW_BACKWARD], ids=ident)
def test_few_samples_of_wide_factors(size, backward):
    c = Case(*size, seed=sum(size[:5]))
    assert plan(c, backward)["factors"] == TENSOR and c.n <= 64
    first = c.run(given=False)
    check(c, first)
    for given in (False, True, True):                   # the blocks' counts are left as they were found
        again = c.run(given=given)
        check(c, again)
        assert torch.equal(again["Y"], first["Y"]) and torch.equal(again["S"], first["S"])
    assert c.plan.sfb_adapter_get_status() == 0


def test_few_samples_of_wide_factors_in_turns():
    sizes = [plan(Case(*s))["factor_blocks"] for s in FEW_FORWARD]
    assert any(b > DRAIN for b in sizes) and any(b <= DRAIN for b in sizes)


@pytest.mark.parametrize("size,backward", ORDERED_FMAS, ids=ident)
def test_samples_in_order_without_the_tensor_cores(size, backward):
    c = Case(*size, seed=5)
    p = plan(c, backward)
    assert p["factors"] == FMAS and p["in_order"] == 1
    check(c, c.run())
    c.ids.copy_(torch.sort(c.ids).values)               # (and the device finds that they are in order already)
    check(c, c.run(given=False))


# sums of more than 12 k-blocks: of the products with the factors (forward, backward), of the shares of the gradients (one or two blocks an SM,
# one half of a tile)
@pytest.mark.parametrize("size,where", [((4_100, 72, 7_000, 3, 16, "runs"), "forward"), ((4_100, 7_000, 72, 3, 16, "mixed"), "backward"),
                                        ((20_000, 40, 1_600, 2, 24, "every"), "forward"), ((7_000, 72, 64, 1, 20, "one"), "shares"),
                                        ((7_000, 72, 64, 1, 16, "one"), "shares"), ((7_000, 136, 64, 1, 100, "one"), "shares"),
                                        ((12_000, 40, 100, 1, 1, "one"), "shares")], ids=ident)
def test_sums_taken_out_in_several_turns(size, where):
    c = Case(*size, seed=sum(size[:5]))
    p = plan(c, where != "forward")
    assert (p["share_blocks"] if where == "shares" else p["factor_blocks"]) > DRAIN
    assert where == "shares" or p["factors"] == TENSOR
    got = c.run()
    check(c, got)
    again = c.run()
    assert all(torch.equal(got[k], again[k]) for k in got)


WANTED = [w for k in (1, 2) for w in itertools.combinations(("dX", "dU", "dV"), k)]


@pytest.mark.parametrize("size", [(40, 300, 520, 6, 20, "mixed"), (16, 25_000, 130, 5, 128, "mixed"), (300, 320, 520, 6, 64, "mixed"), (1_024, 1_000, 9_000, 64, 8, "mixed"),
                                  (1_500, 700, 6_000, 100, 16, "every")], ids=ident)
@pytest.mark.parametrize("want", WANTED, ids="".join)
def test_outputs_that_are_not_wanted(size, want):
    c = Case(*size, seed=7)
    for given in (True, False):
        got = c.run(given=given, want=want)
        check(c, got, ("Y", "S") + want)
        for k in ("dX", "dU", "dV"):
            assert k in want or (got[k] == 7).all(), k
    assert c.plan.sfb_adapter_get_status() == 0


@pytest.mark.parametrize("size,way", [((64, 200, 6_400, 9, 128, "mixed"), (False, TENSOR, 0)), ((16, 130, 25_000, 5, 128, "mixed"), (False, TENSOR, 0)),
                                      ((24, 17_000, 130, 5, 128, "every"), (True, TENSOR, 0)), ((64, 20_001, 130, 9, 128, "mixed"), (True, TENSOR, 0)),
                                      ((1_024, 1_000, 9_000, 64, 8, "mixed"), (True, FMAS, 1)), ((1_024, 9_000, 1_000, 64, 8, "mixed"), (False, FMAS, 1))], ids=ident)
def test_what_is_not_finite_stays_where_it_is(size, way):
    """An adapter and a sample that hold infinities and NaN: the others have the bits they had, and all have them again afterwards."""
    c = Case(*size, seed=sum(size[:5]))
    p = plan(c, way[0])
    assert (p["factors"], p["in_order"]) == way[1:]
    before = c.run()
    U, V, X, dY = (t.clone() for t in (c.U, c.V, c.X, c.dY))
    c.ids[1] = 2                                        # some sample has the adapter
    before = c.run()
    c.U[2, 3, 17], c.U[2, c.rank - 1, 99], c.V[2, 5, 100], c.V[2, 0, 0] = float("inf"), float("nan"), float("nan"), float("-inf")
    bad = c.n // 2
    c.X[bad], c.dY[bad] = float("nan"), float("inf")
    for _ in range(2):
        after = c.run()
        other = c.ids != 2
        other[bad] = False
        for k in ("Y", "S", "dX"):
            assert torch.equal(before[k][other], after[k][other]), k
        owner = int(c.ids[bad])
        keep = [a for a in range(c.adapters) if a not in (2, owner)]
        for k in ("dU", "dV"):
            assert torch.equal(before[k][keep], after[k][keep]), k
        assert torch.isnan(after["Y"][bad]).all()
        assert not torch.isfinite(after["Y"][1][17]) and not torch.isfinite(after["dX"][1][100])
    c.U.copy_(U), c.V.copy_(V), c.X.copy_(X), c.dY.copy_(dY)
    last = c.run()
    assert all(torch.equal(before[k], last[k]) for k in before)


@pytest.mark.parametrize("size", [FEW_FORWARD[1], FEW_BACKWARD[2], ORDERED_FMAS[0][0]], ids=ident)
def test_captured_and_replayed(size):
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        c = Case(*size, seed=9, stream=s)
        got = c.run()
    s.synchronize()
    out = {k: torch.zeros((*v.shape[:-1], -(-v.shape[-1] // 8) * 8 if k in ("Y", "dX") else v.shape[-1]), dtype=v.dtype, device="cuda")[..., : v.shape[-1]]
           for k, v in got.items()}                     # (rows of Y and dX a multiple of 8 entries apart)

    def calls():
        c.plan.sfb_adapter_forward(c.X, c.ids, out["Y"], out["S"])
        c.plan.sfb_adapter_backward(c.dY, c.X, c.ids, out["S"], out["dX"], out["dU"], out["dV"])

    calls()
    g = c.plan.capture(calls)
    c.ids.copy_(torch.flip(c.ids, (0,)))
    torch.cuda.synchronize()
    for _ in range(2):
        with torch.cuda.stream(s):
            g.replay()
    torch.cuda.synchronize()
    check(c, out)
