"""Faults of the adapters' and the clipping's kernels and handles that reading found: each case is one that went wrong, or could.
Bounds: those of test_gpu_adapters and test_gpu_clip unless they are derived at the test."""
import pytest
import torch

import paper_1409_5705_b200 as S
from test_gpu_adapters import Case, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cols", [320, 200, 700])
def test_the_term_in_the_same_stage_of_tile_after_tile(cols):
    """One k-block of the adapters' term a tile, behind five of W (six stages: always the same one), four or eleven: the two warps that hand
    the other CTA's operands on see every phase of that stage.  Many tiles a pair of CTAs, many calls; no wait may run out."""
    c = Case(6000, 3000, cols, 1, 8, "one", seed=cols)
    Y = torch.zeros(c.n, c.rows, dtype=torch.bfloat16, device="cuda")
    Sx = torch.zeros(c.n, c.rank, device="cuda")
    c.plan.sfb_adapter_forward(c.X, c.ids, Y, Sx)
    first = Y.clone()
    check(c, {"Y": Y, "S": Sx}, ("Y", "S"))
    for _ in range(300):
        c.plan.sfb_adapter_forward(c.X, c.ids, Y, Sx)
    assert c.plan.sfb_adapter_get_status() == 0
    assert torch.equal(Y, first)


def test_a_handle_for_no_samples():
    """max_samples = 0: calls of no samples, whose gradients are zeros; one sample is refused."""
    c = Case(3, 40, 48, 2, 4, "one")
    plan = S.Adapters(c.W, c.U, c.V, c.scale, max_samples=0)
    ids = torch.empty(0, dtype=torch.int32, device="cuda")
    dU, dV = torch.ones(2, 4, 40, device="cuda"), torch.ones(2, 4, 48, device="cuda")
    plan.sfb_adapter_forward(c.X[:0], ids, c.dY[:0])
    plan.sfb_adapter_backward(c.dY[:0], c.X[:0], ids, None, c.X[:0], dU, dV)
    assert plan.sfb_adapter_get_status() == 0 and (dU == 0).all() and (dV == 0).all()
    with pytest.raises(S.SfbError):
        plan.sfb_adapter_forward(c.X[:1], c.ids[:1], c.dY[:1])
