"""What once went wrong around lookup, dropout and sampling, on the GPU.  Bounds: those of the operators' own tests."""
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
