"""Lookup, dropout, adapters, sampling, gradients and clipping as they are used together: token ids in, classes out, and a step of the table.  Each
stage against its formula in 64 bits from what the stage before gave; bounds: those of the operators' own tests."""
import pytest
import torch

import paper_1409_5705_b200 as S
from _tokens import mask, sample
from test_gpu_adapters import Case, check
from test_gpu_clip import check as check_clip
from test_gpu_embedding import ULP, gradient_of, ids_of

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


class Step:
    """One model: a table, dropout, an added dropped-out copy, the product with W and each sample's adapter, a draw; and its gradients."""

    def __init__(self, n, stream, p=0.2, tokens=400):
        self.n, self.p, self.tokens, self.stream = n, p, tokens, stream
        c = self.c = Case(n, 300, 264, 5, 12, "runs", seed=n, stream=stream)
        gen = torch.Generator(device="cuda").manual_seed(n + 1)
        self.E = torch.empty(tokens, 264, device="cuda").normal_(0.0, 1.0, generator=gen)
        self.ids, self.rng = ids_of(n, tokens, "skew", n).cuda(), torch.tensor([n, 1 << 33], device="cuda")
        self.u, self.top_p = torch.rand(n, generator=gen, device="cuda"), torch.full((n,), 0.7, device="cuda")
        self.X, self.H = (torch.zeros(n, 264, dtype=BF16, device="cuda") for _ in range(2))
        self.Y = torch.zeros(n, 304, dtype=BF16, device="cuda")[:, :300]
        self.dH, self.dX = torch.zeros_like(self.H), torch.zeros_like(self.X)
        self.dU, self.dV, self.dE = torch.zeros(5, 12, 300, device="cuda"), torch.zeros(5, 12, 264, device="cuda"), torch.zeros_like(self.E)
        self.drawn, self.kept = (torch.zeros(n, dtype=torch.int32, device="cuda") for _ in range(2))
        self.logp, self.norm = torch.zeros(n, device="cuda"), torch.zeros(2, device="cuda")
        self.emb, self.drop = S.Embedding(self.E, n, BF16, scale=0.5, stream=stream), S.Dropout(p, self.rng, stream=stream)
        self.sampler = S.Sampler(300, BF16, n, stream=stream)
        self.clip = S.GradientClip([self.dE, self.dU, self.dV], stream=stream)
        self.dY = c.dY

    def run(self):
        self.emb.sfb_embed_forward(self.ids, self.X, self.drop, 1)
        self.drop.sfb_dropout_apply(self.X, self.H, self.X, call=2)
        self.c.plan.sfb_adapter_forward(self.H, self.c.ids, self.Y)
        self.sampler.sfb_sample(self.Y, self.u, self.drawn, top_p=self.top_p, logp=self.logp, kept=self.kept)
        self.c.plan.sfb_adapter_backward(self.dY, self.H, self.c.ids, None, self.dH, self.dU, self.dV)
        self.drop.sfb_dropout_apply(self.dH, self.dX, self.dH, call=2)
        self.emb.sfb_embed_backward(self.ids, self.dX, self.dE, self.drop, 1)

    def results(self):
        return [t.clone() for t in (self.X, self.H, self.Y, self.drawn, self.kept, self.logp, self.dH, self.dU, self.dV, self.dX, self.dE)]

    def check(self):
        n, first, second = self.n, mask(self.rng, 1, self.n, 264, self.p).cuda(), mask(self.rng, 2, self.n, 264, self.p).cuda()
        want = self.E.double()[self.ids.long().clamp(min=0)] * (self.ids >= 0)[:, None] * 0.5 * first
        assert ((self.X.double() - want).abs() <= want.abs() * (2.0 ** -8 + 3 * ULP)).all()
        for x, y in ((self.X, self.H), (self.dH, self.dX)):
            want = x.double() * second + x.double()
            assert ((y.double() - want).abs() <= want.abs() * (2.0 ** -8 + ULP) + 2 * ULP * (x.double() * second).abs()).all()
        z = self.Y.double().cpu().numpy()
        for i in range(n):
            got = sample(z[i], float(self.u[i]), top_p=float(self.top_p[i]))
            assert (int(self.drawn[i]), int(self.kept[i])) == (got[0], got[2]) and abs(float(self.logp[i]) - got[1]) <= ULP * abs(got[1]) + 1e-12
        sums, most, counts = gradient_of(self.ids, self.dX, self.tokens, 0.5, first)
        assert ((self.dE.double() - sums).abs() <= (counts + 4) * ULP * most).all()


@pytest.mark.parametrize("n", [1, 48, 700])
def test_a_step_and_its_capture(n):
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        step = Step(n, s)
        step.run()
        torch.cuda.synchronize()
        step.check()
        # the products between, by their own test's bounds
        step.c.X = step.H
        check(step.c, {"Y": step.Y, "dX": step.dH, "dU": step.dU, "dV": step.dV}, ("Y", "dX", "dU", "dV"))
        # clipped, and the table moved by the clipped gradient
        before, grads = step.E.clone(), [t.clone() for t in (step.dE, step.dU, step.dV)]
        step.clip.sfb_clip_gradients(0.1, step.norm)
        torch.cuda.synchronize()
        check_clip(grads, [step.dE, step.dU, step.dV], 0.1, step.norm)
        # ... or straight into its rows, with the step in alpha
        step.emb.sfb_embed_backward(step.ids, step.dX, step.E, step.drop, 1, alpha=-0.1, add=True)
        torch.cuda.synchronize()
        assert ((step.E.double() - (before.double() - 0.1 * grads[0].double())).abs() <= 4 * ULP * (before.double().abs() + grads[0].double().abs())).all()
        step.E.copy_(before)
        g = step.c.plan.capture(step.run)
        for i in range(2):                  # other masks, samples and random numbers, without another capture
            step.rng[1] += 3
            step.ids.copy_(ids_of(n, step.tokens, "uniform", 50 + i))
            step.u.uniform_()
            g.replay()
            torch.cuda.synchronize()
            step.check()
            replayed = step.results()
            step.run()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(replayed, step.results()))


def test_two_streams_at_once():
    """Handles of their own on two streams, whose calls run side by side: as one after another."""
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    steps = []
    for k, s in enumerate(streams):
        with torch.cuda.stream(s):
            steps.append(Step(500 + 100 * k, s))
    torch.cuda.synchronize()
    alone = []
    for step in steps:
        step.run()
        torch.cuda.synchronize()
        alone.append(step.results())
    for _ in range(10):
        for step in steps:
            step.run()
    torch.cuda.synchronize()
    for step, want in zip(steps, alone):
        assert all(torch.equal(a, b) for a, b in zip(step.results(), want))
