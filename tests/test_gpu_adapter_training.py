"""Adapters and clipping as they are used together: a worker's factors that were not broadcast as an adapter beside the W of a training
context, and steps of forward pass, gradients, clipping and update on the same handles.  Bounds: those of test_gpu_adapters and test_gpu_clip."""
import pytest
import torch

import paper_1409_5705_b200 as S
from test_gpu_adapters import Case, check
from test_gpu_clip import check as check_clip

pytestmark = pytest.mark.gpu


def test_exported_factors_as_adapters_beside_the_operand_copy():
    """Workers of a context compute factors; each one's view of W, with its own update and without the others', answers samples: the
    adapters are the exported factors, the shared W the context's operand copy."""
    rows, cols, workers, batch, eta = 500, 264, 3, 20, 0.5
    gen = torch.Generator(device="cuda").manual_seed(0)
    W = torch.empty(rows, cols, device="cuda").normal_(0.0, 0.1, generator=gen)
    X = torch.empty(workers * batch, cols, device="cuda").normal_(0.0, 1.0, generator=gen)
    labels = torch.randint(0, rows, (workers * batch,), generator=gen, device="cuda", dtype=torch.int32)
    ctx = S.Context(S.make_config(S.MLR, rows, cols, workers, batch, eta, S.PREC_BF16), W)
    ctx.sfb_compute_factors(-1, X, None, labels)
    U, V = torch.empty(workers, batch, rows, device="cuda"), torch.empty(workers, batch, cols, device="cuda")
    for p in range(workers):
        ctx.sfb_export_factors(p, U[p], V[p])
    c = Case(90, 504, 264, workers, batch, "mixed", seed=1)
    c.rows = rows
    c.W = ctx.operand_copy_as_tensor()[:, :cols]
    pad = torch.full((workers, batch, 504), float("nan"), dtype=torch.bfloat16, device="cuda")
    pad[..., :rows] = U.bfloat16()
    c.U, c.V, c.scale, c.dY = pad[..., :rows], V.bfloat16(), torch.full((workers,), -eta, device="cuda"), c.dY[:, :rows]
    c.plan = S.Adapters(c.W, c.U, c.V, c.scale, max_samples=90)
    got = c.run()
    check(c, got)
    # and against the worker's W itself, (W - eta sum u v^T) x, as near as bf16 operands come: 2^-8 of each of the three roundings
    view = W.double() - eta * torch.einsum("bj,bd->jd", U[1].double(), V[1].double())
    mine = torch.nonzero(c.ids == 1).flatten()
    want = c.X[mine].double() @ view.t()
    room = c.X[mine].double().abs() @ (W.double().abs() + eta * torch.einsum("bj,bd->jd", U[1].double().abs(), V[1].double().abs())).t()
    assert ((got["Y"][mine].double() - want).abs() <= 2.0 ** -8 * (4 * room + want.abs())).all()
    ctx.close()


@pytest.mark.parametrize("n", [48, 700])
def test_steps_on_the_same_handles(n):
    """Forward pass, softmax factor of the loss, gradients, clipping in place, update of U and V in place: three steps, each against the
    formulas from the values that it began with; then the whole step captured and replayed once."""
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        c = Case(n, 300, 264, 5, 12, "runs", seed=n, stream=s)
        c.U.mul_(0.1)
        c.V.mul_(0.1)
        labels = torch.arange(n, device="cuda") % 300
        Y, Sx, dX = torch.zeros(n, 304, dtype=torch.bfloat16, device="cuda")[:, :300], torch.zeros(n, 12, device="cuda"), torch.zeros_like(c.X)
        dU, dV = torch.zeros(5, 12, 300, device="cuda"), torch.zeros(5, 12, 264, device="cuda")
        clip, result = S.GradientClip([dU, dV], stream=s), torch.zeros(2, device="cuda")

        def step():
            c.plan.sfb_adapter_forward(c.X, c.ids, Y, Sx)
            g = torch.softmax(Y.float(), 1)
            g[torch.arange(n, device="cuda"), labels] -= 1
            c.dY.copy_(g)
            c.plan.sfb_adapter_backward(c.dY, c.X, c.ids, Sx, dX, dU, dV)

        for k in range(3):
            before = c.U.clone(), c.V.clone()
            step()
            s.synchronize()
            check(c, {"Y": Y, "S": Sx, "dX": dX, "dU": dU, "dV": dV})
            raw = [dU.clone(), dV.clone()]
            limit = float(0.3 * torch.sqrt(sum(g.double().square().sum() for g in raw)))
            clip.sfb_clip_gradients(limit, result)
            s.synchronize()
            check_clip(raw, [dU, dV], limit, result)
            c.U.sub_(0.1 * dU)
            c.V.sub_(0.1 * dV)
            assert not torch.equal(before[0], c.U) and not torch.equal(before[1], c.V)

    def calls():
        c.plan.sfb_adapter_forward(c.X, c.ids, Y, Sx)
        c.plan.sfb_adapter_backward(c.dY, c.X, c.ids, Sx, dX, dU, dV)
        clip.sfb_clip_gradients(limit, result)

    torch.cuda.synchronize()
    calls()
    s.synchronize()
    eager = [t.clone() for t in (Y, Sx, dX, dU, dV, result)]
    g = c.plan.capture(calls)
    for t in (Y, Sx, dX, dU, dV, result):
        t.zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(eager, (Y, Sx, dX, dU, dV, result)))


def test_two_graphs_of_one_handle_in_turn():
    """Two captured calls share the handle's workspace; replayed in turn, each gives its own results."""
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        c = Case(400, 200, 136, 6, 8, "mixed", seed=3, stream=s)
        d = Case(400, 200, 136, 6, 8, "runs", seed=4, stream=s)
        outs = [(torch.zeros(400, 200, dtype=torch.bfloat16, device="cuda"), torch.zeros(400, 8, device="cuda")) for _ in range(2)]
        few = torch.zeros(30, 200, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    calls = [lambda: c.plan.sfb_adapter_forward(c.X, c.ids, *outs[0]), lambda: c.plan.sfb_adapter_forward(d.X, d.ids, *outs[1]),
             lambda: c.plan.sfb_adapter_forward(d.X[:30], d.ids[:30], few)]
    for f in calls:
        f()
    torch.cuda.synchronize()
    eager = [t.clone() for o in outs for t in o] + [few.clone()]
    graphs = [c.plan.capture(f) for f in calls]
    for _ in range(3):
        for t in [t for o in outs for t in o] + [few]:
            t.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            for g in graphs:
                g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, [t for o in outs for t in o] + [few]))
