"""Faults of the adapters' and the clipping's kernels and handles that reading found: each case is one that went wrong, or could.
Bounds: those of test_gpu_adapters and test_gpu_clip unless they are derived at the test."""
import pytest
import torch

import paper_1409_5705_b200 as S
from test_gpu_adapters import Case, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cols", [320, 200, 576])
def test_the_term_in_the_same_stage_of_tile_after_tile(cols):
    """One k-block of the adapters' term a tile, behind five, four or nine of W, so that it is always in the same one of five or six stages: the
    warps that hand the other CTA's operands on see every phase of it.  Many tiles a pair of CTAs, many calls; no wait may run out."""
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


def two_word_bounds(c):
    """Y and dX with the adapters' term from scale * s in two words, 2^-16 of it, and one rounding to bf16 of the result."""
    U24, U23, U8 = 2.0 ** -24, 2.0 ** -23, 2.0 ** -8
    ids, has, at, sc = c.wide()
    W, U, V, X, dY = (t.double() for t in (c.W, c.U, c.V, c.X, c.dY))
    got = {}
    for name, Z, A, F, G in (("Y", X, W, V, U), ("dX", dY, W.t(), U, V)):
        d = Z.shape[1]
        y, M = Z @ A.t(), Z.abs() @ A.abs().t()
        word = torch.zeros_like(y)
        for a in range(c.adapters):
            i = torch.nonzero(ids == a).flatten()
            p, m = sc[i] * (Z[i] @ F[a].t()), sc[i].abs() * (Z[i].abs() @ F[a].abs().t())
            y[i] += p @ G[a]
            # the words of scale * s and its product's rounding; what s itself is off (see test_gpu_adapters)
            word[i] = (p.abs() * (2.0 ** -16 + U24) + (d / 16 + 16) * U23 * m) @ G[a].abs()
            M[i] += p.abs() @ G[a].abs()
        got[name] = y, U8 * y.abs() + word + (d / 16 + 16 + 2 * 2 * c.rank) * U23 * M
    return got


@pytest.mark.parametrize("size", [(1, 300, 200, 2, 16, "one"), (16, 130, 264, 5, 20, "every"), (30, 700, 120, 30, 33, "mixed"), (64, 1000, 300, 9, 128, "mixed"),
                                  (64, 200, 6400, 9, 128, "mixed"), (100, 515, 777, 100, 8, "every"), (300, 320, 200, 3, 64, "runs"), (513, 260, 300, 5, 128, "mixed"),
                                  (1500, 700, 6000, 100, 16, "every"), (700, 136, 3000, 40, 7, "mixed")], ids=lambda s: "-".join(map(str, s)))
def test_the_term_is_not_held_in_one_word(size):
    """The adapters' term is most of the result, and its parts cancel: one rounding of scale * s to bf16 would be far outside."""
    c = Case(*size, seed=sum(size[:5]))
    c.W.mul_(0.01)
    got = c.run()
    for k, (v, b) in two_word_bounds(c).items():
        off = (got[k].double() - v).abs()
        assert (off <= b).all(), f"{k}: {(off / b.clamp(min=1e-300)).max().item():.3g} of the bound"


@pytest.mark.parametrize("value,count", [(1.174750804901123, 123_456), (1.174750804901123, 200_000), (1.174750804901123, 500_000), (1.6343168020248413, 5_000), (1.6343168020248413, 40_000)])
def test_squares_are_not_rounded_to_32_bits(value, count):
    """Entries whose squares all round the same way in fp32: the norm and the factor are the 64-bit ones, rounded once.  (fp64 sums are
    off by 1e-12 at most; the norms lie further than that from where the rounding turns.)"""
    t = torch.full((count,), value, device="cuda")
    norm = t.double().square().sum().sqrt().item()
    result = torch.zeros(2, device="cuda")
    S.GradientClip([t]).sfb_clip_gradients(1.5, result)
    want = torch.tensor([norm, 1.5 / norm], dtype=torch.float64)
    for near in (want * (1 - 1e-11), want * (1 + 1e-11)):
        assert torch.equal(near.float(), want.float())
    assert torch.equal(result.cpu(), want.float())


@pytest.mark.parametrize("place", ["apart", "inside"])
def test_a_norm_beyond_fp32_is_still_a_factor(place):
    """norm = 6e38 in fp64: result[0] is infinite in fp32, the factor 1 / 6e38 (below fp32's normal numbers: 2^-150 off at most) and applied."""
    src = [torch.full((3,), 3e38, device="cuda"), torch.full((1,), 3e38, dtype=torch.bfloat16, device="cuda")]
    ts = [t.clone() for t in src]
    outs = [torch.zeros_like(t) for t in src] if place == "apart" else None
    result = torch.zeros(2, device="cuda")
    S.GradientClip(src, outs).sfb_clip_gradients(1.0, result)
    norm = sum(t.double().square().sum().item() for t in ts) ** 0.5
    assert result[0] == float("inf") and abs(result[1].item() - 1.0 / norm) <= 2.0 ** -150
    for t, o in zip(ts, outs or src):
        want = t.double() / norm
        assert ((o.double() - want).abs() <= (torch.finfo(t.dtype).eps / 2 + 2.0 ** -24) * want + t.double() * 2.0 ** -150).all()


@pytest.mark.parametrize("kind", ["adapters", "clip"])
def test_memory_of_a_dropped_handle_whose_calls_are_under_way(kind):
    """A handle on a stream of its own is dropped before its call has run: its workspace is not handed out again until it has."""
    s = torch.cuda.Stream()
    c = Case(300, 400, 320, 5, 16, "runs", seed=1)
    Y, Sx = torch.zeros(300, 400, dtype=torch.bfloat16, device="cuda"), torch.zeros(300, 16, device="cuda")
    g, result = torch.full((100_000,), 2.0, device="cuda"), torch.zeros(2, device="cuda")
    torch.cuda.synchronize()
    plan = S.Adapters(c.W, c.U, c.V, c.scale, max_samples=300, stream=s) if kind == "adapters" else S.GradientClip([g], stream=s)
    call = (lambda: plan.sfb_adapter_forward(c.X, c.ids, Y, Sx)) if kind == "adapters" else (lambda: plan.sfb_clip_gradients(1.0, result))
    call()                                              # (kernels are loaded by their first launches, which wait)
    torch.cuda.synchronize()
    g.fill_(2.0)
    with torch.cuda.stream(s):
        torch.cuda._sleep(1)
        s.synchronize()
        torch.cuda._sleep(100_000_000)                  # about 50 ms
    call()
    at, n = plan.workspace.data_ptr(), plan.workspace.numel()
    del plan, call
    again = torch.empty(n, dtype=torch.uint8, device="cuda")
    busy = not s.query()
    torch.cuda.synchronize()
    assert busy and again.data_ptr() != at
    if kind == "adapters":
        check(c, {"Y": Y, "S": Sx}, ("Y", "S"))
    else:
        assert (g * 100_000 ** 0.5 - 1.0).abs().max() <= 2.0 ** -20
