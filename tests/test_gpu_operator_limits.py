"""The adapters and the clipping at the ends of what their handles allow: as many samples and adapters as there may be, results at any 4-byte
offset, tensors of more than 2^31 entries.  Bounds: those of test_gpu_adapters and test_gpu_clip."""
import pytest
import torch

import paper_1409_5705_b200 as S
from test_gpu_adapters import U23, U24, U8, Case, check, padded

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,rows,cols,adapters,rank", [(1 << 22, 16, 24, 3, 2), (300, 40, 72, 65_536, 1), (5_000, 24, 16, 65_536, 3)])
def test_most_samples_and_most_adapters(n, rows, cols, adapters, rank):
    """By samples, not by adapters as elsewhere (65,536 of them take a while).  The gradients' sums over a sample's products are formed in fp64 by
    index; their magnitudes likewise."""
    gen = torch.Generator(device="cuda").manual_seed(n)
    W, U, V = padded((rows, cols), gen, 0.05), padded((adapters, rank, rows), gen, 0.3), padded((adapters, rank, cols), gen, 0.2)
    scale = torch.rand(adapters, generator=gen, device="cuda") * 2 - 0.5
    X, dY = padded((n, cols), gen), padded((n, rows), gen)
    ids = torch.randint(-1, adapters, (n,), generator=gen, device="cuda", dtype=torch.int32)
    plan = S.Adapters(W, U, V, scale, max_samples=n)
    wide = lambda d: torch.full((n, -(-d // 8) * 8), 7.0, dtype=torch.bfloat16, device="cuda")[:, :d]
    Y, dX, Sx = wide(rows), wide(cols), torch.zeros(n, rank, device="cuda")
    dU, dV = torch.full((adapters, rank, rows), 7.0, device="cuda"), torch.full((adapters, rank, cols), 7.0, device="cuda")
    plan.sfb_adapter_forward(X, ids, Y, Sx)
    plan.sfb_adapter_backward(dY, X, ids, Sx, dX, dU, dV)
    assert plan.sfb_adapter_get_status() == 0
    at, has = ids.long().clamp(min=0), (ids >= 0).double()[:, None]
    sc = scale.double()[at][:, None] * has
    count = torch.bincount(at[ids >= 0], minlength=adapters).double()[:, None, None]
    for Z, A, F, G, y, p_got, g, Q in ((X, W, V, U, Y, Sx, dU, dY), (dY, W.t(), U, V, dX, None, dV, X)):
        Zd, Ad, Qd = Z.double(), A.double(), Q.double()
        d = Zd.shape[1]
        p, pm = (torch.zeros(n, rank, dtype=torch.float64, device="cuda") for _ in range(2))
        for r in range(rank):
            f = F[:, r].double()[at]
            p[:, r], pm[:, r] = (Zd * f).sum(1), (Zd * f).abs().sum(1)
        p, pm = p * has, pm * has
        pe = (d / 16 + 16) * U23 * pm
        if p_got is not None:
            assert ((p_got.double() - p).abs() <= pe).all()
        want, M = Zd @ Ad.t(), Zd.abs() @ Ad.abs().t()
        word = torch.zeros_like(want)
        out, mag = torch.zeros(adapters, rank, Qd.shape[1], dtype=torch.float64, device="cuda"), torch.zeros(adapters, rank, Qd.shape[1], dtype=torch.float64, device="cuda")
        err = torch.zeros_like(out)
        for r in range(rank):
            g_r = G[:, r].double()[at]
            want += sc * p[:, r : r + 1] * g_r
            word += sc.abs() * (2.0 ** -16 * p[:, r : r + 1].abs() + pe[:, r : r + 1]) * g_r.abs()
            M += (sc * p[:, r : r + 1] * g_r).abs()
            out[:, r].index_add_(0, at, sc * p[:, r : r + 1] * Qd)
            mag[:, r].index_add_(0, at, (sc * p[:, r : r + 1] * Qd).abs())
            err[:, r].index_add_(0, at, (sc * pe[:, r : r + 1] * Qd).abs())
        bound = U8 * want.abs() + word + (d / 16 + 16 + 4 * rank) * U23 * M
        assert ((y.double() - want).abs() <= bound).all()
        assert ((g.double() - out).abs() <= mag * (2 * U24 + (count / 16 + 16) * U23) + err + U24 * out.abs()).all()


@pytest.mark.parametrize("size", [(40, 300, 520, 6, 20, "mixed"), (300, 320, 520, 6, 64, "mixed"), (3_000, 300, 500, 1, 16, "mixed"), (128, 64, 256, 4, 4, "runs")],
                         ids=lambda s: "-".join(map(str, s)))
def test_results_at_any_offset_of_four_bytes(size):
    """S, dU and dV an entry behind a 16-byte boundary, ids and scale too; what lies around them stays."""
    c = Case(*size, seed=11)
    n, r, a = c.n, c.rank, c.adapters

    def moved(shape, dtype=torch.float32):
        numel = 1
        for k in shape:
            numel *= k
        buf = torch.full((numel + 2,), 9, dtype=dtype, device="cuda")
        return buf, buf[1:-1].view(shape)

    bufs = {k: moved(s) for k, s in (("S", (n, r)), ("dU", (a, r, c.rows)), ("dV", (a, r, c.cols)))}
    (_, ids), (_, scale) = moved((n,), torch.int32), moved((a,))
    ids.copy_(c.ids)
    scale.copy_(c.scale)
    plan = S.Adapters(c.W, c.U, c.V, scale, max_samples=n)
    wide = lambda d: torch.zeros(n, -(-d // 8) * 8, dtype=torch.bfloat16, device="cuda")[:, :d]
    Y, dX = wide(c.rows), wide(c.cols)
    plan.sfb_adapter_forward(c.X, ids, Y, bufs["S"][1])
    plan.sfb_adapter_backward(c.dY, c.X, ids, bufs["S"][1], dX, bufs["dU"][1], bufs["dV"][1])
    check(c, {"Y": Y, "dX": dX, **{k: v for k, (_, v) in bufs.items()}})
    for buf, _ in bufs.values():
        assert buf[0] == 9 and buf[-1] == 9


@pytest.mark.parametrize("shift", [0, 1])
def test_a_tensor_of_more_than_2_31_entries(shift):
    n = (1 << 31) + 12_345
    buf = torch.full((n + 8,), 0.5, dtype=torch.bfloat16, device="cuda")
    t = buf[shift : shift + n]
    t[-1], t[1 << 31] = 3.0, -2.0
    norm = (0.25 * (n - 2) + 13.0) ** 0.5
    result = torch.zeros(2, device="cuda")
    S.GradientClip([t]).sfb_clip_gradients(norm / 4, result)
    assert abs(result[0].item() - norm) <= (U24 + 1e-11) * norm and abs(result[1].item() - 0.25) <= 2.0 ** -24
    # (a factor half a step off 1/4 leaves these values where they are in bf16)
    assert t[-1] == 0.75 and t[1 << 31] == -0.5 and t[0] == 0.125 and (t[: 1 << 20] == 0.125).all() and (t[-10_000:-1] == 0.125).all()
    assert (buf[:shift] == 0.5).all() and (buf[shift + n :] == 0.5).all()
