"""Low-rank adapters beside the shared W on the GPU, entry by entry against the formulas in 64 bits.

Bounds, derived before the first run.  bf16 products are exact in fp32.  A tensor-core instruction contracts 16 products and leaves at
most one unit of the last place, 2^-23 of what the accumulator then holds, which is at most the sum M of the products' magnitudes:
d / 16 instructions leave d / 16 * 2^-23 * M, fp32 sums of parts and ranks less than (16 + rank) * 2^-23 * M more.  A result is rounded
once to bf16 (2^-8 of it) or fp32 (2^-24).  Where the adapter's term goes over the tensor cores, scale * s is rounded to bf16 first:
2^-8 of sum |scale s_t u_t|.  For dU and dV scale * s and scale * t go as three words of bf16, 2^-24 of them
at most, beside one rounding of the product with scale; the contraction is over the adapter's samples.
"""
import pytest
import torch

import paper_1409_5705_b200 as S

pytestmark = pytest.mark.gpu
U24, U23, U8 = 2.0 ** -24, 2.0 ** -23, 2.0 ** -8


def padded(shape, gen, std=1.0, fill=float("nan"), extra=0):
    """bf16 normal values in rows a multiple of 8 entries apart, `fill` between them."""
    pitch = -(-shape[-1] // 8) * 8 + extra
    t = torch.full((*shape[:-1], pitch), fill, dtype=torch.bfloat16, device="cuda")
    t[..., : shape[-1]] = torch.empty(shape, device="cuda").normal_(0.0, std, generator=gen).to(torch.bfloat16)
    return t[..., : shape[-1]]


def draw_ids(mode, n, adapters, gen):
    if mode == "none":
        return torch.full((n,), -1, dtype=torch.int32, device="cuda")
    if mode == "one":
        return torch.full((n,), adapters - 1, dtype=torch.int32, device="cuda")
    if mode == "mixed":
        return torch.randint(-1, adapters, (n,), generator=gen, device="cuda", dtype=torch.int32)
    if mode == "every":                                 # as many adapters in a tile as there are
        return torch.arange(n, device="cuda", dtype=torch.int32) % adapters
    ends = torch.sort(torch.randint(0, n + 1, (2 * adapters,), generator=gen, device="cuda")).values
    which = torch.randint(-1, adapters, (2 * adapters + 1,), generator=gen, device="cuda", dtype=torch.int32)
    return which[torch.bucketize(torch.arange(n, device="cuda"), ends, right=True)]


class Case:
    def __init__(self, n, rows, cols, adapters, rank, mode, seed=0, extra=0, stream=None):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.n, self.rows, self.cols, self.adapters, self.rank = n, rows, cols, adapters, rank
        self.W = padded((rows, cols), gen, 0.05, extra=extra)
        self.U = padded((adapters, rank, rows), gen, 0.3, extra=extra)
        self.V = padded((adapters, rank, cols), gen, 0.2, extra=extra)
        self.scale = torch.rand(adapters, generator=gen, device="cuda") * 2 - 0.5
        self.X = padded((n, cols), gen, 1.0, extra=extra)
        self.dY = padded((n, rows), gen, 1.0, extra=extra)
        self.ids = draw_ids(mode, n, adapters, gen)
        self.plan = S.Adapters(self.W, self.U, self.V, self.scale, max_samples=max(n, 1), stream=stream)

    def wide(self):
        ids = self.ids.long()
        has = ((ids >= 0) & (ids < self.adapters))[:, None]
        at = torch.where(has[:, 0], ids, 0)
        return ids, has, at, self.scale.double()[at][:, None] * has

    def expected(self):
        """{name: (value, bound)}"""
        ids, has, at, sc = self.wide()
        W, U, V, X, dY = (t.double() for t in (self.W, self.U, self.V, self.X, self.dY))
        n, r = self.n, self.rank
        got = {}

        def ranks(Z, F, d):
            p, m = torch.zeros(n, r, dtype=torch.float64, device="cuda"), torch.zeros(n, r, dtype=torch.float64, device="cuda")
            for a in range(self.adapters):
                i = torch.nonzero(ids == a).flatten()
                p[i], m[i] = Z[i] @ F[a].t(), Z[i].abs() @ F[a].abs().t()
            return p, (d / 16 + 16) * U23 * m, m

        def product(Z, A, F, p, pe, pm, d):
            y, M = Z @ A.t(), Z.abs() @ A.abs().t()
            word = torch.zeros_like(y)
            for a in range(self.adapters):
                i = torch.nonzero(ids == a).flatten()
                y[i] += sc[i] * (p[i] @ F[a])
                word[i] = (sc[i].abs() * (U8 * p[i].abs() + pe[i])) @ F[a].abs()
                M[i] += (sc[i] * p[i]).abs() @ F[a].abs()
            return y, U8 * y.abs() + word + (d / 16 + 16 + 2 * r) * U23 * M

        s, se, sm = ranks(X, V, self.cols)
        t, te, tm = ranks(dY, U, self.rows)
        got["S"] = (s, se)
        got["Y"] = product(X, W, U, s, se, sm, self.cols)
        got["dX"] = product(dY, W.t(), V, t, te, tm, self.rows)
        for name, p, pe, Z, like in (("dU", s, se, dY, U), ("dV", t, te, X, V)):
            g, b = torch.zeros_like(like), torch.zeros_like(like)
            for a in range(self.adapters):
                i = torch.nonzero(ids == a).flatten()
                if len(i):
                    g[a] = (sc[i] * p[i]).t() @ Z[i]
                    b[a] = (sc[i].abs() * (p[i].abs() * (2 * U24 + (len(i) / 16 + 16) * U23) + pe[i])).t() @ Z[i].abs()
            got[name] = (g, b + U24 * g.abs())
        return got

    def run(self, given=True, plan=None, want=("dX", "dU", "dV")):
        """All outputs, in buffers with a row more and a gap behind each row that have to stay as they are."""
        plan = plan or self.plan
        mark = 7.0
        out = {"Y": torch.full((self.n + 1, -(-self.rows // 8) * 8 + 8), mark, dtype=torch.bfloat16, device="cuda"),
               "dX": torch.full((self.n + 1, -(-self.cols // 8) * 8 + 8), mark, dtype=torch.bfloat16, device="cuda"),
               "S": torch.full((self.n + 1, self.rank), mark, device="cuda"),
               "dU": torch.full((self.adapters, self.rank, self.rows), mark, device="cuda"),
               "dV": torch.full((self.adapters, self.rank, self.cols), mark, device="cuda")}
        part = {"Y": out["Y"][: self.n, : self.rows], "dX": out["dX"][: self.n, : self.cols], "S": out["S"][: self.n],
                "dU": out["dU"], "dV": out["dV"]}
        plan.sfb_adapter_forward(self.X, self.ids, part["Y"], part["S"])
        plan.sfb_adapter_backward(self.dY, self.X, self.ids, part["S"] if given else None, *(part[k] if k in want else None for k in ("dX", "dU", "dV")))
        torch.cuda.synchronize()
        for k in ("Y", "dX", "S"):
            assert (out[k][self.n :] == mark).all(), k
            assert (out[k][:, part[k].shape[1] :] == mark).all(), k
        return part


def check(case, got, names=("Y", "S", "dX", "dU", "dV")):
    want = case.expected()
    for k in names:
        v, b = want[k]
        off = (got[k].double() - v).abs()
        assert torch.isfinite(got[k]).all(), k
        worst = (off / b.clamp(min=1e-300)).max().item() if off.numel() else 0.0
        assert (off <= b).all(), f"{k}: {worst:.3g} of the bound"


SIZES = [
    # n, rows, cols, adapters, rank, ids
    (1, 10, 8, 1, 1, "one"),
    (1, 1, 1, 1, 1, "one"),
    (1, 1000, 520, 7, 16, "mixed"),
    (2, 129, 65, 3, 4, "mixed"),
    (16, 128, 64, 16, 16, "every"),
    (17, 333, 260, 5, 17, "mixed"),
    (37, 1001, 1999, 37, 16, "every"),
    (64, 257, 4000, 9, 33, "mixed"),
    (100, 515, 777, 100, 8, "every"),
    (128, 64, 256, 4, 4, "runs"),
    (200, 300, 1000, 3, 128, "mixed"),
    (255, 131, 120, 255, 16, "every"),
    (256, 256, 512, 2, 100, "runs"),
    (257, 640, 300, 6, 64, "runs"),
    (700, 1000, 900, 11, 24, "mixed"),
    (1003, 999, 1000, 8, 12, "runs"),
    (2500, 700, 600, 4, 48, "runs"),
    (300, 200, 200, 5, 16, "none"),
    (513, 100, 3001, 300, 16, "every"),
    # up to 64 samples with more rows than 37 tiles of 128: fewer tiles than SMs, more, whole rounds, a k-block each
    (1, 5001, 300, 2, 16, "one"),
    (16, 4900, 70, 5, 5, "mixed"),
    (33, 6000, 999, 8, 24, "mixed"),
    (64, 20001, 130, 9, 128, "mixed"),
    (29, 18944, 264, 29, 8, "every"),
    (40, 300, 9001, 4, 20, "mixed"),
    # operands that are copied first: rows an odd multiple of 16 bytes apart (X and dY; W)
    (70, 5000, 4104, 3, 16, "mixed"),
    (4100, 72, 136, 3, 24, "runs"),
    # many adapters among the samples of a tile: taken in the order of their adapters, or not, as they come
    (1500, 700, 6000, 100, 16, "every"),
    (1501, 700, 6000, 100, 16, "runs"),
    (1502, 6001, 707, 90, 24, "mixed"),
    (333, 9000, 1000, 150, 128, "mixed"),
    (4160, 2100, 4104, 64, 16, "mixed"),
    (1024, 6000, 6000, 100, 20, "none"),
    # few adapters with many samples each, whose gradients are summed in shares
    (3000, 300, 500, 1, 16, "mixed"),
    (2600, 131, 77, 2, 7, "runs"),
    (1700, 100, 900, 2, 100, "every"),
    # samples of few entries, by themselves and in the order of their adapters
    (70, 50, 60, 3, 20, "mixed"),
    (400, 30, 3000, 300, 8, "mixed"),
    # as many samples of one adapter as are taken out of the accumulators in several turns; the widest adapters
    (3000, 300, 200, 1, 20, "one"),
    (900, 136, 264, 2, 128, "mixed"),
]


@pytest.mark.parametrize("size", SIZES, ids=lambda s: "-".join(map(str, s)))
def test_against_the_formulas(size):
    c = Case(*size, seed=sum(size[:5]))
    got = c.run()
    assert c.plan.sfb_adapter_get_status() == 0
    check(c, got)


@pytest.mark.parametrize("size", [SIZES[3], SIZES[6], SIZES[13]], ids=lambda s: "-".join(map(str, s)))
def test_wide_pitches_and_s_not_given(size):
    c = Case(*size, seed=3, extra=24)
    got = c.run(given=False)
    check(c, got)
    # outputs that are not asked for stay as they are
    part = c.run(want=("dV",))
    assert (part["dX"] == 7).all() and (part["dU"] == 7).all() and torch.equal(part["dV"], got["dV"])


@pytest.mark.parametrize("n,rows,cols,adapters", [(5, 300, 520, 6), (40, 300, 520, 6), (300, 300, 520, 6), (1100, 300, 520, 6), (1500, 700, 6000, 100)])
def test_what_is_not_finite_stays_where_it_is(n, rows, cols, adapters):
    """An adapter and a sample that hold infinities and NaN: every result of the others has the bits it had."""
    c = Case(n, rows, cols, adapters, 20, "mixed", seed=n)
    before = c.run()
    c.U[2, 3, 17], c.U[2, 19, 299], c.V[2, 5, 100], c.V[2, 0, 0] = float("inf"), float("nan"), float("nan"), float("-inf")
    bad = n // 2
    c.X[bad], c.dY[bad] = float("nan"), float("inf")
    after = c.run()
    other = (c.ids != 2)
    other[bad] = False
    for k in ("Y", "S", "dX"):
        assert torch.equal(before[k][other], after[k][other]), k
    owner = int(c.ids[bad])
    keep = [a for a in range(adapters) if a not in (2, owner)]
    for k in ("dU", "dV"):
        assert torch.equal(before[k][keep], after[k][keep]), k
    assert torch.isnan(after["Y"][bad]).all()
    mine = c.ids == 2
    mine[bad] = False
    if mine.any():
        assert not torch.isfinite(after["Y"][mine][:, 17]).any() and not torch.isfinite(after["dX"][mine][:, 100]).any()


def test_infinite_products_are_infinite():
    """An infinite s keeps its sign in y and in dU: no NaN from its second word."""
    c = Case(40, 64, 64, 2, 4, "one", seed=1)
    c.X[3] = 0.0
    c.X[3, 5] = float("inf")
    c.V[1], c.U[1] = 1.0, 2.0
    c.W.fill_(1.0)
    c.scale.fill_(1.0)
    c.dY.fill_(1.0)
    got = c.run()
    assert (got["S"][3] == float("inf")).all() and (got["Y"][3] == float("inf")).all()
    assert (got["dU"][1] == float("inf")).all()


@pytest.mark.parametrize("rank", [4, 96])
def test_gradients_of_infinite_entries_are_infinite(rank):
    """An infinite entry of dy or x reaches dU or dV with the sign of the product, whatever the finite factor's lower bits are."""
    n, d = 40, 64
    c = Case(n, d, d, 2, rank, "one", seed=1)
    c.scale.fill_(1.0)
    c.V[1] = c.V[1].abs() + 0.25
    c.U[1] = -c.U[1].abs() - 0.25
    c.X.copy_(c.X.abs())
    c.dY.copy_(c.dY.abs())
    assert c.ids[3] == 1
    c.dY[3, 7] = float("inf")
    got = c.run()                                        # s > 0
    keep = torch.arange(d, device="cuda") != 7
    assert (got["dU"][1][:, 7] == float("inf")).all() and torch.isfinite(got["dU"][1][:, keep]).all()
    c.dY[3, 7], c.X[3, 7] = 1.0, float("inf")
    got = c.run()                                        # t < 0
    assert (got["dV"][1][:, 7] == float("-inf")).all() and torch.isfinite(got["dV"][1][:, keep]).all()


@pytest.mark.parametrize("n,rows,cols,adapters,rank", [(50, 100, 200, 4, 8), (1500, 700, 6000, 100, 16)])
def test_ids_out_of_range_take_no_adapter_and_are_reported(n, rows, cols, adapters, rank):
    c = Case(n, rows, cols, adapters, rank, "mixed", seed=2)
    c.ids[7], c.ids[20], c.ids[49] = adapters, -2, 2 ** 31 - 1
    got = c.run()
    assert c.plan.sfb_adapter_get_status() == S.STATUS_ADAPTER_RANGE
    assert c.plan.sfb_adapter_get_status() == 0
    check(c, got)
    assert (got["S"][[7, 20, 49]] == 0).all()


def test_no_samples():
    c = Case(3, 40, 48, 2, 4, "one")
    e = torch.empty(0, 40, dtype=torch.bfloat16, device="cuda"), torch.empty(0, 48, dtype=torch.bfloat16, device="cuda")
    ids = torch.empty(0, dtype=torch.int32, device="cuda")
    dU, dV = torch.ones(2, 4, 40, device="cuda"), torch.ones(2, 4, 48, device="cuda")
    c.plan.sfb_adapter_forward(e[1], ids, e[0])
    c.plan.sfb_adapter_backward(e[0], e[1], ids, None, e[1], dU, dV)
    torch.cuda.synchronize()
    assert (dU == 0).all() and (dV == 0).all()


def test_the_same_bits_again_and_fewer_samples():
    """Results do not depend on timing; a call of fewer samples than the handle has room for."""
    c = Case(700, 513, 700, 9, 16, "mixed", seed=4)
    a, b = c.run(), c.run()
    assert all(torch.equal(a[k], b[k]) for k in a)
    few = Case(700, 513, 700, 9, 16, "mixed", seed=4)
    few.n, few.X, few.dY, few.ids = 33, few.X[:33], few.dY[:33], few.ids[:33].contiguous()
    check(few, few.run())


def test_captured_and_replayed_with_new_values():
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        c = Case(300, 200, 320, 5, 16, "runs", seed=5, stream=s)
        got = c.run()
    s.synchronize()
    out = {k: torch.zeros_like(v) for k, v in got.items()}

    def calls():
        c.plan.sfb_adapter_forward(c.X, c.ids, out["Y"], out["S"])
        c.plan.sfb_adapter_backward(c.dY, c.X, c.ids, out["S"], out["dX"], out["dU"], out["dV"])

    calls()
    g = c.plan.capture(calls)
    gen = torch.Generator(device="cuda").manual_seed(9)
    c.X.copy_(padded((300, 320), gen))
    c.U.copy_(padded((5, 16, 200), gen, 0.3))
    c.ids.copy_(draw_ids("mixed", 300, 5, gen))
    torch.cuda.synchronize()
    for _ in range(2):
        with torch.cuda.stream(s):
            g.replay()
    torch.cuda.synchronize()
    check(c, out)


def test_two_handles_on_two_streams():
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    a, b = Case(500, 400, 900, 4, 16, "runs", seed=6, stream=s1), Case(60, 1000, 700, 30, 8, "mixed", seed=7, stream=s2)
    torch.cuda.synchronize()
    outs = []
    for c in (a, b):
        outs.append({"Y": torch.zeros(c.n, -(-c.rows // 8) * 8, dtype=torch.bfloat16, device="cuda")[:, : c.rows], "S": torch.zeros(c.n, c.rank, device="cuda")})
    torch.cuda.synchronize()
    for _ in range(20):
        for c, o in zip((a, b), outs):
            c.plan.sfb_adapter_forward(c.X, c.ids, o["Y"], o["S"])
    torch.cuda.synchronize()
    for c, o in zip((a, b), outs):
        check(c, o, ("Y", "S"))


def test_gradients_against_differences():
    """(f(theta + h e) - f(theta - h e)) / 2h for f = <Y, G>, with steps and values that bf16 holds exactly: f is linear in each entry,
    so a difference has no error of its own and only the bounds on Y are left."""
    n, rows, cols, a, r = 24, 40, 48, 3, 4
    c = Case(n, rows, cols, a, r, "mixed", seed=8)
    got = c.run()
    G = c.dY.double()
    _, bound = c.expected()["Y"]

    def f():
        Y = c.run(want=())["Y"].double()
        return (Y * G).sum().item()

    for name, t, at in (("dU", c.U, (1, 2, 7)), ("dV", c.V, (0, 1, 11)), ("dX", c.X, (5, 13)), ("dU", c.U, (2, 0, 39)), ("dV", c.V, (1, 3, 47))):
        old, h = t[at].item(), 64.0
        t[at] = h
        up, yb = f(), c.expected()["Y"][1]
        t[at] = -h
        down = f()
        t[at] = old
        tol = 2 * (yb * G.abs()).sum().item() / (2 * h) + U8 * abs(float(got[name][at]))
        assert abs((up - down) / (2 * h) - float(got[name][at])) <= tol, name
