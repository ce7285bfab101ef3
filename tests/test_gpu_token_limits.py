"""Lookup, gradient, dropout and sampling at the ends of what their handles allow: offsets beyond 2^31 entries, millions of samples, many rows, long
rows; and what the binding refuses.  Bounds: those of the operators' own tests."""
import numpy as np
import pytest
import torch

import paper_1409_5705_b200 as S
from _tokens import mask, sample
from test_gpu_embedding import ULP, check_gradient

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def test_offsets_beyond_2_31():
    """A table of 2.8e9 entries, whose last rows are looked up, and its gradient, in both forms."""
    tokens, dim, n = 70_000, 40_000, 40
    table = torch.empty(tokens, dim, dtype=BF16, device="cuda")
    table[-50:] = torch.randn(50, dim, device="cuda").bfloat16()
    ids = torch.randint(tokens - 50, tokens, (n,), dtype=torch.int32, device="cuda")
    plan, X = S.Embedding(table, 2000), torch.zeros(n, dim, dtype=BF16, device="cuda")
    plan.sfb_embed_forward(ids, X)
    assert torch.equal(X, table[ids.long()])
    del plan, table
    dE = torch.full((tokens, dim), 3.0, device="cuda")
    plan = S.Embedding(torch.empty(tokens, dim, dtype=BF16, device="cuda"), 2000)
    for count in (n, 300):                   # the ways of few and of more samples
        i = ids[torch.arange(count, device="cuda") % n]
        d = torch.randn(count, dim, device="cuda").bfloat16()
        want = torch.zeros(50, dim, dtype=torch.float64, device="cuda").index_add_(0, i.long() - (tokens - 50), d.double())
        size = torch.zeros(50, dim, dtype=torch.float64, device="cuda").index_add_(0, i.long() - (tokens - 50), d.double().abs())
        plan.sfb_embed_backward(i, d, dE)
        assert ((dE[-50:].double() - want).abs() <= (count + 4) * ULP * size).all() and dE[:-50].abs().max() == 0
        plan.sfb_embed_backward(i, d, dE, alpha=-1.0, add=True)
        assert (dE[-50:].abs() <= 2 * (count + 5) * ULP * size).all() and dE[:-50].abs().max() == 0


@pytest.mark.parametrize("n,tokens,dim,kind", [((1 << 22) + 5, 1000, 3, "skew"), (1 << 21, 1 << 21, 2, "uniform"), (1 << 20, 5, 8, "one"), (257, 1 << 24, 1, "runs"), (256, 77, 20_001, "skew")])
@pytest.mark.parametrize("add", [False, True])
def test_many_samples_and_tokens(n, tokens, dim, kind, add):
    check_gradient(n, tokens, dim, kind, BF16, 0.0, add)


@pytest.mark.parametrize("n", [255, 256, 257, 8191, 16384, 16385, 65536, 65537])
def test_where_the_ways_of_the_gradient_change(n):
    check_gradient(n, 300, 40, "skew", BF16, 0.1, False)
    check_gradient(n, 300, 40, "one", F32, 0.0, True)


def test_dropout_of_many_rows_and_long_ones():
    rng = torch.tensor([3, 4], device="cuda")
    for n, cols in ((70_000, 40_000), (40_000_000, 9), (2, 1_400_000_000 // 2)):
        X = torch.ones(n, cols, dtype=BF16, device="cuda")
        S.Dropout(0.3, rng).sfb_dropout_apply(X, X)
        if n > 2:
            assert torch.equal(X[:3].double().cpu(), mask(rng, 0, 3, cols, 0.3).bfloat16().double())
            assert abs((X[-1000:] > 0).double().mean().item() - 0.7) < 6 * (0.21 / (1000 * cols)) ** 0.5
        else:
            assert torch.equal(X[:, :5000].double().cpu(), mask(rng, 0, n, 5000, 0.3).bfloat16().double())
        del X


@pytest.mark.parametrize("n,classes", [(9_000, 262_144), (100_003, 33), (3, 5_000_001), (700, 90_001)])
def test_many_rows_and_long_ones(n, classes):
    Z = torch.empty(n, classes, dtype=BF16, device="cuda").normal_(0.0, 3.0)
    u, ids, logp, kept = torch.rand(n, device="cuda"), torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(n, device="cuda"), torch.empty(n, dtype=torch.int32, device="cuda")
    plan, rows = S.Sampler(classes, BF16, n), sorted({0, 1, n // 2, n - 2, n - 1} & set(range(n)))
    for kw in (dict(), dict(top_p=torch.full((n,), 0.8, device="cuda")), dict(top_k=torch.full((n,), 40, dtype=torch.int32, device="cuda"), min_p=torch.full((n,), 0.05, device="cuda"))):
        plan.sfb_sample(Z, u, ids, logp=logp, kept=kept, **kw)
        assert ((ids >= 0) & (ids < classes) & (kept >= 1) & (logp <= 0)).all()
        for i in rows:
            want = sample(Z[i].double().cpu().numpy(), float(u[i]), **{k: v[i].item() for k, v in kw.items()})
            assert (int(ids[i]), int(kept[i])) == (want[0], want[2]) and abs(float(logp[i]) - want[1]) <= ULP * abs(want[1]) + 1e-12


def test_sampling_twice_is_the_same_bits():
    Z, u = torch.randn(70, 60_000, device="cuda") * 2, torch.rand(70, device="cuda")
    p, k = torch.rand(70, device="cuda"), torch.randint(0, 3000, (70,), device="cuda", dtype=torch.int32)
    plan, got = S.Sampler(60_000, F32, 70), []
    for _ in range(4):
        ids, logp = torch.empty(70, dtype=torch.int32, device="cuda"), torch.empty(70, device="cuda")
        plan.sfb_sample(Z, u, ids, top_p=p, top_k=k, logp=logp)
        got.append((ids, logp))
    assert all(torch.equal(a, b) for g in got[1:] for a, b in zip(got[0], g))


def test_what_the_binding_refuses():
    t = torch.zeros(10, 16, device="cuda")
    emb, drop, i = S.Embedding(t, 8), S.Dropout(0.1, torch.zeros(2, dtype=torch.int64, device="cuda")), torch.zeros(4, dtype=torch.int32, device="cuda")
    x = torch.zeros(4, 16, device="cuda")
    for call in (lambda: emb.sfb_embed_forward(i.long(), x), lambda: emb.sfb_embed_forward(i, x.bfloat16()), lambda: emb.sfb_embed_forward(i, x[:3]),
                 lambda: emb.sfb_embed_forward(i, torch.zeros(16, 4, device="cuda").t()), lambda: emb.sfb_embed_forward(i, x.cpu()), lambda: emb.sfb_embed_forward(i, x, 0.1),
                 lambda: emb.sfb_embed_backward(i, x, t.bfloat16()), lambda: emb.sfb_embed_backward(i, x, t[:9]), lambda: drop.sfb_dropout_apply(x, x.half()),
                 lambda: drop.sfb_dropout_apply(x, x, x[:2]), lambda: drop.sfb_dropout_apply(x.double(), x.double()), lambda: S.Sampler(5, torch.float64, 3),
                 lambda: S.Sampler(16, F32, 4).sfb_sample(x, torch.zeros(4, device="cuda"), i.long()), lambda: S.Sampler(15, F32, 4).sfb_sample(x, torch.zeros(4, device="cuda"), i),
                 lambda: S.Sampler(16, F32, 4).sfb_sample(x, torch.zeros(3, device="cuda"), i), lambda: S.Embedding(t.t()[:, :3], 4), lambda: S.Embedding(t.double(), 4)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: S.Sampler(16, F32, 3).sfb_sample(x, torch.zeros(4, device="cuda"), i), lambda: S.Dropout(1.5, torch.zeros(2, dtype=torch.int64, device="cuda")),
                 lambda: S.Embedding(t, 3).sfb_embed_forward(i, x), lambda: S.Embedding(t, -1), lambda: emb.sfb_embed_backward(i, x, t, alpha=float("nan"))):
        with pytest.raises(S.SfbError):
            call()
    # calls of nothing
    S.Sampler(16, F32, 4).sfb_sample(x[:0], torch.zeros(0, device="cuda"), i[:0])
    drop.sfb_dropout_apply(x[:0], x[:0])
