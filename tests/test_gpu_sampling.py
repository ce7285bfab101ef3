"""Sampling on the GPU against 64 bits: classes and counts are equal; the log-probability is rounded once (2^-24 of it), and the weights
are off by 4e-14, so its argument by less than 1e-12."""
import numpy as np
import pytest
import torch

import paper_1409_5705_b200 as S
from _tokens import sample

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def logits(n, classes, dtype, seed, std=2.0, pitch=0, offset=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    pitch = pitch or classes
    flat = torch.empty(n * pitch + offset, device="cuda").normal_(0.0, std, generator=gen).to(dtype)
    return flat[offset:].view(n, pitch)[:, :classes]


def check(Z, u, **settings):
    """Draws with logp and kept, compares every row, and returns the classes."""
    n, classes = Z.shape
    dev = {k: None if v is None else torch.as_tensor(v, dtype=torch.int32 if k == "top_k" else F32).expand(n).contiguous().cuda() for k, v in settings.items()}
    u = torch.as_tensor(u, dtype=F32).expand(n).contiguous().cuda()
    ids, kept, logp = torch.full((n + 1,), -7, dtype=torch.int32, device="cuda"), torch.full((n + 1,), -7, dtype=torch.int32, device="cuda"), \
        torch.full((n + 1,), 9.0, device="cuda")
    plan = S.Sampler(classes, Z.dtype, n)
    plan.sfb_sample(Z, u, ids[:n], logp=logp[:n], kept=kept[:n], **dev)
    bare = torch.empty(n, dtype=torch.int32, device="cuda")
    plan.sfb_sample(Z, u, bare, **dev)
    assert torch.equal(bare, ids[:n]) and ids[n] == -7 and kept[n] == -7 and logp[n] == 9
    off = {"temperature": 1.0, "top_k": 0, "top_p": 1.0, "min_p": 0.0}
    z, host = Z.double().cpu().numpy(), {k: None if v is None else v.cpu().tolist() for k, v in dev.items()}
    for i in range(n):
        want = sample(z[i], float(u[i]), **{k: host[k][i] if host.get(k) is not None else v for k, v in off.items()})
        got = int(ids[i]), float(logp[i]), int(kept[i])
        assert (got[0], got[2]) == (want[0], want[2]), (i, got, want)
        assert got[1] == want[1] or abs(got[1] - want[1]) <= 2.0 ** -24 * abs(want[1]) + 1e-12, (i, got, want)
    return ids[:n]


def uniform(n, seed):
    return torch.rand(n, generator=torch.Generator().manual_seed(seed))


SIZES = [(1, 1), (3, 2), (2, 7), (5, 100), (40, 1000), (1, 5003), (9, 32_000), (1, 99_999), (2, 325_000), (300, 2047)]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("n,classes", SIZES)
@pytest.mark.parametrize("settings", [dict(), dict(temperature=0.7), dict(top_k=5), dict(top_k=50, top_p=0.9, temperature=0.8), dict(top_p=0.5), dict(top_p=0.99),
                                      dict(min_p=0.05), dict(top_k=1000, top_p=0.95, min_p=0.01, temperature=1.5), dict(temperature=6.0, top_p=0.8),
                                      dict(temperature=0.0)], ids=str)
def test_against_64_bits(n, classes, dtype, settings):
    check(logits(n, classes, dtype, n + classes), uniform(n, classes), **settings)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_each_row_its_own(dtype):
    n, gen = 240, torch.Generator().manual_seed(1)
    k = torch.randint(0, 400, (n,), generator=gen, dtype=torch.int32)
    t, p, m = torch.rand(n, generator=gen) * 2, torch.rand(n, generator=gen) * 1.1, torch.rand(n, generator=gen) * 0.2
    t[::11], p[::7], m[::3], k[::5] = 0.0, 1.0, 0.0, 0
    check(logits(n, 3001, dtype, 5, std=3.0), uniform(n, 2), temperature=t, top_k=k, top_p=p, min_p=m)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("pitch,offset", [(1001, 0), (1008, 0), (1000, 1), (1003, 8)])
def test_strides_and_offsets(dtype, pitch, offset):
    check(logits(20, 1000, dtype, 3, pitch=pitch, offset=offset), uniform(20, 3), top_p=0.9, top_k=300)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("ctas", ["one", "some"])
def test_ties(dtype, ctas):
    """Few values: filters end among equals, of which the first are kept; all equal; two zeros of different sign."""
    classes = 1000 if ctas == "one" else 40_000
    gen = torch.Generator().manual_seed(7)
    Z = torch.randint(-3, 4, (24, classes), generator=gen).to(dtype).cuda()
    Z[:4] = 1.5
    Z[4, ::2], Z[4, 1::2] = 0.0, -0.0
    for settings in (dict(top_k=7), dict(top_k=classes // 2), dict(top_p=0.3), dict(top_p=0.77, top_k=classes // 3), dict(min_p=1.0), dict(min_p=0.3, top_p=0.9)):
        check(Z, uniform(24, 4), **settings)
    check(Z, 0.0, top_k=3)
    check(Z, 1.0 - 2.0 ** -24, top_k=3)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("classes", [9, 1000, 70_000])
def test_masked_rows(dtype, classes):
    """Minus infinity, the type's lowest value, plus infinity, NaN; rows of nothing else."""
    lowest, inf, nan = torch.finfo(dtype).min, float("inf"), float("nan")
    Z = logits(14, classes, dtype, 6)
    Z[0] = -inf
    Z[1] = nan
    Z[2] = lowest
    Z[3] = -inf
    Z[3, classes // 2] = 3.0
    Z[4] = lowest
    Z[4, classes - 1] = 2.0
    Z[5, : classes // 2] = -inf
    Z[6, classes // 3 :] = lowest
    Z[7, ::3] = nan
    Z[8, 4] = inf
    Z[9, 2::3] = inf
    Z[10], Z[10, 5] = lowest, inf
    Z[11] = torch.finfo(dtype).max
    Z[12] = -inf
    Z[12, 1], Z[12, classes - 2] = lowest, lowest
    Z[13, ::2] = nan
    Z[13, 1::2] = -inf
    for settings in (dict(), dict(top_k=3), dict(top_p=0.6), dict(top_k=classes - 2, top_p=0.9999), dict(min_p=0.2), dict(temperature=0.0),
                     dict(temperature=float("inf")), dict(temperature=float("inf"), top_p=0.4), dict(temperature=1e-6, top_p=0.9), dict(temperature=1e30, top_k=classes // 2, top_p=0.5)):
        check(Z, uniform(14, 8), **settings)


def test_settings_that_say_nothing():
    Z, nan = logits(6, 500, F32, 9), float("nan")
    base = check(Z, uniform(6, 1))
    for settings in (dict(top_k=0), dict(top_k=-3), dict(top_k=500), dict(top_k=2 ** 31 - 1), dict(top_p=1.0), dict(top_p=7.0), dict(top_p=nan), dict(min_p=-1.0), dict(min_p=nan)):
        assert torch.equal(base, check(Z, uniform(6, 1), **settings))
    best = Z.argmax(dim=1).int()
    for settings in (dict(temperature=-1.0), dict(temperature=nan), dict(top_k=1), dict(top_p=0.0), dict(top_p=-2.0), dict(min_p=5.0), dict(temperature=1e-30)):
        assert torch.equal(best, check(Z, uniform(6, 1), **settings))


@pytest.mark.parametrize("u", [0.0, 1.0, 2.0, -1.0, float("nan"), 1.0 - 2.0 ** -24])
def test_random_numbers_at_the_ends(u):
    Z = logits(5, 3000, BF16, 3)
    Z[:, -100:] = -30.0                     # (in reach of the last draw, barely)
    Z[1, -50:] = -float("inf")
    Z[2, -70:] = -60000.0                   # weight zero
    check(Z, u)
    check(Z, u, top_k=20)


def test_a_row_that_shared_memory_does_not_hold():
    """Longer than what eight CTAs keep, and of odd length."""
    Z = logits(1, 1_000_003, F32, 2, std=1.5)
    for settings in (dict(), dict(top_k=100_000, top_p=0.9), dict(temperature=3.0, top_p=0.7), dict(temperature=0.0)):
        check(Z, uniform(1, 3), **settings)


@pytest.mark.parametrize("p", [0.001, 0.1, 0.5, 0.9, 0.99, 0.9999])
@pytest.mark.parametrize("std", [0.01, 0.5, 4.0, 30.0])
def test_nuclei_of_any_width(p, std):
    check(logits(12, 20_000, F32, 4, std=std), uniform(12, 5), top_p=p)


def test_draws_follow_the_shares():
    """4,000 draws of 5 classes: a share q is off by sqrt(q (1 - q) / 4000); five of that."""
    z = torch.log(torch.tensor([0.05, 0.4, 0.1, 0.25, 0.2]))
    n = 4000
    ids, u = torch.empty(n, dtype=torch.int32, device="cuda"), uniform(n, 9).cuda()
    S.Sampler(5, F32, n).sfb_sample(z.cuda().expand(n, 5).contiguous(), u, ids)
    got = torch.bincount(ids.long(), minlength=5).double().cpu() / n
    q = z.double().exp()
    assert ((got - q).abs() <= 5 * (q * (1 - q) / n).sqrt()).all()


def test_captured_replayed_and_on_another_stream():
    s, n, classes = torch.cuda.Stream(), 30, 50_000
    Z, u, ids, logp = logits(n, classes, BF16, 1), uniform(n, 2).cuda(), torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(n, device="cuda")
    p = torch.full((n,), 0.8, device="cuda")
    torch.cuda.synchronize()
    plan = S.Sampler(classes, BF16, n, stream=s)
    call = lambda: plan.sfb_sample(Z, u, ids, top_p=p, logp=logp)
    call()
    g = plan.capture(call)
    for step in range(3):
        Z.copy_(logits(n, classes, BF16, 10 + step))
        u.copy_(uniform(n, 20 + step))
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            g.replay()
        torch.cuda.synchronize()
        got = ids.clone()
        assert torch.equal(got, check(Z, u.cpu(), top_p=0.8))
