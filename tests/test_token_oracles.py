"""The generator of the dropout and the sampling's plain form, pinned by hand (no GPU)."""
import numpy as np
import torch

from _tokens import mask, philox, sample


def test_philox_known_answers():
    """The published answers of Philox4x32-10 for all-zero and all-one counters and keys, and for digits of pi."""
    cases = [
        ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
        ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
        ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)),
    ]
    for counter, key, want in cases:
        assert tuple(int(v) for v in philox(np.array(counter, dtype=np.uint64), key)) == want


def test_masks():
    rng = torch.tensor([5, 7], dtype=torch.int64)
    m = mask(rng, 0, 400, 1001, 0.3)
    t = round(float(np.float32(0.3)) * 65536)
    assert set(np.unique(m.numpy())) == {0.0, 65536.0 / (65536 - t)}
    # 400,400 draws: the share of kept ones is off by 0.00072 (one standard deviation); six of them
    assert abs((m > 0).double().mean().item() - (1 - t / 65536)) < 6 * 0.00073
    assert not torch.equal(m, mask(rng, 1, 400, 1001, 0.3))
    assert torch.equal(mask(torch.tensor([5, 6], dtype=torch.int64), 1, 9, 30, 0.3), mask(rng, 0, 9, 30, 0.3))
    assert (mask(rng, 0, 5, 9, 0.0) == 1).all() and (mask(rng, 0, 5, 9, 1.0) == 0).all()


def test_sampling_by_hand():
    z = np.log(np.array([0.1, 0.4, 0.2, 0.3]))
    assert [sample(z, u)[0] for u in (0.0, 0.09, 0.11, 0.49, 0.51, 0.69, 0.71, 0.99, 1.0)] == [0, 0, 1, 1, 2, 2, 3, 3, 3]
    assert sample(z, 0.5, top_k=2)[::2] == (1, 2) and sample(z, 0.6, top_k=2)[0] == 3
    assert sample(z, 0.99, top_p=0.65)[::2] == (3, 2) and sample(z, 0.99, top_p=0.75)[2] == 3
    assert sample(z, 0.0, min_p=0.6)[::2] == (1, 2) and sample(z, 0.3, top_p=0.0) == (1, 0.0, 1)
    assert abs(sample(z, 0.5, top_k=2)[1] - np.log(0.4 / 0.7)) < 1e-12
    assert sample(np.array([2.0, 2.0, 2.0]), 0.9, top_k=2)[::2] == (1, 2)              # ties: the first ones
    assert sample(np.full(3, -np.inf), 0.5) == (-1, -np.inf, 0) and sample(np.array([np.nan, 1.0]), 0.0)[::2] == (1, 1)
    assert sample(np.array([1.0, np.inf, 5.0, np.inf]), 0.6)[0] == 3 and sample(z, 0.9, temperature=0.0) == (1, 0.0, 1)
