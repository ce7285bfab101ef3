"""Plain 64-bit forms of the lookup, its gradient, dropout and sampling, for the tests."""
import numpy as np
import torch


def philox(counter, key):
    """Philox4x32-10 of counters [..., 4] and a key of two words (uint64 arrays that hold 32-bit words)."""
    c = [counter[..., i].astype(np.uint64) for i in range(4)]
    k = [int(key[0]), int(key[1])]
    low = np.uint64(0xFFFFFFFF)
    for _ in range(10):
        a, b = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.stack(c, axis=-1).astype(np.uint32)


def threshold(p):
    return int(np.rint(float(np.float32(p)) * 65536.0))


def mask(rng, call, n, cols, p):
    """m of include/sfb.h, fp64 [n, cols]."""
    seed, offset = (int(v) % (1 << 64) for v in rng.tolist())
    offset = (offset + call) % (1 << 64)
    groups = (cols + 7) // 8
    c = np.zeros((n, groups, 4), dtype=np.uint64)
    c[..., 0], c[..., 1] = np.arange(groups)[None, :], np.arange(n)[:, None]
    c[..., 2], c[..., 3] = offset & 0xFFFFFFFF, offset >> 32
    words = philox(c, (seed & 0xFFFFFFFF, seed >> 32))
    bits = np.stack([words & 0xFFFF, words >> 16], axis=-1).reshape(n, groups * 8)[:, :cols]
    t = threshold(p)
    return torch.from_numpy(np.where(bits >= t, 65536.0 / (65536 - t) if t < 65536 else 0.0, 0.0))


def sample(z, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(class, log-probability, kept) for one row: z in fp64 (numpy)."""
    z = np.where(np.isnan(z), -np.inf, z)
    order = np.lexsort((np.arange(z.size), -z))
    s = z[order]
    finite = int(np.count_nonzero(s > -np.inf))
    if finite == 0:
        return -1, -np.inf, 0
    if not temperature > 0 or top_k == 1 or top_p <= 0:
        return int(order[0]), 0.0, 1
    s = s[:finite]
    with np.errstate(invalid="ignore", over="ignore"):
        d = np.where(s == s[0], 0.0, s - s[0])
        w = np.where(s == s[0], 1.0, 0.0 if np.isinf(s[0]) else np.exp(d / temperature))
    n = min(finite, top_k) if top_k > 0 else finite
    if top_p < 1:
        upto = np.cumsum(w[:n])
        n = min(n, 1 + int(np.searchsorted(upto, top_p * upto[-1], side="left")))
    min_p = min(1.0, max(0.0, min_p)) if min_p == min_p else 0.0
    n = int(np.count_nonzero(w[:n] >= min_p))
    kept = np.sort(order[:n])
    back = np.empty(z.size)
    back[order[:n]] = w[:n]
    upto = np.cumsum(back[kept])
    u = min(1.0, max(0.0, u)) if u == u else 0.0
    i = int(np.searchsorted(upto, u * upto[-1], side="right"))
    if i >= n:
        i = int(np.flatnonzero(back[kept] > 0)[-1])
    return int(kept[i]), float(np.log(back[kept[i]] / upto[-1])), n
