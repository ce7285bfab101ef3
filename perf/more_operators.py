"""The operators on either side of the products with W, as cases that can be timed and compared: token ids become samples on the way
in, logits become answers on the way out.

  lookup    rows of a table for token ids, scaled, perhaps dropped out: the samples that the products take
  gradient  the gradient of that with respect to the table, from the gradients of the samples: written whole, or ("add") added to
            the rows that some token named
  dropout   entries of a matrix dropped by a counter-based generator, the rest rescaled, a residual added
  sample    one class drawn for each row of logits, from given random numbers, after temperature, top-k, top-p and min-p;
            with it the log-probability under what the filters kept, and how many classes they kept

Tokens fall on the table as words do (a few make up much of a text, most are rare); some places are padding (-1).
"filters" of a sampling case: "top" (one setting for all rows, top-k and top-p), "mixed" (each row its own), "none", "flat" (a high
temperature, under which top-p keeps thousands of classes), "greedy".

The generator of "dropout" is Philox4x32-10 (Salmon, Moraes, Dror and Shaw, 2011): key the seed's two words, counter
(column / 8, row, the offset's two words), and 16 bits an entry: entry j of a group of eight takes half j % 2 of word j / 2.  An entry
is kept where its bits are at least t = round(65536 p), and multiplied with 65536 / (65536 - t).
"""
import functools
import math

import numpy as np
import torch

own = False

_TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
_SIZE = {"fp32": 4.0, "bf16": 2.0, "fp16": 2.0}
_MASK = 0xFFFFFFFF


def _lookup(name, n, tokens, dim, table, out, p):
    return {"name": name, "op": "lookup", "n": n, "tokens": tokens, "dim": dim, "table": table, "out": out, "p": p}


def _gradient(name, n, tokens, dim, out, p, add):
    return {"name": name, "op": "gradient", "n": n, "tokens": tokens, "dim": dim, "out": out, "p": p, "add": add}


def _dropout(name, n, cols, dtype, p, residual):
    return {"name": name, "op": "dropout", "n": n, "cols": cols, "dtype": dtype, "p": p, "residual": residual}


def _sample(name, n, classes, dtype, filters):
    return {"name": name, "op": "sample", "n": n, "classes": classes, "dtype": dtype, "filters": filters}


def listed():
    return [
        # the tokens of a few requests, each one step on: latency of a single answer
        _lookup("lookup_serve", 7, 10_000, 5_000, "bf16", "bf16", 0.0),
        # the samples of a training step from the fp32 master table, dropped out on the way
        _lookup("lookup_train", 16_384, 325_000, 2_000, "fp32", "bf16", 0.1),
        # the smallest training step of the repository
        _gradient("gradient_tiny", 128, 1_000, 256, "bf16", 0.0, False),
        # the gradient of a whole table for the optimiser, through the dropout of the lookup
        _gradient("gradient_table", 16_384, 50_000, 2_000, "bf16", 0.1, False),
        # a step that goes straight to the rows of a large table that the minibatch named
        _gradient("gradient_rows", 65_000, 325_000, 1_000, "bf16", 0.0, True),
        # one small layer of samples
        _dropout("dropout_tiny", 128, 256, "bf16", 0.1, False),
        # a layer's output in training, added to the stream that went around it
        _dropout("dropout_residual", 8_192, 5_000, "bf16", 0.1, True),
        # fp32 features of odd width
        _dropout("dropout_large", 16_384, 9_999, "fp32", 0.25, False),
        # one request's next class out of the repository's largest set: latency of a single answer
        _sample("sample_one", 1, 325_000, "bf16", "top"),
        # a batch of requests that arrived together, each with its own settings
        _sample("sample_batch", 64, 325_000, "bf16", "mixed"),
        # many draws at once for a training step's rollouts, from fp32 logits, all classes kept
        _sample("sample_many", 2_048, 10_000, "fp32", "none"),
        # a high temperature, where the filters keep much of an odd-sized set
        _sample("sample_flat", 37, 99_999, "fp32", "flat"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("lookup", "gradient", "dropout", "sample", "sample"))
    while True:
        if op in ("lookup", "gradient"):
            n, tokens, dim = _log(rng, 1, 70_000), _log(rng, 100, 325_000), _log(rng, 16, 10_000)
            p = rng.choice((0.0, 0.0, 0.1, 0.3))
            if n * dim > 66_000_000 or tokens * dim > 650_000_000:
                continue
            if op == "lookup":
                return _lookup(None, n, tokens, dim, rng.choice(sorted(_TYPES)), rng.choice(sorted(_TYPES)), p)
            add = rng.random() < 0.5
            if not add and tokens * dim > 330_000_000:
                continue
            return _gradient(None, n, tokens, dim, rng.choice(sorted(_TYPES)), p, add)
        if op == "dropout":
            n, cols = _log(rng, 1, 40_000), _log(rng, 16, 20_000)
            if n * cols <= 160_000_000:
                return _dropout(None, n, cols, rng.choice(sorted(_TYPES)), rng.choice((0.05, 0.1, 0.25, 0.5)), rng.random() < 0.5)
        else:
            n, classes = _log(rng, 1, 2_048), _log(rng, 100, 400_000)
            if n * classes <= 20_800_000:
                return _sample(None, n, classes, rng.choice(sorted(_TYPES)), rng.choice(("top", "mixed", "mixed", "none", "flat", "greedy")))


# ---- inputs ----------------------------------------------------------------------------------------------------------------------
def _wide(shape, gen, std, dtype):
    """Normal values whose rows start 16 bytes apart or a multiple of that, as the library's operands do."""
    pitch = -(-shape[-1] // 8) * 8
    t = torch.empty((*shape[:-1], pitch), dtype=dtype, device="cuda")
    t.normal_(0.0, std, generator=gen)
    return t[..., : shape[-1]]


@functools.lru_cache(maxsize=None)
def _shares(tokens):
    """How often each token comes up: falling with its number, the first ones a few per cent each."""
    w = 1.0 / (torch.arange(tokens, dtype=torch.float64) + 2.7) ** 1.05
    return w / w.sum()


def _ids(case, gen):
    n, shares = case["n"], _shares(case["tokens"]).cuda()
    at = torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)
    ids = torch.searchsorted(shares.cumsum(0), at).clamp(max=case["tokens"] - 1).int()
    if n > 64:                              # padding behind the texts' ends
        ids[torch.rand(n, generator=gen, device="cuda") < 0.03] = -1
    return ids


def _distinct(case):
    """How many tokens a minibatch names, on average."""
    n = case["n"] * (0.97 if case["n"] > 64 else 1.0)
    return float((1.0 - (1.0 - _shares(case["tokens"])) ** n).sum())


def _settings(case, gen):
    """Temperature, top-k, top-p and min-p of each row; None: not asked for."""
    n, classes, f32 = case["n"], case["classes"], torch.float32
    full = lambda v, t=f32: torch.full((n,), v, dtype=t, device="cuda")
    rand = lambda lo, hi: torch.rand(n, generator=gen, device="cuda") * (hi - lo) + lo
    none = {"temperature": None, "top_k": None, "top_p": None, "min_p": None}
    kind = case["filters"]
    if kind == "none":
        return none
    if kind == "greedy":
        return {**none, "temperature": full(0.0)}
    if kind == "top":
        return {**none, "temperature": full(0.8), "top_k": full(50, torch.int32), "top_p": full(0.9)}
    if kind == "flat":
        return {**none, "temperature": rand(2.5, 5.0), "top_p": rand(0.6, 0.95)}
    temperature, top_p, min_p = rand(0.5, 1.3), rand(0.3, 0.99), rand(0.0, 0.1)
    top_k = torch.randint(1, max(2, min(classes, 2_000)), (n,), generator=gen, device="cuda", dtype=torch.int32)
    which = torch.arange(n, device="cuda")
    temperature[which % 9 == 4] = 0.0       # some requests are answered greedily, some leave a filter out
    top_k[which % 3 == 1] = 0
    top_p[which % 4 == 2] = 1.0
    min_p[which % 2 == 0] = 0.0
    return {"temperature": temperature, "top_k": top_k, "top_p": top_p, "min_p": min_p}


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    state, op = {"case": case}, case["op"]
    if op == "sample":
        n, classes, dtype = case["n"], case["classes"], _TYPES[case["dtype"]]
        # most classes near one another, some far above: what a trained head gives
        z = _wide((n, classes), gen, 2.0, torch.float32)
        z += 6.0 * (torch.rand((n, classes), generator=gen, device="cuda") < 1e-4)
        pitch = -(-classes // 8) * 8
        logits = torch.zeros((n, pitch), dtype=dtype, device="cuda")[:, :classes]
        logits.copy_(z)
        state.update(logits=logits, u=torch.rand(n, generator=gen, device="cuda"), settings=_settings(case, gen),
                     ids=torch.zeros(n, dtype=torch.int32, device="cuda"), logp=torch.zeros(n, device="cuda"),
                     kept=torch.zeros(n, dtype=torch.int32, device="cuda"))
        if own:
            import paper_1409_5705_b200 as S

            state["plan"] = S.Sampler(classes, dtype, max_samples=n)
        return state
    # what the generator of the dropout starts from: a seed, and an offset that a program moves on from step to step
    state.update(p=case["p"], rng=torch.tensor([int(seed) * 7_919 + 12_345, int(seed) % 1_000 + (1 << 33)], dtype=torch.int64).cuda())
    if op == "dropout":
        n, cols, dtype = case["n"], case["cols"], _TYPES[case["dtype"]]
        state.update(X=_wide((n, cols), gen, 1.0, dtype), R=_wide((n, cols), gen, 1.0, dtype) if case["residual"] else None,
                     Y=_wide((n, cols), gen, 0.0, dtype))
        if own:
            import paper_1409_5705_b200 as S

            state["drop"] = S.Dropout(case["p"], state["rng"])
        return state
    n, tokens, dim, out = case["n"], case["tokens"], case["dim"], _TYPES[case["out"]]
    state.update(ids=_ids(case, gen), scale=math.sqrt(dim))
    if op == "lookup":
        table = _wide((tokens, dim), gen, 1.0 / math.sqrt(dim), _TYPES[case["table"]])
        state.update(table=table, X=_wide((n, dim), gen, 0.0, out))
    else:
        # an fp32 table is moved by a step, in place; otherwise its gradient is wanted
        dtable = _wide((tokens, dim), gen, 1.0 / math.sqrt(dim) if case["add"] else 0.0, torch.float32)
        state.update(table=dtable, dX=_wide((n, dim), gen, 1e-3, out), alpha=-0.05 if case["add"] else 1.0)
    if own:
        import paper_1409_5705_b200 as S

        state["drop"] = S.Dropout(case["p"], state["rng"]) if case["p"] > 0 else None
        state["plan"] = S.Embedding(state["table"], max_ids=n, out_dtype=out, scale=state["scale"])
    return state


# ---- the plain form --------------------------------------------------------------------------------------------------------------
def _words(rng, rows, blocks):
    """The generator's four words for each row and group of eight columns, as 64-bit whole numbers."""
    seed, offset = rng[0], rng[1]
    k0, k1 = seed & _MASK, (seed >> 32) & _MASK
    c0 = torch.arange(blocks, device=rng.device)[None, :].expand(rows, blocks)
    c1 = torch.arange(rows, device=rng.device)[:, None].expand(rows, blocks)
    c2, c3 = (offset & _MASK).expand(rows, blocks), ((offset >> 32) & _MASK).expand(rows, blocks)
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57          # 64 bits each: the high word's sign bit is masked off again
        c0, c1, c2, c3 = ((b >> 32) & _MASK) ^ c1 ^ k0, b & _MASK, ((a >> 32) & _MASK) ^ c3 ^ k1, a & _MASK
        k0, k1 = (k0 + 0x9E3779B9) & _MASK, (k1 + 0xBB67AE85) & _MASK
    return c0, c1, c2, c3


def _threshold(p):
    return int(round(float(np.float32(p)) * 65_536.0))


def _factor(rng, rows, cols, p):
    """0 where an entry is dropped, 65536 / (65536 - t) where it is kept."""
    t = _threshold(p)
    words = _words(rng, rows, -(-cols // 8))
    bits = torch.stack([h for w in words for h in (w & 0xFFFF, w >> 16)], dim=-1).view(rows, -1)[:, :cols]
    return (bits >= t).float() * (65_536.0 / (65_536 - t))


def _plain_sample(state):
    z, s = state["logits"].double(), state["settings"]
    n, classes = z.shape
    z = torch.where(torch.isnan(z), -math.inf, z)
    srt, idx = torch.sort(z, dim=1, descending=True, stable=True)
    rank, most = torch.arange(classes, device=z.device)[None, :], srt[:, :1]
    temperature = torch.ones(n, device=z.device) if s["temperature"] is None else s["temperature"]
    warm = (temperature > 0)[:, None]
    below = torch.where(srt == most, 0.0, srt - most) / torch.where(warm, temperature[:, None].double(), 1.0)
    w = torch.where(srt > -math.inf, torch.exp(below), 0.0)
    keep = (srt > -math.inf) & (warm | (rank == 0))
    if s["top_k"] is not None:
        keep &= (rank < s["top_k"][:, None]) | (s["top_k"][:, None] <= 0)
    if s["top_p"] is not None:
        upto = torch.cumsum(w * keep, dim=1)
        p = s["top_p"][:, None].double()
        keep &= (upto - w * keep < p * upto[:, -1:]) | (rank == 0) | (p >= 1)
    if s["min_p"] is not None:
        keep &= (w >= s["min_p"][:, None].double().clamp(max=1.0)) | (rank == 0)
    w = torch.zeros_like(w).scatter_(1, idx, w * keep)
    upto = torch.cumsum(w, dim=1)
    total = upto[:, -1:]
    got = (upto <= state["u"][:, None].double() * total).sum(dim=1, keepdim=True)
    last = (w > 0).double() * (rank + 1)                    # where a random number of 1 would fall
    got = torch.minimum(got, last.amax(dim=1, keepdim=True).long() - 1)
    logp = torch.log(w.gather(1, got.clamp(min=0)) / total)
    return got[:, 0].int(), logp[:, 0].float(), keep.sum(dim=1).int()


def _plain(state):
    case = state["case"]
    op = case["op"]
    if op == "sample":
        return _plain_sample(state)
    if op == "dropout":
        y = state["X"].float() * _factor(state["rng"], case["n"], case["cols"], case["p"])
        if state["R"] is not None:
            y = y + state["R"].float()
        return y.to(_TYPES[case["dtype"]])
    ids, there = state["ids"].long().clamp(min=0), (state["ids"] >= 0)[:, None]
    factor = _factor(state["rng"], case["n"], case["dim"], case["p"]) if case["p"] > 0 else 1.0
    if op == "lookup":
        return (state["table"][ids].float() * state["scale"] * factor * there).to(_TYPES[case["out"]])
    part = state["dX"].float() * (state["scale"] * state["alpha"]) * factor * there
    if not case["add"]:
        state["table"].zero_()
    return state["table"].index_add_(0, ids, part)


def run(state):
    if not own:
        return _plain(state)
    op = state["case"]["op"]
    if op == "sample":
        s = state["settings"]
        state["plan"].sfb_sample(state["logits"], state["u"], state["ids"], s["temperature"], s["top_k"], s["top_p"], s["min_p"],
                                 state["logp"], state["kept"])
        return state["ids"], state["logp"], state["kept"]
    if op == "dropout":
        state["drop"].sfb_dropout_apply(state["X"], state["Y"], state["R"])
        return state["Y"]
    if op == "lookup":
        state["plan"].sfb_embed_forward(state["ids"], state["X"], state["drop"])
        return state["X"]
    state["plan"].sfb_embed_backward(state["ids"], state["dX"], state["table"], state["drop"], alpha=state["alpha"], add=state["case"]["add"])
    return state["table"]


def work(case):
    op, n = case["op"], float(case["n"])
    if op == "sample":
        v = n * case["classes"]
        # an exponential (a dozen operations) and a sum for each class
        return {"bytes": _SIZE[case["dtype"]] * v + 32.0 * n, "flops": 16.0 * v}
    if op == "dropout":
        v = n * case["cols"]
        return {"bytes": _SIZE[case["dtype"]] * v * (3.0 if case["residual"] else 2.0), "flops": 2.0 * v}
    v, rows = n * case["dim"], _distinct(case) * case["dim"]
    if op == "lookup":
        return {"bytes": 4.0 * n + _SIZE[case["table"]] * rows + _SIZE[case["out"]] * v, "flops": v}
    table = 8.0 * rows if case["add"] else 4.0 * case["tokens"] * case["dim"]
    return {"bytes": 4.0 * n + _SIZE[case["out"]] * v + table, "flops": 2.0 * v}


# ---- the definition, in 64 bits --------------------------------------------------------------------------------------------------
def _kept(state, rows, cols, p):
    """The same generator on the host, in words of 32 bits: 1 / (1 - t / 65536) where an entry is kept, else 0."""
    seed, offset = (int(v) & (1 << 64) - 1 for v in state["rng"].tolist())
    groups, low = -(-cols // 8), np.uint64(_MASK)
    out = np.zeros((rows, cols))
    t = _threshold(p)
    for at in range(0, rows, 4_096):
        count = min(4_096, rows - at)
        c = [np.tile(np.arange(groups, dtype=np.uint64), count), np.repeat(np.arange(at, at + count, dtype=np.uint64), groups),
             np.full(count * groups, offset & _MASK, dtype=np.uint64), np.full(count * groups, offset >> 32, dtype=np.uint64)]
        for r in range(10):
            k0, k1 = ((seed & _MASK) + r * 0x9E3779B9) & _MASK, ((seed >> 32) + r * 0xBB67AE85) & _MASK
            x, y = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
            c = [(y >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), y & low, (x >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), x & low]
        half = np.stack([w.astype("<u4") for w in c], axis=-1).view("<u2").reshape(count, groups * 8)[:, :cols]
        out[at : at + count] = np.where(half >= t, 65_536.0 / (65_536 - t), 0.0)
    return torch.from_numpy(out).cuda()


def _exact_row(z, u, temperature, top_k, top_p, min_p):
    order = np.lexsort((np.arange(z.size), -z))
    z = z[order]
    if not z[0] > -np.inf:
        return -1, -np.inf, 0
    if not temperature > 0:
        return int(order[0]), 0.0, 1
    count = int(np.count_nonzero(z > -np.inf))
    w = np.exp((z[:count] - z[0]) / temperature)
    if top_k > 0:
        count = min(count, top_k)
    if top_p < 1:
        ahead = np.cumsum(w[:count])
        count = max(1, min(count, 1 + int(np.searchsorted(ahead, top_p * ahead[-1], side="left"))))
    count = max(1, int(np.count_nonzero(w[:count] >= min(1.0, min_p))))
    left = np.sort(order[:count])
    value = np.zeros(z.size)
    value[order[:count]] = w[:count]
    upto = np.cumsum(value[left])
    i = min(int(np.searchsorted(upto, u * upto[-1], side="right")), count - 1)
    return int(left[i]), float(np.log(value[left[i]] / upto[-1])), count


def exact(case, seed):
    state = prepare(case, seed)
    op, n = case["op"], case["n"]
    if op == "sample":
        s = {k: None if v is None else v.cpu().double().numpy() for k, v in state["settings"].items()}
        at = lambda k, i, off: off if s[k] is None else float(s[k][i])
        u = state["u"].cpu().double().numpy()
        z = state["logits"].float().cpu().numpy()
        rows = [_exact_row(z[i].astype(np.float64), u[i], at("temperature", i, 1.0), int(at("top_k", i, 0)), at("top_p", i, 1.0), at("min_p", i, 0.0))
                for i in range(n)]
        ids, logp, kept = zip(*rows)
        return (torch.tensor(ids, dtype=torch.int32).cuda(), torch.tensor(logp, dtype=torch.float64).cuda(),
                torch.tensor(kept, dtype=torch.int32).cuda())
    if op == "dropout":
        y = state["X"].double() * _kept(state, n, case["cols"], case["p"])
        return y if state["R"] is None else y + state["R"].double()
    ids, dim = state["ids"], case["dim"]
    named = torch.nonzero(ids >= 0).flatten()
    factor = _kept(state, n, dim, case["p"])[named] if case["p"] > 0 else 1.0
    if op == "lookup":
        X = torch.zeros((n, dim), dtype=torch.float64, device="cuda")
        X[named] = state["table"][ids[named].long()].double() * factor * state["scale"]
        return X
    out = state["table"].double() if case["add"] else torch.zeros((case["tokens"], dim), dtype=torch.float64, device="cuda")
    part = state["dX"][named].double() * factor
    return out.index_put_((ids[named].long(),), part * (state["scale"] * state["alpha"]), accumulate=True)
