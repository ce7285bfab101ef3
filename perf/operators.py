"""The operators around the factors that users of this library have it do beside the steps on W, as cases that can be timed and compared.

  forward   the logits of samples against the shared W plus, for each sample, the adapter that its request names: a set of
            `rank` factor pairs kept apart from W.  n = 1 to a few dozen samples is serving, more is a batch or a training step
            (with "save" the products V x that the backward pass takes are returned too)
  backward  the gradients of that: of the samples, and of all adapters' factors
  clip      the global norm over a list of gradient tensors, and their copies rescaled where it is above the limit

"ids" says how the adapters fall on the samples: "runs" (the samples of a request follow one another, some requests without an
adapter) or "mixed" (each sample its own).  "layout" of a clip case: how many tensors share the elements.
"""
import math

import torch

own = False

_TYPES = {"fp32": (torch.float32,), "bf16": (torch.bfloat16,), "mixed": (torch.float32, torch.bfloat16, torch.float16)}
_STD = 1e-3                       # of the gradients


def _adapter(name, op, n, rows, cols, adapters, rank, ids, save=False):
    c = {"op": op, "n": n, "rows": rows, "cols": cols, "adapters": adapters, "rank": rank, "ids": ids}
    if op == "forward":
        c["save"] = save
    return {"name": name, **c} if name else c


def _clip(name, tensors, elements, types, clips):
    c = {"op": "clip", "tensors": tensors, "elements": elements, "types": types, "clips": clips}
    return {"name": name, **c} if name else c


def listed():
    return [
        # one request's sample against a dictionary-sized matrix: latency of a single answer
        _adapter("serve_one", "forward", 1, 10_000, 5_000, 16, 16, "mixed"),
        # a batch of requests that arrived together, each with an adapter of its own, ten thousand classes
        _adapter("serve_mixed", "forward", 37, 10_000, 20_000, 64, 16, "mixed"),
        # the paper-scale matrix: 6.5 GB of W per answer
        _adapter("serve_large", "forward", 64, 325_000, 10_000, 16, 8, "mixed"),
        # a ragged batch of several requests' samples
        _adapter("batch_ragged", "forward", 1_003, 9_999, 20_000, 32, 24, "runs"),
        # the forward half of a training step on many samples, adapters of the largest usual rank
        _adapter("train_forward", "forward", 8_192, 10_000, 5_000, 8, 64, "runs", save=True),
        # the smallest training step of the repository
        _adapter("backward_tiny", "backward", 128, 64, 256, 4, 4, "runs"),
        # a metric-learning-sized map, one sample per client
        _adapter("backward_mixed", "backward", 1_024, 1_000, 20_000, 64, 8, "mixed"),
        # the ordinary training step
        _adapter("backward_mid", "backward", 4_096, 10_000, 20_000, 32, 16, "runs"),
        # the factors of a few small adapters
        _clip("clip_tiny", 8, 5_120, "fp32", True),
        # gradients of many adapters and of the parts around them, of three types
        _clip("clip_many", 600, 40_000_000, "mixed", True),
        # the usual step of a training run in its calm phase: nothing to rescale, copies asked for
        _clip("clip_calm", 64, 21_333_333, "bf16", False),
        # the gradient of a whole parameter matrix of fp32 words
        _clip("clip_large", 12, 500_000_000, "fp32", True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("forward", "forward", "backward", "clip"))
    if op == "clip":
        elements = _log(rng, 1_000, 400_000_000)
        return _clip(None, min(_log(rng, 1, 2_000), elements // 16), elements, rng.choice(sorted(_TYPES)), rng.random() < 0.7)
    while True:
        n, rows, cols = _log(rng, 1, 12_000), _log(rng, 40, 40_000), _log(rng, 40, 24_000)
        adapters, rank = _log(rng, 1, 200), rng.choice((1, 4, 7, 8, 12, 16, 16, 24, 32, 48, 64, 100, 128))
        if n * rows * cols <= 8e11 and adapters * rank <= 4_096 and n * adapters * rank * (rows + cols) <= 1e12:
            return _adapter(None, op, n, rows, cols, adapters, rank, rng.choice(("runs", "mixed")), rng.random() < 0.3)


# ---- inputs ----------------------------------------------------------------------------------------------------------------------
def _wide(shape, gen, std, dtype=torch.bfloat16):
    """Normal values whose rows start 16 bytes apart or a multiple of that, as the library's operands do."""
    pitch = -(-shape[-1] // 8) * 8
    t = torch.empty((*shape[:-1], pitch), dtype=dtype, device="cuda")
    t.normal_(0.0, std, generator=gen)
    return t[..., : shape[-1]]


def _ids(case, gen):
    n, a = case["n"], case["adapters"]
    if case["ids"] == "mixed":
        return torch.randint(0, a, (n,), generator=gen, device="cuda", dtype=torch.int32)
    # runs: requests of unequal lengths one after another, every ninth without an adapter
    requests = max(1, min(n, 2 * a))
    ends = torch.sort(torch.randint(0, n + 1, (requests,), generator=gen, device="cuda")).values
    which = torch.randint(0, a, (requests + 1,), generator=gen, device="cuda", dtype=torch.int32)
    which[8::9] = -1
    return which[torch.bucketize(torch.arange(n, device="cuda"), ends, right=True)]


def _pieces(case):
    """(type, first element, elements) of each tensor within the buffer of its type, and the buffers' lengths.  Some start right
    behind the one before, as in a flattened buffer, others on a 256-byte boundary."""
    types, count, total = _TYPES[case["types"]], case["tensors"], case["elements"]
    weight = [1 + (i * 7_919) % 97 + (400 if i % 50 == 0 else 0) for i in range(count)]
    ends = [total * s // sum(weight) for s in torch.tensor(weight).cumsum(0).tolist()]
    at, got = [0] * len(types), []
    for i in range(count):
        n, k = ends[i] - (ends[i - 1] if i else 0), i % len(types)
        if i % 3 == 0:
            at[k] = -(-at[k] // 128) * 128
        got.append((k, at[k], n))
        at[k] += n
    return got, at


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    state = {"case": case}
    if case["op"] == "clip":
        types, (pieces, lengths) = _TYPES[case["types"]], _pieces(case)
        flat = [torch.empty(max(1, n), dtype=t, device="cuda").normal_(0.0, _STD, generator=gen) for t, n in zip(types, lengths)]
        to = [torch.zeros_like(f) for f in flat]
        state.update(grads=[flat[k][at : at + n] for k, at, n in pieces], outs=[to[k][at : at + n] for k, at, n in pieces], to=to,
                     limit=_STD * math.sqrt(case["elements"]) * (0.37 if case["clips"] else 2.0),
                     result=torch.zeros(2, dtype=torch.float32, device="cuda"))
        if own:
            import paper_1409_5705_b200 as S

            state["plan"] = S.GradientClip(state["grads"], state["outs"])
        return state
    n, rows, cols, a, r = (case[k] for k in ("n", "rows", "cols", "adapters", "rank"))
    state.update(W=_wide((rows, cols), gen, 0.01), U=_wide((a, r, rows), gen, 0.01 / math.sqrt(r)), V=_wide((a, r, cols), gen, 1.0),
                 scale=torch.rand(a, generator=gen, device="cuda") * 1.5 + 0.5, X=_wide((n, cols), gen, 1.0 / math.sqrt(cols)),
                 ids=_ids(case, gen))
    if case["op"] == "forward":
        state.update(Y=_wide((n, rows), gen, 0.0), S=torch.zeros((n, r), device="cuda") if case["save"] else None)
    else:
        state.update(dY=_wide((n, rows), gen, _STD), dX=_wide((n, cols), gen, 0.0), dU=torch.zeros((a, r, rows), device="cuda"),
                     dV=torch.zeros((a, r, cols), device="cuda"), S=_mine(_all(state["X"].float(), state["V"].float()), state["ids"]))
    if own:
        import paper_1409_5705_b200 as S

        state["plan"] = S.Adapters(state["W"], state["U"], state["V"], state["scale"], max_samples=n)
    return state


# ---- the plain form --------------------------------------------------------------------------------------------------------------
def _all(x, f):
    """The products of each sample with every adapter's factors: [n, adapters, rank]."""
    a, r, d = f.shape
    return (x @ f.reshape(a * r, d).t()).view(x.shape[0], a, r)


def _mine(p, ids):
    """Those of each sample's own adapter; zeros for a sample without one."""
    got = p[torch.arange(p.shape[0], device=p.device), ids.long().clamp(min=0)]
    return got * (ids >= 0)[:, None]


def _spread(s, ids, scale):
    """Back to [n, adapters * rank]: scale * s in the place of the sample's own adapter, zeros elsewhere."""
    at = ids.long().clamp(min=0)
    hit = (torch.arange(scale.shape[0], device=ids.device)[None, :] == ids[:, None]).to(s.dtype)
    return (hit[:, :, None] * (scale[at].to(s.dtype)[:, None] * s)[:, None, :]).reshape(s.shape[0], -1)


def _forward(X, W, U, V, scale, ids):
    s = _mine(_all(X, V), ids)
    return X @ W.t() + _spread(s, ids, scale) @ U.reshape(-1, U.shape[-1]), s


def _plain(state):
    X, W, U, V = (state[k].float() for k in ("X", "W", "U", "V"))
    ids, scale = state["ids"], state["scale"]
    if state["case"]["op"] == "forward":
        y, s = _forward(X, W, U, V, scale, ids)
        return (y.to(torch.bfloat16), s) if state["case"]["save"] else y.to(torch.bfloat16)
    dY = state["dY"].float()
    t = _spread(_mine(_all(dY, U), ids), ids, scale)
    s = _spread(state["S"], ids, scale)
    return ((dY @ W + t @ V.reshape(-1, V.shape[-1])).to(torch.bfloat16), (s.t() @ dY).view(U.shape), (t.t() @ X).view(V.shape))


def _plain_clip(state):
    # the sum is long: in 64 bits
    norm = torch.stack([g.double().square().sum() for g in state["grads"]]).sum().sqrt()
    coef = torch.where(norm > state["limit"], state["limit"] / norm, torch.ones_like(norm)).float()
    [o.copy_(g.float() * coef) for g, o in zip(state["grads"], state["outs"])]
    state["result"].copy_(torch.stack([norm.float(), coef]))
    return (*state["to"], state["result"])


def run(state):
    op = state["case"]["op"]
    if not own:
        return _plain_clip(state) if op == "clip" else _plain(state)
    plan = state["plan"]
    if op == "clip":
        plan.sfb_clip_gradients(state["limit"], state["result"])
        return (*state["to"], state["result"])
    if op == "forward":
        plan.sfb_adapter_forward(state["X"], state["ids"], state["Y"], state["S"])
        return (state["Y"], state["S"]) if state["case"]["save"] else state["Y"]
    plan.sfb_adapter_backward(state["dY"], state["X"], state["ids"], state["S"], state["dX"], state["dU"], state["dV"])
    return state["dX"], state["dU"], state["dV"]


def work(case):
    if case["op"] == "clip":
        size = {"fp32": 4.0, "bf16": 2.0, "mixed": 8.0 / 3.0}[case["types"]]
        # read for the norm, written; what is rescaled is a second read only where it no longer is on the chip
        return {"bytes": 2.0 * size * case["elements"], "flops": 3.0 * case["elements"]}
    n, rows, cols, a, r = (float(case[k]) for k in ("n", "rows", "cols", "adapters", "rank"))
    used = min(a, n)                        # adapters that some sample names, at most
    factors = 2.0 * used * r * (rows + cols)
    if case["op"] == "forward":
        return {"bytes": 2.0 * (rows * cols + n * cols + n * rows) + factors + (4.0 * n * r if case["save"] else 0.0),
                "flops": 2.0 * n * rows * cols + 2.0 * n * r * (rows + cols)}
    return {"bytes": 2.0 * (rows * cols + 2.0 * n * cols + n * rows) + factors + 4.0 * n * r + 4.0 * a * r * (rows + cols),
            "flops": 2.0 * n * rows * cols + 4.0 * n * r * (rows + cols)}


# ---- the definition, in 64 bits --------------------------------------------------------------------------------------------------
def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "clip":
        total = sum(float(torch.linalg.vector_norm(g, dtype=torch.float64)) ** 2 for g in state["grads"])
        norm = math.sqrt(total)
        coef = min(1.0, state["limit"] / norm)
        to = [torch.zeros(f.shape, dtype=torch.float64, device="cuda") for f in state["to"]]
        for (k, at, n), g in zip(_pieces(case)[0], state["grads"]):
            to[k][at : at + n] = g.double() * coef
        return (*to, torch.tensor([norm, coef], dtype=torch.float64))
    n, rows, cols, r = (case[k] for k in ("n", "rows", "cols", "rank"))
    X, ids, scale = state["X"].double(), state["ids"], state["scale"].double()
    S = torch.zeros((n, r), dtype=torch.float64, device="cuda")
    groups = [(a, torch.nonzero(ids == a).flatten()) for a in range(case["adapters"])]
    step = max(1, int(2e8) // cols)         # rows of W at a time
    if case["op"] == "forward":
        Y = torch.empty((n, rows), dtype=torch.float64, device="cuda")
        for at in range(0, rows, step):
            Y[:, at : at + step] = X @ state["W"][at : at + step].double().t()
        for a, i in groups:
            if len(i):
                S[i] = X[i] @ state["V"][a].double().t()
                Y[i] += scale[a] * (S[i] @ state["U"][a].double())
        return (Y, S) if case["save"] else Y
    dY = state["dY"].double()
    dX = torch.zeros((n, cols), dtype=torch.float64, device="cuda")
    for at in range(0, rows, step):
        dX += dY[:, at : at + step] @ state["W"][at : at + step].double()
    dU = torch.zeros(state["dU"].shape, dtype=torch.float64, device="cuda")
    dV = torch.zeros(state["dV"].shape, dtype=torch.float64, device="cuda")
    for a, i in groups:
        if len(i):
            t = dY[i] @ state["U"][a].double().t()
            dX[i] += scale[a] * (t @ state["V"][a].double())
            dU[a] = scale[a] * (state["S"][i].double().t() @ dY[i])
            dV[a] = scale[a] * (t.t() @ X[i])
    return dX, dU, dV
