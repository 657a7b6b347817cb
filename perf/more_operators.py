"""What learns and answers beside a shared head, as cases for a timing harness.

Points of several sources share one projection; each source's own part of it is
small.  Three operators, each a case family here:

* ``adapted``: a shared linear map with a low-rank adapter per row, chosen by the
  row's id: ``y_i = w x_i + f_g up_g (down_g x_i)``, forward (``infer``) or with
  the gradient (``train``);
* ``orthogonal``: a weight's update along its orthogonalised momentum by
  Newton-Schulz products (``step``), or the orthogonalising alone (``map``);
* ``choose``: logits with penalties for ids already given, biases and bit masks
  of the ids allowed, and the id, its log probability and the log sum of each row.

Point counts, widths and class counts are those of the repository's workloads
(n up to 20000 here, d = 16 .. 784, up to 1024 clusters) in fp32, and generic
projections and vocabularies in 16 bits.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
QUINTIC = (3.4445, -4.7750, 2.0315)
EPS = 1e-7
MOMENTUM, RATE, KEEP = 0.95, 0.02, 0.999
REPEAT, PRESENCE, FREQUENCY, SCALE = 1.2, 0.25, 0.125, 0.8
# Products of one case at most: of a projection, of an orthogonalising's first Gram matrix.
MAX_PRODUCTS, MAX_PRODUCTS_F32 = 1.4e11, 1.7e10
MAX_GRAM, MAX_GRAM_F32 = 6.9e10, 4.0e9
MAX_LOGITS = 6.8e7


def listed():
    return [
        # One point of one source through a small head: the call's latency.
        _adapted("adapt-one", "infer", 1, 784, 64, 8, 8, "f32"),
        # A serving step: each request's token has an adapter of its own.
        _adapted("adapt-few", "infer", 32, 4096, 4096, 32, 16, "bf16"),
        # A training step on image-like points of eight sources.
        _adapted("adapt-points", "train", 20000, 784, 1024, 8, 8, "f32", drop=0.1),
        # Odd sizes throughout, rows at any address, binary16.
        _adapted("adapt-ragged", "train", 3001, 1001, 777, 5, 12, "f16", pad=3, drop=0.3),
        # A training batch through a wide projection.
        _adapted("adapt-wide", "train", 8192, 4096, 4096, 16, 32, "bf16"),
        # The adapters' own update: a stack of flat matrices.
        _orthogonal("ortho-adapters", "step", 8, 8, 784, "f32"),
        # A head over the engine's largest number of clusters.
        _orthogonal("ortho-head", "step", 1, 1024, 784, "f32"),
        # Odd sizes, binary16, the orthogonalising alone.
        _orthogonal("ortho-ragged", "map", 3, 777, 1001, "f16", pad=5),
        # A wide projection's update.
        _orthogonal("ortho-wide", "step", 1, 4096, 4096, "bf16"),
        # One token's answer from a vocabulary.
        _choose("choose-one", 1, 32768, 64, 8, 1, "bf16"),
        # New points of an ordinary data set, each held to the clusters open to it.
        _choose("choose-points", 20000, 64, 0, 0, 16, "f32", offset=True),
        # A serving batch over a large vocabulary with long histories.
        _choose("choose-wide", 512, 131072, 1024, 32, 16, "bf16"),
    ]


def draw(rng):
    """One more case of the listed ones' ranges; none costs more than the largest of them."""
    op = rng.choice(["adapted", "adapted", "orthogonal", "choose"])
    dtype = rng.choice(["f32", "f16", "bf16"])
    pad = rng.choice([0, 0, 0, 1, 8])
    if op == "adapted":
        what = rng.choice(["infer", "train", "train"])
        d = _width(rng, 16, 1024 if dtype == "f32" else 4096)
        m = _width(rng, 7, 1024 if dtype == "f32" else 4096)
        rank = _log_between(rng, 1, 64)
        adapters = _log_between(rng, 1, min(64, 1024 // rank))
        products = MAX_PRODUCTS_F32 if dtype == "f32" else MAX_PRODUCTS
        n = _log_between(rng, 1, int(min(20000, products // (d * m))))
        case = _adapted("", what, n, d, m, adapters, rank, dtype, pad, rng.choice([0.0, 0.1, 0.5]))
    elif op == "orthogonal":
        what = rng.choice(["step", "step", "map"])
        top = 1024 if dtype == "f32" else 4096
        m, n = _width(rng, 4, top), _width(rng, 4, top)
        gram = MAX_GRAM_F32 if dtype == "f32" else MAX_GRAM
        batch = _log_between(rng, 1, int(max(1, min(16, gram // (min(m, n) ** 2 * max(m, n))))))
        case = _orthogonal("", what, batch, m, n, dtype, pad)
    else:
        V = _log_between(rng, 7, 131072)
        n = _log_between(rng, 1, int(min(20000, MAX_LOGITS // V)))
        given = rng.choice([0, _log_between(rng, 1, 1024)])
        biases = rng.choice([0, _log_between(rng, 1, min(64, V))])
        masks = rng.choice([0, _log_between(rng, 1, 16)])
        case = _choose("", n, V, given, biases, masks, dtype, pad, rng.random() < 0.5)
    return {key: v for key, v in case.items() if key != "name"}


def _log_between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width: two in three are a multiple of 8."""
    d = _log_between(rng, lo, hi)
    return d if rng.random() < 0.34 else (d + 7) // 8 * 8


def _adapted(name, what, n, d, m, adapters, rank, dtype, pad=0, drop=0.0):
    return {"name": name, "op": "adapted", "what": what, "n": n, "d": d, "m": m, "adapters": adapters, "rank": rank,
            "dtype": dtype, "pad": pad, "drop": drop}


def _orthogonal(name, what, batch, m, n, dtype, pad=0):
    return {"name": name, "op": "orthogonal", "what": what, "batch": batch, "m": m, "n": n, "steps": 5, "dtype": dtype,
            "pad": pad}


def _choose(name, n, classes, given, biases, masks, dtype, pad=0, offset=False):
    return {"name": name, "op": "choose", "n": n, "classes": classes, "given": given, "biases": biases, "masks": masks,
            "dtype": dtype, "pad": pad, "offset": offset}


# ------------------------------------------------------------------ inputs

def _data(case, seed):
    """A case's inputs on the GPU, from the seed alone."""
    gen = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 31)

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=gen)

    def uniform(*shape):
        return torch.rand(*shape, device="cuda", generator=gen)

    dtype, pad = DTYPES[case["dtype"]], case["pad"]

    def table(values):  # the first columns of a table `pad` wider
        t = torch.empty((*values.shape[:-1], values.shape[-1] + pad), device="cuda", dtype=dtype)[..., :values.shape[-1]]
        return t.copy_(values)

    n = case["n"]
    if case["op"] == "adapted":
        d, m, s, r = case["d"], case["m"], case["adapters"], case["rank"]
        ids = (s * uniform(n) ** 1.5).long().clamp_(max=s - 1)  # some sources have more points than others
        ids = torch.where(uniform(n) < case["drop"], -1, ids).to(torch.int32)
        return {"x": table(normal(n, d)), "w": table(normal(m, d) / math.sqrt(d)),
                "down": (normal(s, r, d) / math.sqrt(d)).to(dtype), "up": (normal(s, m, r) / math.sqrt(2 * r)).to(dtype),
                "factor": 0.5 + uniform(s), "ids": ids, "dy": table(normal(n, m) / math.sqrt(n))}
    if case["op"] == "orthogonal":
        shape = (case["batch"], case["m"], n)
        few = max(1, min(shape[1:]) // 4)  # a gradient's few strong directions, and noise
        g = torch.bmm(normal(shape[0], shape[1], few), normal(shape[0], few, n)) / math.sqrt(few) + 0.2 * normal(*shape)
        data = {"g": table(1e-3 * g)}
        if case["what"] == "step":
            data["w"] = table(normal(*shape) / math.sqrt(n))
            data["v"] = 1e-3 * (2 * g + normal(*shape))
        return data
    V = case["classes"]
    data = {"z": table(3 * normal(n, V)), "offset": None, "given": None, "bias_ids": None, "bias": None, "masks": None,
            "mask_ids": None}
    if case["offset"]:  # log shares of the clusters; about one in twenty is empty
        kept = uniform(V) >= 0.05
        kept[0] = True
        data["offset"] = torch.where(kept, torch.log(0.05 + uniform(V)), -math.inf)
    if case["given"]:  # skewed, as ids in use are, so that some come many times; the rows' lists differ in length
        ids = (V * uniform(n, case["given"]) ** 3).long().clamp_(max=V - 1)
        there = torch.arange(case["given"], device="cuda")[None, :] < case["given"] * (0.25 + uniform(n, 1))
        data["given"] = torch.where(there, ids, -1).to(torch.int32)
    if case["biases"]:  # different ids of each row
        b = case["biases"]
        first = torch.randint(0, V, (n, 1), device="cuda", generator=gen)
        ids = (first + (V // b) * torch.arange(b, device="cuda")[None, :]) % V
        data["bias_ids"] = torch.where(uniform(n, b) < 0.1, -1, ids).to(torch.int32)
        data["bias"] = 2 * normal(n, b)
    if case["masks"]:
        words = (V + 31) // 32
        data["masks"] = torch.randint(-2 ** 31, 2 ** 31, (case["masks"], words), device="cuda", generator=gen).to(torch.int32)
        data["mask_ids"] = torch.randint(-1, case["masks"], (n,), device="cuda", generator=gen).to(torch.int32)
    return data


_handle = None


def _context():
    """The engine's context on the current stream, kept as a program keeps it."""
    global _handle
    from paper_2601_17136_amd import kkm
    if _handle is None:
        _handle = kkm.kkm_create(kkm.current_stream_handle())
    return _handle


def prepare(case, seed):
    state = _data(case, seed)
    state["case"] = case
    like = {"device": "cuda", "dtype": DTYPES[case["dtype"]]}
    if case["op"] == "adapted":
        state["y"] = torch.empty((case["n"], case["m"]), **like)
        if case["what"] == "train":
            state.update(dx=torch.empty((case["n"], case["d"]), **like), ddown=torch.empty_like(state["down"]),
                         dup=torch.empty_like(state["up"]))
    elif case["op"] == "orthogonal":
        if case["what"] == "map":
            state["y"] = torch.empty((case["batch"], case["m"], case["n"]), **like)
    else:
        state.update(out=torch.empty((case["n"], case["classes"]), **like),
                     ids=torch.empty(case["n"], device="cuda", dtype=torch.int32),
                     logp=torch.empty(case["n"], device="cuda"), lse=torch.empty(case["n"], device="cuda"),
                     repeat=torch.tensor(REPEAT, device="cuda"))
    if own:
        state["ctx"] = _context()
    return state


# ------------------------------------------------------------------ one pass

def run(state):
    return {"adapted": _run_adapted, "orthogonal": _run_orthogonal, "choose": _run_choose}[state["case"]["op"]](state)


def _run_adapted(s):
    train = s["case"]["what"] == "train"
    if own:
        from paper_2601_17136_amd import kkm
        kkm.kkm_adapted_linear(s["ctx"], s["x"], s["w"], s["down"], s["up"], s["ids"], s["y"], factor=s["factor"])
        if not train:
            return s["y"]
        kkm.kkm_adapted_linear_grad(s["ctx"], s["x"], s["w"], s["down"], s["up"], s["ids"], s["dy"], s["dx"],
                                    s["ddown"], s["dup"], factor=s["factor"])
        return s["y"], s["dx"], s["ddown"], s["dup"]
    x, w, dtype = s["x"].float(), s["w"].float(), s["x"].dtype
    adapters, rank, d = s["down"].shape
    m = s["up"].shape[1]
    # every adapter's product, of which a row keeps its own
    mine = s["ids"][:, None] == torch.arange(adapters, device="cuda")[None, :]
    weight = torch.where(mine, s["factor"][None, :], 0.0)[:, :, None]
    down = s["down"].float().reshape(adapters * rank, d)
    up = s["up"].float().transpose(1, 2).reshape(adapters * rank, m)
    t = ((x @ down.t()).view(-1, adapters, rank) * weight).view(-1, adapters * rank)
    y = (x @ w.t() + t @ up).to(dtype)
    if not train:
        return y
    dy = s["dy"].float()
    u = ((dy @ up.t()).view(-1, adapters, rank) * weight).view(-1, adapters * rank)
    dx = (dy @ w + u @ down).to(dtype)
    ddown = (u.t() @ x).view(adapters, rank, d).to(dtype)
    dup = (t.t() @ dy).view(adapters, rank, m).transpose(1, 2).contiguous().to(dtype)
    return y, dx, ddown, dup


def _run_orthogonal(s):
    step = s["case"]["what"] == "step"
    if own:
        from paper_2601_17136_amd import kkm
        coef = [QUINTIC] * s["case"]["steps"]
        if not step:
            kkm.kkm_orthogonalize(s["ctx"], s["g"], s["y"], coef=coef, eps=EPS)
            return s["y"]
        kkm.kkm_orthogonal_step(s["ctx"], s["w"], s["g"], s["v"], RATE, momentum=MOMENTUM, keep=KEEP, coef=coef, eps=EPS)
        return s["w"], s["v"]
    x = s["g"].float()
    if step:
        s["v"].mul_(MOMENTUM).add_(x)
        x = x + MOMENTUM * s["v"]
    # the sum of squares in 64 bits: a sum over all entries
    x = x / (torch.sqrt((x.double() ** 2).sum((1, 2), keepdim=True)) + EPS).float()
    tall = x.shape[1] > x.shape[2]
    x = x.transpose(1, 2).contiguous() if tall else x
    a, b, c = QUINTIC
    for _ in range(s["case"]["steps"]):
        gram = torch.bmm(x, x.transpose(1, 2).contiguous())
        x = a * x + torch.bmm(b * gram + c * torch.bmm(gram, gram), x)
    x = x.transpose(1, 2).contiguous() if tall else x
    if not step:
        return x.to(s["g"].dtype)
    s["w"].copy_(KEEP * s["w"].float() - RATE * x)
    return s["w"], s["v"]


def _run_choose(s):
    if own:
        from paper_2601_17136_amd import kkm
        kkm.kkm_choose(s["ctx"], s["z"], s["out"], s["ids"], s["logp"], s["lse"], scale=SCALE, offset=s["offset"],
                       given=s["given"], repeat=REPEAT, presence=PRESENCE, frequency=FREQUENCY, bias_ids=s["bias_ids"],
                       bias=s["bias"], masks=s["masks"], mask_ids=s["mask_ids"])
        return s["out"], s["ids"], s["logp"], s["lse"]
    u = s["z"].float()
    n, V = u.shape
    if s["given"] is not None:
        there = s["given"] >= 0
        count = torch.zeros_like(u).scatter_add_(1, s["given"].clamp(min=0).long(), there.float())
        seen = torch.where(u > 0, u / s["repeat"], u * REPEAT) - (PRESENCE + count * FREQUENCY)
        u = torch.where(count > 0, seen, u)
    if s["offset"] is not None:
        u = u + s["offset"]
    if s["bias"] is not None:
        u = u.scatter_add(1, s["bias_ids"].clamp(min=0).long(), torch.where(s["bias_ids"] >= 0, s["bias"], 0.0))
    u = u * SCALE
    if s["masks"] is not None:
        words = s["masks"][s["mask_ids"].clamp(min=0).long()]
        bits = (words[:, :, None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1
        allowed = bits.view(n, -1)[:, :V].bool() | (s["mask_ids"] < 0)[:, None]
        u = torch.where(allowed, u, -math.inf)
    top = u.max(1, keepdim=True).values
    some = top[:, 0] > -math.inf
    at = torch.where(u == top, torch.arange(V, device="cuda"), V).min(1).values
    ids = torch.where(some, at, -1).to(torch.int32)
    logsum = torch.log(torch.exp(u - torch.where(some[:, None], top, 0.0)).sum(1))
    logp = torch.where(some, -logsum, -math.inf)
    return u.to(s["z"].dtype), ids, logp, top[:, 0] + torch.where(some, logsum, 0.0)


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    n, size = case["n"], {"f32": 4, "f16": 2, "bf16": 2}[case["dtype"]]
    if case["op"] == "adapted":
        d, m, r = case["d"], case["m"], case["rank"]
        low = min(case["adapters"], n) * r * (d + m)  # the adapters that rows have
        passes = 2 if case["what"] == "train" else 1  # (train: dy read and dx written beside x and y; the adapters' gradients)
        return {"bytes": size * (passes * (n * (d + m) + low) + m * d) + 4 * n + 4 * case["adapters"],
                "flops": 2 * n * (d * m + r * (d + m)) * passes + (2 * n * r * (d + m) if passes > 1 else 0)}
    if case["op"] == "orthogonal":
        short, entries = min(case["m"], n), case["m"] * n * case["batch"]
        # Gram and square are symmetric, so half of each; of flat matrices all steps' squares alone and one product
        flat, square = short * entries, case["batch"] * short ** 3
        flops = min(case["steps"] * (3 * flat + square), 3 * flat + 4 * case["steps"] * square)
        return {"bytes": entries * (3 * size + 8 if case["what"] == "step" else 2 * size), "flops": flops}
    V = case["classes"]
    words = case["masks"] * ((V + 31) // 32)
    return {"bytes": 2 * size * n * V + 4 * n * (case["given"] + 2 * case["biases"] + 4) + 4 * words +
            (4 * V if case["offset"] else 0), "flops": 8 * n * V}


# ------------------------------------------------------------------ the definitions in 64 bits

def exact(case, seed):
    s = _data(case, seed)
    return {"adapted": _exact_adapted, "orthogonal": _exact_orthogonal, "choose": _exact_choose}[case["op"]](case, s)


def _exact_adapted(case, s):
    x, w, dy = s["x"].double(), s["w"].double(), s["dy"].double()
    y, dx = torch.mm(x, w.t().contiguous()), torch.mm(dy, w)
    ddown, dup = torch.zeros_like(s["down"], dtype=torch.float64), torch.zeros_like(s["up"], dtype=torch.float64)
    for g in range(case["adapters"]):
        rows = torch.nonzero(s["ids"] == g)[:, 0]
        low, high, f = s["down"][g].double(), s["up"][g].double(), s["factor"][g].double()
        xg, dyg = x[rows], dy[rows]
        y[rows] += f * torch.mm(torch.mm(xg, low.t().contiguous()), high.t().contiguous())
        back = torch.mm(dyg, high)
        dx[rows] += f * torch.mm(back, low)
        ddown[g] = f * torch.mm(back.t().contiguous(), xg)
        dup[g] = f * torch.mm(dyg.t().contiguous(), torch.mm(xg, low.t().contiguous()))
    return (y, dx, ddown, dup) if case["what"] == "train" else y


def _exact_orthogonal(case, s):
    g = s["g"].double()
    if case["what"] == "step":
        v = s["v"].double() * MOMENTUM + g
        u = g + v * MOMENTUM
    else:
        u = g
    x = u / (torch.linalg.matrix_norm(u)[:, None, None] + EPS)
    a, b, c = QUINTIC
    for i in range(case["batch"]):
        y = x[i] if case["m"] <= case["n"] else x[i].t().contiguous()
        for _ in range(case["steps"]):
            back = torch.mm(torch.mm(y, y.t().contiguous()), y)  # x x' x, then x x' (b . + c x x' .)
            y = a * y + b * back + c * torch.mm(torch.mm(y, y.t().contiguous()), back)
        x[i] = y if case["m"] <= case["n"] else y.t()
    if case["what"] == "map":
        return x
    return s["w"].double() * KEEP - RATE * x, v


def _exact_choose(case, s):
    n, V = case["n"], case["classes"]
    outs, logps, lses = [], [], []
    step = max(1, 2 ** 24 // V)
    for lo in range(0, n, step):
        hi = min(lo + step, n)
        u = s["z"][lo:hi].double()
        if s["given"] is not None:
            ids = s["given"][lo:hi].long()
            count = torch.zeros(hi - lo, V + 1, device="cuda", dtype=torch.float64)
            count.scatter_add_(1, torch.where(ids < 0, V, ids), torch.ones_like(ids, dtype=torch.float64))
            count = count[:, :V]
            u = torch.where(count > 0, u * torch.where(u > 0, 1 / REPEAT, REPEAT) - PRESENCE - FREQUENCY * count, u)
        add = torch.zeros(hi - lo, V + 1, device="cuda", dtype=torch.float64)
        if s["bias"] is not None:
            ids = s["bias_ids"][lo:hi].long()
            add.scatter_(1, torch.where(ids < 0, V, ids), s["bias"][lo:hi].double())
        u = u + add[:, :V]
        if s["offset"] is not None:
            u = u + s["offset"].double()
        u = u * SCALE
        if s["masks"] is not None:
            which = s["mask_ids"][lo:hi].long()
            v = torch.arange(V, device="cuda")
            gone = (s["masks"][which.clamp(min=0)][:, v // 32].long() >> (v % 32)) % 2 == 0
            u = u.masked_fill(gone & (which >= 0)[:, None], -math.inf)
        lse = torch.logsumexp(u, dim=1)
        best = u.amax(1)
        outs.append(u)
        lses.append(lse)
        logps.append(torch.where(best > -math.inf, best - lse, -math.inf))
    return torch.cat(outs), None, torch.cat(logps), torch.cat(lses)
