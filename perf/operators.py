"""What is trained on the engine's clusterings, as cases for a timing harness.

A model that learns cluster ids ends in three operators, each a case family here:

* ``layer_norm``: normalised features, forward (``infer``) or with the gradient (``train``);
* ``head``: softmax cross entropy of ``scale * H W^T + offset`` with ids, over few
  classes or a large vocabulary; the loss alone (``infer``) or with the gradient;
* ``distill``: the same head against a teacher's top logits, here the nearest
  clusters of each point.

Point counts, widths and class counts are those of the repository's workloads
(n up to 60000, d = 16 .. 784, k = 7 .. 1024 clusters) in fp32, and generic
vocabulary heads in 16 bits.  Targets of large vocabularies are skewed, as ids
in use are; some rows are unlabelled, some classes left out.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-5
# Binary16 gradients are scaled, as a binary16 training loop scales its loss.
LOSS_SCALE = {"f32": 1.0, "f16": 4096.0, "bf16": 1.0}
# Classes times points of one head case (the plain form stores that many fp32
# logits several times), and the products of a 16-bit and an fp32 one.
MAX_LOGITS, MAX_PRODUCTS, MAX_PRODUCTS_F32 = 3.0e8, 1.0e12, 1.2e11


def listed():
    return [
        # One point on its way to the head: the call's latency.
        _norm("norm-one", "infer", 1, 784, "f32"),
        # The features of an image-like data set, a training step.
        _norm("norm-points", "train", 20000, 784, "f32"),
        # Columns of a wider table, odd width: no row is aligned.
        _norm("norm-ragged", "train", 40001, 301, "f16", pad=6),
        # Wide 16-bit activations: the largest batch.
        _norm("norm-wide", "train", 16384, 4096, "bf16"),
        # One token scored against a vocabulary: W's bytes count.
        _head("head-one", "infer", 1, 2048, 32768, "bf16"),
        # Cluster ids as labels, few classes; empty clusters left out, part of the points unlabelled.
        _head("head-points", "train", 60000, 780, 10, "f32", drop=0.1, offset=True),
        # Odd sizes throughout, binary16.
        _head("head-ragged", "train", 3001, 1001, 10007, "f16", drop=0.05),
        # A training batch over a large vocabulary.
        _head("head-vocab", "train", 8192, 4096, 32768, "bf16", drop=0.02),
        # A few points scored against the engine's largest number of clusters.
        _distill("distill-few", "infer", 16, 784, 1024, 16, "f32"),
        # Soft assignments of an ordinary data set: the 8 nearest of 64 clusters.
        _distill("distill-points", "train", 20000, 784, 64, 8, "f32", drop=0.1),
        # Odd sizes, binary16, rows with fewer pairs than others.
        _distill("distill-ragged", "train", 1777, 1000, 20011, 20, "f16", drop=0.2),
        # A teacher's top 32 of a large vocabulary.
        _distill("distill-vocab", "train", 4096, 2048, 50000, 32, "bf16", drop=0.05),
    ]


def draw(rng):
    """One more case of the listed ones' ranges; none costs more than the largest of them."""
    op = rng.choice(["layer_norm", "head", "head", "distill", "distill"])
    what = rng.choice(["infer", "train", "train"])
    dtype = rng.choice(["f32", "f16", "bf16"])
    pad = rng.choice([0, 0, 0, 1, 8])
    if op == "layer_norm":
        d = _width(rng, 8, 8192)
        case = _norm("", what, _log_between(rng, 1, min(60000, 16384 * 4096 // d)), d, dtype, pad)
    else:
        d = _width(rng, 16, 4096)
        points = dtype == "f32"
        classes = _log_between(rng, 2, 1024) if points else _log_between(rng, 64, 65536)
        products = MAX_PRODUCTS_F32 if points else MAX_PRODUCTS
        n_max = int(min(60000, MAX_LOGITS // classes, products // (classes * d)))
        n = _log_between(rng, 1, n_max)
        drop = rng.choice([0.0, 0.05, 0.5])
        offset = rng.random() < 0.3
        if op == "head":
            case = _head("", what, n, d, classes, dtype, pad, drop, offset)
        else:
            case = _distill("", what, n, d, classes, _log_between(rng, 1, min(64, classes)), dtype, pad, drop, offset)
    return {key: v for key, v in case.items() if key != "name"}


def _log_between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A number of features: two in three are a multiple of 8."""
    d = _log_between(rng, lo, hi)
    return d if rng.random() < 0.34 else (d + 7) // 8 * 8


def _norm(name, what, n, d, dtype, pad=0):
    return {"name": name, "op": "layer_norm", "what": what, "n": n, "d": d, "dtype": dtype, "pad": pad}


def _head(name, what, n, d, classes, dtype, pad=0, drop=0.0, offset=False):
    return {"name": name, "op": "head", "what": what, "n": n, "d": d, "classes": classes, "dtype": dtype, "pad": pad,
            "drop": drop, "offset": offset}


def _distill(name, what, n, d, classes, m, dtype, pad=0, drop=0.0, offset=False):
    return {"name": name, "op": "distill", "what": what, "n": n, "d": d, "classes": classes, "m": m, "dtype": dtype,
            "pad": pad, "drop": drop, "offset": offset}


# ------------------------------------------------------------------ inputs

def _data(case, seed):
    """A case's inputs on the GPU, from the seed alone."""
    gen = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 29)

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=gen)

    def uniform(*shape):
        return torch.rand(*shape, device="cuda", generator=gen)

    n, d, dtype = case["n"], case["d"], DTYPES[case["dtype"]]

    def rows():  # n x d, the first d columns of a table d + pad wide
        return torch.empty((n, d + case["pad"]), device="cuda", dtype=dtype)[:, :d]

    if case["op"] == "layer_norm":
        x, dy = rows(), rows()
        x.copy_(normal(n, d) * (0.5 + uniform(n, 1)) + normal(n, 1))
        dy.copy_(normal(n, d) * (LOSS_SCALE[case["dtype"]] / n))
        return {"x": x, "dy": dy, "weight": 1 + 0.1 * normal(d), "bias": 0.1 * normal(d)}
    V = case["classes"]
    h = rows()
    h.copy_(normal(n, d))
    w = (normal(V, d) * (2.0 / math.sqrt(d))).to(dtype)
    offset = None
    kept = torch.ones(V, dtype=torch.bool, device="cuda")
    if case["offset"]:  # log shares of the clusters; about one in twenty is empty
        kept = uniform(V) >= 0.05
        kept[0] = True
        offset = torch.where(kept, torch.log(0.05 + uniform(V)), -math.inf)
    names = torch.nonzero(kept)[:, 0]  # the classes that are there
    dropped = uniform(n) < case["drop"]
    dloss = (0.5 + uniform(n)) * (LOSS_SCALE[case["dtype"]] / n)
    data = {"h": h, "w": w, "offset": offset, "dloss": dloss, "scale": 1.0}
    if case["op"] == "head":
        ids = names[(names.numel() * uniform(n) ** 3).long().clamp_(max=names.numel() - 1)]
        data["ids"] = torch.where(dropped, -1, ids).to(torch.int32)
        return data
    m = case["m"]
    first = torch.randint(0, names.numel(), (n, 1), device="cuda", generator=gen)
    step = max(names.numel() // m, 1)  # m different classes of each row (with -1 beyond those there are)
    j = torch.arange(m, device="cuda")[None, :]
    top_ids = names[(first + step * j) % names.numel()]
    here = (j * step < names.numel()) & (uniform(n, m) >= 0.5 * case["drop"]) & ~dropped[:, None]
    top_logits = torch.sort(4 * uniform(n, m), dim=1, descending=True).values
    data["top_ids"] = torch.where(here, top_ids, -1).to(torch.int32).contiguous()
    data["top_logits"] = torch.where(here, top_logits, -math.inf).contiguous()
    data["teacher_scale"] = 0.5
    data["scale"] = 0.5
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
    f32 = {"device": "cuda", "dtype": torch.float32}
    n = case["n"]
    if case["op"] == "layer_norm":
        state.update(y=torch.empty_like(state["x"], memory_format=torch.contiguous_format),
                     mean=torch.empty(n, **f32), rstd=torch.empty(n, **f32))
        if case["what"] == "train":
            state.update(dx=torch.empty_like(state["y"]), dweight=torch.empty_like(state["weight"]),
                         dbias=torch.empty_like(state["bias"]))
    else:
        state.update(loss=torch.empty(n, **f32), lse=torch.empty(n, **f32))
        if case["what"] == "train":
            state.update(dh=torch.empty((n, case["d"]), device="cuda", dtype=state["h"].dtype),
                         dw=torch.empty_like(state["w"]))
    if own:
        state["ctx"] = _context()
    return state


# ------------------------------------------------------------------ one pass

def run(state):
    case = state["case"]
    return {"layer_norm": _run_norm, "head": _run_head, "distill": _run_distill}[case["op"]](
        state, case["what"] == "train")


def _run_norm(s, train):
    if own:
        from paper_2601_17136_amd import kkm
        kkm.kkm_layer_norm(s["ctx"], s["x"], s["weight"], s["bias"], EPS, s["y"], s["mean"], s["rstd"])
        if train:
            kkm.kkm_layer_norm_grad(s["ctx"], s["x"], s["weight"], s["dy"], s["mean"], s["rstd"], s["dx"],
                                    s["dweight"], s["dbias"])
            return s["y"], s["mean"], s["rstd"], s["dx"], s["dweight"], s["dbias"]
        return s["y"], s["mean"], s["rstd"]
    x = s["x"].float()
    mean = x.mean(1, keepdim=True)
    centred = x - mean
    rstd = 1.0 / torch.sqrt((centred * centred).mean(1, keepdim=True) + EPS)
    xhat = centred * rstd
    y = (xhat * s["weight"] + s["bias"]).to(s["x"].dtype)
    if not train:
        return y, mean[:, 0], rstd[:, 0]
    dy = s["dy"].float()
    g = dy * s["weight"]
    dx = rstd * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
    return y, mean[:, 0], rstd[:, 0], dx.to(s["x"].dtype), (dy * xhat).sum(0), dy.sum(0)


def _run_head(s, train):
    if own:
        from paper_2601_17136_amd import kkm
        if train:
            kkm.kkm_head_grad(s["ctx"], s["h"], s["w"], s["ids"], s["dloss"], s["loss"], s["lse"], s["dh"], s["dw"],
                              scale=s["scale"], offset=s["offset"])
            return s["loss"], s["lse"], s["dh"], s["dw"]
        kkm.kkm_head_loss(s["ctx"], s["h"], s["w"], s["ids"], s["loss"], s["lse"], scale=s["scale"],
                          offset=s["offset"])
        return s["loss"], s["lse"]
    logits, lse = _logits(s)
    ids = s["ids"].long()
    labelled = ids >= 0
    at = ids.clamp(min=0)[:, None]
    loss = torch.where(labelled, lse - logits.gather(1, at)[:, 0], 0.0)
    if not train:
        return loss, lse
    p = torch.exp(logits - lse[:, None])
    p.scatter_add_(1, at, -torch.ones_like(at, dtype=torch.float32))
    return (loss, lse) + _products(s, p, torch.where(labelled, s["dloss"], 0.0))


def _run_distill(s, train):
    if own:
        from paper_2601_17136_amd import kkm
        if train:
            kkm.kkm_distill_grad(s["ctx"], s["h"], s["w"], s["top_ids"], s["top_logits"], s["dloss"], s["loss"],
                                 s["lse"], s["dh"], s["dw"], scale=s["scale"], offset=s["offset"],
                                 teacher_scale=s["teacher_scale"])
            return s["loss"], s["lse"], s["dh"], s["dw"]
        kkm.kkm_distill_loss(s["ctx"], s["h"], s["w"], s["top_ids"], s["top_logits"], s["loss"], s["lse"],
                             scale=s["scale"], offset=s["offset"], teacher_scale=s["teacher_scale"])
        return s["loss"], s["lse"]
    logits, lse = _logits(s)
    ids = s["top_ids"].long()
    t = torch.where(ids >= 0, s["teacher_scale"] * s["top_logits"], -math.inf)
    there = t > -math.inf
    top = t.max(1, keepdim=True).values
    e = torch.where(there, torch.exp(t - torch.where(top > -math.inf, top, 0.0)), 0.0)
    total = e.sum(1, keepdim=True)
    some = total[:, 0] > 0
    q = e / torch.where(total > 0, total, 1.0)
    at = ids.clamp(min=0)
    each = q * (torch.log(torch.where(q > 0, q, 1.0)) - logits.gather(1, at) + lse[:, None])
    loss = torch.where(q > 0, each, 0.0).sum(1)
    if not train:
        return loss, lse
    p = torch.exp(logits - lse[:, None])
    p.scatter_add_(1, at, -q)
    return (loss, lse) + _products(s, p, torch.where(some, s["dloss"], 0.0))


def _logits(s):
    """The plain form's logits, n x classes in fp32, and their log sums of exponentials."""
    logits = s["scale"] * (s["h"].float() @ s["w"].float().t())
    if s["offset"] is not None:
        logits = logits + s["offset"]
    top = logits.max(1, keepdim=True).values
    return logits, (top + torch.log(torch.exp(logits - top).sum(1, keepdim=True)))[:, 0]


def _products(s, p, dloss):
    """dH and dW from the logits' gradient before its rows' factors."""
    g = p * (dloss * s["scale"])[:, None]
    return (g @ s["w"].float()).to(s["h"].dtype), (g.t() @ s["h"].float()).to(s["w"].dtype)


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    n, d, size = case["n"], case["d"], {"f32": 4, "f16": 2, "bf16": 2}[case["dtype"]]
    train = case["what"] == "train"
    if case["op"] == "layer_norm":
        # x read, y written (train: dy read, dx written too); statistics, weight, bias and their gradients
        return {"bytes": n * d * size * (4 if train else 2) + 8 * n + 4 * d * (4 if train else 2),
                "flops": n * d * (18 if train else 8)}
    V = case["classes"]
    pairs = 8 * case["m"] if case["op"] == "distill" else 4
    return {"bytes": (n + V) * d * size * (2 if train else 1) + n * (pairs + 8 + (4 if train else 0)) +
            (4 * V if case["offset"] else 0),
            "flops": n * V * d * (6 if train else 2)}


# ------------------------------------------------------------------ the definitions in 64 bits

def exact(case, seed):
    s = _data(case, seed)
    if case["op"] == "layer_norm":
        return _exact_norm(case, s)
    rows = max(1, min(case["n"], 2 ** 26 // case["classes"]))
    h, w = s["h"].double(), s["w"].double()
    losses, lses, dhs, dw = [], [], [], torch.zeros_like(w)
    for a in range(0, case["n"], rows):
        b = min(a + rows, case["n"])
        z = torch.mm(h[a:b], w.t().contiguous()).mul_(s["scale"])
        if s["offset"] is not None:
            z += s["offset"].double()
        logp = torch.log_softmax(z, dim=1)
        target = torch.zeros_like(z)
        if case["op"] == "head":
            i = torch.nonzero(s["ids"][a:b] >= 0)[:, 0]
            target[i, s["ids"][a:b][i].long()] = 1.0
            entropy = torch.zeros(b - a, device="cuda", dtype=torch.float64)
        else:
            gone = s["top_ids"][a:b] < 0
            t = (s["top_logits"][a:b].double() * s["teacher_scale"]).masked_fill(gone, -math.inf)
            q = torch.softmax(t, dim=1).nan_to_num(0.0).masked_fill(gone, 0.0)
            target.scatter_add_(1, s["top_ids"][a:b].long().masked_fill(gone, 0), q)
            entropy = torch.special.entr(q).sum(1)
        losses.append(-(torch.where(target > 0, target * logp, 0.0)).sum(1) - entropy)
        lses.append(torch.logsumexp(z, dim=1))
        if case["what"] == "train":
            mass = target.sum(1, keepdim=True)  # 1, or 0 where a row has no target
            g = (logp.exp_() * mass.round() - target) * (s["dloss"][a:b].double() * s["scale"])[:, None]
            dhs.append(torch.mm(g, w))
            dw += torch.mm(g.t().contiguous(), h[a:b])
    out = (torch.cat(losses), torch.cat(lses))
    return out + (torch.cat(dhs), dw) if case["what"] == "train" else out


def _exact_norm(case, s):
    x, w, b = s["x"].double(), s["weight"].double(), s["bias"].double()
    var, mean = torch.var_mean(x, dim=1, correction=0)
    rstd = torch.rsqrt(var + EPS)
    z = (x - mean[:, None]) * rstd[:, None]
    out = (torch.addcmul(b, z, w), mean, rstd)
    if case["what"] == "infer":
        return out
    dy = s["dy"].double()
    dz = dy * w
    d = case["d"]
    dx = (dz * d - dz.sum(1, keepdim=True) - z * (dz * z).sum(1, keepdim=True)) * (rstd[:, None] / d)
    return out + (dx, torch.linalg.vecdot(dy, z, dim=0), dy.sum(0))
