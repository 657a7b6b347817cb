"""Plain 64-bit forms of layer norm and the class head's losses, with error
bounds for the kernels.

The bounds follow from the arithmetic the kernels state: operands as given,
fp32 sums (U = 2^-24 a rounding; the matrix cores' sums may truncate, so 2 U,
twice per instruction of 16 terms), G in the operands' type, one rounding of
what is stored.  fp32 operands are three bfloat16 parts: six plane products, so
six times the instructions, and 2^-23 of each product left out."""
import torch

U = 2.0 ** -24
UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
# Smallest step of what is stored (binary16 has a narrow range).
STEP = {torch.float32: 0.0, torch.float16: 2.0 ** -24, torch.bfloat16: 0.0}


def sum_error(terms, dtype):
    """Relative error of a matrix-core sum of so many products, of the sum of their sizes."""
    segs = 6 if dtype == torch.float32 else 1
    return (2 * segs * (terms / 16 + 4) + 4) * 2 * U


def head(h, w, q, dloss, scale, offset):
    """(loss, lse, dh, dw, bounds) of targets q (n x classes, rows that sum to 1 or 0)."""
    dtype = h.dtype
    h, w, q, dloss = h.double().cpu(), w.double().cpu(), q.double().cpu(), dloss.double().cpu()
    n, d = h.shape
    V = w.shape[0]
    off = torch.zeros(V, dtype=torch.float64) if offset is None else offset.double().cpu()
    kept = off > -1e30  # (the type's lowest value leaves a class out as well)
    off = torch.where(kept, off, -torch.inf)
    has = q.sum(1) > 0
    h = torch.where((has & (dloss != 0))[:, None] | torch.isfinite(h), h, 0.0)
    w = torch.where(kept[:, None], w, 0.0)
    z = scale * (h @ w.t()) + off
    dz = abs(scale) * (h.abs() @ w.abs().t()) * sum_error(d, dtype) + 4 * U * torch.where(kept, z.abs() + off.abs(), 0.0)
    dz = dz.amax(1)  # an entry's error, row by row
    lse = torch.logsumexp(z, 1)
    alive = lse > -torch.inf
    base = torch.where(alive, lse, 0.0)[:, None]
    terms = torch.where(q > 0, q * (torch.log(q) - z + base), 0.0)
    loss = torch.where(has, terms.sum(1), 0.0)
    loss = torch.where(has & ~alive, torch.inf, loss)
    size = torch.where(alive, lse.abs(), 0.0) + torch.where((q > 0) & kept, q * (torch.log(q.clamp(min=1e-300)).abs() + z.abs()), 0.0).sum(1)
    tol_loss = 3 * dz + (16 + V / 64) * 2 * U * size + (V / 64 + 16) * 2 * U
    p = torch.where(alive[:, None], torch.exp(z - base), 0.0)
    c = torch.where(has & alive, dloss, 0.0)[:, None] * scale
    G = torch.where(kept, p - q, 0.0) * c
    # an entry's error: the logits' and the sum's, a rounding to the operands' type
    rel = 4 * dz[:, None] + (V / 64 + 32) * 2 * U
    low = STEP[dtype] * dloss.abs().max() * 2.0 ** -12 * abs(scale)
    dG = (p * rel + q * 8 * U) * c.abs() + G.abs() * (UNIT[dtype] if dtype != torch.float32 else 2 * U) + low
    dG = torch.where(c != 0, dG, 0.0)
    dh, dw = G @ w, G.t() @ h
    tol = []
    for left, dleft, right, out, K in ((G, dG, w, dh, V), (G.t(), dG.t(), h, dw, n)):
        tol.append((dleft.abs() + left.abs() * (sum_error(K, dtype) + 40 * U)) @ right.abs()
                   + UNIT[dtype] * out.abs() + STEP[dtype])
    return dict(loss=loss, lse=lse, dh=dh, dw=dw, tol_loss=tol_loss, tol_lse=dz + (16 + V / 64) * 2 * U * (1 + size),
                tol_dh=tol[0], tol_dw=tol[1])


def one_hot(ids, V):
    q = torch.zeros(ids.numel(), V, dtype=torch.float64)
    ids = ids.cpu().long()
    i = torch.nonzero(ids >= 0)[:, 0]
    q[i, ids[i]] = 1.0
    return q


def teacher(top_ids, top_logits, scale, V):
    ids, t = top_ids.cpu().long(), top_logits.double().cpu() * scale
    t = torch.where(ids >= 0, t, -torch.inf)
    q = torch.softmax(t, 1)
    q = torch.where(t > -torch.inf, q, 0.0)
    return torch.zeros(ids.shape[0], V, dtype=torch.float64).scatter_add_(1, ids.clamp(min=0), q)


def layer_norm(x, weight, bias, eps, dy):
    dtype = x.dtype
    x, dy = x.double().cpu(), dy.double().cpu()
    n, d = x.shape
    w = torch.ones(d, dtype=torch.float64) if weight is None else weight.double().cpu()
    b = torch.zeros(d, dtype=torch.float64) if bias is None else bias.double().cpu()
    mu = x.mean(1, keepdim=True)
    var = ((x - mu) ** 2).mean(1, keepdim=True)
    r = 1 / torch.sqrt(var + eps)
    xh = (x - mu) * r
    g = dy * w
    mg, mgx = g.mean(1, keepdim=True), (g * xh).mean(1, keepdim=True)
    # a thread adds up to max(32, d/256) terms, a tree of 8 joins them
    L = 48 + d / 256
    dmu = L * U * x.abs().mean(1, keepdim=True)
    drel = 2 * (L + 8) * U + r * dmu + (r * dmu) ** 2  # of r
    dxh = r * dmu + xh.abs() * (drel + 4 * U) + 2 * U * r * (x - mu).abs() + r * U * mu.abs()
    dg = 2 * U * g.abs()
    sums = mg.abs() * 0 + g.abs().mean(1, keepdim=True) * (L + 4) * 2 * U
    sumx = (g * xh).abs().mean(1, keepdim=True) * (L + 8) * 2 * U + (g.abs() * dxh).mean(1, keepdim=True)
    ddx = r * (dg + sums + dxh * mgx.abs() + (xh.abs() + dxh) * sumx + 8 * U * (g.abs() + mg.abs() + (xh * mgx).abs()))
    dx = r * (g - mg - xh * mgx)
    ddx = ddx + dx.abs() * (drel + 4 * U) + r * (mg.abs() + xh.abs() * mgx.abs()) * drel
    rows = (n / 64 + 64) * 2 * U
    y = xh * w + b
    wtype = torch.float32 if weight is None else weight.dtype
    dw, db = (dy * xh).sum(0), dy.sum(0)
    return dict(y=y, mean=mu[:, 0], rstd=r[:, 0], dx=dx, dw=dw, db=db,
                tol_y=w.abs() * dxh + 4 * U * (y.abs() + b.abs()) + UNIT[dtype] * y.abs() + STEP[dtype],
                tol_mean=dmu[:, 0] + 4 * U * mu[:, 0].abs(), tol_rstd=(r * (drel + 8 * U))[:, 0],
                tol_dx=ddx + UNIT[dtype] * dx.abs() + STEP[dtype],
                tol_dw=(dy.abs() * dxh).sum(0) + rows * (dy * xh).abs().sum(0) + UNIT[wtype] * dw.abs() + STEP[wtype],
                tol_db=rows * dy.abs().sum(0) + UNIT[wtype] * db.abs() + STEP[wtype])


def check(name, got, ref, tol):
    got = got.double().cpu()
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    fin = torch.isfinite(ref)
    same = torch.isnan(ref) & torch.isnan(got) | (ref == got)
    assert bool(same[~fin].all()), f"{name}: infinities or NaN differ"
    if not fin.any():
        return 0.0
    err = torch.where(fin, (got - torch.where(fin, ref, 0.0)).abs(), 0.0)
    bad = ~(err <= tol) & fin
    assert not bool(bad.any()), (f"{name}: {int(bad.sum())} of {bad.numel()} beyond the bound; worst "
                                 f"{float((err / tol.clamp(min=1e-300))[bad].max()):.3g} of it at "
                                 f"{torch.nonzero(bad)[0].tolist()}")
    return float((err / tol.clamp(min=1e-300)).max())
