"""Plain forms of the adapted projection, the orthogonalised update and answers
from logits, with error bounds for the kernels that follow from the arithmetic
they state (U = 2^-24, half a step of fp32)."""
import torch

U = 2.0 ** -24
UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
STEP = {torch.float32: 0.0, torch.float16: 2.0 ** -24, torch.bfloat16: 0.0}  # smallest step of what is stored


def rows(n, d, dtype, pad, values):
    """n x d values as the columns [pad // 2, ..) of a table d + pad wide, NaN beside them."""
    t = torch.full((n, d + pad), float("nan"), device=values.device, dtype=dtype)[:, pad // 2:pad // 2 + d]
    t.copy_(values)
    return t


# ------------------------------------------------------------------ answers from logits

def choose(z, scale, offset=None, given=None, repeat=1.0, presence=0.0, frequency=0.0, bias_ids=None, bias=None,
           masks=None, mask_ids=None):
    """(u, ids, logp, lse, bound of lse and logp): u in fp32 with the stated operations (so ids are exact),
    the sums in 64 bits."""
    f32 = torch.float32
    z = z.float().cpu()
    n, V = z.shape
    scale, repeat, presence, frequency = (torch.tensor(v, dtype=f32) for v in (scale, repeat, presence, frequency))
    u = z.clone()
    gone = torch.zeros(n, V, dtype=torch.bool)
    if given is not None:
        given = given.cpu()
        for i in range(n):
            ids = given[i][(given[i] >= 0) & (given[i] < V)].long()
            count = torch.bincount(ids, minlength=V).float()
            seen = torch.where(u[i] > 0, u[i] / repeat, u[i] * repeat) - (presence + count * frequency)
            u[i] = torch.where(count > 0, seen, u[i])
    if offset is not None:
        u = u + offset.cpu()[None, :]
        gone |= (offset.cpu() == -torch.inf)[None, :]
    if bias_ids is not None:
        for i in range(n):
            last = {int(v): float(b) for v, b in zip(bias_ids[i].cpu(), bias[i].cpu()) if 0 <= v < V}
            for v, b in last.items():
                u[i, v] = u[i, v] + torch.tensor(b, dtype=f32)
                gone[i, v] |= b == -float("inf")
    u = u * scale
    lost = torch.zeros(n, dtype=torch.bool)
    if masks is not None:
        v = torch.arange(V)
        bits = (masks.cpu().long()[:, v // 32] >> (v % 32)) & 1 == 0
        for i in range(n):
            k = i if mask_ids is None else int(mask_ids[i])
            if k >= masks.shape[0]:
                lost[i] = True
            elif k >= 0:
                gone[i] |= bits[k]
    u = torch.where(lost[:, None], torch.nan, u)
    u = torch.where(gone & ~lost[:, None], -torch.inf, u)
    d = u.double()
    nan = torch.isnan(d).any(1)
    top = torch.where(nan, 0.0, torch.nan_to_num(d, nan=0.0, posinf=torch.inf, neginf=-torch.inf).amax(1))
    first = torch.where(d == top[:, None], torch.arange(V), V).amin(1)
    ids = torch.where(nan | (top == -torch.inf), -1, first).to(torch.int32)
    terms = torch.where(d == top[:, None], 1.0, torch.exp(d - torch.where(top == -torch.inf, 0.0, top)[:, None]))
    s = torch.log(terms.sum(1))
    none = top == -torch.inf
    logp = torch.where(nan, torch.nan, torch.where(none, -torch.inf, -s))
    lse = torch.where(nan, torch.nan, torch.where(none, -torch.inf, top + s))
    # a term: the difference and its product with log2 e rounded (x e^-x is at most 0.37), the exponential 2 steps;
    # the sum: 16 terms of a lane, 6 levels of lanes, 4 wavefronts, up to 512 slices by lanes and levels again; the
    # logarithm 2 steps of itself, the sum with the largest logit one rounding
    tol = (4 * 0.37 + 4 + 16 + 6 + 4 + 8 + 6) * U + 4 * U * s.abs()
    return u, ids, logp, lse, tol, tol + U * lse.abs()


# ------------------------------------------------------------------ orthogonalised updates

def newton(u, coef, eps, dtype=torch.float32):
    """The steps in 64 bits, and a bound of the result's error in the Frobenius norm.

    A step x -> p(x) of the singular values carries an error of X on by at most the
    largest |p'| (also of the parts that mix two singular vectors, whose factors are
    differences and sums of p over those of s).  To it each step adds its own: two
    binary16 parts leave 2^-22 of an operand and the product without lo lo 2^-22 more,
    A, A^2 and B once each; fp32 sums of K terms on the matrix cores 2 U at each of
    3 K / 16 instructions, of sizes that the norms' products bound.  A bfloat16 result's
    Gram matrices and products with B take X by its hi part alone, 2^-11 of it off."""
    x = u.double()
    if x.numel() < 10 ** 6:
        x = x.cpu()
    tall = x.shape[0] > x.shape[1]
    if tall:
        x = x.t().contiguous()
    x = x / (x.norm() + eps)
    S, K = x.shape
    err, top = (4 * U + 2.0 ** -22) * float(x.norm()), 1.0
    for a, b, c in coef:
        s = torch.linspace(0, top, 2001, dtype=torch.float64)
        slope = float((a + 3 * b * s ** 2 + 5 * c * s ** 4).abs().max())
        A = x @ x.t().contiguous()
        an, xn = float(A.norm()), float(x.norm())
        rel = lambda terms: 3 * 2.0 ** -22 + 2 * U * (3 * terms / 16 + 4)
        one = 2.0 ** -11 if dtype == torch.bfloat16 else 0.0
        dA = (rel(K) + 2 * one) * xn * top
        B = b * A + c * (A @ A)
        # (|X Y| <= |X| times Y's largest singular value)
        dB = (abs(b) + 2 * abs(c) * top ** 2) * dA + abs(c) * rel(S) * an * an + 2.0 ** -22 * (abs(b) * an + abs(c) * an * an)
        new = a * x + B @ x
        beta = float((b * s ** 2 + c * s ** 4).abs().max())  # the norm of B
        local = dB * top + one * beta * xn + rel(S) * float(B.norm()) * xn + (2.0 ** -21) * (abs(a) * xn + float(new.norm()))
        err = slope * err + local
        top = max(float((a * s + b * s ** 3 + c * s ** 5).abs().max()), 1e-30) * (1 + 1e-6)
        x = new
    return (x.t() if tall else x).cpu(), float(err)


def slope_of(coef):
    """How far the steps carry an error of X = u / |u| at most."""
    slope, top = 1.0, 1.0
    for a, b, c in coef:
        s = torch.linspace(0, top, 2001, dtype=torch.float64)
        slope *= float((a + 3 * b * s ** 2 + 5 * c * s ** 4).abs().max())
        top = max(float((a * s + b * s ** 3 + c * s ** 5).abs().max()), 1e-30) * (1 + 1e-6)
    return slope


# ------------------------------------------------------------------ adapted projection

def _sums(terms, dtype):
    from model_reference import sum_error
    return sum_error(terms, dtype)


def adapted(x, w, down, up, ids, factor, dy):
    """(y, dx, ddown, dup and a bound of each, entry by entry) in 64 bits, where the inputs are."""
    dtype = x.dtype
    x, w, down, up, dy = (v.double() for v in (x, w, down, up, dy))
    n, d = x.shape
    m = w.shape[0]
    s, r, _ = down.shape
    f = torch.ones(s, dtype=torch.float64, device=x.device) if factor is None else factor.double()
    out = {"y": x @ w.t(), "dx": dy @ w, "ddown": torch.zeros_like(down), "dup": torch.zeros_like(up)}
    tol = {"y": _sums(d, dtype) * (x.abs() @ w.abs().t()), "dx": _sums(m, dtype) * (dy.abs() @ w.abs()),
           "ddown": torch.zeros_like(down), "dup": torch.zeros_like(up)}
    for g in range(s):
        i = torch.nonzero(ids == g)[:, 0]
        if i.numel() == 0:
            continue
        # t and u: a sum of the width, times f; the second product r terms more; a gradient the rows' sum
        t, u = f[g] * (x[i] @ down[g].t()), f[g] * (dy[i] @ up[g])
        dt = f[g].abs() * (_sums(d, torch.float32) + 4 * U) * (x[i].abs() @ down[g].abs().t())
        du = f[g].abs() * (_sums(m, torch.float32) + 4 * U) * (dy[i].abs() @ up[g].abs())
        # (of 16-bit rows t and u are two parts of the rows' type, 16 or 22 bits, in y and dx, and two bfloat16 parts in
        # the adapters' gradients)
        low = (r + 8) * 2 * U + {torch.float32: 0.0, torch.float16: 2.0 ** -21, torch.bfloat16: 2.0 ** -16}[dtype]
        rows = (i.numel() / 4 + 40) * 2 * U + (0.0 if dtype == torch.float32 else 2.0 ** -16)
        out["y"][i] += t @ up[g].t()
        tol["y"][i] += (dt + low * t.abs()) @ up[g].abs().t()
        out["dx"][i] += u @ down[g]
        tol["dx"][i] += (du + low * u.abs()) @ down[g].abs()
        out["ddown"][g] = u.t() @ x[i]
        tol["ddown"][g] = (du + rows * u.abs()).t() @ x[i].abs()
        out["dup"][g] = dy[i].t() @ t
        tol["dup"][g] = dy[i].abs().t() @ (dt + rows * t.abs())
    bad = torch.nonzero(ids >= s)[:, 0]
    out["y"][bad] = torch.nan
    out["dx"][bad] = torch.nan
    for k, v in out.items():
        tol[k] += (UNIT[dtype] + 4 * U) * v.abs() + STEP[dtype]
    return out, tol


def check(name, got, want, tol):
    got = got.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want)), name
    fine = ~torch.isnan(want)
    off = (got - want).abs()[fine]
    worst = float((off / tol[fine].clamp(min=1e-300)).max()) if off.numel() else 0.0
    assert worst <= 1, (name, worst)
    return worst
