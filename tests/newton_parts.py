"""How near the tiled orthogonalised update has to come: no further from 64 bits than twice fp32 products of the same
steps, before the one rounding to the result's type.

An entry of two binary16 parts is at most 2^-22 of itself off and a product without lo lo 2^-22 more, where fp32
entries are 2^-24 off and a sum of K terms up to K 2^-24; both errors are carried through the steps alike."""
import torch

U = 2.0 ** -24
BITS = {torch.float32: 24, torch.float16: 11, torch.bfloat16: 8}


def _steps(x, coef, product):
    tall = x.shape[0] > x.shape[1]
    x = x.t().contiguous() if tall else x
    for a, b, c in coef:
        A = product(x, x.t().contiguous())
        B = b * A + c * product(A, A) if c else b * A
        x = a * x + product(B, x)
    return x.t().contiguous() if tall else x


def exact(u, coef, eps):
    u = u.double()
    return _steps(u / (u.norm() + eps), coef, torch.mm)


def fp32(u, coef, eps):
    x = (u.double() / (u.double().norm() + eps)).float()
    return _steps(x, coef, torch.mm).double()


def parts(u, coef, eps, count):
    """The steps in 64 bits, every factor of a product held as `count` binary16 parts at a power of two."""
    def split(v):
        scale = 2.0 ** (14 - torch.ceil(torch.log2(v.abs().max())))
        hi = (v * scale).half().double()
        lo = (v * scale - hi).half().double() if count == 2 else torch.zeros_like(hi)
        return hi / scale, lo / scale

    def product(p, q):
        (ph, pl), (qh, ql) = split(p), split(q)
        return ph @ qh + (ph @ ql + pl @ qh)

    u = u.double()
    return _steps(u / (u.norm() + eps), coef, product)


def beyond(got, want):
    """The norm of what `got` is off by past half a step of its type."""
    _, e = torch.frexp(got.double())
    half = torch.where(got == 0, 0.0, torch.exp2((e - BITS[got.dtype] - 1).double()))  # (a zero is not rounded to)
    if got.dtype == torch.float16:
        half = half.clamp(min=2.0 ** -25)
    return float(((got.double() - want).abs() - half).clamp(min=0.0).norm())


def room(u, want, coef, eps):
    """What `beyond` may be: twice fp32 products' error, and four roundings of fp32 at the end."""
    return 2 * float((fp32(u, coef, eps) - want).norm()) + 4 * U * float(want.norm())
