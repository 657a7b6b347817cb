"""Heads at the ends of what the arguments allow: more work-items than one launch
can have, in the scores, the copies of operands, the sums and the zeros."""
import pytest

import model_reference as ref
from test_gpu_model import ctx  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _normal(n, d, seed, size, dtype=torch.bfloat16):
    """n x d normal values, made in parts."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = torch.empty(n, d, device="cuda", dtype=dtype)
    for i in range(0, n, 1 << 17):
        part = out[i:i + (1 << 17)]
        part.copy_(torch.randn(part.shape, device="cuda", generator=g) * size)
    return out


def _check_rows(h, w, ids, loss, lse, rows):
    """The loss of some rows, against 64 bits."""
    hd = h[rows].double()
    z = torch.cat([torch.mm(hd, w[i:i + (1 << 16)].double().t().contiguous()) for i in range(0, w.shape[0], 1 << 16)], 1)
    dz = float((hd.abs().sum(1) * w.abs().max().double()).max()) * ref.sum_error(h.shape[1], h.dtype)
    want = torch.logsumexp(z, 1)
    V = w.shape[0]
    tol = dz + (16 + V / 64) * 2 * ref.U * (1 + want.abs())
    assert bool(((lse[rows].double() - want).abs() <= tol).all())
    want_loss = want - z.gather(1, ids[rows].long()[:, None])[:, 0]
    assert bool(((loss[rows].double() - want_loss).abs() <= 3 * tol).all())
    return z, want


def test_scores_of_most_rows_by_many_classes(ctx):
    """2^21 rows by 2^18 + 77 classes: 2^32 work-items and more."""
    from paper_2601_17136_amd import kkm
    n, V, d = kkm.KKM_MAX_ROWS, (1 << 18) + 77, 8
    print(f"[gpu] scores n={n} V={V} d={d}", flush=True)
    h, w = _normal(n, d, 91, 1.0), _normal(V, d, 92, 0.5)
    ids = torch.randint(0, V, (n,), device="cuda", dtype=torch.int32)
    loss, lse = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    kkm.kkm_head_loss(ctx, h, w, ids, loss, lse)
    rows = torch.tensor([0, 1, 127, 128, 255, 256, n // 2 - 1, n // 2, n - 257, n - 2, n - 1], device="cuda")
    ids[rows[0]] = V - 1
    kkm.kkm_head_loss(ctx, h, w, ids, loss, lse)
    _check_rows(h, w, ids, loss, lse, rows)
    assert torch.isfinite(loss).all() and torch.isfinite(lse).all()


def test_copies_of_many_rows(ctx):
    """2^21 classes of 4097 features, whose rows are copied for the matrix cores: 9e9 entries."""
    from paper_2601_17136_amd import kkm
    n, V, d = 70, kkm.KKM_MAX_ROWS, 4097
    print(f"[gpu] copies n={n} V={V} d={d}", flush=True)
    h, w = _normal(n, d, 93, 1.0), _normal(V, d, 94, 0.03)
    w[V - 1] = w[V - 1] * 8
    ids = torch.randint(0, V, (n,), device="cuda", dtype=torch.int32)
    ids[3] = V - 1
    loss, lse = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    kkm.kkm_head_loss(ctx, h, w, ids, loss, lse)
    _check_rows(h, w, ids, loss, lse, torch.arange(n, device="cuda"))


def test_sums_of_many_rows(ctx):
    """dh of 2^21 rows of 2100 over two pieces of the classes: 4.4e9 sums."""
    from paper_2601_17136_amd import kkm
    n, V, d = kkm.KKM_MAX_ROWS, 300, 2100
    print(f"[gpu] sums n={n} V={V} d={d}", flush=True)
    h, w = _normal(n, d, 95, 1.0), _normal(V, d, 96, 0.04)
    ids = torch.randint(0, V, (n,), device="cuda", dtype=torch.int32)
    dloss = torch.rand(n, device="cuda") + 0.5
    loss, lse, dh = torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.full_like(h, float("nan"))
    kkm.kkm_head_grad(ctx, h, w, ids, dloss, loss, lse, dh, None)
    rows = torch.tensor([0, 1, 255, 256, 1 << 20, (1 << 20) + 1, n - 300, n - 2, n - 1], device="cuda")
    _check_rows(h, w, ids, loss, lse, rows)
    r = ref.head(h[rows], w, ref.one_hot(ids[rows], V), dloss[rows], 1.0, None)
    ref.check("dh", dh[rows], r["dh"], r["tol_dh"])
    assert all(bool(torch.isfinite(dh[i:i + (1 << 17)]).all()) for i in range(0, n, 1 << 17))


def test_zeros_of_many_classes(ctx):
    """No rows: dw of 2^21 classes of 2050 features is zero, 4.3e9 entries of it."""
    from paper_2601_17136_amd import kkm
    V, d = kkm.KKM_MAX_ROWS, 2050
    w, h = torch.empty(V, d, device="cuda", dtype=torch.bfloat16), torch.empty(0, d, device="cuda", dtype=torch.bfloat16)
    dw = torch.full_like(w, 3.0)
    e = torch.empty(0, device="cuda")
    kkm.kkm_head_grad(ctx, h, w, e.to(torch.int32), e, e, e, None, dw)
    assert not any(bool(dw[i:i + (1 << 17)].any()) for i in range(0, V, 1 << 17))
