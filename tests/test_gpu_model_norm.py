"""Layer norm: rows of one value, whose differences from the mean are all
rounding, and more rows than a launch has groups for."""
import pytest

import model_reference as ref
from test_gpu_model import DTYPES, _gen, ctx  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("d", [7, 257, 300, 780, 1000, 1023, 3001, 8000, 9001, 20000])
def test_rows_of_one_value(ctx, d):
    """xh = 0, the mean is the value, and no gradient goes to the weight."""
    from paper_2601_17136_amd import kkm
    eps, L = 1e-5, 48 + d / 256  # L: a sum's roundings
    values = torch.tensor([1000.0, 30000.0, -30000.1, 0.1, 3.0, 1.0 / 3, 65537.0, 1e6], device="cuda")
    x = values[:, None].repeat(1, d).contiguous()
    b, dy = (torch.randn(*s, device="cuda", generator=_gen(d)) for s in ((d,), (8, d)))
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = torch.empty(8, device="cuda"), torch.empty(8, device="cuda")
    dw, db = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    kkm.kkm_layer_norm(ctx, x, None, b, eps, y, mean, rstd)
    # x - mu is off by the sum's roundings, once in mu and once more in what is left of it
    left = (L * ref.U) ** 2 * values.abs().double()
    assert torch.equal(mean, values)
    assert bool(((y - b).abs().double() <= (left / eps ** 0.5)[:, None] + 2 * ref.U * b.abs().double()).all())
    var = (L * ref.U * values.abs().double()) ** 2 * 4 * L * ref.U
    assert bool(((rstd.double() * eps ** 0.5 - 1).abs() <= var / eps + 8 * ref.U).all())
    kkm.kkm_layer_norm_grad(ctx, x, torch.ones(d, device="cuda"), dy, mean, rstd, dx, dw, db)
    assert not dw.any()
    g = dy.double()
    tol = (2 * g.abs() + (L + 8) * 2 * g.abs().mean(1, keepdim=True)) * ref.U * 8 / eps ** 0.5
    want = rstd.double()[:, None] * (g - g.mean(1, keepdim=True))
    assert bool(((dx.double() - want).abs() <= tol).all())


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("d", [780, 3001, 9001, 20000])
def test_rows_of_one_value_in_16_bits(ctx, d, dtype):
    from paper_2601_17136_amd import kkm
    t, eps, L = DTYPES[dtype], 1e-5, 48 + d / 256
    values = torch.tensor([1000.0, 30000.0, 0.1, 1.0 / 3], device="cuda").to(t)
    x = values[:, None].repeat(1, d).contiguous()
    y, mean, rstd = torch.empty_like(x), torch.empty(4, device="cuda"), torch.empty(4, device="cuda")
    kkm.kkm_layer_norm(ctx, x, None, None, eps, y, mean, rstd)
    assert torch.equal(mean, values.float())
    left = (L * ref.U) ** 2 * values.abs().double() / eps ** 0.5
    assert bool((y.abs().double() <= (left * 1.01 + ref.STEP[t])[:, None]).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,d", [(9001, 301), (5001, 784), (2500, 4096), (1100, 20000)])
def test_more_rows_than_groups(ctx, n, d, dtype):
    """Each group of lanes goes over several rows, the next on its way while one is summed."""
    from paper_2601_17136_amd import kkm
    t, g = DTYPES[dtype], _gen(n + d)
    print(f"[gpu] layer norm n={n} d={d} {dtype}", flush=True)
    x = (torch.randn(n, d, device="cuda", generator=g) * 2 + torch.randn(n, 1, device="cuda", generator=g) * 3).to(t)
    dy = torch.randn(n, d, device="cuda", generator=g).to(t)
    w, b = 1 + 0.3 * torch.randn(d, device="cuda", generator=g), torch.randn(d, device="cuda", generator=g)
    y, dx, dw, db = torch.empty_like(x), torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
    mean, rstd = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    kkm.kkm_layer_norm(ctx, x, w, b, 1e-3, y, mean, rstd)
    kkm.kkm_layer_norm_grad(ctx, x, w, dy, mean, rstd, dx, dw, db)
    r = ref.layer_norm(x, w, b, 1e-3, dy)
    for name, got in (("y", y), ("mean", mean), ("rstd", rstd), ("dx", dx), ("dw", dw), ("db", db)):
        ref.check(name, got, r[name], r["tol_" + name])
