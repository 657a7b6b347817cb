"""Classes that are left out have no gradient, also beside rows that are NaN."""
import pytest

from test_gpu_model import DTYPES, _head_case, _outputs, _teacher, ctx  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("m", [0, 3])
@pytest.mark.parametrize("spoil", ["id", "h", "dloss"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,d,V", [(150, 40, 90), (150, 40, 50), (4200, 40, 50), (40, 40, 90), (2600, 640, 1300),
                                   (300, 640, 9000)])
def test_gradient_of_a_class_that_is_left_out(ctx, n, d, V, dtype, spoil, m):
    """An id past the classes, a NaN in a row of h and in its weight: NaN in dw, but not in the rows of dw left out."""
    from paper_2601_17136_amd import kkm
    print(f"[gpu] left out n={n} d={d} V={V} {dtype} {spoil} m={m}", flush=True)
    h, w, off, ids, dloss, g, kept = _head_case(n, d, V, dtype, 81, offset=True)
    said, fn = (ids,), kkm.kkm_head_grad
    if m:
        said, fn = _teacher(n, V, m, g, kept), kkm.kkm_distill_grad
        said[0][7] = kept[:m].to(torch.int32)
        said[1][7] = 0.5
    if spoil == "id":
        said[0].view(n, -1)[7, 0] = V
    elif spoil == "h":
        h[7, 3] = float("nan")
    else:
        dloss[7] = float("nan")
    loss, lse, dh, dw = _outputs(h, w)
    fn(ctx, h, w, *said, dloss, loss, lse, dh, dw, offset=off)
    out = off == -float("inf")
    assert not dw[out].any() and torch.isnan(dw[~out]).any()
    assert torch.isnan(dh[7]).all() and torch.isfinite(dh[8:]).all() and torch.isfinite(dh[:7]).all()
    alone = torch.empty_like(dw)
    fn(ctx, h, w, *said, dloss, loss, lse, None, alone, offset=off)
    assert not alone[out].any()
