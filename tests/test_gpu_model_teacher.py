"""A teacher's logits and scale at their ends: scale 0 and below, logits of -inf
and of the type's lowest value."""
import pytest

import model_reference as ref
from test_gpu_model import DTYPES, _head_case, _outputs, ctx  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
LOWEST = torch.finfo(torch.float32).min


@pytest.mark.parametrize("scale", [0.0, -0.8, 2.0])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,d,V,m", [(150, 40, 90, 9), (150, 40, 50, 20), (40, 40, 90, 9), (2600, 640, 1300, 9),
                                     (300, 40, 1100, 70), (2600, 640, 1300, 70)])
def test_pairs_of_each_scale(ctx, n, d, V, m, dtype, scale):
    from paper_2601_17136_amd import kkm
    print(f"[gpu] teacher scale {scale} n={n} d={d} V={V} m={m} {dtype}", flush=True)
    h, w, _, _, dloss, g, _ = _head_case(n, d, V, dtype, 71)
    ids = torch.argsort(torch.rand(n, V, device="cuda", generator=g), dim=1)[:, :m]  # each class once
    logits = 3 * torch.randn(n, m, device="cuda", generator=g)
    gone = torch.rand(n, m, device="cuda", generator=g)
    ids = torch.where(gone < 0.1, -1, ids)
    logits = torch.where(gone > 0.8, -float("inf"), logits)
    logits[6, ::2] = LOWEST
    logits[7] = LOWEST  # all alike: q is uniform
    logits[9] = -float("inf")
    ids = ids.to(torch.int32).contiguous()
    there = (ids >= 0) & (logits > -float("inf"))
    s = torch.where(there, logits.double() * scale, -torch.inf)
    parts = torch.where(there, torch.softmax(s, 1), 0.0)
    q = torch.zeros(n, V, device="cuda", dtype=torch.float64).scatter_add_(1, ids.long().clamp(min=0), parts)
    loss, lse, dh, dw = _outputs(h, w)
    kkm.kkm_distill_grad(ctx, h, w, ids, logits, dloss, loss, lse, dh, dw, scale=0.5, teacher_scale=scale)
    r = ref.head(h, w, q, dloss, 0.5, None)
    for name, got in (("loss", loss), ("lse", lse), ("dh", dh), ("dw", dw)):
        ref.check(name, got, r[name], r["tol_" + name])
    assert loss[9] == 0 and not dh[9].any()
    alone = torch.empty_like(loss)
    kkm.kkm_distill_loss(ctx, h, w, ids, logits, alone, lse, scale=0.5, teacher_scale=scale)
    assert torch.equal(alone, loss)
