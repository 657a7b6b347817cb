"""Rows whose mask id is none of the masks, beside offsets and biases that leave classes out."""
import pytest

import learn_reference as ref
from test_gpu_choose import DTYPES, INF, _check, _run, ctx  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [1, 15, 33, 600, 1030, 5000, 70001])
def test_a_lost_row_is_nan(ctx, V, dtype):  # noqa: F811
    g = torch.Generator(device="cuda").manual_seed(V)
    z = ref.rows(6, V, DTYPES[dtype], 3, torch.randn(6, V, device="cuda", generator=g))
    masks = torch.randint(-2 ** 31, 2 ** 31, (3, (V + 31) // 32), device="cuda", generator=g).int()
    masks[2] = 0
    mask_ids = torch.tensor([3, 1, 2 ** 31 - 1, -1, 2, 4], dtype=torch.int32, device="cuda")
    lost = torch.tensor([True, False, True, False, False, True], device="cuda")
    some, every = torch.zeros(V, device="cuda"), torch.full((V,), -INF, device="cuda")
    some[::3] = -INF
    bias_ids = torch.tensor([[0, V - 1, V // 2]] * 6, dtype=torch.int32, device="cuda")
    bias = torch.tensor([[-INF, 1.0, -INF]] * 6, device="cuda")
    for offset in (None, some, every):
        for lists in ({}, {"bias_ids": bias_ids, "bias": bias}):
            kw = dict(masks=masks, mask_ids=mask_ids, offset=offset, scale=0.5, **lists)
            got = _run(ctx, z, 1, **kw)
            _check(z, got, kw)
            out, ids, logp, lse = got
            assert torch.isnan(out[lost]).all() and torch.isnan(logp[lost]).all() and torch.isnan(lse[lost]).all()
            assert bool((ids[lost] == -1).all()) and not torch.isnan(lse[~lost]).any()
            alone = _run(ctx, z, out=False, **kw)
            assert torch.isnan(alone[2][lost]).all() and torch.isnan(alone[3][lost]).all()
