"""Rows' weights (dloss) in the head's gradient: what rows that take no part
hold, weights that are no numbers, and weights of very different sizes."""
import pytest

import model_reference as ref
from test_gpu_model import DTYPES, _head_case, _outputs, _teacher, ctx  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

# each form the head runs in: little work, few classes, few rows, tiles
FORMS = [(150, 40, 90), (150, 40, 50), (40, 40, 90), (2600, 640, 1300)]


def _call(ctx, m, h, w, said, dloss, off=None):
    from paper_2601_17136_amd import kkm
    out = _outputs(h, w)
    (kkm.kkm_distill_grad if m else kkm.kkm_head_grad)(ctx, h, w, *said, dloss, *out, offset=off)
    return out


def _targets(n, V, m, ids, g, kept):
    """Ids or pairs, and three rows that have none."""
    none = [5, 17, 33]
    if not m:
        ids[none] = -1
        return (ids,), none
    top, logits = _teacher(n, V, m, g, kept)
    top[none[0]] = -1
    logits[none[1:]] = -float("inf")
    return (top, logits), none


@pytest.mark.parametrize("m", [0, 3])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,d,V", FORMS)
def test_weights_of_rows_without_a_target(ctx, n, d, V, dtype, m):
    """Whatever weight such a row has, every result has the bits it has with weight 0 there."""
    print(f"[gpu] weights of rows without a target n={n} d={d} V={V} {dtype} m={m}", flush=True)
    h, w, off, ids, dloss, g, kept = _head_case(n, d, V, dtype, 61, offset=True)
    said, none = _targets(n, V, m, ids, g, kept)
    dloss[none] = 0.0
    want = _call(ctx, m, h, w, said, dloss, off)
    assert torch.isfinite(want[2]).all() and torch.isfinite(want[3]).all() and want[3].any()
    for weights in ((float("nan"), 1.0, 1.0), (float("inf"), -float("inf"), 0.0), (1e30, -1e-30, 3e38)):
        dloss[none] = torch.tensor(weights, device="cuda")
        got = _call(ctx, m, h, w, said, dloss, off)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), weights


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,d,V", FORMS)
def test_a_weight_that_is_no_number_spoils_its_own_row(ctx, n, d, V, dtype, bad):
    print(f"[gpu] weight {bad} n={n} d={d} V={V} {dtype}", flush=True)
    h, w, _, ids, dloss, _, _ = _head_case(n, d, V, dtype, 62)
    dloss[7] = 0.0
    want = _call(ctx, 0, h, w, (ids,), dloss)
    dloss[7] = bad
    got = _call(ctx, 0, h, w, (ids,), dloss)
    others = [i for i in range(n) if i != 7]
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert torch.equal(got[2][others], want[2][others])
    assert not torch.isfinite(got[2][7]).any()


@pytest.mark.parametrize("m", [0, 5])
@pytest.mark.parametrize("n,d,V", [(700, 216, 1100), (701, 217, 1101), (2600, 640, 1300), (900, 400, 20000)])
def test_rows_weights_of_many_sizes(ctx, n, d, V, m):
    """Binary16: a row of a ten thousand millionth of the largest weight has as exact a dh as the others."""
    print(f"[gpu] weights of many sizes n={n} d={d} V={V} m={m}", flush=True)
    h, w, _, ids, dloss, g, kept = _head_case(n, d, V, "f16", 63, drop=0.1)
    said, q = (ids,), ref.one_hot(ids, V)
    if m:
        said = _teacher(n, V, m, g, kept)
        q = ref.teacher(*said, 1.0, V)
    power = torch.arange(n, device="cuda") % 10
    dloss = torch.sign(dloss) * 10.0 ** (5 - power)
    dh = _call(ctx, m, h, w, said, dloss)[2]
    for p in range(10):
        rows = torch.nonzero(power == p)[:, 0]
        r = ref.head(h[rows], w, q[rows.cpu()], dloss[rows], 1.0, None)
        ref.check(f"dh of weight 1e{5 - p}", dh[rows], r["dh"], r["tol_dh"])


@pytest.mark.parametrize("factor", [1.0, 2.0 ** -20, 2.0 ** 10])
@pytest.mark.parametrize("n,d,V", [(700, 216, 1100), (701, 217, 1101), (2600, 640, 1300)])
def test_features_of_light_rows_alone(ctx, n, d, V, factor):
    """Binary16: half of the features are other than 0 in four light rows alone (1e-7 of the others'
    weight), so that these columns of dw are theirs."""
    print(f"[gpu] features of light rows n={n} d={d} V={V} factor={factor}", flush=True)
    h, w, _, ids, dloss, _, _ = _head_case(n, d, V, "f16", 64)
    light = torch.zeros(n, dtype=torch.bool, device="cuda")
    light[[3, n // 3, n // 2, n - 1]] = True
    a = d // 2
    h[:, :a] *= 0.1
    h[:, a:] *= 30.0
    w[:, :a] *= 10.0
    w[:, a:] /= 30.0
    h[~light, a:] = 0.0
    h[light, :a] = 0.0
    dloss = torch.where(light, 3e-3, 3e4) * torch.sign(dloss) * factor
    dw = _call(ctx, 0, h, w, (ids,), dloss)[3]
    q = ref.one_hot(ids, V)
    want, tol, top = 0.0, 0.0, -1e9
    for part in (light, ~light):
        rows = torch.nonzero(part)[:, 0]
        r = ref.head(h[rows], w, q[rows.cpu()], dloss[rows], 1.0, None)
        want, tol = want + r["dw"], tol + r["tol_dw"]
        top = max(top, float(torch.log2(dloss[rows].abs().max() * h[rows].abs().max())) + 2)
    # the copy of h that dw is multiplied from holds it times its weight, 15 bits above 1 at the most:
    # a step is 2^-24, so that half of one is 2^(top - 40) of a row's weight times its entry of h
    tol = tol + 2.0 ** (top - 40) * (n * 1.0 / V + 4)
    ref.check("dw", dw[:, a:], want[:, a:], tol[:, a:])
