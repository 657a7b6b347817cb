"""Many steps of matrices that lack rank: what roundings leave beside a zero singular value must not grow past the steps'
own range, and rows that are alike stay so."""
import pytest

import newton_parts as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
EPS = 1e-7


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.fail("GPU test on a machine without a GPU")
    from paper_2601_17136_amd import kkm
    c = kkm.kkm_create(kkm.current_stream_handle())
    yield c
    kkm.kkm_destroy(c)


def _matrix(m, n, rank, alike):
    """Rows (or columns, of a tall one) that repeat `rank` of them, or combinations of these, rounded."""
    g = torch.Generator(device="cuda").manual_seed(m + n + rank)
    S, K = min(m, n), max(m, n)
    base = torch.randn(rank, K, device="cuda", generator=g)
    x = base[torch.arange(S, device="cuda") % rank] if alike else torch.randn(S, rank, device="cuda", generator=g) @ base
    return (x if m <= n else x.t()).contiguous()


def _exact_of_alike(x, rank, coef):
    """Rows i, i + rank, .. are alike: with c_i of them, x = E B, E having orthonormal columns of entries 1 / sqrt(c_i)
    and B rows sqrt(c_i) x_i, so that the steps are those of B (which has full rank: library products of x itself do
    not keep its rows alike)."""
    tall = x.shape[0] > x.shape[1]
    x = (x.t() if tall else x).double()
    at = torch.arange(x.shape[0]) % rank
    root = torch.bincount(at, minlength=rank)[:rank, None].double().sqrt()
    y = (ref.exact(x[:rank] * root, coef, EPS) / root)[at]
    return (y.t() if tall else y).contiguous()


FLAT = [(8, 784, 4), (784, 8, 3), (16, 100, 3), (33, 900, 2), (64, 64, 32), (64, 784, 10), (64, 64, 1), (5, 9, 5), (40, 300, 40)]


@pytest.mark.parametrize("steps", [6, 12, 16, 20, 32])
@pytest.mark.parametrize("m,n,rank", FLAT)
def test_rows_that_are_alike(ctx, m, n, rank, steps):
    """Products of the steps so far times 2^-53 a stage, and X's own: 2^-39 of the result at most for each of 6 stages
    of sums of 64 terms, beside the one rounding to fp32."""
    from paper_2601_17136_amd import kkm
    x = _matrix(m, n, rank, True)
    coef = [kkm.KKM_QUINTIC] * steps
    y = torch.empty_like(x)
    print(f"[gpu] {m} x {n}, rank {rank}, {steps} steps", flush=True)
    kkm.kkm_orthogonalize(ctx, x, y, coef=coef, eps=EPS)
    want = _exact_of_alike(x.cpu(), min(rank, m, n), coef)
    assert ref.beyond(y.cpu(), want) <= 6 * 64 * 2.0 ** -39 * float(want.norm())


@pytest.mark.parametrize("steps", [12, 20, 32])
@pytest.mark.parametrize("m,n,rank", FLAT + [(100, 300, 40), (300, 100, 7), (70, 70, 1)])
def test_combinations(ctx, m, n, rank, steps):
    """Singular values that roundings of the entries alone make: the result's stay in the steps' range, 1.25 at most."""
    from paper_2601_17136_amd import kkm
    for alike in (False, True):
        x = _matrix(m, n, rank, alike)
        y = torch.empty_like(x)
        kkm.kkm_orthogonalize(ctx, x, y, coef=[kkm.KKM_QUINTIC] * steps, eps=EPS)
        assert torch.isfinite(y).all()
        assert float(torch.linalg.svdvals(y.double().cpu()).max()) <= 1.25


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_steps_of_a_batch_in_stages(ctx, dtype):
    """A batch, row strides, in place, and an update, in several stages; the same bits each time."""
    from paper_2601_17136_amd import kkm
    coef = [kkm.KKM_QUINTIC] * 14
    g = torch.Generator(device="cuda").manual_seed(4)
    for m, n in ((12, 50), (50, 12)):
        wide = torch.full((5, m, n + 3), 7.0, device="cuda", dtype=dtype)
        x = wide[:, :, 1:n + 1]
        x.copy_(torch.randn(5, m, n, device="cuda", generator=g))
        y = torch.empty(5, m, n, device="cuda", dtype=dtype)
        kkm.kkm_orthogonalize(ctx, x, y, coef=coef, eps=EPS)
        for i in range(5):
            want = ref.exact(x[i].cpu(), coef, EPS)
            assert ref.beyond(y[i].cpu(), want) <= 2.0 ** -23 * float(want.norm())  # (rounded to fp32, then to the type)
        w, v = torch.zeros_like(y), torch.zeros(5, m, n, device="cuda")
        kkm.kkm_orthogonal_step(ctx, w, x, v, 1.0, momentum=0.0, nesterov=False, coef=coef, eps=EPS)
        assert torch.equal(-w, y) and torch.equal(v, x.float())
        kkm.kkm_orthogonalize(ctx, x, x, coef=coef, eps=EPS)
        assert torch.equal(x, y) and bool((wide[:, :, 0] == 7.0).all()) and bool((wide[:, :, n + 1:] == 7.0).all())


def test_zero_rows_and_zero_matrices_in_stages(ctx):
    from paper_2601_17136_amd import kkm
    x = torch.randn(3, 20, 90, device="cuda", generator=torch.Generator(device="cuda").manual_seed(9))
    x[0], x[1, 5:] = 0.0, 0.0
    y = torch.empty_like(x)
    kkm.kkm_orthogonalize(ctx, x, y, coef=[kkm.KKM_QUINTIC] * 32, eps=EPS)
    assert not y[0].any() and not y[1, 5:].any() and torch.isfinite(y).all()
    want = ref.exact(x[1].cpu(), [kkm.KKM_QUINTIC] * 32, EPS)
    assert ref.beyond(y[1].cpu(), want) <= 6 * 64 * 2.0 ** -39 * float(want.norm())
