"""Results on top of inputs that are still read when they are written: refused, with everything left as it was."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.fail("GPU test on a machine without a GPU")
    from paper_2601_17136_amd import kkm
    c = kkm.kkm_create(kkm.current_stream_handle())
    yield c
    kkm.kkm_destroy(c)


def _refused(call, tensors):
    from paper_2601_17136_amd import kkm
    was = [t.clone() for t in tensors]
    with pytest.raises(kkm.KKMError) as e:
        call()
    assert e.value.code == kkm.KKM_ERR_ARG
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(tensors, was))


@pytest.mark.parametrize("n,d", [(1, 16), (10, 16), (400, 100)])
def test_adapted(ctx, n, d):
    from paper_2601_17136_amd import kkm

    def normal(*shape):
        return torch.randn(*shape, device="cuda")

    x, w, down, up, dy = normal(n, d), normal(d, d), normal(3, d, d), normal(3, d, d), normal(n, d)
    ids = torch.zeros(n, dtype=torch.int32, device="cuda")
    every = (x, w, down, up, dy)
    for y in (x, w[:n] if n <= d else None, down[0][:n] if n <= d else None, up[0][:n] if n <= d else None):
        if y is not None:
            _refused(lambda: kkm.kkm_adapted_linear(ctx, x, w, down, up, ids, y), every)
    for kw in (dict(dx=x), dict(dx=dy), dict(ddown=down), dict(ddown=up), dict(dup=down), dict(dup=up)):
        _refused(lambda: kkm.kkm_adapted_linear_grad(ctx, x, w, down, up, ids, dy, **kw), every)
    one = normal(3, d, d)
    _refused(lambda: kkm.kkm_adapted_linear_grad(ctx, x, w, down, up, ids, dy, ddown=one, dup=one), (*every, one))
    if n <= d:
        _refused(lambda: kkm.kkm_adapted_linear_grad(ctx, x, w, down, up, ids, dy, dx=one[0][:n], ddown=one), (*every, one))
    # columns of one table, side by side, are apart
    table = torch.zeros(n, 2 * d, device="cuda")
    table[:, :d] = x
    y = torch.empty(n, d, device="cuda")
    kkm.kkm_adapted_linear(ctx, x, w, down, up, ids, y)
    kkm.kkm_adapted_linear(ctx, table[:, :d], w, down, up, ids, table[:, d:])
    assert torch.equal(table[:, d:], y) and torch.equal(table[:, :d], x)


@pytest.mark.parametrize("m,n", [(8, 100), (80, 100)])
def test_momentum(ctx, m, n):
    from paper_2601_17136_amd import kkm
    w, g = torch.randn(m, n, device="cuda"), torch.randn(m, n, device="cuda")
    _refused(lambda: kkm.kkm_orthogonal_step(ctx, w, g, g, 0.1), (w, g))
    _refused(lambda: kkm.kkm_orthogonal_step(ctx, w, g, w, 0.1), (w, g))
