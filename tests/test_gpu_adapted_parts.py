"""The bits that the adapted projection keeps of down x and up^T dy beside 16-bit matrices: sums that cancel all but
the last ones, exact in fp32."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
# Three numbers of one bit each, of which two parts of the type do not hold the sum: 8 bits a part of bfloat16, 11 of binary16.
BITS = {"f16": (1.0, 2.0 ** -12, 2.0 ** -23), "bf16": (1.0, 2.0 ** -9, 2.0 ** -20)}
S = 2.0 ** 10  # what the last bit is multiplied by, so that each type holds it


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.fail("GPU test on a machine without a GPU")
    from paper_2601_17136_amd import kkm
    c = kkm.kkm_create(kkm.current_stream_handle())
    yield c
    kkm.kkm_destroy(c)


def _zeros(dtype, *shape):
    return torch.zeros(*shape, device="cuda", dtype=dtype)


def _spread(bits, dtype):
    """(a, b), a . b = their sum, each entry a normal number of the type."""
    a, b = torch.ones(3, device="cuda"), torch.tensor(bits, device="cuda")
    a[2], b[2] = 2.0 ** -11, bits[2] * 2.0 ** 11
    return a.to(dtype), b.to(dtype)


SHAPES = [(300, 200, 256, 3, 2), (3000, 96, 1024, 5, 40), (8200, 64, 2048, 2, 17), (2100, 1000, 1040, 60, 128)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,d,m,s,r", SHAPES)
def test_second_products(ctx, n, d, m, s, r, dtype):
    """t = (1 + b + c, -(1 + b)) beside up = (S, S): S c is left; dx from u likewise."""
    from paper_2601_17136_amd import kkm
    t, bits = DTYPES[dtype], BITS[dtype]
    print(f"[gpu] second products n={n} d={d} m={m} adapters={s} rank={r} {dtype}", flush=True)
    a, b = _spread(bits, t)
    ids = (torch.arange(n, device="cuda") % (s + 1) - 1).int()
    want = torch.where(ids >= 0, S * bits[2], 0.0)[:, None]
    x, w = _zeros(t, n, d), _zeros(t, m, d)
    down, up, y = _zeros(t, s, r, d), _zeros(t, s, m, r), _zeros(t, n, m)
    x[:, :3], down[:, 0, :3], down[:, 1, :2] = a, b, -b[:2]
    up[:, :, :2] = S
    kkm.kkm_adapted_linear(ctx, x, w, down, up, ids, y)
    assert torch.equal(y.float(), want.expand(n, m))
    dy, dx = _zeros(t, n, m), _zeros(t, n, d)
    down, up = _zeros(t, s, r, d), _zeros(t, s, m, r)
    dy[:, :3], up[:, :3, 0], up[:, :2, 1] = a, b, -b[:2]
    down[:, :2] = S
    kkm.kkm_adapted_linear_grad(ctx, x, w, down, up, ids, dy, dx)
    assert torch.equal(dx.float(), want.expand(n, d))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,d,m,s,r", [(80, 40, 48, 2, 20), (3000, 96, 1024, 5, 40), (2400, 1000, 1040, 60, 128)])
def test_adapters_gradients(ctx, n, d, m, s, r, dtype):
    """Rows in pairs of coefficients 1 + b + c and -(1 + b): S c is left of each pair."""
    from paper_2601_17136_amd import kkm
    t, bits = DTYPES[dtype], BITS["bf16"]  # (two bfloat16 parts do not hold these)
    print(f"[gpu] adapters' gradients n={n} d={d} m={m} adapters={s} rank={r} {dtype}", flush=True)
    a, b = _spread(bits, t)
    n = n // (2 * s) * (2 * s)
    ids = (torch.arange(n, device="cuda") // 2 % s).int()
    want = n // (2 * s) * S * bits[2]
    w = _zeros(t, m, d)
    for side in ("ddown", "dup"):
        x, dy, down, up = _zeros(t, n, d), _zeros(t, n, m), _zeros(t, s, r, d), _zeros(t, s, m, r)
        rows = dy if side == "ddown" else x
        rows[::2, :3], rows[1::2, :2] = a, -a[:2]
        if side == "ddown":
            up[:, :3, r - 1] = b
            x[:] = S
        else:
            down[:, r - 1, :3] = b
            dy[:] = S
        out = torch.full_like(down if side == "ddown" else up, 7.0)
        kkm.kkm_adapted_linear_grad(ctx, x, w, down, up, ids, dy, **{side: out})
        mine = out[:, r - 1] if side == "ddown" else out[:, :, r - 1]
        assert bool((mine.float() == want).all()), (side, float(mine.float().min()), want)
        assert int((out != 0).sum()) == mine.numel()
