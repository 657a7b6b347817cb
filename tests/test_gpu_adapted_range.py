"""The tiled fp32 projection: rows of every size, entries of one row of very different sizes, zeros, infinities and NaN.

An entry is two binary16 parts at a power of two of its row: at most 2^-22 of itself off, or 2^-50 of the row's largest,
and a product without lo lo 2^-22 more.  The sums are fp32 on the matrix cores, 2 U at each instruction of 16 terms."""
import pytest

import learn_reference as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
U = ref.U


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.fail("GPU test on a machine without a GPU")
    from paper_2601_17136_amd import kkm
    c = kkm.kkm_create(kkm.current_stream_handle())
    yield c
    kkm.kkm_destroy(c)


def _project(x, w, down, up, ids):
    """y = x w^T + up down x in 64 bits, and the bound of the kernel's error."""
    x, w, down, up = (v.double() for v in (x, w, down, up))
    d, s = x.shape[1], down.shape[0]
    y, size = x @ w.t(), x.abs() @ w.abs().t()
    rows, cols = x.abs(), w.abs()
    tol = (3 * 2.0 ** -22 + (2 * (d / 16 + 4) + 8) * 2 * U) * size + 1.01 * 2.0 ** -50 * (
        rows.amax(1)[:, None] * cols.sum(1)[None, :] + rows.sum(1)[:, None] * cols.amax(1)[None, :])
    for g in range(s):
        i = torch.nonzero(ids == g)[:, 0]
        t = x[i] @ down[g].t()
        dt = (2 * (d / 4 + 4) + 8) * 2 * U * (rows[i] @ down[g].abs().t())  # fp32 sums, 4 terms an instruction
        y[i] += t @ up[g].t()
        tol[i] += (dt + (down.shape[1] + 8) * 2 * U * t.abs()) @ up[g].abs().t()
    return y, tol + 5 * U * y.abs()


def _both(ctx, x, w, down, up, ids):
    """y of x, and the same from the gradient: dx of dy = x with w and the adapters turned."""
    from paper_2601_17136_amd import kkm
    y, dx, none = (torch.zeros(x.shape[0], w.shape[0], device="cuda") for _ in range(3))
    kkm.kkm_adapted_linear(ctx, x, w, down, up, ids, y)
    kkm.kkm_adapted_linear_grad(ctx, none, w.t().contiguous(), up.transpose(1, 2).contiguous(),
                                down.transpose(1, 2).contiguous(), ids, x, dx)
    return {"y": y, "dx": dx}


SHAPES = [(1500, 2100, 1030, 4, 8), (300, 4096, 2050, 60, 16), (2049, 200, 901, 3, 33), (20000, 784, 1024, 8, 8),
          (130, 1000, 90, 130, 17)]


def _case(n, d, m, s, r):
    g = torch.Generator(device="cuda").manual_seed(n + d)

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=g)

    ids = torch.randint(-1, s, (n,), device="cuda", generator=g).int()
    return normal(n, d), normal(m, d) / d ** 0.5, normal(s, r, d) / d ** 0.5, normal(s, m, r) / r ** 0.5, ids


@pytest.mark.parametrize("n,d,m,s,r", SHAPES)
def test_rows_of_every_size(ctx, n, d, m, s, r):
    x, w, down, up, ids = _case(n, d, m, s, r)
    x *= torch.exp2((torch.arange(n, device="cuda") * 37 % 161 - 100).float())[:, None]
    cols = torch.exp2((torch.arange(m, device="cuda") * 29 % 61 - 20).float())
    w, up = w * cols[:, None], up * cols[None, :, None]
    x[5], w[7], up[:, 7] = 0.0, 0.0, 0.0
    print(f"[gpu] rows of every size n={n} d={d} m={m}", flush=True)
    want, tol = _project(x, w, down, up, ids)
    for k, got in _both(ctx, x, w, down, up, ids).items():
        worst = ref.check(k, got, want, tol)
        print(f"      {k} {worst:.2g} of the bound", flush=True)
        assert not got[5].any() and not got[:, 7].any()


@pytest.mark.parametrize("n,d,m,s,r", SHAPES)
def test_features_of_every_size(ctx, n, d, m, s, r):
    """Features down to 2^-26 of the largest, whose weights make up for it."""
    x, w, down, up, ids = _case(n, d, m, s, r)
    size = torch.exp2(-(torch.arange(d, device="cuda") * 11 % 27).float())
    x, w, down = x * size, w / size, down / size
    print(f"[gpu] features of every size n={n} d={d} m={m}", flush=True)
    want, tol = _project(x, w, down, up, ids)
    for k, got in _both(ctx, x, w, down, up, ids).items():
        print(f"      {k} {ref.check(k, got, want, tol):.2g} of the bound", flush=True)


@pytest.mark.parametrize("n,d,m,s,r", SHAPES)
def test_infinities_and_nan_stay_in_their_rows(ctx, n, d, m, s, r):
    x, w, down, up, ids = _case(n, d, m, s, r)
    want, tol = _project(x, w, down, up, ids)
    x[3, 1], x[n - 1, d - 1], w[m - 1, 0] = float("inf"), float("nan"), float("-inf")
    lost = torch.zeros_like(want, dtype=torch.bool)
    lost[3], lost[n - 1], lost[:, m - 1] = True, True, True
    for k, got in _both(ctx, x, w, down, up, ids).items():
        assert torch.isnan(got[lost]).all()  # (an infinite entry has no parts)
        ref.check(k, got[~lost], want[~lost], tol[~lost])


@pytest.mark.parametrize("n,d,m,s,r", SHAPES + [(2100, 4096, 1024, 2, 4)])
def test_beside_fp32_products(ctx, n, d, m, s, r):
    """No further from 64 bits than twice a library's fp32 product, which a product of one part each is not."""
    x, w, down, up, ids = _case(n, d, m, s, r)
    ids.fill_(-1)
    want = x.double() @ w.double().t()
    room = 2 * float(((x @ w.t()).double() - want).norm()) + 2 * U * float(want.norm())
    one = x.half().double() @ w.half().double().t()
    assert float((one - want).norm()) > 4 * room
    for k, got in _both(ctx, x, w, down, up, ids).items():
        off = float((got.double() - want).norm())
        print(f"[gpu] {k} n={n} d={d} m={m}: {off / room:.2g} of the room", flush=True)
        assert off <= room
