"""The adapted projection and its gradient against the formulas in 64 bits, at the sizes, strides and ids where
they can go wrong."""
import pytest

import learn_reference as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
NAN = float("nan")


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.fail("GPU test on a machine without a GPU")
    from paper_2601_17136_amd import kkm
    c = kkm.kkm_create(kkm.current_stream_handle())
    yield c
    kkm.kkm_destroy(c)


def _case(n, d, m, s, r, dtype, seed, pad=0, drop=0.2):
    t, g = DTYPES[dtype], torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=g)

    x, dy = ref.rows(n, d, t, pad, normal(n, d)), ref.rows(n, m, t, (pad + 1) % 4, normal(n, m) / n ** 0.5)
    w = ref.rows(m, d, t, (pad + 2) % 5, normal(m, d) / d ** 0.5)
    down, up = (normal(s, r, d) / d ** 0.5).to(t), (normal(s, m, r) / r ** 0.5).to(t)
    ids = torch.randint(0, s, (n,), device="cuda", generator=g)
    ids = torch.where(torch.rand(n, device="cuda", generator=g) < drop, -3, ids).int()
    return x, w, down, up, ids, 0.5 + torch.rand(s, device="cuda", generator=g), dy


def _outputs(x, w, down, up, pad=0):
    n, d = x.shape
    m = w.shape[0]
    return (ref.rows(n, m, x.dtype, pad, torch.zeros(n, m, device="cuda")),
            ref.rows(n, d, x.dtype, (pad + 3) % 4, torch.zeros(n, d, device="cuda")),
            torch.full_like(down, 9.0), torch.full_like(up, 9.0))


def _run(ctx, x, w, down, up, ids, f, dy, pad=0):
    from paper_2601_17136_amd import kkm
    y, dx, ddown, dup = _outputs(x, w, down, up, pad)
    kkm.kkm_adapted_linear(ctx, x, w, down, up, ids, y, factor=f)
    kkm.kkm_adapted_linear_grad(ctx, x, w, down, up, ids, dy, dx, ddown, dup, factor=f)
    return {"y": y, "dx": dx, "ddown": ddown, "dup": dup}


def _check(case, got):
    want, tol = ref.adapted(*case)
    worst = [ref.check(k, got[k], want[k], tol[k]) for k in want]
    print(f"      of the bounds: {', '.join(f'{v:.2g}' for v in worst)}", flush=True)


# rows, width, columns, adapters, rank
DIRECT = [(1, 1, 1, 1, 1), (1, 784, 64, 8, 8), (1, 1001, 333, 3, 16), (1, 70, 40, 2, 17), (5, 7, 3, 2, 1), (3, 100, 1000, 40, 17), (16, 33, 65, 5, 16), (17, 64, 16, 1, 5),
          (31, 300, 130, 31, 33), (33, 54, 7, 2, 3), (64, 256, 300, 9, 64), (65, 65, 65, 3, 2), (100, 784, 10, 4, 8),
          (257, 48, 200, 1, 100), (1000, 130, 64, 7, 128), (3000, 16, 17, 20, 4), (700, 301, 129, 90, 12),
          (40, 2000, 2100, 3, 8), (2500, 40, 30, 1024, 2)]
TILED = [(1500, 2100, 1030, 4, 8), (300, 4096, 2050, 60, 16), (4100, 700, 801, 9, 33), (4096, 304, 2048, 3, 64),
         (2049, 1000, 1111, 300, 5), (8200, 520, 600, 2, 128), (5001, 1001, 777, 5, 12)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,d,m,s,r", DIRECT + TILED)
def test_adapted(ctx, n, d, m, s, r, dtype):
    pad = (n + d + m) % 4
    print(f"[gpu] adapted n={n} d={d} m={m} adapters={s} rank={r} {dtype} pad={pad}", flush=True)
    case = _case(n, d, m, s, r, dtype, n * 131 + d + m, pad)
    got = _run(ctx, *case, pad=pad)
    _check(case, got)
    again = _run(ctx, *case)  # the same bits
    assert all(torch.equal(got[k], again[k]) for k in got)


@pytest.mark.parametrize("n,d,m", [(50, 64, 72), (300, 96, 50), (2100, 1000, 1040)])
def test_parts_of_the_gradient(ctx, n, d, m):
    """Each output alone has the bits it has beside the others."""
    from paper_2601_17136_amd import kkm
    case = x, w, down, up, ids, f, dy = _case(n, d, m, 3, 10, "bf16", 5)
    got = _run(ctx, *case)
    for k in ("dx", "ddown", "dup"):
        one = {k: torch.full_like(got[k], 3.0)}
        kkm.kkm_adapted_linear_grad(ctx, x, w, down, up, ids, dy, factor=f, **one)
        assert torch.equal(one[k], got[k]), k
    kkm.kkm_adapted_linear_grad(ctx, x, w, down, up, ids, dy, factor=f)  # nothing asked for


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,d,m", [(40, 64, 72), (300, 96, 50), (2100, 1000, 1040)])
def test_ids_that_are_none_and_adapters_of_nan(ctx, n, d, m, dtype):
    """Rows without an adapter, of an id past the last, adapters without rows, and one of NaN."""
    x, w, down, up, ids, f, dy = _case(n, d, m, 6, 9, dtype, 7)
    ids = torch.randint(-1, 3, (n,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).int()
    ids[::7] = 5
    ids[3], ids[n - 1], ids[n // 2] = 6, 2 ** 31 - 1, -2 ** 31
    down[4:], up[4:], f[4:] = NAN, NAN, NAN  # 4 has no rows
    case = (x, w, down, up, ids, f, dy)
    got = _run(ctx, *case)
    mine = ids == 5
    assert torch.isnan(got["y"][mine]).all() and torch.isnan(got["dx"][mine]).all()
    assert torch.isnan(got["ddown"][5]).all() and torch.isnan(got["dup"][5]).all()
    assert not got["ddown"][3:5].any() and not got["dup"][3:5].any()
    want, tol = ref.adapted(*case)
    for k in ("y", "dx"):
        ref.check(k, got[k][~mine], want[k][~mine], tol[k][~mine])
    for k in ("ddown", "dup"):
        ref.check(k, got[k][:3], want[k][:3], tol[k][:3])
    # a row of NaN stays its own, and spoils its adapter's gradients alone
    ids[::7] = 0
    down[4:], up[4:], f[4:] = 0.0, 0.0, 1.0
    row = int(torch.nonzero(ids == 1)[2])
    x[row], dy[row] = NAN, NAN
    got = _run(ctx, x, w, down, up, ids, f, dy)
    assert torch.isnan(got["y"]).all(1).sum() == 3 and torch.isnan(got["y"][row]).all()
    assert torch.isnan(got["dx"]).all(1).sum() == 3 and torch.isnan(got["dx"][row]).all()
    for k in ("ddown", "dup"):
        assert torch.isnan(got[k][1]).all() and not torch.isnan(got[k][[0, 2, 3, 4, 5]]).any()


def test_no_rows_and_no_factor(ctx):
    case = _case(0, 30, 20, 4, 5, "f32", 3)
    got = _run(ctx, *case)
    assert not got["ddown"].any() and not got["dup"].any()
    case = list(_case(90, 30, 20, 4, 5, "f32", 4))
    case[5] = None
    _check(case, _run(ctx, *case))


@pytest.mark.parametrize("dtype", DTYPES)
def test_one_row_of_each_id(ctx, dtype):
    """A row by itself: of each adapter, of none, and of an id past the last, NaN in the other adapters."""
    from paper_2601_17136_amd import kkm
    x, w, down, up, _, f, dy = _case(1, 130, 50, 4, 7, dtype, 21)
    for g in (-1, 0, 3, 4, 2 ** 31 - 1, -2 ** 31):
        ids = torch.tensor([g], dtype=torch.int32, device="cuda")
        d2, u2, f2 = (torch.full_like(t, NAN) for t in (down, up, f))
        if 0 <= g < 4:
            d2[g], u2[g], f2[g] = down[g], up[g], f[g]
        y = torch.empty(1, 50, device="cuda", dtype=x.dtype)
        kkm.kkm_adapted_linear(ctx, x, w, d2, u2, ids, y, factor=f2)
        want, tol = ref.adapted(x, w, down, up, ids, f, dy)
        ref.check("y", y, want["y"], tol["y"])


def test_all_rows_without_an_adapter(ctx):
    for n, d, m in ((30, 40, 50), (2100, 1000, 1040)):
        case = list(_case(n, d, m, 4, 5, "bf16", 4, drop=2.0))
        got = _run(ctx, *case)
        _check(case, got)
        assert not got["ddown"].any() and not got["dup"].any()


def test_rows_far_apart(ctx):
    """Rows whose offsets pass 32 bits, of the direct form and of the tiles."""
    from paper_2601_17136_amd import kkm
    for n, d, m in ((70, 64, 72), (2200, 1000, 1000)):
        x, w, down, up, ids, f, dy = _case(n, d, m, 3, 8, "bf16", 9)
        ld = (1 << 32) // (2 * n) // 8 * 8 + 8 * d
        far = torch.empty(n * ld, device="cuda", dtype=torch.bfloat16).as_strided((n, d), (ld, 1))
        far.copy_(x)
        y, y2 = torch.empty(n, m, device="cuda", dtype=torch.bfloat16), torch.empty(n, m, device="cuda", dtype=torch.bfloat16)
        kkm.kkm_adapted_linear(ctx, x, w, down, up, ids, y, factor=f)
        kkm.kkm_adapted_linear(ctx, far, w, down, up, ids, y2, factor=f)
        assert torch.equal(y, y2)
        a, b = torch.empty_like(down), torch.empty_like(down)
        kkm.kkm_adapted_linear_grad(ctx, x, w, down, up, ids, dy, ddown=a, factor=f)
        kkm.kkm_adapted_linear_grad(ctx, far, w, down, up, ids, dy, ddown=b, factor=f)
        assert torch.equal(a, b)


@pytest.mark.parametrize("s", [1, 1000])
def test_two_million_rows(ctx, s):
    """The largest n: the rows' order by many workgroups."""
    from paper_2601_17136_amd import kkm
    n, d, m, r = 1 << 21, 16, 24, 2
    x, w, down, up, ids, f, dy = _case(n, d, m, s, r, "f16", 13)
    y, ddown = torch.empty(n, m, device="cuda", dtype=torch.float16), torch.empty_like(down)
    kkm.kkm_adapted_linear(ctx, x, w, down, up, ids, y, factor=f)
    kkm.kkm_adapted_linear_grad(ctx, x, w, down, up, ids, dy, ddown=ddown, factor=f)
    at = ids.clamp(min=0).long()
    on = (ids >= 0).double()[:, None]
    xd, wd = x.double(), w.double()
    t = torch.stack([(xd * down[at, k].double()).sum(1) for k in range(r)], 1) * f[at].double()[:, None] * on
    want, size = xd @ wd.t(), xd.abs() @ wd.abs().t()
    for k in range(r):
        want += t[:, k:k + 1] * up[at, :, k].double()
        size += t[:, k:k + 1].abs() * up[at, :, k].double().abs()
    off = (y.double() - want).abs()
    assert bool((off <= want.abs() * (2.0 ** -11 + 4 * ref.U) + 64 * ref.U * size + 2.0 ** -20 * size + 2.0 ** -24).all())
    u = torch.stack([(dy.double() * up[at, :, k].double()).sum(1) for k in range(r)], 1) * f[at].double()[:, None] * on
    for k in range(r):
        sums = torch.zeros(s, d, dtype=torch.float64, device="cuda").index_add_(0, at, u[:, k:k + 1] * xd)
        sizes = torch.zeros(s, d, dtype=torch.float64, device="cuda").index_add_(0, at, (u[:, k:k + 1] * xd).abs())
        rows = n / s / 4 + 2000
        off = (ddown[:, k].double() - sums).abs()
        assert bool((off <= sums.abs() * 2.0 ** -11 + (rows * 2 * ref.U + 2.0 ** -16) * sizes + 2.0 ** -24).all())


def test_gradient_against_differences(ctx):
    """<dy, y(p + h q) - y(p - h q)> = 2 h <dp, q>, exact but for roundings: y is linear in each of x, down and up."""
    from paper_2601_17136_amd import kkm
    x, w, down, up, ids, f, dy = _case(120, 70, 90, 5, 6, "f32", 11)
    got = _run(ctx, x, w, down, up, ids, f, dy)
    g = torch.Generator(device="cuda").manual_seed(2)
    for k, name in ((0, "dx"), (2, "ddown"), (3, "dup")):
        p = [x.contiguous(), w, down, up]
        q = torch.randn(p[k].shape, device="cuda", generator=g)
        ends = []
        for h in (0.5, -0.5):
            moved = list(p)
            moved[k] = p[k] + h * q
            y = torch.empty(120, 90, device="cuda")
            kkm.kkm_adapted_linear(ctx, moved[0], moved[1], moved[2], moved[3], ids, y, factor=f)
            ends.append(y.double())
        slope = float(((ends[0] - ends[1]) * dy.double()).sum())
        size = float(((ends[0].abs() + ends[1].abs()) * dy.double().abs()).sum())
        want = float((got[name].double() * q.double()).sum())
        # y of about 70 + 6 terms and the gradient of 120: each entry's roundings, by the sizes that enter
        room = 400 * ref.U * (size + float((got[name].double().abs() * q.double().abs()).sum()))
        assert abs(slope - want) <= room, (name, slope, want, room)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,r", [(1, 1), (1, 20), (9, 1), (9, 3), (90, 3)])
def test_an_infinite_factor(ctx, n, r, dtype):
    """Rows straight from memory: f down x is infinite, of one sign in all of the rank, and
    so is the row's y; another adapter's rows are as they were."""
    from paper_2601_17136_amd import kkm
    d, m, dtype = 24, 10, DTYPES[dtype]
    x = torch.ones(n, d, device="cuda", dtype=dtype)
    w = torch.ones(m, d, device="cuda", dtype=dtype)
    down, up = torch.ones(2, r, d, device="cuda", dtype=dtype), torch.ones(2, m, r, device="cuda", dtype=dtype)
    up[:, 1::2] = -1
    f = torch.tensor([float("inf"), 0.5], device="cuda")
    ids = (torch.arange(n, device="cuda") % 2).to(torch.int32)
    y = torch.zeros(n, m, device="cuda", dtype=dtype)
    kkm.kkm_adapted_linear(ctx, x, w, down, up, ids, y, factor=f)
    sign = up[0, :, 0].float()
    want = torch.where(ids[:, None] == 0, sign * float("inf"), d + 0.5 * r * d * sign)
    assert torch.equal(y.float(), want.expand(n, m))  # (small whole numbers and halves: exact in each type)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,d,m,s,r", [(200, 700, 130, 190, 64), (70, 900, 300, 66, 128), (130, 1000, 90, 130, 17),
                                       (97, 1300, 70, 1000, 33), (600, 3000, 2000, 300, 48)])
def test_many_adapters_in_a_tile(ctx, n, d, m, s, r, dtype):
    """Runs of one to three rows in tiles, ranks of two to eight steps, rows without an adapter and of none of them."""
    x, w, down, up, ids, f, dy = _case(n, d, m, s, r, dtype, n + m, drop=0.1)
    ids[5], ids[n - 1] = s, s + 7
    case = (x, w, down, up, ids, f, dy)
    got = _run(ctx, *case)
    lost = ids >= s
    assert torch.isnan(got["y"][lost]).all() and torch.isnan(got["dx"][lost]).all()
    want, tol = ref.adapted(*case)
    for k in ("y", "dx"):
        ref.check(k, got[k][~lost], want[k][~lost], tol[k][~lost])
    for k in ("ddown", "dup"):
        ref.check(k, got[k], want[k], tol[k])
