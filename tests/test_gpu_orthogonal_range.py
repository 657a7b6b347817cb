"""Rows, columns and whole matrices far below the rest, in the tiled orthogonalised update."""
import pytest

import newton_parts as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.fail("GPU test on a machine without a GPU")
    from paper_2601_17136_amd import kkm
    c = kkm.kkm_create(kkm.current_stream_handle())
    yield c
    kkm.kkm_destroy(c)


def _run(ctx, x, eps):
    from paper_2601_17136_amd import kkm
    y = torch.empty_like(x)
    kkm.kkm_orthogonalize(ctx, x, y, eps=eps)
    coef = [kkm.KKM_QUINTIC] * 5
    # A stored entry of X is at most 2^-50 of the bound on X's singular values off, whatever its own size, and the steps
    # carry that on by 3.4445 each; the operands of later steps add a geometric series' rest, a half of it, and B its own.
    floor = 3 * 3.4445 ** 5 * 2.0 ** -50
    return y, ref.exact(x, coef, eps), ref.fp32(x, coef, eps), floor


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("scale", [1e-3, 1e-5, 1e-7])
@pytest.mark.parametrize("m,n", [(256, 400), (400, 256), (130, 90), (1000, 1100)])
def test_small_rows_and_columns(ctx, m, n, scale, dtype):
    for side in (0, 1):
        x = torch.randn(m, n, device="cuda", generator=torch.Generator(device="cuda").manual_seed(m))
        part = (slice(None, None, 2), slice(None)) if side == 0 else (slice(None), slice(None, None, 2))
        x[part] *= scale
        x = x.to(DTYPES[dtype])
        y, want, plain, floor = _run(ctx, x, 1e-7)
        own = want[part]
        room = 2 * float((plain[part] - own).norm()) + 4 * ref.U * float(own.norm()) + floor * own.numel() ** 0.5
        off = ref.beyond(y[part], own)
        print(f"[gpu] {m} x {n} {dtype} {scale} of side {side}: {off / room:.2g} of the room", flush=True)
        assert off <= room
        assert room < 1e-4 * float(own.norm())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("norm", [1e-9, 1e-11, 1e-13])
@pytest.mark.parametrize("m,n", [(256, 400), (400, 256), (130, 90)])
def test_a_norm_far_below_eps(ctx, m, n, norm, dtype):
    x = torch.randn(m, n, device="cuda", generator=torch.Generator(device="cuda").manual_seed(n))
    x = (x * (norm / x.norm())).to(DTYPES[dtype])
    y, want, plain, floor = _run(ctx, x, 1e-7)
    room = 2 * float((plain - want).norm()) + 4 * ref.U * float(want.norm()) + floor * want.numel() ** 0.5
    off = ref.beyond(y, want)
    print(f"[gpu] {m} x {n} {dtype} norm {norm}: {off / room:.2g} of the room", flush=True)
    assert off <= room
    assert room < 1e-4 * float(want.norm())
