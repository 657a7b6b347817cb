"""The tiled orthogonalised update beside fp32 products of the same steps, in every type and in tiles of every shape."""
import pytest

import newton_parts as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-7


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.fail("GPU test on a machine without a GPU")
    from paper_2601_17136_amd import kkm
    c = kkm.kkm_create(kkm.current_stream_handle())
    yield c
    kkm.kkm_destroy(c)


def _near(got, u, coef):
    want = ref.exact(u, coef, EPS)
    off, room = ref.beyond(got, want), ref.room(u, want, coef, EPS)
    print(f"      {off / room:.2g} of the room", flush=True)
    assert off <= room, (off, room)


SHAPES = [(2, 65, 65), (3, 66, 130), (2, 130, 66), (1, 128, 128), (2, 129, 257), (2, 257, 65), (1, 300, 301), (1, 520, 700),
          (1, 1000, 65), (3, 777, 1001), (1, 1300, 1200), (1, 2050, 1700), (1, 2050, 4100), (1, 4100, 2050), (1, 600, 9000),
          (1, 4096, 4096)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("batch,m,n", SHAPES)
def test_map(ctx, batch, m, n, dtype):
    from paper_2601_17136_amd import kkm
    print(f"[gpu] orthogonalize {batch} x {m} x {n} {dtype}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(m * 7 + n)
    x = torch.randn(batch, m, n, device="cuda", generator=g).to(DTYPES[dtype])
    y = torch.empty_like(x)
    kkm.kkm_orthogonalize(ctx, x, y, eps=EPS)
    for i in range(batch):
        _near(y[i], x[i], [kkm.KKM_QUINTIC] * 5)


@pytest.mark.parametrize("coef", ["cubic", "mixed"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n", [(90, 70), (300, 500), (1100, 900)])
def test_other_steps(ctx, m, n, dtype, coef):
    from paper_2601_17136_amd import kkm
    steps = {"cubic": [kkm.KKM_CUBIC] * 12,
             "mixed": [(3.0, -3.2, 1.2), kkm.KKM_CUBIC, (0.5, 0.25, 0.0), (-1.0, 0.5, -0.125)]}[coef]
    x = torch.randn(m, n, device="cuda", generator=torch.Generator(device="cuda").manual_seed(m)).to(DTYPES[dtype])
    y = torch.empty_like(x)
    kkm.kkm_orthogonalize(ctx, x, y, coef=steps, eps=EPS)
    _near(y, x, steps)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n", [(65, 90), (300, 200), (129, 640), (1000, 1500)])
def test_step(ctx, m, n, dtype):
    """w = 0 w - X: the update alone."""
    from paper_2601_17136_amd import kkm
    g, t = torch.Generator(device="cuda").manual_seed(m + 3 * n), DTYPES[dtype]
    w, grad = (torch.randn(m, n, device="cuda", generator=g).to(t) for _ in range(2))
    v = torch.randn(m, n, device="cuda", generator=g)
    kkm.kkm_orthogonal_step(ctx, w, grad, v, 1.0, momentum=0.5, keep=0.0, eps=EPS)
    _near(-w, grad.double() + 0.5 * v.double(), [kkm.KKM_QUINTIC] * 5)
