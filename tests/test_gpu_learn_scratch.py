"""Contexts whose budget is what include/kkm.h says that a call's scratch takes."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
MB = 1 << 20


def _up(v, to):
    return -(-v // to) * to


def _within(budget, call):
    from paper_2601_17136_amd import kkm
    if not torch.cuda.is_available():
        pytest.fail("GPU test on a machine without a GPU")
    c = kkm.kkm_create(kkm.current_stream_handle(), budget)
    try:
        call(kkm, c)
        torch.cuda.synchronize()
    finally:
        kkm.kkm_destroy(c)


@pytest.mark.parametrize("batch,m,n,steps", [(1, 65, 65, 5), (1, 100, 100, 5), (3, 777, 1001, 5), (1, 65, 3000, 5), (1, 3000, 3000, 5),
                                             (1, 4352, 4352, 5), (1, 4097, 4097, 5), (300, 400, 400, 5), (1, 64, 64, 5),
                                             (1, 5, 100000, 5), (1, 200000, 64, 12), (900, 60, 700, 12)])
def test_updates(batch, m, n, steps):
    if min(m, n) > 64:
        one = 24 * _up(m, 32) * _up(n, 32)
        budget = one * max(1, min(batch, (1 << 30) // one)) + (32 * MB if batch == 1 else 0) + MB
    else:
        budget = max(256 * MB if batch > 1 else 0, 3 * MB + (8 * m * n if steps > 6 else 0))
    x = torch.randn(batch, m, n, device="cuda").bfloat16()
    y = torch.zeros_like(x)
    print(f"[gpu] {batch} x {m} x {n}: {budget} bytes", flush=True)
    _within(budget, lambda kkm, c: kkm.kkm_orthogonalize(c, x, y, coef=[kkm.KKM_QUINTIC] * steps))
    assert y.any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("n,d,m,s,r", [(1, 20, 30, 1, 1), (64, 300, 200, 5, 7), (300, 1001, 777, 1024, 3), (5001, 1001, 777, 5, 12),
                                       (20000, 784, 1024, 8, 8), (2049, 4100, 1000, 40, 100), (300000, 20, 40, 1000, 16)])
def test_adapted(n, d, m, s, r, dtype):
    size = 4 if dtype == torch.float32 else 2
    pad = 32 if size == 4 else 8
    R = next(v for v in (16, 32, 64, 128) if r <= v)
    low = s * r * (d + m)
    forward = 16 * n + 4 * n * R + MB + (n + m) * (_up(d, pad) * size + 4)
    pieces = min(1024, -(-n // 64)) + min(s, n)
    grad = (16 * n + 8 * n * R + MB + size * (d * _up(m, 8) + low) + (n + d) * (_up(m, pad) * size + 4)
            + 4 * pieces * r * (d + m))

    def normal(*shape):
        return (torch.randn(*shape, device="cuda") * 0.1).to(dtype)

    x, w, down, up, dy = normal(n, d + 1)[:, 1:], normal(m, d + 1)[:, 1:], normal(s, r, d), normal(s, m, r), normal(n, m + 1)[:, 1:]
    ids = torch.randint(-1, s, (n,), device="cuda").int()
    y, dx, ddown, dup = normal(n, m).zero_(), normal(n, d).zero_(), torch.zeros_like(down), torch.zeros_like(up)
    print(f"[gpu] {n} x {d} to {m}, {s} of {r} {dtype}: {forward} and {grad} bytes", flush=True)
    _within(forward, lambda kkm, c: kkm.kkm_adapted_linear(c, x, w, down, up, ids, y))
    _within(grad, lambda kkm, c: kkm.kkm_adapted_linear_grad(c, x, w, down, up, ids, dy, dx, ddown, dup))
    assert y.any() and dx.any()


@pytest.mark.parametrize("n,V", [(3, 4096), (1, 32768), (100, 70001)])
def test_answers(n, V):
    z, ids = torch.randn(n, V, device="cuda"), torch.empty(n, dtype=torch.int32, device="cuda")
    _within(max(256, 16 * n * -(-V // 4096)), lambda kkm, c: kkm.kkm_choose(c, z, ids=ids))
    assert torch.equal(ids.long(), z.argmax(1))
