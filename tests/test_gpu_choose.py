"""Answers from logits against the stated operations, at the sizes, lists and masks where they can go wrong."""
import pytest

import learn_reference as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
INF = float("inf")


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.fail("GPU test on a machine without a GPU")
    from paper_2601_17136_amd import kkm
    c = kkm.kkm_create(kkm.current_stream_handle())
    yield c
    kkm.kkm_destroy(c)


def _same(a, b):
    return torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(torch.nan_to_num(a), torch.nan_to_num(b))


def _run(ctx, z, pad=0, out=True, **kw):
    from paper_2601_17136_amd import kkm
    n, V = z.shape
    o = ref.rows(n, V, z.dtype, pad, torch.zeros(n, V, device="cuda")) if out else None
    ids = torch.full((n,), 77, dtype=torch.int32, device="cuda")
    logp, lse = torch.full((n,), 7.0, device="cuda"), torch.full((n,), 7.0, device="cuda")
    kkm.kkm_choose(ctx, z, o, ids, logp, lse, **kw)
    return o, ids, logp, lse


def _check(z, got, kw):
    out, ids, logp, lse = got
    u, want, wlogp, wlse, tol_p, tol_l = ref.choose(z, kw.get("scale", 1.0), **{k: v for k, v in kw.items() if k != "scale"})
    if out is not None:
        assert _same(out.cpu().float(), u.to(z.dtype).float())
    assert torch.equal(ids.cpu(), want)
    for name, g, w, tol in (("logp", logp, wlogp, tol_p), ("lse", lse, wlse, tol_l)):
        g = g.cpu().double()
        assert torch.equal(torch.isnan(g), torch.isnan(w)), name
        fine = torch.isfinite(w)
        assert torch.equal(g[~fine & ~torch.isnan(w)], w[~fine & ~torch.isnan(w)]), name
        off = (g - w).abs()[fine]
        assert bool((off <= tol[fine]).all()), (name, float((off / tol[fine]).max()))


def _lists(n, V, given, biases, masks, g):
    kw = {}
    if given:
        ids = (V * torch.rand(n, given, device="cuda", generator=g) ** 2).int()
        drop = torch.rand(n, given, device="cuda", generator=g)
        ids = torch.where(drop < 0.2, -1, torch.where(drop > 0.95, V + 3, ids))
        kw.update(given=ids.int(), repeat=1.3, presence=0.4, frequency=0.3)
    if biases:
        ids = torch.randint(-2, V + 1, (n, biases), device="cuda", generator=g)
        kw.update(bias_ids=ids.int(), bias=torch.randn(n, biases, device="cuda", generator=g))
    if masks:
        words = (V + 31) // 32 + 1
        m = torch.randint(-2 ** 31, 2 ** 31, (masks, words), device="cuda", generator=g).int()
        m[0] = 0
        kw.update(masks=m, mask_ids=torch.randint(-1, masks, (n,), device="cuda", generator=g).int())
    return kw


SIZES = [(1, 1), (1, 7), (3, 15), (17, 16), (5, 33), (33, 64), (7, 255), (20, 256), (6, 257), (5, 1000), (4, 1024),
         (3, 1025), (3, 4096), (5, 4097), (2, 8199), (1, 32768), (2, 70001)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,V", SIZES)
def test_choose(ctx, n, V, dtype):
    g = torch.Generator(device="cuda").manual_seed(n * 131 + V)
    pad = (n + V) % 4
    print(f"[gpu] choose n={n} V={V} {dtype} pad={pad}", flush=True)
    z = ref.rows(n, V, DTYPES[dtype], pad, 3 * torch.randn(n, V, device="cuda", generator=g))
    offset = torch.randn(V, device="cuda", generator=g)
    offset[torch.rand(V, device="cuda", generator=g) < 0.1] = -INF
    for k, (given, biases, masks) in enumerate([(0, 0, 0), (9, 0, 0), (0, 5, 0), (0, 0, 3), (70, 300, 4)]):
        kw = _lists(n, V, given, biases, masks, g)
        if k % 2:
            kw["offset"] = offset
        kw["scale"] = 0.7
        got = _run(ctx, z, (pad + 1) % 3, **kw)
        _check(z, got, kw)
        again = _run(ctx, z, out=False, **kw)  # the same bits without the logits
        assert torch.equal(again[1], got[1]) and _same(again[2], got[2]) and _same(again[3], got[3])


def test_ties_go_to_the_lowest_id(ctx):
    for V in (40, 700, 9000):
        z = torch.zeros(3, V, device="cuda")
        z[1, V - 1] = z[1, V // 2] = 2.0
        z[2, :V // 2] = -1.0
        got = _run(ctx, z)
        assert got[1].tolist() == [0, V // 2, V // 2]
        _check(z, got, {})


def test_rows_with_nothing_left_infinities_and_nan(ctx):
    for V in (33, 600, 5000):
        z = torch.randn(9, V, device="cuda", generator=torch.Generator(device="cuda").manual_seed(V))
        masks = torch.full((4, (V + 31) // 32), -1, dtype=torch.int32, device="cuda")
        masks[0] = 0
        masks[2, 0] = ~2  # all but id 1
        mask_ids = torch.tensor([0, 1, -1, 2, 2, 4, 1, 1, 1], dtype=torch.int32, device="cuda")
        z[0, 3] = float("nan")  # masked with the rest of the row
        z[2, 5] = float("nan")
        z[3, 1] = float("nan")  # masked
        z[4, 1] = INF           # masked
        z[6, V - 1] = INF
        z[6, 7] = INF
        z[7] = -INF
        z[8, 2:] = -INF
        kw = dict(masks=masks, mask_ids=mask_ids)
        got = _run(ctx, z, **kw)
        _check(z, got, kw)
        assert got[1].tolist()[0] == -1 and got[1][2] == -1 and got[1][5] == -1 and got[1][6] == 7 and got[1][7] == -1
        # biases and offsets of -inf leave an id out, whatever its logit
        offset = torch.zeros(V, device="cuda")
        offset[5] = -INF
        bias_ids = torch.full((9, 2), 7, dtype=torch.int32, device="cuda")
        bias = torch.tensor([[1.0, -INF]], device="cuda").repeat(9, 1)
        kw = dict(offset=offset, bias_ids=bias_ids, bias=bias, scale=2.0)
        got = _run(ctx, z, **kw)
        _check(z, got, kw)
        assert got[1][6] == V - 1


def test_penalties_of_each_sign_and_of_many_repeats(ctx):
    V = 50
    z = torch.linspace(-2, 2, V, device="cuda").repeat(4, 1)
    given = torch.full((4, 5000), 49, dtype=torch.int32, device="cuda")
    given[1, ::2] = 0
    given[2] = torch.arange(5000, device="cuda") % V
    given[3] = -1
    for repeat, presence, frequency in ((2.0, 0.0, 0.0), (0.5, 0.0, 0.0), (1.0, 1.0, 0.0), (1.0, 0.0, 0.001),
                                        (1.7, -0.3, -0.01)):
        kw = dict(given=given, repeat=repeat, presence=presence, frequency=frequency)
        _check(z, _run(ctx, z, **kw), kw)


def test_in_place_and_a_mask_of_each_row(ctx):
    from paper_2601_17136_amd import kkm
    g = torch.Generator(device="cuda").manual_seed(8)
    for V in (100, 9001):
        z = ref.rows(5, V, torch.bfloat16, 3, torch.randn(5, V, device="cuda", generator=g))
        masks = torch.randint(-2 ** 31, 2 ** 31, (5, (V + 31) // 32), device="cuda", generator=g).int()
        kw = dict(masks=masks, scale=1.5)
        want = _run(ctx, z, **kw)
        beside = z.clone()
        ids = torch.empty(5, dtype=torch.int32, device="cuda")
        kkm.kkm_choose(ctx, z, z, ids, None, None, **kw)
        assert _same(z.float(), want[0].float()) and torch.equal(ids, want[1])
        _check(beside, want, kw)


def test_no_rows(ctx):
    z = torch.empty(0, 40, device="cuda")
    assert all(t is None or t.numel() == 0 for t in _run(ctx, z))


def test_more_rows_than_a_launch_takes_at_once(ctx):
    """A slice a workgroup: 1.05 million rows of five."""
    free, _ = torch.cuda.mem_get_info()
    n, V = (1 << 20) + 5, 4096 * 4 + 1
    if free < 3 * n * V * 2:
        pytest.skip("not enough memory")
    z = torch.zeros(n, V, device="cuda", dtype=torch.bfloat16)
    at = torch.arange(n, device="cuda") * 7919 % V
    z[torch.arange(n, device="cuda"), at] = 1.0
    ids, lse = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(n, device="cuda")
    from paper_2601_17136_amd import kkm
    kkm.kkm_choose(ctx, z, None, ids, None, lse)
    assert torch.equal(ids.long(), at)
    assert float((lse - torch.log(torch.tensor(V - 1 + 2.718281828459045))).abs().max()) < 1e-5


def test_refusals_of_what_a_row_would_overwrite_or_lose(ctx):
    from paper_2601_17136_amd import kkm
    buf = torch.randn(400, device="cuda")
    was = buf.clone()
    z, out = buf.as_strided((6, 8), (8, 1)), buf.as_strided((6, 8), (9, 1))
    with pytest.raises(kkm.KKMError):
        kkm.kkm_choose(ctx, z, out=out)
    with pytest.raises(ValueError):
        kkm.kkm_choose(ctx, z, lse=torch.empty(6, device="cuda"), bias=torch.zeros(6, 2, device="cuda"))
    assert torch.equal(buf, was)
