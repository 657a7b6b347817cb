"""Layer norm and the class head's losses against their 64-bit forms, at the
sizes, strides and masks where they can go wrong."""
import pytest

import model_reference as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.fail("GPU test on a machine without a GPU")
    from paper_2601_17136_amd import kkm
    c = kkm.kkm_create(kkm.current_stream_handle())
    yield c
    kkm.kkm_destroy(c)


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _rows(n, d, dtype, pad, values):
    """n x d values as the columns [pad // 2, ..) of a table d + pad wide."""
    t = torch.full((n, d + pad), float("nan"), device="cuda", dtype=dtype)[:, pad // 2:pad // 2 + d]
    t.copy_(values)
    return t


# ------------------------------------------------------------------ layer norm

NORM = [(1, 1), (1, 7), (2, 64), (5, 33), (3, 255), (4, 256), (9, 257), (130, 301), (2050, 54), (700, 784),
        (65, 1025), (17, 2049), (5, 4097), (6, 8192), (3, 8193), (2, 20000)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,d", NORM)
def test_layer_norm(ctx, n, d, dtype):
    from paper_2601_17136_amd import kkm
    t, g = DTYPES[dtype], _gen(n * 131 + d)
    pad = (n + d) % 4
    wtype = t if d % 2 else torch.float32
    print(f"[gpu] layer norm n={n} d={d} {dtype} pad={pad}", flush=True)
    x = _rows(n, d, t, pad, torch.randn(n, d, device="cuda", generator=g) * 2 + torch.randn(n, 1, device="cuda", generator=g) * 3)
    dy = _rows(n, d, t, 3 - pad, torch.randn(n, d, device="cuda", generator=g))
    w = (1 + 0.3 * torch.randn(d, device="cuda", generator=g)).to(wtype)
    b = torch.randn(d, device="cuda", generator=g).to(wtype)
    y, dx = _rows(n, d, t, 2 * pad, torch.zeros(n, d)), _rows(n, d, t, pad, torch.zeros(n, d))
    mean, rstd = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    dw, db = torch.empty_like(w), torch.empty_like(b)
    eps = 1e-3
    kkm.kkm_layer_norm(ctx, x, w, b, eps, y, mean, rstd)
    kkm.kkm_layer_norm_grad(ctx, x, w, dy, mean, rstd, dx, dw, db)
    r = ref.layer_norm(x, w, b, eps, dy)
    for name, got in (("y", y), ("mean", mean), ("rstd", rstd), ("dx", dx), ("dw", dw), ("db", db)):
        ref.check(name, got, r[name], r["tol_" + name])
    # the same bits again, in place, and with only a part of the gradient
    y2, dx2, dw2 = x.clone(), dy.clone(), torch.empty_like(w)
    kkm.kkm_layer_norm_grad(ctx, x, w, dx2, mean, rstd, dx2, dw2, None)
    kkm.kkm_layer_norm(ctx, y2, w, b, eps, y2)
    assert torch.equal(y2, y) and torch.equal(dx2, dx) and torch.equal(dw2, dw)
    db2 = torch.empty_like(b)
    kkm.kkm_layer_norm_grad(ctx, x, w, dy, mean, rstd, None, None, db2)
    assert torch.equal(db2, db)


def test_layer_norm_without_weight_or_rows(ctx):
    from paper_2601_17136_amd import kkm
    g = _gen(5)
    x, dy = torch.randn(40, 100, device="cuda", generator=g), torch.randn(40, 100, device="cuda", generator=g)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = torch.empty(40, device="cuda"), torch.empty(40, device="cuda")
    kkm.kkm_layer_norm(ctx, x, None, None, 1e-5, y, mean, rstd)
    kkm.kkm_layer_norm_grad(ctx, x, None, dy, mean, rstd, dx)
    r = ref.layer_norm(x, None, None, 1e-5, dy)
    ref.check("y", y, r["y"], r["tol_y"])
    ref.check("dx", dx, r["dx"], r["tol_dx"])
    none = torch.empty(0, 100, device="cuda")
    dw, db = torch.full((100,), 7.0, device="cuda"), torch.full((100,), 7.0, device="cuda")
    kkm.kkm_layer_norm(ctx, none, None, None, 1e-5, none)
    kkm.kkm_layer_norm_grad(ctx, none, None, none, mean[:0], rstd[:0], none, dw, db)
    assert not dw.any() and not db.any()


def test_layer_norm_rows_of_one_value_and_infinite_rows(ctx):
    """A constant row has xh = 0; a row with an infinity or NaN spoils itself alone."""
    from paper_2601_17136_amd import kkm
    x = torch.randn(6, 300, device="cuda", generator=_gen(6))
    x[1] = 1000.0
    x[2, 5] = float("inf")
    x[3, 299] = float("nan")
    y, mean, rstd = torch.empty_like(x), torch.empty(6, device="cuda"), torch.empty(6, device="cuda")
    b = torch.randn(300, device="cuda", generator=_gen(7))
    kkm.kkm_layer_norm(ctx, x, None, b, 1e-5, y, mean, rstd)
    fine = [0, 1, 4, 5]
    r = ref.layer_norm(x[fine], None, b, 1e-5, x[fine])
    ref.check("y", y[fine], r["y"], r["tol_y"])
    assert torch.isnan(y[3]).all() and torch.isnan(y[2, 5])


# ------------------------------------------------------------------ the head

def _head_case(n, d, V, dtype, seed, pad=0, offset=False, drop=0.0):
    t, g = DTYPES[dtype], _gen(seed)
    h = _rows(n, d, t, pad, torch.randn(n, d, device="cuda", generator=g))
    w = _rows(V, d, t, pad, torch.randn(V, d, device="cuda", generator=g) * (2 / d ** 0.5))
    off = None
    if offset:
        off = torch.randn(V, device="cuda", generator=g)
        off[torch.rand(V, device="cuda", generator=g) < 0.2] = -float("inf")
        off[V // 2] = 0.25
    kept = torch.arange(V, device="cuda") if off is None else torch.nonzero(off > -float("inf"))[:, 0]
    ids = kept[torch.randint(0, kept.numel(), (n,), device="cuda", generator=g)]
    ids = torch.where(torch.rand(n, device="cuda", generator=g) < drop, -100, ids).to(torch.int32)
    dloss = torch.randn(n, device="cuda", generator=g)
    return h, w, off, ids, dloss, g, kept


def _outputs(h, w, pad=0):
    n, d = h.shape
    dev = {"device": "cuda"}
    return (torch.empty(n, **dev), torch.empty(n, **dev), _rows(n, d, h.dtype, pad, torch.zeros(n, d)),
            _rows(w.shape[0], d, h.dtype, pad, torch.zeros(w.shape[0], d)))


def _check_head(r, loss, lse, dh, dw):
    worst = [ref.check(name, got, r[name], r["tol_" + name])
             for name, got in (("loss", loss), ("lse", lse), ("dh", dh), ("dw", dw)) if got is not None]
    print(f"      of the bounds: {', '.join(f'{x:.2g}' for x in worst)}", flush=True)


HEAD = [(1, 1, 1), (1, 5, 3), (2, 8, 2), (3, 64, 130), (5, 7, 1000), (33, 100, 17), (64, 54, 7), (127, 65, 129),
        (128, 128, 128), (130, 16, 257), (257, 784, 10), (300, 301, 64), (700, 72, 300), (1030, 24, 65),
        (2000, 19, 32), (999, 130, 16), (16, 300, 4100), (17, 64, 5000), (64, 40, 16400), (65, 65, 65), (1, 2048, 700),
        (1500, 2100, 1030), (777, 4000, 1100), (5000, 56, 4000)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,d,V", HEAD)
def test_head(ctx, n, d, V, dtype):
    from paper_2601_17136_amd import kkm
    pad = (0, 0, 3, 8)[(n + d + V) % 4]
    print(f"[gpu] head n={n} d={d} V={V} {dtype} pad={pad}", flush=True)
    h, w, off, ids, dloss, _, _ = _head_case(n, d, V, dtype, n + 31 * d + 7 * V, pad, offset=V > 2 and V % 2 == 1,
                                             drop=0.2 if n > 2 else 0.0)
    loss, lse, dh, dw = _outputs(h, w, pad)
    scale = 1.0 if d % 2 else 0.7
    kkm.kkm_head_grad(ctx, h, w, ids, dloss, loss, lse, dh, dw, scale=scale, offset=off)
    r = ref.head(h, w, ref.one_hot(ids, V), dloss, scale, off)
    _check_head(r, loss, lse, dh, dw)
    loss2, lse2, dh2, dw2 = _outputs(h, w)
    kkm.kkm_head_loss(ctx, h, w, ids, loss2, lse2, scale=scale, offset=off)
    assert torch.equal(loss2, loss) and torch.equal(lse2, lse)
    kkm.kkm_head_grad(ctx, h, w, ids, dloss, loss2, lse2, dh2, None, scale=scale, offset=off)
    kkm.kkm_head_grad(ctx, h, w, ids, dloss, loss2, lse2, None, dw2, scale=scale, offset=off)
    assert torch.equal(dh2, dh) and torch.equal(dw2, dw)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,d,V", [(3000, 40, 4500), (8200, 72, 1600)])
def test_head_of_many_rows_and_classes(ctx, n, d, V, dtype):
    from paper_2601_17136_amd import kkm
    print(f"[gpu] head n={n} d={d} V={V} {dtype}", flush=True)
    h, w, off, ids, dloss, _, _ = _head_case(n, d, V, dtype, 11, drop=0.1, offset=V == 1600)
    loss, lse, dh, dw = _outputs(h, w)
    kkm.kkm_head_grad(ctx, h, w, ids, dloss, loss, lse, dh, dw, offset=off)
    _check_head(ref.head(h, w, ref.one_hot(ids, V), dloss, 1.0, off), loss, lse, dh, dw)


@pytest.mark.parametrize("n,d,V,dtype", [(300, 8, 100003, "f32"), (300, 8, 270001, "bf16"), (1000, 24, 140000, "f16")])
def test_head_in_pieces_of_the_classes(ctx, n, d, V, dtype):
    """More classes than one piece of G holds: dh is summed over the pieces."""
    from paper_2601_17136_amd import kkm
    print(f"[gpu] head n={n} d={d} V={V} {dtype}", flush=True)
    h, w, off, ids, dloss, _, _ = _head_case(n, d, V, dtype, 12)
    ids[0], ids[1] = 0, V - 1
    loss, lse, dh, dw = _outputs(h, w)
    kkm.kkm_head_grad(ctx, h, w, ids, dloss, loss, lse, dh, dw)
    _check_head(ref.head(h, w, ref.one_hot(ids, V), dloss, 1.0, off), loss, lse, dh, dw)


# (each form the head runs in: few classes, few rows, little work, tiles)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,d,V", [(150, 40, 90), (150, 40, 50), (40, 40, 90), (2600, 640, 1300)])
def test_head_masks(ctx, n, d, V, dtype):
    """What a mask covers may hold anything: classes left out with NaN rows of w,
    rows without a label or of weight 0 with NaN in h, rows that see no class."""
    from paper_2601_17136_amd import kkm
    print(f"[gpu] head masks n={n} d={d} V={V} {dtype}", flush=True)
    h, w, _, ids, dloss, _, _ = _head_case(n, d, V, dtype, 13)
    off = torch.zeros(V, device="cuda")
    off[10:30] = -float("inf")
    off[40] = torch.finfo(torch.float32).min
    w[12] = float("nan")
    w[13] = float("inf")
    ids = torch.where((ids >= 10) & (ids < 30) | (ids == 40), 3, ids).to(torch.int32)
    ids[5], ids[6], ids[7] = -1, -1, 15  # without a label; a class that is left out
    dloss[8] = 0.0
    h[5, 3], h[8, 1] = float("nan"), float("inf")
    loss, lse, dh, dw = _outputs(h, w)
    kkm.kkm_head_grad(ctx, h, w, ids, dloss, loss, lse, dh, dw, offset=off)
    assert loss[5] == 0 and loss[6] == 0 and loss[7] == float("inf")
    assert not dh[5].any() and not dh[6].any() and not dh[8].any()
    assert not dw[10:30].any() and not dw[40].any()
    r = ref.head(h, w, ref.one_hot(ids, V), dloss, 1.0, off)
    rows = [i for i in range(n) if i not in (5, 8)]
    ref.check("loss", loss[rows], r["loss"][rows], r["tol_loss"][rows])
    ref.check("lse", lse[rows], r["lse"][rows], r["tol_lse"][rows])
    ref.check("dh", dh, r["dh"], r["tol_dh"])
    ref.check("dw", dw, r["dw"], r["tol_dw"])
    off[:] = -float("inf")
    kkm.kkm_head_grad(ctx, h, w, ids, dloss, loss, lse, dh, dw, offset=off)
    assert (lse == -float("inf")).all() and not dh.any() and not dw.any()
    assert loss[5] == 0 and loss[9] == float("inf")
    ids[:] = -1
    kkm.kkm_head_grad(ctx, h, w, ids, dloss, loss, lse, dh, dw)
    assert not loss.any() and not dh.any() and not dw.any()


def test_head_reports_an_id_out_of_range(ctx):
    from paper_2601_17136_amd import kkm
    h, w, _, ids, dloss, _, _ = _head_case(20, 16, 9, "f32", 14)
    ids[4] = 9
    loss, lse, dh, dw = _outputs(h, w)
    kkm.kkm_head_grad(ctx, h, w, ids, dloss, loss, lse, dh, dw)
    assert torch.isnan(loss[4]) and torch.isfinite(loss[torch.arange(20, device="cuda") != 4]).all()
    assert torch.isnan(dh[4]).all() and torch.isfinite(dh[3]).all() and torch.isnan(dw).any()


def test_head_of_no_rows(ctx):
    from paper_2601_17136_amd import kkm
    h, w = torch.empty(0, 12, device="cuda"), torch.randn(5, 12, device="cuda")
    dw = torch.full_like(w, 3.0)
    e = torch.empty(0, device="cuda")
    kkm.kkm_head_loss(ctx, h, w, e.to(torch.int32), e, e)
    kkm.kkm_head_grad(ctx, h, w, e.to(torch.int32), e, e, e, h, dw)
    assert not dw.any()


@pytest.mark.parametrize("dtype", DTYPES)
def test_head_of_large_logits(ctx, dtype):
    """Logits of hundreds: one class has all of a row's probability."""
    from paper_2601_17136_amd import kkm
    h, w, _, ids, dloss, _, _ = _head_case(200, 64, 150, dtype, 15)
    h *= 16
    w *= 8
    loss, lse, dh, dw = _outputs(h, w)
    kkm.kkm_head_grad(ctx, h, w, ids, dloss, loss, lse, dh, dw)
    assert all(torch.isfinite(t).all() for t in (loss, lse, dh, dw))
    r = ref.head(h, w, ref.one_hot(ids, 150), dloss, 1.0, None)
    ref.check("loss", loss, r["loss"], r["tol_loss"])
    ref.check("lse", lse, r["lse"], r["tol_lse"])


def test_head_gradient_against_differences(ctx):
    """The gradient of sum(dloss * loss) along a direction, against the loss on both sides of it."""
    from paper_2601_17136_amd import kkm
    n, d, V, eps = 50, 30, 40, 2.0 ** -6
    h, w, _, ids, dloss, g, _ = _head_case(n, d, V, "f32", 16, drop=0.1)
    loss, lse, dh, dw = _outputs(h, w)
    kkm.kkm_head_grad(ctx, h, w, ids, dloss, loss, lse, dh, dw, scale=0.5)
    uh, uw = torch.randn(n, d, device="cuda", generator=g), torch.randn(V, d, device="cuda", generator=g)
    uh /= uh.norm()
    uw /= uw.norm()
    for grad, dirh, dirw in ((dh, uh, 0 * uw), (dw, 0 * uh, uw)):
        side = []
        for e in (-eps, eps):
            kkm.kkm_head_loss(ctx, h + e * dirh, w + e * dirw, ids, loss, lse, scale=0.5)
            side.append(float((dloss.double() * loss.double()).sum()))
        slope = float((grad.double() * (dirh if grad is dh else dirw).double()).sum())
        # the third derivative of a log sum of exponentials of logits that move by at most s per
        # unit is below s^3; a loss is off by less than 2e-5
        s = 0.5 * float((h.norm(dim=1).max() if grad is dw else w.norm(dim=1).max()))
        tol = float(dloss.abs().sum()) * ((2 * s) ** 3 * eps ** 2 / 6 + 2e-5 / eps)
        assert abs((side[1] - side[0]) / (2 * eps) - slope) <= tol, (side, slope, tol)


# ------------------------------------------------------------------ distillation

def _teacher(n, V, m, g, kept):
    ids = kept[torch.randint(0, kept.numel(), (n, m), device="cuda", generator=g)].to(torch.int32)
    logits = 3 * torch.randn(n, m, device="cuda", generator=g)
    gone = torch.rand(n, m, device="cuda", generator=g)
    ids = torch.where(gone < 0.1, -1, ids)
    logits = torch.where(gone > 0.9, -float("inf"), logits)
    if n > 3:
        ids[2] = -1
        logits[3] = -float("inf")
    return ids.to(torch.int32).contiguous(), logits.contiguous()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,d,V,m", [(1, 1, 1, 1), (1, 6, 5, 3), (4, 17, 9, 12), (50, 54, 7, 7), (130, 33, 257, 64),
                                     (65, 120, 1000, 65), (40, 8, 300, 256), (600, 784, 64, 8), (300, 100, 513, 20), (100, 60, 2050, 200), (1200, 2050, 1001, 70)])
def test_distill(ctx, n, d, V, m, dtype):
    from paper_2601_17136_amd import kkm
    pad = (0, 8, 1)[(n + d) % 3]
    print(f"[gpu] distill n={n} d={d} V={V} m={m} {dtype} pad={pad}", flush=True)
    h, w, off, _, dloss, g, kept = _head_case(n, d, V, dtype, 3 * n + d + V, pad, offset=m == 20)
    ids, logits = _teacher(n, V, m, g, kept)
    loss, lse, dh, dw = _outputs(h, w, pad)
    kkm.kkm_distill_grad(ctx, h, w, ids, logits, dloss, loss, lse, dh, dw, scale=0.5, offset=off, teacher_scale=0.8)
    r = ref.head(h, w, ref.teacher(ids, logits, 0.8, V), dloss, 0.5, off)
    # each pair's own terms: a class named twice has q log q of its parts
    q = torch.softmax(torch.where(ids >= 0, logits.double() * 0.8, -torch.inf), 1).nan_to_num(0.0).cpu()
    both = ref.teacher(ids, logits, 0.8, V)
    r["loss"] = r["loss"] + (torch.special.entr(both).sum(1) - torch.special.entr(q).sum(1))
    _check_head(r, loss, lse, dh, dw)
    if n > 3:
        assert loss[2] == 0 and loss[3] == 0 and not dh[2].any() and not dh[3].any()
    loss2, lse2, dh2, _ = _outputs(h, w)
    kkm.kkm_distill_loss(ctx, h, w, ids, logits, loss2, lse2, scale=0.5, offset=off, teacher_scale=0.8)
    assert torch.equal(loss2, loss) and torch.equal(lse2, lse)
    kkm.kkm_distill_grad(ctx, h, w, ids, logits, dloss, loss2, lse2, dh2, None, scale=0.5, offset=off,
                         teacher_scale=0.8)
    assert torch.equal(dh2, dh)


def test_distill_of_one_pair_is_the_loss_with_ids(ctx):
    from paper_2601_17136_amd import kkm
    h, w, off, ids, dloss, _, _ = _head_case(90, 48, 70, "bf16", 21, offset=True, drop=0.2)
    a, b = _outputs(h, w), _outputs(h, w)
    kkm.kkm_head_grad(ctx, h, w, ids, dloss, *a, offset=off)
    kkm.kkm_distill_grad(ctx, h, w, ids[:, None].contiguous(), torch.full((90, 1), -4.5, device="cuda"), dloss, *b,
                         offset=off)
    assert all(torch.equal(x, y) for x, y in zip(a, b))


# ------------------------------------------------------------------ streams, graphs, memory

def test_another_stream_than_the_contexts(ctx):
    """Inputs made, and outputs read, on torch's current stream; the context on another."""
    from paper_2601_17136_amd import kkm
    side = torch.cuda.Stream()
    h, w, _, ids, dloss, _, _ = _head_case(2000, 256, 3000, "bf16", 31)
    want = _outputs(h, w)
    kkm.kkm_head_grad(ctx, h, w, ids, dloss, *want)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        other = kkm.kkm_create(kkm.current_stream_handle())
    try:
        assert kkm.kkm_get_stream(other) == side.cuda_stream
        for _ in range(3):
            h2 = (h.float() * 2).to(h.dtype) / 2  # on the current stream, as are the reads below
            got = _outputs(h2, w)
            kkm.kkm_head_grad(other, h2, w, ids, dloss, *got)
            copies = [t.clone() for t in got]
            del h2, got
            assert all(torch.equal(x, y) for x, y in zip(copies, want))
    finally:
        kkm.kkm_destroy(other)


def test_replayed_graph():
    """A captured step of all three, replayed on new inputs."""
    from paper_2601_17136_amd import kkm
    n, d, V, m = 500, 96, 700, 5
    g = _gen(41)
    x = torch.randn(n, d, device="cuda", generator=g)
    w = torch.randn(V, d, device="cuda", generator=g) * 0.2
    gamma, beta = torch.ones(d, device="cuda"), torch.zeros(d, device="cuda")
    ids, logits = _teacher(n, V, m, g, torch.arange(V, device="cuda"))
    label = ids[:, 0].contiguous()
    dloss = torch.full((n,), 1.0 / n, device="cuda")
    y, dh, dx = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    dw, dw2, dh2 = torch.empty_like(w), torch.empty_like(w), torch.empty_like(x)
    mean, rstd, loss, lse = (torch.empty(n, device="cuda") for _ in range(4))
    dg, db = torch.empty_like(gamma), torch.empty_like(beta)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        c = kkm.kkm_create(kkm.current_stream_handle())

        def step():
            kkm.kkm_layer_norm(c, x, gamma, beta, 1e-5, y, mean, rstd)
            kkm.kkm_head_grad(c, y, w, label, dloss, loss, lse, dh, dw)
            kkm.kkm_distill_grad(c, y, w, ids, logits, dloss, loss, lse, dh2, dw2)
            kkm.kkm_layer_norm_grad(c, x, gamma, dh, mean, rstd, dx, dg, db)

        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step()
        outs = (y, loss, lse, dh, dw, dh2, dw2, dx, dg, db)
        for k in range(4):
            x.copy_(torch.randn(n, d, device="cuda", generator=g))
            torch.cuda.synchronize()
            step()
            want = [t.clone() for t in outs]
            for t in outs:
                t.fill_(float("nan"))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(outs, want)), k
    torch.cuda.synchronize()
    kkm.kkm_destroy(c)


def test_workspace_counts_against_the_budget_and_goes_with_a_build():
    from paper_2601_17136_amd import datagen, kkm
    c = kkm.kkm_create(kkm.current_stream_handle(), 64 << 20)
    try:
        h, w, _, ids, dloss, _, _ = _head_case(2000, 64, 100, "f32", 51)
        out = _outputs(h, w)
        kkm.kkm_head_grad(c, h, w, ids, dloss, *out)
        big = torch.randn(200000, 64, device="cuda")
        bigids = torch.zeros(200000, dtype=torch.int32, device="cuda")
        with pytest.raises(kkm.KKMError) as e:
            kkm.kkm_head_grad(c, big, w, bigids, big[:, 0].contiguous(), *_outputs(big, w))
        assert e.value.code == kkm.KKM_ERR_OOM
        kkm.kkm_head_grad(c, h, w, ids, dloss, *out)
        X = torch.from_numpy(datagen.make_points(2, n=2600, d=24)[0]).cuda()
        kkm.kkm_build_kernel(c, X, 2600, 24, kkm.KKM_LINEAR, kkm.make_params(mode=kkm.KKM_MODE_RESIDENT))
        assert kkm.kkm_get_info(c)["bytes_total"] <= 64 << 20
        J = kkm.kkm_objective(c, torch.zeros(2600, dtype=torch.int32, device="cuda"), 1)
        small = _head_case(60, 20, 10, "f32", 52)
        kkm.kkm_head_grad(c, small[0], small[1], small[3], small[4], *_outputs(small[0], small[1]))
        assert kkm.kkm_objective(c, torch.zeros(2600, dtype=torch.int32, device="cuda"), 1) == J
    finally:
        kkm.kkm_destroy(c)


# ------------------------------------------------------------------ few classes of many rows

@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,d,V,m", [(4096, 1, 1, 0), (4111, 33, 5, 3), (5000, 780, 10, 0), (4200, 513, 31, 40),
                                     (9001, 1000, 16, 0), (6002, 900, 3, 7), (4999, 512, 32, 0), (4500, 257, 17, 5),
                                     (4100, 1024, 12, 2), (4101, 1025, 12, 2)])
def test_few_classes_of_many_rows(ctx, n, d, V, m, dtype):
    """The same loss from each call, rows without a label that hold infinities, a label past the classes."""
    from paper_2601_17136_amd import kkm
    pad = (0, 3, 8)[(n + d + V) % 3]
    print(f"[gpu] few classes n={n} d={d} V={V} m={m} {dtype} pad={pad}", flush=True)
    h, w, off, ids, dloss, g, kept = _head_case(n, d, V, dtype, n + 5 * d + V, pad, offset=V > 2 and d % 2 == 1,
                                                drop=0.15)
    more = dict(scale=0.6, offset=off)
    if m:
        top, logits = _teacher(n, V, m, g, kept)
        more["teacher_scale"] = 0.9
        fwd, bwd, said = kkm.kkm_distill_loss, kkm.kkm_distill_grad, (top, logits)
        q = ref.teacher(top, logits, 0.9, V)
        none = 2
    else:
        ids[7] = -1
        fwd, bwd, said = kkm.kkm_head_loss, kkm.kkm_head_grad, (ids,)
        q = ref.one_hot(ids, V)
        none = 7
    loss, lse, dh, dw = _outputs(h, w, pad)
    bwd(ctx, h, w, *said, dloss, loss, lse, dh, dw, **more)
    r = ref.head(h, w, q, dloss, 0.6, off)
    if m:  # each pair's own terms: a class named twice has q log q of its parts
        parts = torch.softmax(torch.where(top >= 0, logits.double() * 0.9, -torch.inf), 1).nan_to_num(0.0).cpu()
        r["loss"] = r["loss"] + (torch.special.entr(q).sum(1) - torch.special.entr(parts).sum(1))
    _check_head(r, loss, lse, dh, dw)
    assert loss[none] == 0 and not dh[none].any()
    # the loss alone, one gradient alone: the same bits
    a = _outputs(h, w)
    fwd(ctx, h, w, *said, *a[:2], **more)
    assert torch.equal(a[0], loss) and torch.equal(a[1], lse)
    bwd(ctx, h, w, *said, dloss, *a[:2], a[2], None, **more)
    bwd(ctx, h, w, *said, dloss, *a[:2], None, a[3], **more)
    assert torch.equal(a[2], dh) and torch.equal(a[3], dw)
    # an infinity in a row that takes no part reaches no other row's results
    h2 = h.clone()
    h2[none] = float("inf")
    b = _outputs(h, w)
    bwd(ctx, h2, w, *said, dloss, *b, **more)
    assert torch.equal(b[3], dw) and not b[2][none].any()
    # a label past the classes: NaN for its row, and in dW
    first = said[0].clone()
    first.view(n, -1)[11, 0] = V
    if m:
        logits[11, 0] = 0.5
    bwd(ctx, h, w, first, *said[1:], dloss, *b, **more)
    assert torch.isnan(b[0][11]) and torch.isnan(b[3]).any()
    assert torch.equal(b[0][:11], loss[:11]) and torch.equal(b[2][12:], dh[12:])


# ------------------------------------------------------------------ rows far apart

def _far(values, ld):
    """The rows `ld` elements apart: past 32 bits for the last."""
    n, d = values.shape
    t = torch.empty((n - 1) * ld + d, device="cuda", dtype=values.dtype).as_strided((n, d), (ld, 1))
    assert (n - 1) * ld > 2 ** 31
    return t.copy_(values)


@pytest.mark.parametrize("n,d,V,dtype,ld", [(2100, 48, 10, "bf16", 2 ** 20 + 8), (2100, 64, 100, "f16", 2 ** 20 + 8),
                                            (1300, 64, 90, "f32", 2 ** 21 - 5), (2100, 264, 2000, "bf16", 2 ** 20 + 8),
                                            (1100, 264, 2000, "bf16", 2 ** 21 + 8), (1100, 250, 2000, "f32", 2 ** 21)])
def test_rows_of_h_far_apart(ctx, n, d, V, dtype, ld):
    from paper_2601_17136_amd import kkm
    print(f"[gpu] far h n={n} d={d} V={V} {dtype} ld={ld}", flush=True)
    h, w, off, ids, dloss, _, _ = _head_case(n, d, V, dtype, n + d, offset=True, drop=0.1)
    want, got = _outputs(h, w), list(_outputs(h, w))
    kkm.kkm_head_grad(ctx, h, w, ids, dloss, *want, offset=off)
    got[2] = _far(torch.zeros_like(h), ld)
    kkm.kkm_head_grad(ctx, _far(h, ld), w, ids, dloss, *got, offset=off)
    assert all(torch.equal(x, y) for x, y in zip(got, want))


@pytest.mark.parametrize("n,V,d,dtype", [(16, 2100, 72, "bf16"), (200, 2100, 72, "f16"), (2000, 2100, 264, "bf16")])
def test_rows_of_w_far_apart(ctx, n, V, d, dtype):
    from paper_2601_17136_amd import kkm
    print(f"[gpu] far w n={n} d={d} V={V} {dtype}", flush=True)
    h, w, _, _, dloss, g, kept = _head_case(n, d, V, dtype, n + d)
    ids, logits = _teacher(n, V, 5, g, kept)
    want, got = _outputs(h, w), list(_outputs(h, w))
    kkm.kkm_distill_grad(ctx, h, w, ids, logits, dloss, *want)
    got[3] = _far(torch.zeros_like(w), 2 ** 20 + 8)
    kkm.kkm_distill_grad(ctx, h, _far(w, 2 ** 20 + 8), ids, logits, dloss, *got)
    assert all(torch.equal(x, y) for x, y in zip(got, want))


@pytest.mark.parametrize("n,d,dtype", [(2100, 300, "bf16"), (2100, 3001, "f16"), (2100, 20000, "bf16")])
def test_layer_norm_of_rows_far_apart(ctx, n, d, dtype):
    from paper_2601_17136_amd import kkm
    print(f"[gpu] far norm n={n} d={d} {dtype}", flush=True)
    ld, dev = 2 ** 20 + 8, {"device": "cuda"}
    x, dy = (torch.randn(n, d, generator=_gen(d + k), **dev).to(DTYPES[dtype]) for k in (0, 1))
    w, b = torch.randn(d, generator=_gen(5), **dev), torch.randn(d, generator=_gen(6), **dev)
    outs = []
    for far in (False, True):
        place = (lambda t: _far(t, ld)) if far else (lambda t: t)
        y, dx = place(torch.zeros_like(x)), place(torch.zeros_like(x))
        mean, rstd, dw, db = (torch.empty(k, **dev) for k in (n, n, d, d))
        kkm.kkm_layer_norm(ctx, place(x), w, b, 1e-5, y, mean, rstd)
        kkm.kkm_layer_norm_grad(ctx, place(x), w, place(dy), mean, rstd, dx, dw, db)
        outs.append([t.clone() for t in (y, mean, rstd, dx, dw, db)])
    assert all(torch.equal(x, y) for x, y in zip(*outs))


# ------------------------------------------------------------------ logits kept for a part of the classes

@pytest.mark.parametrize("n,d,V,m,dtype", [(4096, 2056, 20000, 0, "bf16"), (5001, 1111, 40007, 3, "f16"),
                                           (9000, 320, 9001, 0, "f32"), (66000, 1100, 1300, 2, "bf16")])
def test_head_of_more_logits_than_are_kept(ctx, n, d, V, m, dtype):
    """Rows and classes on both sides of what is kept, against the formulas on a part of each."""
    from paper_2601_17136_amd import kkm
    print(f"[gpu] kept in part n={n} d={d} V={V} m={m} {dtype}", flush=True)
    h, w, off, ids, dloss, g, kept = _head_case(n, d, V, dtype, n + V, offset=True, drop=0.1)
    more, out = dict(scale=0.7, offset=off), _outputs(h, w)
    if m:
        ids, logits = _teacher(n, V, m, g, kept)
        kkm.kkm_distill_grad(ctx, h, w, ids, logits, dloss, *out, teacher_scale=0.9, **more)
        t = torch.where(ids >= 0, logits.double() * 0.9, -torch.inf)
        q = torch.softmax(t, 1).nan_to_num(0.0)
    else:
        kkm.kkm_head_grad(ctx, h, w, ids, dloss, *out, **more)
        q = (ids >= 0).double()[:, None]
        ids = ids[:, None]
    loss, lse, dh, dw = out
    # G in blocks of rows, in 64 bits on the GPU (plain products of two matrices)
    wd = torch.where((off > -torch.inf)[:, None], w.double(), 0.0)
    want_dw = torch.zeros(V, d, device="cuda", dtype=torch.float64)
    size_dw = torch.zeros(V, d, device="cuda", dtype=torch.float64)
    unit = ref.UNIT[h.dtype] if h.dtype != torch.float32 else 2 * ref.U
    for i in range(0, n, 2048):
        r = slice(i, min(i + 2048, n))
        hd = h[r].double()
        z = 0.7 * (hd @ wd.t().contiguous()) + off.double()
        L = torch.logsumexp(z, 1)
        has = q[r].sum(1) > 0
        # an entry's error: a logit's, the sum's, one rounding to the operands' type
        dz = (0.7 * (hd.abs() @ wd.abs().t().contiguous())).amax(1) * ref.sum_error(d, h.dtype) + 1e-5
        assert bool(((lse[r].double() - L).abs() <= dz + (16 + V / 64) * 2 * ref.U * (1 + L.abs())).all())
        c = torch.where(has, dloss[r].double(), 0.0)[:, None] * 0.7
        G = torch.exp(z - L[:, None])
        dG = G * (4 * dz[:, None] + (V / 64 + 32) * 2 * ref.U)
        at = ids[r].long().clamp(min=0)
        G.scatter_add_(1, at, -q[r])
        dG.scatter_add_(1, at, 8 * ref.U * q[r])
        G, dG = G * c, dG * c.abs() + (G * c).abs() * unit
        dG = dG + ref.STEP[h.dtype] * dloss.abs().max() * 2.0 ** -12 * (c != 0)
        G, dG = torch.where(c != 0, G, 0.0), torch.where(c != 0, dG, 0.0)
        want, size = G @ wd, (dG + G.abs() * (ref.sum_error(V, h.dtype) + 40 * ref.U)) @ wd.abs()
        assert bool(((dh[r].double() - want).abs() <= size + ref.UNIT[h.dtype] * want.abs() + ref.STEP[h.dtype]).all())
        want_dw += G.t().contiguous() @ hd
        size_dw += (dG + G.abs() * (ref.sum_error(n, h.dtype) + 40 * ref.U)).t().contiguous() @ hd.abs()
    assert bool(((dw.double() - want_dw).abs() <= size_dw + ref.UNIT[h.dtype] * want_dw.abs() + ref.STEP[h.dtype]).all())
    # one gradient alone, and the loss alone, have the same bits
    b = _outputs(h, w)
    if m:
        kkm.kkm_distill_loss(ctx, h, w, ids, logits, *b[:2], teacher_scale=0.9, **more)
        assert torch.equal(b[0], loss) and torch.equal(b[1], lse)
        kkm.kkm_distill_grad(ctx, h, w, ids, logits, dloss, *b[:2], None, b[3], teacher_scale=0.9, **more)
    else:
        one = ids[:, 0].contiguous()
        kkm.kkm_head_loss(ctx, h, w, one, *b[:2], **more)
        assert torch.equal(b[0], loss) and torch.equal(b[1], lse)
        kkm.kkm_head_grad(ctx, h, w, one, dloss, *b[:2], None, b[3], **more)
    assert torch.equal(b[3], dw)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,d,V,m", [(2500, 8, 9000, 4), (2500, 33, 3000, 5), (2100, 64, 2100, 33), (2100, 65, 2100, 64),
                                     (1500, 127, 2000, 65), (1400, 300, 1400, 17), (900, 1025, 1500, 100),
                                     (2500, 20, 9001, 256)])
def test_distill_of_many_pairs_of_short_and_long_rows(ctx, n, d, V, m, dtype):
    test_distill(ctx, n, d, V, m, dtype)
