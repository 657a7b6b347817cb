"""Refusals of the model operators: the C ABI's checks, which run on the host, and the binding's."""
import ctypes

import pytest

from paper_2601_17136_amd import kkm

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("args,ok", [
    ((kkm.KKM_F32, 10, 5, 5, kkm.KKM_F32, 1e-5), True),
    ((kkm.KKM_BF16, 0, 1, 8, kkm.KKM_BF16, 1e-5), True),
    ((kkm.KKM_F16, 10, 5, 5, kkm.KKM_F32, 1e-5), True),
    ((3, 10, 5, 5, kkm.KKM_F32, 1e-5), False),
    ((kkm.KKM_F32, 10, 5, 5, kkm.KKM_F16, 1e-5), False),
    ((kkm.KKM_F16, 10, 5, 5, kkm.KKM_BF16, 1e-5), False),
    ((kkm.KKM_F32, -1, 5, 5, kkm.KKM_F32, 1e-5), False),
    ((kkm.KKM_F32, 2 ** 31, 5, 5, kkm.KKM_F32, 1e-5), False),
    ((kkm.KKM_F32, 10, 0, 5, kkm.KKM_F32, 1e-5), False),
    ((kkm.KKM_F32, 10, kkm.KKM_MAX_FEATURES + 1, 2 ** 21, kkm.KKM_F32, 1e-5), False),
    ((kkm.KKM_F32, 10, 5, 4, kkm.KKM_F32, 1e-5), False),
    ((kkm.KKM_F32, 10, 5, 5, kkm.KKM_F32, 0.0), False),
    ((kkm.KKM_F32, 10, 5, 5, kkm.KKM_F32, -1.0), False),
    ((kkm.KKM_F32, 10, 5, 5, kkm.KKM_F32, float("nan")), False),
    ((kkm.KKM_F32, 10, 5, 5, kkm.KKM_F32, float("inf")), False),
])
def test_norm_argument_checks(args, ok):
    rc = kkm.kkm_check_norm_args(*args)
    assert rc == (kkm.KKM_OK if ok else kkm.KKM_ERR_ARG)
    assert ok or kkm.kkm_last_error()


def _head(**kw):
    a = dict(type=kkm.KKM_F32, d=8, n=10, classes=4, h=None, ldh=8, w=None, ldw=8, offset=None, scale=1.0)
    a.update(kw)
    return kkm.kkm_head(*[a[f] for f, _ in kkm.kkm_head._fields_])


@pytest.mark.parametrize("change,ok", [
    ({}, True), ({"n": 0}, True), ({"scale": -2.0}, True), ({"ldh": 100}, True), ({"type": 7}, False),
    ({"d": 0}, False), ({"d": kkm.KKM_MAX_FEATURES + 1}, False), ({"n": -1}, False),
    ({"n": kkm.KKM_MAX_ROWS + 1}, False), ({"classes": 0}, False), ({"classes": kkm.KKM_MAX_ROWS + 1}, False),
    ({"ldh": 7}, False), ({"ldw": 7}, False), ({"scale": float("nan")}, False), ({"scale": float("inf")}, False),
])
def test_head_argument_checks(change, ok):
    rc = kkm.kkm_check_head_args(_head(**change))
    assert rc == (kkm.KKM_OK if ok else kkm.KKM_ERR_ARG)
    assert ok or kkm.kkm_last_error()


@pytest.mark.parametrize("m,scale,n,ok", [(1, 1.0, 10, True), (256, 0.5, 10, True), (0, 1.0, 10, False),
                                          (257, 1.0, 10, False), (8, float("nan"), 10, False),
                                          (256, 1.0, kkm.KKM_MAX_ROWS, True)])
def test_teacher_argument_checks(m, scale, n, ok):
    rc = kkm.kkm_check_head_args(_head(n=n), kkm.kkm_teacher(None, None, m, scale))
    assert rc == (kkm.KKM_OK if ok else kkm.KKM_ERR_ARG)


def test_limits_match_the_header():
    import os
    src = open(os.path.join(os.path.dirname(kkm.__file__), "..", "include", "kkm.h")).read()
    assert f"#define KKM_MAX_TOP {kkm.KKM_MAX_TOP}" in src
    assert "#define KKM_MAX_FEATURES (1 << 20)" in src and kkm.KKM_MAX_FEATURES == 1 << 20
    assert "#define KKM_MAX_ROWS (1 << 21)" in src and kkm.KKM_MAX_ROWS == 1 << 21


def test_null_context_is_rejected_without_a_gpu():
    L, h = kkm.lib(), _head()
    t = kkm.kkm_teacher(None, None, 1, 1.0)
    assert L.kkm_layer_norm(None, 0, 1, 1, None, 1, 0, None, None, 1e-5, None, 1, None, None) == kkm.KKM_ERR_ARG
    assert L.kkm_layer_norm_grad(None, 0, 1, 1, None, 1, 0, None, None, None, None, 1, None, 1, None,
                                 None) == kkm.KKM_ERR_ARG
    assert L.kkm_head_loss(None, ctypes.byref(h), None, None, None) == kkm.KKM_ERR_ARG
    assert L.kkm_head_grad(None, ctypes.byref(h), None, None, None, None, None, 8, None, 8) == kkm.KKM_ERR_ARG
    assert L.kkm_distill_loss(None, ctypes.byref(h), ctypes.byref(t), None, None) == kkm.KKM_ERR_ARG
    assert L.kkm_distill_grad(None, ctypes.byref(h), ctypes.byref(t), None, None, None, None, 8, None,
                              8) == kkm.KKM_ERR_ARG
    assert L.kkm_get_stream(None, None) == kkm.KKM_ERR_ARG
    assert L.kkm_check_head_args(None, None) == kkm.KKM_ERR_ARG


def test_binding_refuses_host_tensors_and_wrong_dtypes():
    x = torch.zeros(3, 4)
    with pytest.raises(TypeError):
        kkm.kkm_layer_norm(None, x, None, None, 1e-5, x)
    with pytest.raises(TypeError):
        kkm.kkm_head_loss(None, x, x, torch.zeros(3, dtype=torch.int32), x[:, 0], x[:, 0])
    with pytest.raises(TypeError):
        kkm._type_code(torch.float64, "x")


@pytest.mark.gpu
def test_calls_refuse_wrong_arguments():
    """On a GPU: every refusal leaves the outputs alone and the context usable."""
    if not torch.cuda.is_available():
        pytest.fail("GPU test on a machine without a GPU")
    c = kkm.kkm_create(kkm.current_stream_handle())
    try:
        f = dict(device="cuda")
        h, w, ids = torch.randn(6, 8, **f), torch.randn(5, 8, **f), torch.zeros(6, dtype=torch.int32, **f)
        loss, lse = torch.zeros(6, **f), torch.zeros(6, **f)
        ok = lambda **kw: kkm.kkm_head_loss(c, kw.get("h", h), kw.get("w", w), kw.get("ids", ids),
                                            kw.get("loss", loss), lse, scale=kw.get("scale", 1.0),
                                            offset=kw.get("offset"))
        for kw, exc in [(dict(w=w.half()), TypeError), (dict(w=torch.randn(5, 9, **f)), ValueError),
                        (dict(ids=ids.long()), TypeError), (dict(ids=ids[:5]), ValueError),
                        (dict(loss=loss.half()), TypeError), (dict(h=h.t().contiguous().t()), ValueError),
                        (dict(h=h[0]), ValueError), (dict(offset=torch.zeros(4, **f)), ValueError),
                        (dict(scale=float("nan")), kkm.KKMError), (dict(h=h[:, :0], w=w[:, :0]), kkm.KKMError),
                        (dict(w=w[:0]), kkm.KKMError)]:
            with pytest.raises(exc):
                ok(**kw)
        with pytest.raises(ValueError):
            kkm.kkm_head_loss(c, h[:1].expand(6, 8), w, ids, loss, lse)
        with pytest.raises(ValueError):
            kkm.kkm_head_grad(c, h, w, ids, loss, loss, lse, dh=h[:5], dw=None)
        with pytest.raises(kkm.KKMError):
            kkm.kkm_distill_loss(c, h, w, torch.zeros(6, 300, dtype=torch.int32, **f), torch.zeros(6, 300, **f), loss, lse)
        with pytest.raises(ValueError):
            kkm.kkm_distill_loss(c, h, w, ids[:, None][:5], torch.zeros(5, 1, **f), loss, lse)
        with pytest.raises(kkm.KKMError):
            kkm.kkm_layer_norm(c, h, None, None, 0.0, torch.empty_like(h))
        with pytest.raises(TypeError):
            kkm.kkm_layer_norm(c, h.half(), torch.ones(8, **f).bfloat16(), torch.ones(8, **f), 1e-5, h.half())
        with pytest.raises(kkm.KKMError):
            kkm.kkm_layer_norm(c, h.half(), torch.ones(8, **f).bfloat16(), None, 1e-5, h.half())
        assert not loss.any()
        ok()
        assert (loss > 0).all()
    finally:
        kkm.kkm_destroy(c)
