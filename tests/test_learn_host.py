"""Refusals of the operators beside a shared head: the C ABI's checks, which run on the host, and the binding's."""
import ctypes

import pytest

from paper_2601_17136_amd import kkm

torch = pytest.importorskip("torch")
NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("coef,eps,args,ok", [
    ([kkm.KKM_QUINTIC] * 5, 1e-7, (0, 1, 8, 8), True), ([kkm.KKM_QUINTIC] * 32, 1e-7, (2, 0, 1, 1), True),
    ([kkm.KKM_CUBIC] * 30, 1e-30, (1, 3, 5, 9), True), ([], 1e-7, (0, 1, 8, 8), False),
    ([kkm.KKM_QUINTIC] * 33, 1e-7, (0, 1, 8, 8), False), ([kkm.KKM_QUINTIC], 0.0, (0, 1, 8, 8), False),
    ([kkm.KKM_QUINTIC], NAN, (0, 1, 8, 8), False), ([kkm.KKM_QUINTIC], INF, (0, 1, 8, 8), False),
    ([(NAN, 0, 0)], 1e-7, (0, 1, 8, 8), False), ([(1, INF, 0)], 1e-7, (0, 1, 8, 8), False),
    ([(3, 0, 0)] * 7, 1e-7, (0, 1, 8, 8), True), ([(3, 0, 0)] * 8, 1e-7, (0, 1, 8, 8), False),
    ([kkm.KKM_QUINTIC], 1e-7, (3, 1, 8, 8), False), ([kkm.KKM_QUINTIC], 1e-7, (0, -1, 8, 8), False),
    ([kkm.KKM_QUINTIC], 1e-7, (0, kkm.KKM_MAX_ROWS + 1, 8, 8), False), ([kkm.KKM_QUINTIC], 1e-7, (0, 1, 0, 8), False),
    ([kkm.KKM_QUINTIC], 1e-7, (0, 1, 8, 0), False), ([kkm.KKM_QUINTIC], 1e-7, (0, 1, kkm.KKM_MAX_FEATURES + 1, 8), False),
    ([kkm.KKM_QUINTIC], 1e-7, (0, 1, 8, kkm.KKM_MAX_FEATURES + 1), False),
])
def test_newton_argument_checks(coef, eps, args, ok):
    rc = kkm.kkm_check_newton_args(kkm._newton_args(coef, eps), *args)
    assert rc == (kkm.KKM_OK if ok else kkm.KKM_ERR_ARG)
    assert ok or kkm.kkm_last_error()


def _adapted(**kw):
    a = dict(type=kkm.KKM_BF16, d=8, n=10, m=4, x=None, ldx=8, w=None, ldw=8, adapters=3, rank=2, down=None, up=None,
             ids=None, factor=None)
    a.update(kw)
    return kkm.kkm_adapted(*[a[f] for f, _ in kkm.kkm_adapted._fields_])


@pytest.mark.parametrize("change,ok", [
    ({}, True), ({"n": 0}, True), ({"ldx": 100}, True), ({"type": -1}, False), ({"d": 0}, False),
    ({"d": kkm.KKM_MAX_FEATURES + 1}, False), ({"n": -1}, False), ({"n": kkm.KKM_MAX_ROWS + 1}, False), ({"m": 0}, False),
    ({"m": kkm.KKM_MAX_FEATURES + 1}, False), ({"ldx": 7}, False), ({"ldw": 7}, False), ({"adapters": 0}, False),
    ({"adapters": kkm.KKM_MAX_ADAPTERS}, True), ({"adapters": kkm.KKM_MAX_ADAPTERS + 1}, False), ({"rank": 0}, False),
    ({"rank": kkm.KKM_MAX_RANK}, True), ({"rank": kkm.KKM_MAX_RANK + 1}, False),
])
def test_adapted_argument_checks(change, ok):
    rc = kkm.kkm_check_adapted_args(_adapted(**change))
    assert rc == (kkm.KKM_OK if ok else kkm.KKM_ERR_ARG)
    assert ok or kkm.kkm_last_error()


def _choice(**kw):
    a = dict(type=kkm.KKM_F32, classes=70, n=10, z=None, ldz=70, scale=1.0, offset=None, given=None, ngiven=0, repeat=1.0,
             presence=0.0, frequency=0.0, bias_ids=None, bias=None, nbias=0, masks=None, words=0, nmasks=0, mask_ids=None)
    a.update(kw)
    return kkm.kkm_choice(*[a[f] for f, _ in kkm.kkm_choice._fields_])


@pytest.mark.parametrize("change,ok", [
    ({}, True), ({"n": 0}, True), ({"ldz": 100}, True), ({"type": 3}, False), ({"n": -1}, False),
    ({"n": kkm.KKM_MAX_ROWS + 1}, False), ({"classes": 0}, False), ({"classes": kkm.KKM_MAX_ROWS + 1}, False),
    ({"ldz": 69}, False), ({"scale": 0.0}, False), ({"scale": -1.0}, False), ({"scale": NAN}, False),
    ({"scale": INF}, False), ({"ngiven": -1}, False), ({"ngiven": kkm.KKM_MAX_GIVEN}, True),
    ({"ngiven": kkm.KKM_MAX_GIVEN + 1}, False), ({"repeat": 0.0}, False), ({"repeat": NAN}, False),
    ({"presence": INF}, False), ({"frequency": NAN}, False), ({"presence": -2.0, "frequency": -1.0}, True),
    ({"nbias": -1}, False), ({"nbias": kkm.KKM_MAX_BIASES}, True), ({"nbias": kkm.KKM_MAX_BIASES + 1}, False),
    ({"masks": 16, "words": 3, "nmasks": 10}, True), ({"masks": 16, "words": 2, "nmasks": 10}, False),
    ({"masks": 16, "words": 3, "nmasks": 9}, False), ({"masks": 16, "words": 3, "nmasks": 0, "mask_ids": 16}, True),
    ({"masks": 16, "words": 3, "nmasks": -1, "mask_ids": 16}, False), ({"mask_ids": 16}, False),
])
def test_choice_argument_checks(change, ok):
    rc = kkm.kkm_check_choice_args(_choice(**change))
    assert rc == (kkm.KKM_OK if ok else kkm.KKM_ERR_ARG)
    assert ok or kkm.kkm_last_error()


def test_masks_that_are_not_there_have_no_negative_count():
    assert kkm.kkm_check_choice_args(_choice(nmasks=-5)) == kkm.KKM_ERR_ARG
    assert kkm.kkm_check_choice_args(_choice(nmasks=7)) == kkm.KKM_OK


def test_limits_match_the_header():
    import os
    src = open(os.path.join(os.path.dirname(kkm.__file__), "..", "include", "kkm.h")).read()
    assert f"#define KKM_MAX_STEPS {kkm.KKM_MAX_STEPS}" in src and f"#define KKM_MAX_BIASES {kkm.KKM_MAX_BIASES}" in src
    assert f"#define KKM_MAX_RANK {kkm.KKM_MAX_RANK}" in src
    assert f"#define KKM_MAX_ADAPTERS {kkm.KKM_MAX_ADAPTERS}" in src
    assert "#define KKM_MAX_GIVEN ((1 << 20) - 1)" in src and kkm.KKM_MAX_GIVEN == (1 << 20) - 1


def test_null_context_is_rejected_without_a_gpu():
    L, w, q = kkm.lib(), kkm._newton_args([kkm.KKM_CUBIC], 1e-7), _choice()
    assert L.kkm_orthogonalize(None, ctypes.byref(w), 0, 1, 1, 1, None, 1, 1, None, 1, 1) == kkm.KKM_ERR_ARG
    assert L.kkm_orthogonal_step(None, ctypes.byref(w), 0, 1, 1, 1, None, 1, 1, None, 1, 1, None, 0.9, 1, 0.1,
                                 1.0) == kkm.KKM_ERR_ARG
    assert L.kkm_choose(None, ctypes.byref(q), None, 70, None, None, None) == kkm.KKM_ERR_ARG
    a = _adapted()
    assert L.kkm_adapted_linear(None, ctypes.byref(a), None, 4) == kkm.KKM_ERR_ARG
    assert L.kkm_adapted_linear_grad(None, ctypes.byref(a), None, 4, None, 8, None, None) == kkm.KKM_ERR_ARG
    assert L.kkm_check_adapted_args(None) == kkm.KKM_ERR_ARG
    assert L.kkm_check_newton_args(None, 0, 1, 1, 1) == kkm.KKM_ERR_ARG
    assert L.kkm_check_choice_args(None) == kkm.KKM_ERR_ARG


def test_binding_refuses_host_tensors_and_wrong_shapes():
    x = torch.zeros(3, 4)
    with pytest.raises(TypeError):
        kkm.kkm_orthogonalize(None, x, x)
    with pytest.raises(TypeError):
        kkm.kkm_orthogonal_step(None, x, x, x, 0.1)
    with pytest.raises(TypeError):
        kkm.kkm_choose(None, x)
    with pytest.raises(TypeError):
        kkm.kkm_adapted_linear(None, x, x, x[None], x[None], x[:, 0].int(), x)
    with pytest.raises(ValueError):
        kkm._newton_args([(1.0, 2.0)], 1e-7)


@pytest.mark.gpu
def test_calls_refuse_wrong_arguments():
    """On a GPU: every refusal leaves the outputs alone and the context usable."""
    if not torch.cuda.is_available():
        pytest.fail("GPU test on a machine without a GPU")
    c = kkm.kkm_create(kkm.current_stream_handle())
    try:
        f = dict(device="cuda")
        x, y, v = torch.randn(2, 6, 8, **f), torch.zeros(2, 6, 8, **f), torch.zeros(2, 6, 8, **f)
        for bad, exc in [((x, y[:1]), ValueError), ((x, y.half()), TypeError), ((x[0], y), ValueError),
                         ((x.transpose(1, 2), y.transpose(1, 2)), ValueError), ((x[0, 0], y[0, 0]), ValueError),
                         ((x[:1].expand(2, 6, 8), y), ValueError), ((x[:, :1].expand(2, 6, 8), y), ValueError),
                         ((x[:, :0], y[:, :0]), kkm.KKMError), ((x.double(), y.double()), TypeError)]:
            with pytest.raises(exc):
                kkm.kkm_orthogonalize(c, *bad)
        for kw in (dict(eps=0.0), dict(coef=[]), dict(coef=[(9.0, 0.0, 0.0)] * 5)):
            with pytest.raises(kkm.KKMError):
                kkm.kkm_orthogonalize(c, x, y, **kw)
        with pytest.raises(TypeError):
            kkm.kkm_orthogonal_step(c, y, x, v.half(), 0.1)
        with pytest.raises(ValueError):
            kkm.kkm_orthogonal_step(c, y, x, v[:1], 0.1)
        with pytest.raises(TypeError):
            kkm.kkm_orthogonal_step(c, y, x.half(), v, 0.1)
        with pytest.raises(kkm.KKMError):
            kkm.kkm_orthogonal_step(c, y, x, v, float("nan"))
        assert not y.any() and not v.any()
        p, w, down, up = torch.randn(6, 8, **f), torch.randn(5, 8, **f), torch.randn(3, 2, 8, **f), torch.randn(3, 5, 2, **f)
        q, one = torch.zeros(6, 5, **f), torch.zeros(6, dtype=torch.int32, **f)
        good = dict(x=p, w=w, down=down, up=up, ids=one, y=q)
        for kw, exc in [(dict(w=w.half()), TypeError), (dict(w=w[:, :7]), ValueError), (dict(down=down[:, :, :7]), ValueError),
                        (dict(down=down[0]), ValueError), (dict(down=down[:2]), ValueError), (dict(up=up[:, :4]), ValueError),
                        (dict(up=up.half()), TypeError), (dict(down=down.transpose(0, 1).contiguous().transpose(0, 1)), ValueError),
                        (dict(ids=one.long()), TypeError), (dict(ids=one[:5]), ValueError), (dict(y=q[:, :4]), ValueError),
                        (dict(factor=torch.ones(2, **f)), ValueError), (dict(factor=torch.ones(3, **f).half()), TypeError),
                        (dict(down=down[:, :0], up=up[:, :, :0]), kkm.KKMError)]:
            with pytest.raises(exc):
                kkm.kkm_adapted_linear(c, **{**good, **kw})
        assert not q.any()
        for kw, exc in [(dict(dx=p[:5]), ValueError), (dict(ddown=down[:2]), ValueError), (dict(dup=up.half()), TypeError),
                        (dict(dy=q[:5]), ValueError)]:
            with pytest.raises(exc):
                kkm.kkm_adapted_linear_grad(c, **{"dy": q, **{k: v for k, v in good.items() if k != "y"}, **kw})
        kkm.kkm_adapted_linear(c, **good)
        assert q.any()
        z, ids = torch.randn(6, 40, **f), torch.zeros(6, dtype=torch.int32, **f)
        out, lists = torch.zeros(6, 40, **f), torch.zeros(6, 3, dtype=torch.int32, **f)
        for kw, exc in [(dict(out=out.half()), TypeError), (dict(out=out[:5]), ValueError), (dict(ids=ids.long()), TypeError),
                        (dict(ids=ids[:5]), ValueError), (dict(given=lists[:5]), ValueError),
                        (dict(given=lists.long()), TypeError), (dict(bias_ids=lists), ValueError),
                        (dict(bias_ids=lists, bias=torch.zeros(6, 2, **f)), ValueError),
                        (dict(offset=torch.zeros(39, **f)), ValueError), (dict(scale=0.0), kkm.KKMError),
                        (dict(masks=lists[:, :1].contiguous()), kkm.KKMError), (dict(masks=ids), ValueError),
                        (dict(mask_ids=ids), kkm.KKMError), (dict(masks=lists[:3], mask_ids=ids[:3]), ValueError),
                        (dict(masks=lists[:3].float(), mask_ids=ids), TypeError), (dict(repeat=0.0), kkm.KKMError)]:
            with pytest.raises(exc):
                kkm.kkm_choose(c, z, **{"out": out, **kw})
        assert not out.any()
        kkm.kkm_choose(c, z, out, ids)
        assert torch.equal(out, z) and torch.equal(ids.long(), z.argmax(1))
        kkm.kkm_orthogonalize(c, x, y)
        assert y.any()
    finally:
        kkm.kkm_destroy(c)
