"""Coefficients of steps as the binding takes them."""
import pytest

from paper_2601_17136_amd import kkm

np = pytest.importorskip("numpy")


@pytest.mark.parametrize("coef", [[(1.0, 2.0)], [(1.0, 2.0), (3.0, 4.0, 5.0, 6.0)], [(1.0, 2.0, 3.0), ()], [(), (1.0,) * 6]])
def test_each_step_has_three(coef):
    with pytest.raises(ValueError):
        kkm._newton_args(coef, 1e-7)


@pytest.mark.parametrize("coef", [[(1.0, 2.0, 3.0)], ((1, 2, 3), [4, 5, 6]), np.ones((4, 3)), []])
def test_steps_of_any_sequence(coef):
    a = kkm._newton_args(coef, 1e-7)
    assert a.steps == len(coef) and [a.coef[i] for i in range(3 * a.steps)] == [float(v) for s in coef for v in s]
