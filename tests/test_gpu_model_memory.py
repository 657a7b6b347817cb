"""The model operators' scratch beside a build, in budgets that hold little more
than kkm_plan asks for."""
import numpy as np
import pytest

from gpu_helpers import Engine
from paper_2601_17136_amd import datagen

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _operator(ctx, scratch):
    """The loss of ten rows over as many classes as take about this much scratch
    (16 scores a class, and the rows' sums of each 16 of them)."""
    from paper_2601_17136_amd import kkm
    f = {"device": "cuda"}
    V = int(scratch / (64 + 5))
    h, w = torch.ones(10, 16, **f), torch.zeros(V, 16, **f)
    loss, lse = torch.empty(10, **f), torch.empty(10, **f)
    kkm.kkm_head_loss(ctx, h, w, torch.zeros(10, dtype=torch.int32, **f), loss, lse)
    assert bool(((lse - np.log(V)).abs() < 1e-5).all())


@pytest.mark.parametrize("mode", ["resident", "packed", "onthefly"])
def test_a_rebuild_of_the_same_shape_gives_the_scratch_back(mode):
    from paper_2601_17136_amd import kkm
    X = datagen.make_points(2, n=2600, d=24)[0]
    with Engine(X, "linear", mode=mode, mem_budget=1 << 30) as eng:
        held = eng.info()["bytes_total"]
        _operator(eng.ctx, 8 << 20)
        assert eng.info()["bytes_total"] > held + (7 << 20)
        kkm.kkm_build_kernel(eng.ctx, eng.X, 2600, 24, kkm.KKM_LINEAR, kkm.make_params(mode=kkm.MODES[mode]))
        assert eng.info()["bytes_total"] == held
