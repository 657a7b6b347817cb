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


def _same(a, b):
    return all(np.array_equal(a[key], b[key]) for key in ("E", "D", "z", "cl", "counts")) and a["J"] == b["J"]


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


@pytest.mark.parametrize("mode", ["resident", "packed", "onthefly"])
@pytest.mark.parametrize("kind", ["linear", "gauss"])
def test_the_scratch_makes_way_for_updates_and_seeding(kind, mode):
    """An operator between a build and the first update, in a budget of exactly the plan."""
    from paper_2601_17136_amd import kkm
    n, d, k = 1500, 40, 60
    X = datagen.make_points(2, n=n, d=d)[0]
    cl = datagen.random_init(n, k, 5)
    _, need = kkm.kkm_plan(n, d, k, kkm.KINDS[kind], 1 << 40, kkm.MODES[mode])
    u = np.random.default_rng(1).random(k)
    more = need + 24 * n + 16384  # room for the seeding scratch of n points: 16 bytes each and the centers
    with Engine(X, kind, 1.0 / d, mode=mode, mem_budget=need, k_hint=k) as eng:
        want = eng.step(cl, k)
        fixups = eng.info()["fixups"]
    with Engine(X, kind, 1.0 / d, mode=mode, mem_budget=more, k_hint=k) as eng:
        eng.step(cl, k)
        seeds = eng.seed(k, u)
    with Engine(X, kind, 1.0 / d, mode=mode, mem_budget=need, k_hint=k) as eng:
        held = eng.info()["bytes_total"]
        _operator(eng.ctx, 0.9 * (need - held))
        assert eng.info()["bytes_total"] > held
        got = eng.step(cl, k)
        assert eng.info()["bytes_total"] <= need and eng.info()["fixups"] == fixups
        assert _same(got, want)
    with Engine(X, kind, 1.0 / d, mode=mode, mem_budget=more, k_hint=k) as eng:
        eng.step(cl, k)
        _operator(eng.ctx, 0.9 * (more - eng.info()["bytes_total"]))
        again = eng.seed(k, u)
        assert all(np.array_equal(a, b) for a, b in zip(again, seeds))


def test_an_operator_takes_nothing_of_the_builds():
    """On the fly the updates multiply the split points: an operator that finds no
    room beside them is refused, and the next update has the same bits."""
    from paper_2601_17136_amd import kkm
    n, d, k = 2000, 90, 7
    X = datagen.make_points(2, n=n, d=d)[0]
    cl = datagen.random_init(n, k, 5)
    _, need = kkm.kkm_plan(n, d, k, kkm.KKM_LINEAR, 1 << 40, kkm.KKM_MODE_ONTHEFLY)
    split = 2048 * (6 * 64 + 8)
    budget = need + split + 60000
    with Engine(X, "linear", mode="onthefly", mem_budget=budget, k_hint=k) as eng:
        first = eng.step(cl, k)
        held = eng.info()["bytes_total"]
        assert held > need  # the split points are there
        with pytest.raises(kkm.KKMError) as e:
            _operator(eng.ctx, budget - held + split // 2)
        assert e.value.code == kkm.KKM_ERR_OOM
        assert eng.info()["bytes_total"] == held
        assert _same(eng.step(cl, k), first)
        _operator(eng.ctx, (budget - held) // 2)
        assert _same(eng.step(cl, k), first)


def test_a_captured_call_that_lacks_scratch_is_refused():
    """Nothing is freed or made within a capture: what the context holds stays usable."""
    from paper_2601_17136_amd import kkm
    stream, f = torch.cuda.Stream(), {"device": "cuda"}
    h, w, ids = torch.randn(700, 24, **f), torch.randn(90, 24, **f), torch.zeros(700, dtype=torch.int32, **f)
    loss, lse, small = torch.empty(700, **f), torch.empty(700, **f), torch.empty(70, **f)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        c = kkm.kkm_create(kkm.current_stream_handle())
        kkm.kkm_build_kernel(c, h, 700, 24, kkm.KKM_LINEAR, kkm.make_params(mode=kkm.KKM_MODE_RESIDENT))
        built = kkm.kkm_get_info(c)["bytes_total"]
        kkm.kkm_head_loss(c, h[:70], w, ids[:70], small, lse[:70])
        want, held = small.clone(), kkm.kkm_get_info(c)["bytes_total"]
        assert held > built
        with pytest.raises(kkm.KKMError) as e:
            with torch.cuda.graph(torch.cuda.CUDAGraph(), stream=stream):
                kkm.kkm_head_loss(c, h, w, ids, loss, lse)
        assert e.value.code == kkm.KKM_ERR_STATE
        assert kkm.kkm_get_info(c)["bytes_total"] == held
        kkm.kkm_head_loss(c, h[:70], w, ids[:70], small, lse[:70])
        assert torch.equal(small, want)
        kkm.kkm_head_loss(c, h, w, ids, loss, lse)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            kkm.kkm_head_loss(c, h, w, ids, loss, lse)
        want = loss.clone()
        for _ in range(3):
            loss.fill_(float("nan"))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(loss, want)
    torch.cuda.synchronize()
    kkm.kkm_destroy(c)
