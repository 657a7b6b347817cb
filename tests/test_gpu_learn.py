"""The adapted projection, the orthogonalised update and answers from logits together: a model's step and its
answers against 64 bits, streams, graphs, scratch, memory beside the outputs."""
import os
import sys

import pytest

import learn_reference as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
F32, I32 = torch.float32, torch.int32


def _kkm():
    if not torch.cuda.is_available():
        pytest.fail("GPU test on a machine without a GPU")
    from paper_2601_17136_amd import kkm
    return kkm


class _Step:
    """A model's step and its answers: features, the head's loss, gradients, updates, masked ids."""

    def __init__(self, n=300, d=96, m=80, V=50, s=5, r=12, dtype=F32, seed=3):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def normal(*shape):
            return torch.randn(*shape, device="cuda", generator=g)

        self.x, self.w, self.head = normal(n, d).to(dtype), (normal(m, d) / d ** 0.5).to(dtype), normal(V, m).to(dtype)
        self.down, self.up = (normal(s, r, d) / d ** 0.5).to(dtype), (normal(s, m, r) / r ** 0.5).to(dtype)
        self.source = torch.randint(-1, s, (n,), device="cuda", generator=g).int()
        self.ids = torch.randint(0, V, (n,), device="cuda", generator=g).int()
        self.masks = torch.randint(-2 ** 31, 2 ** 31, (3, (V + 31) // 32), device="cuda", generator=g).int()
        self.mask_ids = torch.randint(-1, 3, (n,), device="cuda", generator=g).int()
        self.given = torch.randint(-1, V, (n, 6), device="cuda", generator=g).int()
        self.v_down, self.v_up = normal(s, r, d) * 1e-3, normal(s, m, r) * 1e-3
        self.y, self.dy = torch.empty(n, m, device="cuda", dtype=dtype), torch.empty(n, m, device="cuda", dtype=dtype)
        self.dx, self.z = torch.empty_like(self.x), torch.empty(n, V, device="cuda", dtype=dtype)
        self.dw = torch.empty_like(self.head)
        self.ddown, self.dup = torch.empty_like(self.down), torch.empty_like(self.up)
        self.loss, self.lse, self.logp, self.total = (torch.empty(n, device="cuda") for _ in range(4))
        self.dloss = torch.full((n,), 1.0 / n, device="cuda")
        self.picked = torch.empty(n, dtype=I32, device="cuda")
        self.none, self.empty = torch.full((n,), -1, dtype=I32, device="cuda"), torch.zeros(1, 1, m, device="cuda", dtype=dtype)
        self.flat = torch.zeros(1, V, 1, device="cuda", dtype=dtype)

    def run(self, c):
        kkm = _kkm()
        kkm.kkm_adapted_linear(c, self.x, self.w, self.down, self.up, self.source, self.y)
        kkm.kkm_head_grad(c, self.y, self.head, self.ids, self.dloss, self.loss, self.lse, self.dy, self.dw)
        kkm.kkm_adapted_linear_grad(c, self.x, self.w, self.down, self.up, self.source, self.dy, self.dx, self.ddown,
                                    self.dup)
        kkm.kkm_orthogonal_step(c, self.down, self.ddown, self.v_down, 0.02)
        kkm.kkm_orthogonal_step(c, self.up, self.dup, self.v_up, 0.02)
        # the head's logits: the projection of rows without an adapter
        kkm.kkm_adapted_linear(c, self.y, self.head, self.empty, self.flat, self.none, self.z)
        kkm.kkm_choose(c, self.z, self.z, self.picked, self.logp, self.total, scale=0.8, given=self.given, repeat=1.2,
                       presence=0.1, frequency=0.1, masks=self.masks, mask_ids=self.mask_ids)

    def outputs(self):
        return (self.y, self.loss, self.dy, self.dx, self.ddown, self.dup, self.down, self.up, self.v_down, self.v_up,
                self.z, self.picked, self.logp, self.total)

    def state(self):
        return (self.down, self.up, self.v_down, self.v_up)


def test_a_step_and_its_answers():
    """Every output of a step against the formulas, each from the step's own inputs."""
    kkm = _kkm()
    c = kkm.kkm_create(kkm.current_stream_handle())
    try:
        for dtype in (F32, torch.bfloat16):
            s = _Step(dtype=dtype)
            down, up, v_down, v_up = (t.clone() for t in s.state())
            s.run(c)
            want, tol = ref.adapted(s.x, s.w, down, up, s.source, None, s.dy)
            for name in ("y", "dx", "ddown", "dup"):
                ref.check(name, getattr(s, name), want[name], tol[name])
            z = s.y.double() @ s.head.double().t()
            p = torch.softmax(z, 1)
            p[torch.arange(p.shape[0]), s.ids.long()] -= 1
            dy = (p / p.shape[0]) @ s.head.double()
            assert float((s.dy.double() - dy).norm()) <= (1e-4 if dtype == F32 else 8e-3) * float(dy.norm())
            for w0, g, v0, w1, v1 in ((down, s.ddown, v_down, s.down, s.v_down), (up, s.dup, v_up, s.up, s.v_up)):
                v = 0.95 * v0.double() + g.double()
                assert float((v1.double() - v).abs().max()) <= 4 * ref.U * float(v.abs().max())
                for i in range(w0.shape[0]):
                    u = g[i].double() + 0.95 * v1[i].double()
                    o, _ = ref.newton(u, [kkm.KKM_QUINTIC] * 5, 1e-7)
                    new = w0[i].double().cpu() - 0.02 * o
                    # (short sides of 12: 64 bits, u's entries and the result rounded to fp32)
                    room = 0.02 * ref.slope_of([kkm.KKM_QUINTIC] * 5) * 8 * ref.U + 3 * ref.U * float(new.norm())
                    assert float((w1[i].double().cpu() - new).norm()) <= room + ref.UNIT[dtype] * float(new.norm())
            logits = torch.empty_like(s.z)
            kkm.kkm_adapted_linear(c, s.y, s.head, s.empty, s.flat, s.none, logits)
            u, ids, logp, lse, tol_p, tol_l = ref.choose(logits, 0.8, given=s.given, repeat=1.2, presence=0.1, frequency=0.1,
                                                         masks=s.masks, mask_ids=s.mask_ids)
            assert torch.equal(s.picked.cpu(), ids) and torch.equal(s.z.cpu(), u.to(dtype))
            fine = torch.isfinite(lse)
            assert bool(((s.total.cpu().double() - lse).abs() <= tol_l)[fine].all())
            assert bool(((s.logp.cpu().double() - logp).abs() <= tol_p)[fine].all())
    finally:
        kkm.kkm_destroy(c)


@pytest.mark.parametrize("dtype", [F32, torch.float16, torch.bfloat16])
def test_replayed_graph(dtype):
    """A captured step replayed on new inputs, with eager steps and synchronizations between the replays."""
    kkm = _kkm()
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        c = kkm.kkm_create(kkm.current_stream_handle())
        s = _Step(n=2500, d=200, m=260, V=9000, s=7, r=70, dtype=dtype)
        start = [t.clone() for t in s.state()]

        def reset():
            for t, v in zip(s.state(), start):
                t.copy_(v)

        s.run(c)
        reset()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            s.run(c)
        g = torch.Generator(device="cuda").manual_seed(5)
        for k in range(4):
            s.x.copy_(torch.randn(s.x.shape, device="cuda", generator=g))
            s.source.copy_(torch.randint(-1, 8, s.source.shape, device="cuda", generator=g))
            torch.cuda.synchronize()
            reset()
            s.run(c)
            want = [t.clone() for t in s.outputs()]
            torch.cuda.synchronize()
            for t in s.outputs():
                t.fill_(-3)
            reset()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            for a, b in zip(s.outputs(), want):
                assert torch.equal(torch.nan_to_num(a.float(), 7), torch.nan_to_num(b.float(), 7)), k
    torch.cuda.synchronize()
    kkm.kkm_destroy(c)


def test_another_stream_than_the_contexts_and_two_at_once():
    kkm = _kkm()
    here = kkm.kkm_create(kkm.current_stream_handle())
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        there = kkm.kkm_create(kkm.current_stream_handle())
    try:
        a, b = _Step(dtype=torch.bfloat16, n=2500, m=300), _Step(dtype=torch.bfloat16, n=2500, m=300)
        for _ in range(3):
            for k in (a, b):  # the same work on both, at the same time
                k.x.copy_((k.x.float() * 1.5).to(k.x.dtype))  # on the current stream, as are the reads below
            a.run(here)
            b.run(there)
            assert all(torch.equal(torch.nan_to_num(p.float(), 7), torch.nan_to_num(q.float(), 7))
                       for p, q in zip(a.outputs(), b.outputs()))
    finally:
        kkm.kkm_destroy(there)
        kkm.kkm_destroy(here)


def test_memory_beside_the_outputs_stays():
    """Columns past an output's own, and rows after its last, are left as they were."""
    kkm = _kkm()
    c = kkm.kkm_create(kkm.current_stream_handle())
    try:
        for dtype in (F32, torch.bfloat16):
            for n, d, m in ((5, 33, 17), (70, 100, 90), (700, 301, 333)):
                g = torch.Generator(device="cuda").manual_seed(n)
                x, w = torch.randn(n, d, device="cuda", generator=g).to(dtype), torch.randn(m, d, device="cuda", generator=g).to(dtype)
                down, up = torch.randn(2, 3, d, device="cuda", generator=g).to(dtype), torch.randn(2, m, 3, device="cuda", generator=g).to(dtype)
                ids = torch.randint(0, 2, (n,), device="cuda", generator=g).int()

                def around(rows, cols):  # a matrix inside a larger one
                    t = torch.full((rows + 2, cols + 5), 77.0, device="cuda", dtype=dtype)
                    return t, t[1:rows + 1, 2:cols + 2]

                ty, y = around(n, m)
                tx, dx = around(n, d)
                to, o = around(n, m)
                tw, v = around(m, d)
                kkm.kkm_adapted_linear(c, x, w, down, up, ids, y)
                kkm.kkm_adapted_linear_grad(c, x, w, down, up, ids, y, dx)
                kkm.kkm_choose(c, y, o, given=ids[:, None].contiguous(), presence=1.0)
                kkm.kkm_orthogonalize(c, w, v)
                for t, inner in ((ty, y), (tx, dx), (to, o), (tw, v)):
                    assert not bool((inner == 77.0).all())
                    inner.fill_(77.0)
                    assert bool((t == 77.0).all())
    finally:
        kkm.kkm_destroy(c)


def test_scratch_counts_against_the_budget_and_a_capture_needs_it():
    kkm = _kkm()
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        c = kkm.kkm_create(kkm.current_stream_handle(), 16 << 20)
        try:
            x = torch.randn(2000, 2000, device="cuda")
            y = torch.full_like(x, 5.0)
            with pytest.raises(kkm.KKMError) as e:  # 24 bytes an entry
                kkm.kkm_orthogonalize(c, x, y)
            assert e.value.code == kkm.KKM_ERR_OOM and bool((y == 5.0).all())
            small, out = torch.randn(100, 200, device="cuda"), torch.empty(100, 200, device="cuda")
            caught = None
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                out.fill_(1.0)
                try:
                    kkm.kkm_orthogonalize(c, small, out)
                except kkm.KKMError as err:
                    caught = err
            assert caught is not None and caught.code == kkm.KKM_ERR_STATE
            kkm.kkm_orthogonalize(c, small, out)
            want = out.clone()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                kkm.kkm_orthogonalize(c, small, out)
            for _ in range(3):
                out.fill_(0.0)
                graph.replay()
                torch.cuda.synchronize()
                assert torch.equal(out, want)
        finally:
            torch.cuda.synchronize()
            kkm.kkm_destroy(c)


def test_matrices_far_apart():
    """Matrices of a batch, and rows, whose offsets pass 32 bits."""
    kkm = _kkm()
    c = kkm.kkm_create(kkm.current_stream_handle())
    try:
        stride = (1 << 31) + 512
        for m, n in ((20, 100), (100, 90)):
            x = torch.randn(3, m, n, device="cuda").bfloat16()
            far = torch.empty(2 * stride + m * n, device="cuda", dtype=torch.bfloat16).as_strided((3, m, n), (stride, n, 1))
            far.copy_(x)
            y, y2 = torch.empty_like(x), torch.empty_like(x)
            kkm.kkm_orthogonalize(c, x, y)
            kkm.kkm_orthogonalize(c, far, y2)
            assert torch.equal(y, y2)
            kkm.kkm_orthogonalize(c, far, far)
            assert torch.equal(far, y)
            del far
    finally:
        kkm.kkm_destroy(c)


def test_example():
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    from examples import adapt_sources
    out = adapt_sources.run(points=1200, new=200, steps=6, log=lambda *a: None)
    for name in ("shared", "adapters"):
        assert len(out[name]) == 6 and all(v == v and abs(v) != float("inf") for v in out[name])
    assert all(0.0 <= v <= 1.0 for v in out["agree"])
