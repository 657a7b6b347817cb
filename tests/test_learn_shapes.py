"""What the binding says to tensors of the right number of entries in another order."""
import pytest

from paper_2601_17136_amd import kkm

torch = pytest.importorskip("torch")
F32 = torch.float32


class _Device:
    """Stands in for a device tensor."""
    is_cuda, dtype = True, F32

    def __init__(self, *shape):
        self.shape = torch.Size(shape)

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 4096


@pytest.mark.parametrize("got,want,ok", [
    ((2, 6, 8), (2, 6, 8), True), ((96,), (2, 6, 8), True), ((1, 6, 8), (6, 8), True), ((6, 1), (1, 6), True),
    ((2, 8, 6), (2, 6, 8), False), ((6, 2, 8), (2, 6, 8), False), ((12, 8), (2, 6, 8), False), ((8, 6), (6, 8), False)])
def test_shapes(got, want, ok):
    if ok:
        assert kkm._shaped(_Device(*got), F32, "v", torch.Size(want)) == 4096
    else:
        with pytest.raises(ValueError):
            kkm._shaped(_Device(*got), F32, "v", torch.Size(want))


def test_addresses_and_none_pass():
    assert kkm._shaped(None, F32, "v", (2, 3)) is None and kkm._shaped(64, F32, "v", (2, 3)) == 64


@pytest.mark.gpu
def test_calls():
    """On a GPU: refused before anything is written."""
    if not torch.cuda.is_available():
        pytest.fail("GPU test on a machine without a GPU")
    c = kkm.kkm_create(kkm.current_stream_handle())
    try:
        f = dict(device="cuda")
        x, w, down, up = torch.randn(6, 8, **f), torch.randn(5, 8, **f), torch.randn(3, 2, 8, **f), torch.randn(3, 5, 2, **f)
        ids, dy = torch.zeros(6, dtype=torch.int32, **f), torch.randn(6, 5, **f)
        for kw in (dict(ddown=torch.zeros(3, 8, 2, **f)), dict(dup=torch.zeros(3, 2, 5, **f)), dict(dup=torch.zeros(2, 3, 5, **f))):
            with pytest.raises(ValueError):
                kkm.kkm_adapted_linear_grad(c, x, w, down, up, ids, dy, **kw)
            assert not next(iter(kw.values())).any()
        p, g, v = torch.randn(2, 6, 8, **f), torch.randn(2, 6, 8, **f), torch.zeros(2, 8, 6, **f)
        was = p.clone()
        with pytest.raises(ValueError):
            kkm.kkm_orthogonal_step(c, p, g, v, 0.1)
        assert not v.any() and torch.equal(p, was)
        z, lists, out = torch.randn(6, 40, **f), torch.zeros(6, 3, dtype=torch.int32, **f), torch.zeros(6, 40, **f)
        with pytest.raises(ValueError):
            kkm.kkm_choose(c, z, out, bias_ids=lists, bias=torch.ones(3, 6, **f))
        assert not out.any()
        flat = torch.zeros(96, **f)
        kkm.kkm_orthogonal_step(c, p, g, flat, 0.1)
        kkm.kkm_orthogonal_step(c, was, g, v.view(2, 6, 8), 0.1)
        assert torch.equal(flat, v.view(-1)) and torch.equal(p, was)
    finally:
        kkm.kkm_destroy(c)
