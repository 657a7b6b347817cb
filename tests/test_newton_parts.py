"""The measure of the tiled orthogonalised update's accuracy tells a right result from wrong ones."""
import pytest

import newton_parts as ref

torch = pytest.importorskip("torch")
from paper_2601_17136_amd import kkm  # noqa: E402

COEF = [kkm.KKM_QUINTIC] * 5


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("m,n", [(65, 65), (66, 130), (257, 65), (129, 257), (300, 301)])
def test_what_passes(m, n, dtype):
    u = torch.randn(m, n, generator=torch.Generator().manual_seed(m + n)).to(dtype)
    want = ref.exact(u, COEF, 1e-7)
    room = ref.room(u, want, COEF, 1e-7)
    for fine in (want, ref.parts(u, COEF, 1e-7, 2), ref.fp32(u, COEF, 1e-7)):
        assert ref.beyond(fine.to(dtype), want) <= room
    for wrong in (torch.zeros_like(want), ref.exact(u, COEF[:4], 1e-7), ref.parts(u, COEF, 1e-7, 1),
                  ref.exact(u.bfloat16() if dtype != torch.bfloat16 else (u.double() * (1 + 2.0 ** -9 * torch.randn(m, n))), COEF, 1e-7)):
        assert ref.beyond(wrong.to(dtype), want) > 4 * room


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_half_a_step(dtype):
    """A rounded value is nothing beyond it, a zero or a neighbour of it is, at every size."""
    want = torch.exp2(torch.arange(-13, 4).double()) * 1.3
    got = want.to(dtype)
    assert ref.beyond(got, want) == 0.0
    for i in range(want.numel()):
        off = got.clone()
        off[i] = 0.0
        assert ref.beyond(off, want) >= 0.9 * float(want[i]) - 2.0 ** -24
        off[i] = got[i] * (1 + 2 * torch.finfo(dtype).eps)
        assert ref.beyond(off, want) > 0.5 * torch.finfo(dtype).eps * float(want[i])
