"""GPU tests of the norm's autograd layer: second derivatives are refused, and the weight gradient is within the bound of
the sum that the kernels form."""
import numpy as np
import pytest

import plain64 as P
from test_gpu_rmsnorm import TYPES, B, _inputs, _np  # noqa: F401  (B is a fixture)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def test_second_derivatives_are_refused(B):
    from paper_2209_04161_amd import modules
    x, r, w = _inputs(4, 33, "float32", 1)
    for t in (x, r, w):
        t.requires_grad_()
    y, h = modules.rms_norm(x, w, residual=r)
    (g,) = torch.autograd.grad((y * y).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        ((y * y).sum() + (g * g).sum()).backward()


@pytest.mark.parametrize("typ", TYPES)
@pytest.mark.parametrize("rows,n", [(1, 7), (63, 64), (1024, 33), (1025, 1024), (3000, 200), (4100, 1500)])
def test_weight_gradient_within_the_bound_of_its_sum(B, rows, n, typ):
    """An owner adds its rows one after the other (a row to each of 1024 workgroups, or of 4096 waves up to 1024
    elements, in turn), 64 threads each add up to 64 owners, six levels add those: each term passes at most
    ceil(rows / owners) + 64 + 6 additions, and two roundings (h rstd, and the first sum's) of its own."""
    x, r, w = _inputs(rows, n, typ, rows + n)
    dy, _, _ = _inputs(rows, n, typ, rows + n + 1)
    f = B.amsim_rmsnorm_fwd(x, w, 1e-5, residual=r, rstd=True)
    _, dw = B.amsim_rmsnorm_bwd(dy, f.h, w, f.rstd)
    _, want, _, size = P.rmsnorm_bwd(_np(dy), _np(f.h), _np(w), _np(f.rstd))
    owners = 4096 if n <= 1024 else 1024
    assert np.all(np.abs(_np(dw) - want) <= (-(-rows // owners) + 64 + 6 + 2) * P.EPS32 * size)
