"""GPU tests of where the attention writes: any layout of tokens and heads whose elements lie apart, and no other."""
import pytest

from test_gpu_cache8 import B, Batch, _t  # noqa: F401  (B is a fixture)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("new", [1, 3, 40])
def test_layouts_of_the_result(B, new):
    bt = Batch(B, [90], [new], 2, 64, 32, new)
    q = _t(bt.rng.normal(0, 1, (new, 4, 64)))
    want = bt.attend(q)
    empty = lambda *s: torch.full(s, 7.0, device="cuda")  # noqa: E731
    for out in (empty(4, new, 64).transpose(0, 1), empty(new, 4, 65)[:, :, :64], empty(new, 9, 64)[:, ::2][:, :4],
                empty(5, new, 80)[:4, :, 3:67].transpose(0, 1), empty(new * 2, 4, 64)[::2]):
        bt.attend(q, out=out)
        assert torch.equal(out, want)
    wrong = [empty(new, 1, 64).expand(new, 4, 64), torch.as_strided(empty(new * 300), (new, 4, 64), (300, 32, 1))]
    if new > 1:
        wrong += [empty(1, 4, 64).expand(new, 4, 64), torch.as_strided(empty(new * 300), (new, 4, 64), (255, 64, 1))]
    for out in wrong:
        with pytest.raises(ValueError):
            bt.attend(q, out=out)
