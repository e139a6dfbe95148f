"""GPU tests of what Decoder8 takes from the model that it is made of: the weights as they were, and nothing of the model
itself."""
import copy
import gc
import weakref

import numpy as np
import pytest

from test_gpu_decoder import _model, _x

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _serve(served, x):
    cache = served.cache(pages=2)
    s = cache.add()
    return served(x, cache, cache.extend([(s, x.shape[0])]))


def test_training_on_leaves_the_served_model_as_it_was():
    from paper_2209_04161_amd import decoder
    model = _model()
    served = decoder.Decoder8(model)
    x = _x(40, 1)
    want = _serve(served, x)
    with torch.no_grad():
        for p in model.parameters():
            p += 0.5
    assert torch.equal(_serve(served, x), want)


def test_a_conversion_of_the_served_model_leaves_the_trained_one():
    from paper_2209_04161_amd import decoder
    model = _model()
    before = [p.detach().clone() for p in model.parameters()]
    decoder.Decoder8(model).half()
    assert all(p.dtype == torch.float32 and torch.equal(p, b) for p, b in zip(model.parameters(), before))


def test_the_trained_model_can_be_given_up():
    from paper_2209_04161_amd import decoder
    model = _model()
    parts = [weakref.ref(m) for m in model.modules()] + [weakref.ref(p) for p in model.parameters()]
    served = decoder.Decoder8(model)
    del model
    gc.collect()
    assert not any(r() is not None for r in parts)
    x = _x(33, 2)
    again = copy.deepcopy(served)
    assert torch.equal(_serve(again, x), _serve(served, x))
    assert np.isfinite(_serve(again, x).cpu().numpy()).all()
