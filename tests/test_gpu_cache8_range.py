"""GPU tests of the cache's attention at values near both ends of FP32's range: the sums of P times values stay those of
P up to 1, however P is held.

Tolerances are those of plain64.attention (derived there) and the result type's rounding; below 2^-112 a page's scale
and below 2^-126 a result may read as zero, 127 and 1 of them."""
import numpy as np
import pytest

import plain64 as P
from test_gpu_cache8 import B, Batch, _np, _t  # noqa: F401  (B is a fixture)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("typ", ["float32", "bfloat16"])
@pytest.mark.parametrize("magnitude", [2e35, 1e33, 1e-28, 1e-30])
@pytest.mark.parametrize("length,new,d,page", [(200, 1, 64, 64), (1000, 1, 128, 32), (5000, 1, 64, 64), (700, 40, 64, 32),
                                               (300, 2, 256, 64), (3000, 70, 128, 64)])
def test_large_and_small_values(B, length, new, d, page, magnitude, typ):
    bt = Batch(B, [length], [new], 2, d, page, length)
    bt.vs[bt.used] = np.float32(magnitude / 127) * bt.rng.uniform(0.1, 1.0, (len(bt.used), 2)).astype(np.float32)
    q = _t(bt.rng.normal(0, 1, (new, 4, d)), typ)
    got = _np(bt.attend(q))
    want, tol = P.attention(bt.k, bt.v, bt.ks, bt.vs, bt.table, bt.lengths, bt.starts, _np(q), d ** -0.5,
                            terms16=typ != "float32")
    assert np.all(np.abs(got - want) <= tol + 1.01 * P.U[typ] * np.abs(want) + 127 * 2.0 ** -112)
