"""GPU tests of the attention of many rows where the value scales of a sequence's pages lie far apart: a row whose
pages are small beside others that it does not see, teams and chunks of keys of either kind.

Tolerances are those of plain64.attention (derived there) and the result type's rounding."""
import numpy as np
import pytest

from test_gpu_cache8 import TYPES, B, Batch, _np, _t  # noqa: F401  (B is a fixture)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _rows(bt, got, q, typ, see, window=0):
    """Checks the rows of sequence 0 that `see` names against the definition."""
    import plain64 as P
    want, tol = P.attention(bt.k, bt.v, bt.ks, bt.vs, bt.table, bt.lengths, bt.starts, _np(q), bt.d ** -0.5, True, window,
                            terms16=typ != "float32")
    tol = tol + 1.01 * P.U[typ] * np.abs(want) + 2.0 ** -24 * (typ == "float16")
    assert np.all(np.abs(_np(got) - want)[see] <= tol[see])
    assert np.abs(want[see]).max() > 0


@pytest.mark.parametrize("typ", TYPES)
@pytest.mark.parametrize("small,large", [(1e-3, 1e18), (1e-20, 1e10), (1e-30, 1e34), (0.02, 1e5)])
@pytest.mark.parametrize("d,heads,page", [(64, 1, 32), (128, 1, 64), (192, 1, 64), (128, 1, 32)])
def test_a_large_page_after_the_rows(B, d, heads, page, small, large, typ):
    """A later page, of keys that the first rows do not see, is the one whose scale is large."""
    bt = Batch(B, [160], [160], heads, d, page, d + page)
    bt.vs[bt.table[0, :-1]] = small
    bt.vs[bt.table[0, 64 // page]] = large
    q = _t(bt.rng.normal(0, 1, (160, heads, d)), typ)
    got = bt.attend(q)
    _rows(bt, got, q, typ, slice(0, 64))
    if typ != "float16":
        _rows(bt, got, q, typ, slice(64, 160))


@pytest.mark.parametrize("typ", ["float32", "bfloat16"])
def test_a_large_page_with_many_workgroups(B, typ):
    """One team of waves to a workgroup."""
    bt = Batch(B, [130], [130], 130, 64, 64, 9)
    bt.vs[bt.table[0, :-1]] = 1e-20
    bt.vs[bt.table[0, 1]] = 1e10
    q = _t(bt.rng.normal(0, 1, (130, 130, 64)), typ)
    _rows(bt, bt.attend(q), q, typ, slice(0, 130))


@pytest.mark.parametrize("typ", TYPES)
@pytest.mark.parametrize("small,large", [(1e-3, 1e18), (1e-20, 1e10), (1e-30, 1e34)])
@pytest.mark.parametrize("d,page", [(64, 32), (128, 64), (256, 128)])
def test_a_large_page_that_the_window_has_left(B, d, page, small, large, typ):
    bt = Batch(B, [300], [300], 1, d, page, d + page)
    bt.vs[bt.table[0, :-1]] = small
    bt.vs[bt.table[0, 0]] = large
    q = _t(bt.rng.normal(0, 1, (300, 1, d)), typ)
    got = bt.attend(q, window=20)
    _rows(bt, got, q, typ, slice(page + 20, 300), 20)
    if typ != "float16":
        _rows(bt, got, q, typ, slice(0, 300), 20)


@pytest.mark.parametrize("typ", ["float32", "bfloat16"])
@pytest.mark.parametrize("step", [2.0 ** -30, 2.0 ** -12, 2.0 ** 12, 2.0 ** 30])
@pytest.mark.parametrize("new", [64, 600])
def test_scales_that_rise_and_fall(B, new, step, typ):
    """Page after page, up or down by a factor, to the ends of what a scale can be, over several tiles of rows."""
    bt = Batch(B, [600], [new], 1, 64, 64, new)
    scale = 1.0 if step < 1 else 2.0 ** -60
    for p in bt.table[0, :10]:
        bt.vs[p] = scale
        scale = min(max(scale * step, 2.0 ** -100), 2.0 ** 100)
    q = _t(bt.rng.normal(0, 1, (new, 3, 64)), typ)
    _rows(bt, bt.attend(q), q, typ, slice(0, new))


@pytest.mark.parametrize("typ", ["float32", "bfloat16"])
def test_chunks_of_small_and_of_large_pages(B, typ):
    """Long contexts whose chunks of keys hold pages of one kind, or of both."""
    bt = Batch(B, [5000], [70], 1, 64, 64, 1)
    q = _t(bt.rng.normal(0, 1, (70, 2, 64)), typ)
    for large in (slice(0, 16), slice(20, 21), slice(77, 78), slice(0, 78, 3)):
        bt.vs[bt.table[0, :-1]] = 1e-25
        bt.vs[bt.table[0, :78][large]] = 1e12
        _rows(bt, bt.attend(q), q, typ, slice(0, 70))
        _rows(bt, bt.attend(q, window=400), q, typ, slice(0, 70), 400)
