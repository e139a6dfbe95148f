"""GPU tests of wrong lengths and starts: what the calls do with them is what they do with the numbers cut to the
tensors, and nothing beside the tensors is written.

Tolerances are those of plain64.attention (derived there) and FP32's rounding."""
import numpy as np
import pytest

import plain64 as P
from test_gpu_cache8 import B, Batch, _np, _t  # noqa: F401  (B is a fixture)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

BIG = 2 ** 31 - 1
# lengths, starts as they are given; what they are cut to: lengths, first new row and new rows of each sequence
CASES = [
    ([BIG, -7], [0, 1, 3], [160, 0], [0, 1], [1, 2]),
    ([100, 70], [0, BIG, 3], [100, 70], [0, 3], [2, 0]),
    ([100, 70], [-4, 1, 900], [100, 70], [0, 1], [1, 2]),
    ([100, 1], [1, 0, 3], [100, 1], [1, 0], [0, 2]),
    ([1, 128], [0, 2, 3], [1, 128], [0, 2], [2, 1]),
]


def _guarded(t, fill):
    """t inside a larger tensor of `fill`: (the view, the whole)."""
    big = torch.full((t.shape[0] + 4,) + tuple(t.shape[1:]), fill, dtype=t.dtype, device="cuda")
    view = big[2:-2]
    view.copy_(t)
    return view, big


def _guards_whole(pairs, fills):
    return all(bool((big[:2] == f).all()) and bool((big[-2:] == f).all()) for (_, big), f in zip(pairs, fills))


@pytest.mark.parametrize("rows", [1, 40])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_numbers_are_cut_to_the_tensors(B, case, rows):
    """`rows` query heads to a key head: the attention of few rows and that of many."""
    given, starts, lens, first, news = CASES[case]
    bt = Batch(B, [100, 160], [1, 2], 1, 64, 32, 20 + case)  # pages for up to 160 tokens each
    spare = [p for p in range(bt.pages) if p not in set(bt.used.tolist())]
    bt.table = bt.table[:, :5].copy()
    bt.table[0, 4] = spare[0]
    bt.ks[spare[0]] = bt.vs[spare[0]] = 0.01
    fills = (77, 77, 7.0, 7.0)
    pairs = [_guarded(t, f) for t, f in zip(bt.cache(), fills)]
    cache = B.Cache8(*(view for view, _ in pairs))
    table = torch.from_numpy(bt.table).cuda()
    dl = torch.tensor(given, dtype=torch.int32, device="cuda")
    ds = torch.tensor(starts, dtype=torch.int32, device="cuda")
    q = _t(bt.rng.normal(0, 1, (3, rows, 64)))
    out, big = _guarded(torch.full((3, rows, 64), 7.0, device="cuda"), 7.0)
    B.amsim_cache_attention(cache, table, dl, q, ds, 2, 160, out=out)
    want = np.full((3, rows, 64), 7.0)
    tol = np.zeros((3, rows, 64))
    for b in range(2):
        if news[b]:
            at = slice(first[b], first[b] + news[b])
            want[at], tol[at] = P.attention(bt.k, bt.v, bt.ks, bt.vs, bt.table[b:b + 1], [lens[b]], [0, news[b]],
                                            _np(q)[at], 64 ** -0.5, terms16=False)
    assert np.all(np.abs(_np(out) - want) <= tol + 2 * P.EPS32 * np.abs(want))
    assert _guards_whole([(out, big)], (7.0,)) and _guards_whole(pairs, fills)
    x = _t(bt.rng.normal(0, 1, (3, 1, 64)))
    B.amsim_cache_append(cache, table, dl, x, x, ds, 2)
    wk, wks, wv, wvs = bt.k, bt.ks, bt.v, bt.vs
    for b in range(2):
        if news[b]:
            rows_b = _np(x)[first[b]:first[b] + news[b]]
            args = (bt.table[b:b + 1], [lens[b]], [0, news[b]], rows_b)
            wk, wks = P.append32(wk, wks, False, *args)
            wv, wvs = P.append32(wv, wvs, True, *args)
    for got, w in zip(cache, (wk, wv, wks, wvs)):
        np.testing.assert_array_equal(_np(got), w)
    assert _guards_whole(pairs, fills)
