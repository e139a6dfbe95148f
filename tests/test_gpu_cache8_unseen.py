"""GPU tests of the attention of many rows beside pages that no row of a tile sees: a page past a sequence's end or
before its window, whose number is a page of the cache and whose scales are finite and as large as memory may hold.

Tolerances are those of plain64.attention (derived there) and the result type's rounding."""
import numpy as np
import pytest

from test_gpu_cache8 import TYPES, B, Batch, _t  # noqa: F401  (B is a fixture)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _foreign(bt, value, window=0):
    """Entries past a sequence's pages name a spare page; its scales, and those of the pages that no new token sees,
    are `value`."""
    spare = [p for p in range(bt.pages) if p not in set(bt.used.tolist())]
    for b, (length, new) in enumerate(zip(bt.lengths, bt.news)):
        held = -(-length // bt.page)
        bt.table[b, held:] = spare[b % len(spare)]
        first = max(0, length - new - window + 1) if window else 0
        for p in bt.table[b, :min(held, first // bt.page)]:
            bt.ks[p] = bt.vs[p] = value
    bt.ks[spare] = bt.vs[spare] = value


@pytest.mark.parametrize("typ", TYPES)
@pytest.mark.parametrize("value", [1e6, 1e12, 1e30])
@pytest.mark.parametrize("d,heads", [(64, 1), (128, 2), (192, 1)])
def test_pages_past_the_end(B, d, heads, value, typ):
    """Pages of 32 tokens, sequences that end in the first half of a tile of 64 keys."""
    lengths, news = [90, 32, 145, 70], [40, 32, 100, 35]
    bt = Batch(B, lengths, news, heads, d, 32, d)
    q = _t(bt.rng.normal(0, 1, (bt.total, heads, d)), typ)
    clean = bt.attend(q)
    _foreign(bt, value)
    got = bt.attend(q)
    bt.check(q, got, typ)
    assert torch.equal(got, clean)


@pytest.mark.parametrize("typ", TYPES)
@pytest.mark.parametrize("value", [1e12, 1e30])
@pytest.mark.parametrize("d,window", [(64, 30), (128, 20), (256, 35)])
def test_pages_before_the_window(B, d, window, value, typ):
    """The first keys that the window leaves lie in the second half of a tile of 64."""
    bt = Batch(B, [300, 299], [40, 38], 1, d, 32, d + window)
    q = _t(bt.rng.normal(0, 1, (bt.total, 2, d)), typ)
    clean = bt.attend(q, window=window)
    _foreign(bt, value, window)
    got = bt.attend(q, window=window)
    bt.check(q, got, typ, True, window)
    assert torch.equal(got, clean)


@pytest.mark.parametrize("typ", TYPES)
def test_pages_past_the_end_of_long_sequences(B, typ):
    """Chunks of keys with a team or two, and with more workgroups than compute units."""
    bt = Batch(B, [5000, 2080], [70, 33], 1, 64, 32, 3)
    q = _t(bt.rng.normal(0, 1, (bt.total, 2, 64)), typ)
    _foreign(bt, 1e30)
    bt.check(q, bt.attend(q), typ)
    bt = Batch(B, [97] * 9, [97] * 9, 30, 64, 32, 4)
    q = _t(bt.rng.normal(0, 1, (bt.total, 30, 64)), typ)
    _foreign(bt, 1e30)
    bt.check(q, bt.attend(q), typ)
    assert np.isfinite(bt.vs).all()
