"""GPU tests of calls of more workgroups than one launch takes: the same bits as calls on parts of the batch."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def B():
    from paper_2209_04161_amd import binding
    binding.lib()
    return binding


def _randn(seed, *shape, dtype=torch.float16):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, device="cuda", generator=g, dtype=dtype)


def test_many_short_rows(B):
    """2^26 rows and some, of 8 elements, four to a workgroup of 256 threads."""
    rows, n = (1 << 26) + 5, 8
    x = _randn(1, rows, n)
    q, s = B.amsim_quantize_rows(x)
    w = torch.linspace(0.5, 2.0, n, device="cuda")
    f = B.amsim_rmsnorm_fwd(x, w, 1e-5, residual=x, q8=True, rstd=True)
    for lo, hi in ((0, 1000), ((1 << 21) - 7, (1 << 21) + 9), ((1 << 25) - 3, (1 << 25) + 5), (rows - 1001, rows)):
        p, t = B.amsim_quantize_rows(x[lo:hi])
        assert torch.equal(q[lo:hi], p) and torch.equal(s[lo:hi], t)
        part = B.amsim_rmsnorm_fwd(x[lo:hi], w, 1e-5, residual=x[lo:hi], q8=True, rstd=True)
        assert all(torch.equal(a[lo:hi], b) for a, b in zip(f, part))
    # every row was written: the largest integer of a row of scale s is 127
    assert torch.equal(q.abs().amax(1) == 127, s > 0)


def test_many_sequences(B):
    """2^24 pairs of sequence and head and more, the sequences' pages shared: one key each, or two."""
    batch, heads, d, page, pages = (1 << 19) + 3, 32, 16, 32, 5
    g = torch.Generator(device="cuda").manual_seed(2)
    k = torch.randint(-127, 128, (pages, heads, page, d), dtype=torch.int8, device="cuda", generator=g)
    v = torch.randint(-127, 128, (pages, heads, d, page), dtype=torch.int8, device="cuda", generator=g)
    scale = torch.rand((pages, heads), device="cuda", generator=g) * 0.02
    cache = B.Cache8(k, v, scale, scale + 0.01)
    table = torch.randint(0, pages, (batch, 1), dtype=torch.int32, device="cuda", generator=g)
    lens = torch.randint(1, 3, (batch,), dtype=torch.int32, device="cuda", generator=g)
    starts = torch.arange(batch + 1, dtype=torch.int32, device="cuda")
    q = _randn(3, batch, heads, d)
    out = B.amsim_cache_attention(cache, table, lens, q, starts, 1, 2)
    for lo in range(0, batch, 100001):
        hi = min(batch, lo + 100001)
        part = B.amsim_cache_attention(cache, table[lo:hi], lens[lo:hi], q[lo:hi], starts[:hi - lo + 1], 1, 2)
        assert torch.equal(out[lo:hi], part)


def test_an_append_of_many_pages(B):
    """Sequences of one new token beside one of 2050, whose pages set the number of workgroups for each."""
    batch, heads, d, page, long = 4096, 32, 16, 32, 2050
    news = [1] * (batch - 1) + [long]
    each = -(-long // page)
    total, pages = sum(news), batch - 1 + each
    table = torch.zeros((batch, each), dtype=torch.int32)
    table[:, 0] = torch.arange(batch)
    table[-1] = torch.arange(batch - 1, pages)
    table = table.cuda()
    lens = torch.tensor(news, dtype=torch.int32, device="cuda")
    starts = torch.arange(batch + 1, dtype=torch.int32, device="cuda")
    starts[-1] = total
    x, y = _randn(4, total, heads, d), _randn(5, total, heads, d)

    def empty():
        return B.Cache8(torch.zeros((pages, heads, page, d), dtype=torch.int8, device="cuda"),
                        torch.zeros((pages, heads, d, page), dtype=torch.int8, device="cuda"),
                        torch.zeros((pages, heads), device="cuda"), torch.zeros((pages, heads), device="cuda"))

    got, want = empty(), empty()
    B.amsim_cache_append(got, table, lens, x, y, starts, long)
    half = batch // 2
    B.amsim_cache_append(want, table[:half], lens[:half], x[:half], y[:half], starts[:half + 1], 1)
    B.amsim_cache_append(want, table[half:], lens[half:], x[half:], y[half:], (starts[half:] - half).contiguous(), long)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert bool((got.k_scale > 0).all())
