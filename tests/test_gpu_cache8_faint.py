"""GPU tests of the attention of many rows whose weight lies in many faint keys, in pages of zeros or of values far
smaller than another page's.

Every sequence holds one key of score s, the other n of score 0: with p = e^-s the result is
(x0 + p n x1) / (1 + n p) for the values x0 of the first key and x1 of all others.  Tolerance: a score is off
by at most (d + 8) 2^-24 s, p by twice that and 2^-21, each P is rounded to 11 bits (2^-11; 22 for FP32), in the sums'
ratio at most twice, the sums by (n / 64 + 80) 2^-23, then the result's type.  P is held down to 2^-39 of the
largest: n 2^-39 of the sum."""
import math

import numpy as np
import pytest

import plain64 as P
from test_gpu_cache8 import TYPES, B, _np  # noqa: F401  (B is a fixture)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

D = 64


@pytest.mark.parametrize("typ", TYPES)
@pytest.mark.parametrize("length,s", [(4096, 13.6), (16384, 13.6), (16384, 10.0), (16384, 16.0)])
@pytest.mark.parametrize("ratio", [0.0, 2.0 ** -22, 2.0 ** -19, 2.0 ** -10, 2.0 ** -40])
@pytest.mark.parametrize("page", [32, 64])
def test_one_key_and_many_faint_ones(B, page, ratio, length, s, typ):
    batch, heads, new = 64, 4, 33  # so many workgroups that each takes all keys
    pages = length // page
    k = torch.zeros((pages, heads, page, D), dtype=torch.int8, device="cuda")
    v = torch.full((pages, heads, D, page), 100, dtype=torch.int8, device="cuda")
    k[0, :, 0] = 100
    v[0] = 0
    v[0, :, :, 0] = 127
    ks = torch.full((pages, heads), s / (100 * D * 0.125), device="cuda")
    vs = torch.full((pages, heads), 0.02 * ratio, device="cuda")
    vs[0] = 0.02
    table = torch.arange(pages, dtype=torch.int32, device="cuda").repeat(batch, 1)
    lens = torch.full((batch,), length, dtype=torch.int32, device="cuda")
    starts = torch.arange(batch + 1, dtype=torch.int32, device="cuda") * new
    q = torch.ones((batch * new, heads, D), device="cuda").to(getattr(torch, typ))
    got = _np(B.amsim_cache_attention(B.Cache8(k, v, ks, vs), table, lens, q, starts, new, length, scale=0.125))
    n = np.arange(length - new, length, dtype=np.float64)  # keys that each new token sees beside the first
    score = 100.0 * D * 0.125 * float(ks[0, 0])
    p = math.exp(-score)
    x0, x1 = 127 * float(vs[0, 0]), 100 * float(vs[1, 0])
    want = (x0 + p * (n - page + 1) * x1) / (1 + n * p)
    rel = (2 * (D + 8) * P.EPS32 * score + 2.0 ** -21 + (2.0 ** -20 if typ == "float32" else 2.0 ** -10)
           + (n / 64 + 80) * 2 * P.EPS32 + n * 2.0 ** -39)
    tol = (rel + 1.01 * P.U[typ]) * want + 2.0 ** -24 * (typ == "float16")
    got = got.reshape(batch, new, heads, D).astype(np.float64)
    off = np.abs(got - want[None, :, None, None])
    assert np.all(off <= tol[None, :, None, None]), float((off / tol[None, :, None, None]).max())
