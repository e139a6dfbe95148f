"""Host-side checks of what the 8-bit decoder's calls refuse at their limits, before anything is launched (no GPU)."""
import ctypes
import os

import pytest

from paper_2209_04161_amd import binding as B


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(B.library_path()):
        from paper_2209_04161_amd import build
        build.build()
    return B.lib()


def test_products_of_more_threads_than_a_launch_takes_are_refused(L):
    p, nb = 4096, ctypes.c_size_t(-1).value

    def gemm(m, n, k, lda, ldb, a=p):
        return L.amsim_gemm_i8(m, n, k, a, lda, p, p, ldb, p, None, B.AMSIM_BF16, p, n, p, nb, None)

    # 2^26 tiles of 64 x 64, whose rows lie at any address
    assert gemm(1 << 19, 1 << 19, 16, 17, 17) == B.AMSIM_ERR_UNSUPPORTED
    # 2^33 pieces of 16 bytes to copy
    assert gemm(1 << 20, 1 << 20, 65537, 65537, 65537) == B.AMSIM_ERR_UNSUPPORTED


def test_a_scale_that_is_no_finite_number_is_refused(L):
    """As a NaN it would be lost in the maximum that keeps a factor above zero: weights alike for every key."""
    p = 4096
    cache = B.amsim_cache8(p, p, p, p, 4, 32, 2, 64)

    def attend(scale, new):
        return L.amsim_cache_attention(ctypes.byref(cache), 1, p, 200, p, p, new, new, 5000, B.AMSIM_F32, 4, p, 256, 64,
                                       scale, 1, 0, p, 256, 64, p, 1 << 40, None)

    for new in (1, 100):
        for scale in (float("nan"), float("inf"), float("-inf"), 3e38):
            assert attend(scale, new) == B.AMSIM_ERR_INVALID_ARG
