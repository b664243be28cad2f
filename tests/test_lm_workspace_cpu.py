"""Workspace sizes of the local step's operators over the whole range of sizes (host only)."""

import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_2504_17672_b200 import build
    build.build()
    from paper_2504_17672_b200 import binding
    return binding.library()


def test_sizes_that_the_calls_refuse_have_no_workspace(lib):
    for V, D, T in ((2 ** 30 + 1, 8, 8), (8, 2 ** 31, 8), (8, 8, 2 ** 27 + 1), (2 ** 40, 2 ** 40, 2 ** 40), (-1, 8, 8), (8, -1, 8), (8, 8, -1)):
        assert lib.cocodc_lm_embed_grad_workspace(V, D, T) == 0, (V, D, T)
    for T, D, F in ((2 ** 31, 8, 8), (8, 2 ** 31, 8), (8, 8, 2 ** 31), (2 ** 40, 8, 2 ** 40), (2 ** 32, 8, 2 ** 30), (-1, 8, 8), (8, -1, 8), (8, 8, -1)):
        assert lib.cocodc_lm_glu_grad_workspace(T, D, F) == 0, (T, D, F)


def test_the_largest_sizes_do_not_wrap(lib):
    """Exact integers: what the kernels are known to write, at sizes whose byte counts come near 2^64."""
    most = 2 ** 31 - 1
    for T, F in ((most, most), (most, 1), (1, most), (2 ** 30 + 5, 2 ** 31 - 9)):
        assert lib.cocodc_lm_glu_grad_workspace(T, 8, F) >= 4 * T * ((F + 7) // 8 * 8)
    for V, D, T in ((2 ** 30, most, 2 ** 27), (2 ** 30, 1, 2 ** 27), (1, most, 2 ** 27)):
        assert lib.cocodc_lm_embed_grad_workspace(V, D, T) >= 4 * V + 8 * T + T // 128 * 2 * D * 4
