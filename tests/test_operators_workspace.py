"""Scratch that the matrix operators ask for, on the CPU."""
import ctypes
import os

import pytest

import paper_1802_02422_amd as ivf


@pytest.fixture(autouse=True, scope="module")
def library():
    if not os.path.exists(ivf.library_path()):
        from paper_1802_02422_amd.build import build_library
        build_library()


def test_orthogonalising_small_matrices_needs_none_for_them():
    """One launch takes matrices up to 128 x 128 through all steps: what is asked for does not grow with their number."""
    for rows, cols in ((1, 1), (96, 96), (128, 128), (128, 3)):
        for batch in (0, 1, 4096, 1 << 20):
            assert 0 < ivf.ivf_orthogonalise_workspace(batch, rows, cols) <= 1 << 14
    # past that: five matrices in two terms
    assert 5 * 2 * 2 * 256 * 256 <= ivf.ivf_orthogonalise_workspace(1, 256, 256) <= 6 * 2 * 2 * 256 * 256


def test_products_with_4_bit_rows_need_none_for_rows_of_no_whole_words():
    """b's values are expanded only for rows that are copied straight into LDS: of a multiple of eight components, on 16-byte boundaries."""
    import torch
    assert ivf.ivf_mx4_rows_product_workspace(4096, 8192, 1024, dtype=torch.bfloat16) == 8192 * 1024 * 2
    assert ivf.ivf_mx4_rows_product_workspace(4096, 8192, 1023, dtype=torch.bfloat16) == 0
    # through the pointer (refused for the one without room, before anything is launched)
    P, lib = ctypes.c_void_p(4096), ivf.load_library()
    assert lib.ivf_mx4_rows_product(P, 1024, 4096, 2, P, P, 8192, 1024, 0, P, 8192, 2, None, 0, None) == -1
    assert "workspace" in ivf.ivf_last_error()
