"""Scratch that the matrix operators ask for, on the CPU."""
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
