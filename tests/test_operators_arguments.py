"""What the binding of the matrix operators refuses before it looks at a device: every wrong argument is an IvfError (on the CPU)."""
import os

import pytest
import torch

import paper_1802_02422_amd as ivf

T = torch.zeros


@pytest.fixture(autouse=True, scope="module")
def library():
    if not os.path.exists(ivf.library_path()):
        from paper_1802_02422_amd.build import build_library
        build_library()


ROWS = ivf.Mx4Rows(T(4, 16, dtype=torch.uint8), T(4, 1, dtype=torch.uint8), 6)
BAD = {
    "rows_list": lambda: ivf.ivf_grouped_product([[1.0]], T(2, 3, 4), T(3, dtype=torch.int32)),
    "rows_none": lambda: ivf.ivf_grouped_product(None, T(2, 3, 4), T(3, dtype=torch.int32)),
    "rows_number": lambda: ivf.ivf_grouped_product(torch.tensor(1.0), T(2, 3, 4), T(3, dtype=torch.int32)),
    "matrices_list": lambda: ivf.ivf_grouped_product(T(2, 4), [1.0], T(3, dtype=torch.int32)),
    "offsets_list": lambda: ivf.ivf_grouped_gradient(T(2, 3), T(2, 4), [0, 2]),
    "offsets_number": lambda: ivf.ivf_grouped_gradient(T(2, 3), T(2, 4), torch.tensor(0, dtype=torch.int32)),
    "gradient_list": lambda: ivf.ivf_grouped_gradient([1.0], T(2, 4), T(2, dtype=torch.int32)),
    "matrix_list": lambda: ivf.ivf_orthogonalise([[1.0]], [(1.5, -0.5, 0.0)]),
    "quantise_list": lambda: ivf.ivf_mx4_quantise([[1.0]]),
    "not_4_bits": lambda: ivf.ivf_mx4_expand(T(4, 16)),
    "codes_list": lambda: ivf.ivf_mx4_expand(ivf.Mx4Rows([1], T(4, 1, dtype=torch.uint8), 6)),
    "codes_flat": lambda: ivf.ivf_mx4_expand(ivf.Mx4Rows(T(64, dtype=torch.uint8), T(4, dtype=torch.uint8), 6)),
    "one_side": lambda: ivf.ivf_mx4_product(ROWS, T(4, 6)),
    "other_side": lambda: ivf.ivf_mx4_rows_product(T(4, 6), T(4, 6)),
    "rows_list_4_bits": lambda: ivf.ivf_mx4_rows_product([[1.0]], ROWS),
}


@pytest.mark.parametrize("which", BAD)
def test_refused(which):
    with pytest.raises(ivf.IvfError):
        BAD[which]()
