"""The largest numbers of matrices and columns fit a launch: their sizes pass and the workspace is looked at next."""
import ctypes

import paper_2510_00236_b200 as pe
from paper_2510_00236_b200 import build as pe_build


def test_many_small_matrices_and_very_long_ones():
    pe_build.build_library()
    lib = pe.load_library()
    buf = ctypes.create_string_buffer(4096)
    p = (ctypes.addressof(buf) + 255) & ~255
    for count, rows, cols in ((65535, 1, 1048576), (1, 1 << 30, 1), (63, 1, 1 << 30), (1, 1 << 18, (1 << 18) - 1)):
        assert lib.pe_orthogonalize_f32(p, count, rows, cols, 5, p, p, 1 << 11, None) == 9      # PE_ERR_WORKSPACE
    assert lib.pe_orthogonalize_f32(p, 64, 1, 1 << 30, 5, p, p, 1 << 11, None) == 2              # PE_ERR_DIM
