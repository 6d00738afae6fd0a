"""Sizes whose products would need more thread blocks than a launch has are refused before anything is enqueued."""
import ctypes

import paper_2510_00236_b200 as pe
from paper_2510_00236_b200 import build as pe_build


def test_more_tiles_than_a_launch_has():
    pe_build.build_library()
    lib = pe.load_library()
    buf = ctypes.create_string_buffer(4096)
    p = (ctypes.addressof(buf) + 255) & ~255
    # 65535 matrices of 1 x 1048577: 16385 tiles of 64 columns each, two blocks a tile
    assert lib.pe_orthogonalize_f32(p, 65535, 1, 1048577, 5, p, p, 1 << 11, None) == 2
    assert lib.pe_orthogonalize_f32(p, 65534, 1, 1048576, 5, p, p, 1 << 11, None) == 9       # fits: then the workspace is looked at
