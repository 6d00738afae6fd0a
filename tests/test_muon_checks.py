"""What the orthogonalised update refuses, before anything touches a GPU."""
import ctypes

import pytest
import torch

import paper_2510_00236_b200 as pe
from paper_2510_00236_b200 import build as pe_build


@pytest.fixture(scope="module")
def lib():
    pe_build.build_library()
    return pe.load_library()


@pytest.fixture(scope="module")
def p16():
    buf = ctypes.create_string_buffer(1 << 16)
    p16.keep = buf
    return (ctypes.addressof(buf) + 255) & ~255


def test_library_validates_orthogonalize(lib, p16):
    for f in (lib.pe_orthogonalize, lib.pe_orthogonalize_f32):
        def call(G=p16, count=1, rows=8, cols=8, steps=5, out=p16, ws=p16, n=1 << 15):
            return f(G, count, rows, cols, steps, out, ws, n, None)
        assert call(G=None) == 1 and call(out=None) == 1
        assert call(count=-1) == 2 and call(rows=0) == 2 and call(cols=-3) == 2 and call(count=65536) == 2
        assert call(rows=1 << 20, cols=1 << 20) == 2 and call(steps=0) == 2 and call(steps=101) == 2
        assert call(G=p16 + 2) == 3 and call(out=p16 + 2) == 3 and call(ws=p16 + 128) == 3
        assert call(ws=None) == 9 and call(n=100) == 9


def test_library_validates_muon_step(lib, p16):
    f = ctypes.c_float

    def call(theta=p16, lp=None, m=p16, g=p16, count=1, rows=8, cols=8, B=4, steps=5, ws=p16, n=1 << 15):
        return lib.muon_step(theta, lp, m, g, count, rows, cols, B, f(1.0), f(0.1), f(0.9), 1, steps, f(1.0), f(0.0), ws, n, None)
    assert call(theta=None) == 1 and call(m=None) == 1 and call(g=None) == 1
    assert call(B=0) == 2 and call(rows=0) == 2 and call(steps=0) == 2
    assert call(theta=p16 + 4) == 3 and call(lp=p16 + 2) == 3 and call(ws=p16 + 16) == 3
    assert call(ws=None) == 9 and call(n=8) == 9


def test_workspace_bytes(lib):
    need = pe.pe_orthogonalize_workspace_bytes
    assert need(0, 8, 8) == 0 and need(1, 0, 8) == 0 and need(-1, 8, 8) == 0
    assert need(2, 100, 300) == need(2, 300, 100)
    # two operands of two halves per entry (rows padded to 8), A and Q alike
    assert need(1, 512, 2048) >= 2 * 4 * 512 * 2048 + 2 * 4 * 512 * 512


def test_binding_refuses_what_the_library_cannot_see():
    G = torch.zeros(2, 8, 16)
    with pytest.raises(TypeError):
        pe.pe_orthogonalize(G.half())
    with pytest.raises(TypeError):
        pe.pe_orthogonalize_f32(G.to(torch.bfloat16))
    with pytest.raises(ValueError, match="G must"):
        pe.pe_orthogonalize(G.transpose(1, 2))
    with pytest.raises(ValueError, match="G must"):
        pe.pe_orthogonalize(torch.zeros(8))
    with pytest.raises(ValueError, match="out"):
        pe.pe_orthogonalize(G, out=torch.zeros(2, 16, 8))
    with pytest.raises(TypeError):
        pe.pe_orthogonalize(G, out=G.to(torch.bfloat16))
    with pytest.raises(ValueError, match="workspace"):
        pe.pe_orthogonalize(G, workspace=torch.zeros(1 << 16, dtype=torch.uint8)[::2])
    with pytest.raises(TypeError):
        pe.muon_step(G.to(torch.bfloat16), G, G, 4, lr=0.1, beta=0.9)
    with pytest.raises(ValueError, match="sum_g"):
        pe.muon_step(G, G.clone(), G[:1], 4, lr=0.1, beta=0.9)
    with pytest.raises(TypeError):
        pe.muon_step(G, G.clone(), G.clone(), 4, lr=0.1, beta=0.9, theta_lp=G.clone())
    with pytest.raises(pe.PestatsError):                # tensors on the CPU
        pe.pe_orthogonalize(G)


def test_the_shapes_whose_precision_is_tested_take_every_kind_of_product(lib):
    """Widths of tiles and slices follow an estimate of the time: should it change, the list of shapes has to change with it."""
    from test_gpu_muon_pairs import PRECISE
    taken = set()
    for count, rows, cols in PRECISE:
        for product in range(3):
            width, slices, _, at_a_time = pe.pe_plan_query(pe.PLAN_ORTHOGONALIZE, product, count, 1, cols, rows, 148)
            taken.add((product, at_a_time, width, slices > 1))
    assert taken >= {(product, at_a_time, width, False) for product in range(3) for at_a_time in (1, 2) for width in (64, 128, 256)}
    # X X^T in slices; the other products never are
    assert taken >= {(0, 1, 64, True), (0, 1, 256, True), (0, 2, 64, True), (0, 2, 128, True), (0, 2, 256, True)}
    assert not any(sliced for product, _, _, sliced in taken if product)


def test_plan_queries_of_the_orthogonalised_update(lib):
    for bad in ((3, 1, 64, 64), (-1, 1, 64, 64), (0, 65536, 1, 1), (0, 1, 1 << 30, 1 << 30)):
        with pytest.raises(pe.PestatsError):
            pe.pe_plan_query(pe.PLAN_ORTHOGONALIZE, bad[0], bad[1], 1, bad[3], bad[2], 148)
    assert pe.pe_plan_query(pe.PLAN_ORTHOGONALIZE, 0, 3, 1, 128, 64, 148)[0] == 0 and pe.pe_plan_query(pe.PLAN_ORTHOGONALIZE, 0, 3, 1, 64, 128, 148)[0] == 0
    assert pe.pe_plan_query(pe.PLAN_ORTHOGONALIZE, 0, 1, 1, 129, 64, 148)[0] > 0
