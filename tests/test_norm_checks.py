"""What the normalisation layers' entry points refuse, before anything touches a GPU."""
import ctypes

import pytest
import torch

import paper_2510_00236_b200 as pe
from paper_2510_00236_b200 import build as pe_build

BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def lib():
    pe_build.build_library()
    return pe.load_library()


@pytest.fixture(scope="module")
def p16():
    buf = ctypes.create_string_buffer(1 << 16)
    p16.keep = buf
    return (ctypes.addressof(buf) + 255) & ~255


def test_library_validates_the_forward_pass(lib, p16):
    for f, al in ((lib.pe_norm_forward, 2), (lib.pe_norm_forward_f32, 2)):
        assert f(None, None, None, 4, 8, 0, 1e-5, p16, None, None, None) == 1           # PE_ERR_NULL
        assert f(p16, None, None, 4, 8, 0, 1e-5, None, None, None, None) == 1
        assert f(p16, None, None, -1, 8, 0, 1e-5, p16, None, None, None) == 2           # PE_ERR_DIM
        assert f(p16, None, None, 4, 0, 0, 1e-5, p16, None, None, None) == 2
        assert f(p16, None, None, 1 << 38, 8, 0, 1e-5, p16, None, None, None) == 2
        assert f(p16, None, None, 4, 8, 0, -1.0, p16, None, None, None) == 2
        assert f(p16, None, None, 4, 8, 0, float("nan"), p16, None, None, None) == 2
        assert f(p16, None, None, 4, 8, 2, 1e-5, p16, None, None, None) == 5            # PE_ERR_PHI
        assert f(p16 + al, None, None, 4, 8, 0, 1e-5, p16, None, None, None) == 3       # PE_ERR_ALIGN
        assert f(p16, p16 + 2, None, 4, 8, 0, 1e-5, p16, None, None, None) == 3
        assert f(p16, None, None, 4, 8, 0, 1e-5, p16, None, p16 + 1, None) == 3


def test_library_validates_the_backward_pass(lib, p16):
    for f in (lib.pe_norm_backward, lib.pe_norm_backward_f32):
        def call(x=p16, dy=p16, gain=None, mean=p16, rstd=p16, B=2, T=3, d=8, kind=0, phi=1, acc=0, dx=p16, gs=None, gt=None, bs=None, bt=None, ws=p16, n=1 << 15):
            return f(x, dy, gain, mean, rstd, B, T, d, kind, phi, acc, dx, gs, gt, bs, bt, ws, n, None)
        assert call(x=None) == 1 and call(dy=None) == 1 and call(rstd=None) == 1 and call(mean=None) == 1
        assert call(dx=None) == 1                                                        # nothing to compute
        assert call(B=-1) == 2 and call(T=-1) == 2 and call(d=0) == 2 and call(B=1 << 30, T=1 << 10) == 2
        assert call(kind=3) == 5 and call(phi=3) == 5 and call(phi=-1) == 5
        assert call(x=p16 + 2) == 3 and call(dx=p16 + 2) == 3 and call(gs=p16 + 2) == 3 and call(mean=p16 + 1) == 3


def test_library_validates_the_packed_backward_pass(lib, p16):
    def call(offs=p16, B=2, rows=6, d=8, dx=p16):
        return lib.pe_norm_backward_ragged(p16, p16, None, p16, p16, offs, B, rows, d, 0, 1, 0, dx, None, None, None, None, p16, 1 << 15, None)
    assert call(offs=None) == 1 and call(rows=1 << 31) == 2 and call(B=-1) == 2 and call(offs=p16 + 2) == 3 and call(dx=None) == 1


def test_workspace_bytes(lib):
    need = pe.pe_norm_backward_workspace_bytes
    assert need(0, 64) == 0 and need(-1, 64) == 0 and need(16, 0) == 0
    assert need(128, 64) % 256 == 0
    # rows wider than a block leave their two means there
    assert need(1000, 8192) >= 8 * 1000
    # never more than the elements of 592 blocks, their flags and the means
    for rows, d in ((1 << 18, 2048), (1 << 20, 64), (1 << 12, 4096), (1 << 12, 16384)):
        assert need(rows, d) <= 592 * 8 * d * 4 + 8 * rows + (1 << 14)


def test_binding_refuses_what_the_library_cannot_see():
    x = torch.zeros(2, 3, 16, dtype=BF16)
    r = torch.zeros(2, 3)
    with pytest.raises(TypeError):
        pe.pe_norm_forward(x.half())
    with pytest.raises(TypeError):
        pe.pe_norm_forward_f32(x)
    with pytest.raises(ValueError, match="contiguous"):
        pe.pe_norm_forward(x.transpose(0, 1))
    with pytest.raises(ValueError, match="gain"):
        pe.pe_norm_forward(x, torch.zeros(15))
    with pytest.raises(ValueError, match="gain"):
        pe.pe_norm_forward(x, torch.zeros(16, dtype=BF16))
    with pytest.raises(ValueError, match="bias"):
        pe.pe_norm_forward(x, None, torch.zeros(16, device="meta"))
    with pytest.raises(ValueError, match="rstd"):
        pe.pe_norm_forward(x, rstd=torch.zeros(6))
    with pytest.raises(TypeError):
        pe.pe_norm_forward(x, out=torch.zeros(2, 3, 16))
    with pytest.raises(KeyError):
        pe.pe_norm_forward(x, kind="group")
    with pytest.raises(ValueError, match="B, T, d"):
        pe.pe_norm_backward(x[0], x[0], None, r[0], r[0], "square")
    with pytest.raises(ValueError, match="mean"):
        pe.pe_norm_backward(x, x.clone(), None, None, r, "square")
    with pytest.raises(ValueError, match="dy"):
        pe.pe_norm_backward(x, x[:1], None, r, r, "square")
    with pytest.raises(ValueError, match="overlap"):
        pe.pe_norm_backward(x, x.clone(), None, r, r, "square", dx=x)
    with pytest.raises(ValueError, match="accumulate"):
        pe.pe_norm_backward(x, x.clone(), None, r, r, "square", accumulate=True)
    with pytest.raises(ValueError, match="gain_stat"):
        pe.pe_norm_backward(x, x.clone(), None, r, r, "square", gain_stat=torch.zeros(17))
    with pytest.raises(ValueError, match="workspace"):
        pe.pe_norm_backward(x, x.clone(), None, r, r, "square", workspace=torch.zeros(4096, dtype=torch.uint8)[::2])
    with pytest.raises(ValueError, match="seq_offsets"):
        pe.pe_norm_backward_ragged(x[0], x[1], None, r[0], r[0], torch.zeros(3, dtype=torch.int64), "square")
    with pytest.raises(pe.PestatsError):                # tensors on the CPU
        pe.pe_norm_forward(x)
    with pytest.raises(pe.PestatsError):
        pe.pe_norm_backward(x, x.clone(), None, r, r, "square")


def test_rows_too_wide_are_refused(lib, p16):
    """Before anything is enqueued; the widest that is taken passes on to the workspace, or to the device that is missing here."""
    for f in (lib.pe_norm_backward, lib.pe_norm_backward_f32):
        for d, refused in (((1 << 28) + 1, True), ((1 << 31) - 1, True), (1 << 28, False), (65535 * 2048 + 8, False)):
            status = f(p16, p16, None, p16, p16, 1, 1, d, 0, 1, 0, p16, None, None, None, None, p16, 1 << 10, None)
            assert (status == 2) == refused, d
    for f in (lib.pe_norm_forward, lib.pe_norm_forward_f32):
        for d, refused in (((1 << 31) - 1024, True), ((1 << 31) - 1, True), ((1 << 31) - 1025, False)):
            assert (f(p16, None, None, 1, d, 0, 1e-5, p16, None, None, None) == 2) == refused, d
    need = pe.pe_norm_backward_workspace_bytes
    assert need(1, (1 << 28) + 1) == 0 and need(1, (1 << 31) - 1) == 0
    assert need(1, 1 << 28) >= 8 * 4 * (1 << 28)


def test_workspace_of_rows_wider_than_a_cluster(lib):
    """Beyond 32768 features the two means of every row are kept there, 8 bytes; below, nothing grows with the rows once every SM has its blocks."""
    need = pe.pe_norm_backward_workspace_bytes
    for d in (32776, 40000, 100001):
        assert need(3000000, d) - need(1000000, d) == 16000000
    for d in (64, 2048, 4096, 8192, 32768):
        assert need(3000000, d) == need(1000000, d)
