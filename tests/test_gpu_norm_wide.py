"""Rows of several thousand features: slices of a row in the blocks of a cluster, and rows too wide for that; long examples and short ones."""
import pytest
import torch

import paper_2510_00236_b200 as pe
from test_gpu_norm import DEV, DT, EPS, _check_backward, _rows, _stats
from norm_reference import assert_within, forward, half_step

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("B,T,d", [(3, 70, 5000), (2, 40, 8192), (40, 1, 8200), (1, 33, 16384), (3, 5, 24003), (2, 7, 32768), (2, 5, 32776), (2, 3, 40001), (3, 2, 65536)])
def test_backward_of_wide_rows(B, T, d, dtype, kind):
    x, dy, gain, _ = _rows(B, T, d, DT[dtype], d + B)
    mean, rstd = _stats(x, kind)
    got = pe.pe_norm_backward(x, dy, gain, mean, rstd, "square", kind=kind)
    _check_backward(got, x, dy, gain, mean, rstd, list(range(0, B * T + 1, T)), "square", kind)
    again = pe.pe_norm_backward(x, dy, gain, mean, rstd, "square", kind=kind)
    assert all(torch.equal(a, b) for a, b in zip(got, again) if a is not None)


@pytest.mark.parametrize("phi", ["square", "sign", "identity"])
@pytest.mark.parametrize("B,T,d", [(40, 100, 2048), (9, 1000, 512), (3, 3001, 1024), (700, 33, 320), (2000, 1, 2048), (900, 2, 4096), (37, 129, 1000), (50, 64, 3001)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_backward_of_many_rows(B, T, d, phi, dtype):
    """Every worker has several turns, examples that end inside them, at their borders and in none."""
    x, dy, gain, _ = _rows(B, T, d, DT[dtype], d + T)
    mean, rstd = _stats(x, "layer")
    got = pe.pe_norm_backward(x, dy, gain, mean, rstd, phi)
    _check_backward(got, x, dy, gain, mean, rstd, list(range(0, B * T + 1, T)), phi, "layer")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("rows,d", [(40001, 64), (9000, 512), (3001, 2048), (5003, 1001), (1700, 4096), (1500, 3333), (100003, 24), (2500, 1536)])
def test_forward_of_many_rows(rows, d, dtype, kind):
    x, _, gain, bias = _rows(1, rows, d, DT[dtype], rows)
    for gn, bs in ((gain, bias), (None, None)):
        y, mean, rstd = pe.pe_norm_forward(x, gn, bs, kind=kind, eps=EPS)
        ry, rm, rr, y_off, m_off, r_off = forward(x.double(), gn, bs, kind, EPS)
        assert_within("y", y, ry, y_off, half_step(DT[dtype]))
        assert_within("rstd", rstd, rr, r_off)
        if mean is not None:
            assert_within("mean", mean, rm, m_off)


def test_rows_at_the_ends_of_a_buffer():
    """Tensors that begin and end inside a 16-byte word: the words around them stay as they were, and theirs is all that counts."""
    B, T, d = 5, 7, 333
    x, dy, gain, bias = _rows(B, T, d, torch.float32, 3)
    n = x.numel()
    for shift in (1, 2, 3):
        store = [torch.full((n + 8,), float("nan"), device=DEV) for _ in range(4)]
        views = [t[shift:shift + n].view(B, T, d) for t in store]
        views[0].copy_(x)
        views[1].copy_(dy)
        mean, rstd = _stats(x, "layer")
        got = pe.pe_norm_backward(views[0], views[1], gain, mean, rstd, "square", dx=views[2])
        _check_backward(got, x, dy, gain, mean, rstd, list(range(0, B * T + 1, T)), "square", "layer")
        pe.pe_norm_forward(views[0], gain, bias, out=views[3])
        for t in store:
            assert torch.isnan(t[:shift]).all() and torch.isnan(t[shift + n:]).all() and not torch.isnan(t[shift:shift + n]).any()


def _same_pattern(got, want):
    """NaN, and infinities of either sign, at the same places."""
    got, want = got.double(), want.double()
    return torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got == float("inf"), want == float("inf")) and torch.equal(got == -float("inf"), want == -float("inf"))


# many rows (the forward ring) and few; threads whose last features are out of range, aligned fp32 rows among them; slices of rows
INFINITE = [(13001, 333, "bf16"), (13001, 333, "fp32"), (40, 333, "fp32"), (9, 100, "fp32"), (70, 1004, "fp32"), (5, 4609, "bf16"), (5, 5004, "fp32"), (1, 33001, "fp32"), (200001, 21, "bf16")]


@pytest.mark.parametrize("rows,d,dtype", INFINITE)
def test_infinities_under_rms(rows, d, dtype):
    """An infinity in a row makes its rstd zero: that feature is NaN, every other one the bias, whichever feature it is."""
    x, _, gain, bias = _rows(1, rows, d, DT[dtype], d)
    x = x[0]
    where = {k * (rows // 5): c for k, c in enumerate((0, 1, d // 2, d - 2, d - 1)) if rows >= 5} or {0: d // 2}
    clean, _, r0 = pe.pe_norm_forward(x, gain, bias, kind="rms", eps=EPS)
    for row, c in where.items():
        x[row, c] = -float("inf") if c & 1 else float("inf")
    y, _, r = pe.pe_norm_forward(x, gain, bias, kind="rms", eps=EPS)
    for row, c in where.items():
        want = bias.to(DT[dtype]).clone()
        want[c] = float("nan")
        assert float(r[row]) == 0.0 and torch.equal(torch.isnan(y[row]), torch.isnan(want)) and torch.equal(y[row].nan_to_num(nan=0.0), want.nan_to_num(nan=0.0))
        y[row], r[row] = clean[row], r0[row]
    assert torch.equal(y, clean) and torch.equal(r, r0)


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("rows,d,dtype", INFINITE)
def test_infinite_gradients(rows, d, dtype, kind):
    """dx where dy holds an infinity: infinite or NaN just where the formula is."""
    x, dy, gain, _ = _rows(1, rows, d, DT[dtype], d + 1)
    mean, rstd = _stats(x, kind)
    dy[0, 0, 0] = float("inf")
    dy[0, rows // 2, d - 1] = -float("inf")
    dy[0, rows - 1, d // 2] = float("inf")
    dx, gain_sum, *_ = pe.pe_norm_backward(x, dy, gain, mean, rstd, "square", kind=kind)
    hit = sorted({0, rows // 2, rows - 1})
    xs, ds, r = x[0, hit].double(), dy[0, hit].double(), rstd[0, hit, None].double()
    h = (xs - (mean[0, hit, None].double() if kind == "layer" else 0.0)) * r
    w = ds * gain.double()
    want = r * (w - h * (w * h).mean(1, keepdim=True) - (w.mean(1, keepdim=True) if kind == "layer" else 0.0))
    assert _same_pattern(dx[0, hit], want)
    others = torch.ones(rows, dtype=torch.bool, device=DEV)
    others[hit] = False
    assert torch.isfinite(dx[0, others]).all()
    finite = torch.ones(d, dtype=torch.bool, device=DEV)
    finite[[0, d - 1, d // 2]] = False
    assert torch.isfinite(gain_sum[finite]).all() and not torch.isfinite(gain_sum[~finite]).any()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("B,T,d", [(3, 3001, 8192), (1100, 3, 12292), (2, 1200, 32768), (5, 601, 24003)])
def test_slices_that_exchange_sums_over_dozens_of_turns(B, T, d, dtype, kind):
    """4 bf16 rows or 2 fp32 ones a turn, 15 to 74 clusters: at least 24 turns, so that the ring and both words of the exchange are used over and over.
    (A cluster's sums go over at most 3000 / 15 rows and the joins, fewer than the additions that the bound is made for.)"""
    x, dy, gain, _ = _rows(B, T, d, DT[dtype], d + B)
    mean, rstd = _stats(x, kind)
    got = pe.pe_norm_backward(x, dy, gain, mean, rstd, "square", kind=kind)
    assert pe.pe_get_async_status(DEV) == (0, 0)
    _check_backward(got, x, dy, gain, mean, rstd, list(range(0, B * T + 1, T)), "square", kind)
    for _ in range(3):
        again = pe.pe_norm_backward(x, dy, gain, mean, rstd, "square", kind=kind)
        assert all(torch.equal(a, b) for a, b in zip(got, again) if a is not None)


@pytest.mark.parametrize("B,T,d", [(3, 40, 64), (700, 33, 320), (40, 100, 2048), (5, 70, 8192), (3, 50, 40000)])
def test_what_the_workspace_holds_before_does_not_matter(B, T, d):
    x, dy, gain, _ = _rows(B, T, d, torch.bfloat16, 11)
    mean, rstd = _stats(x, "layer")
    need = pe.pe_norm_backward_workspace_bytes(B * T, d)
    got = [pe.pe_norm_backward(x, dy, gain, mean, rstd, "square", workspace=torch.full((need,), fill, dtype=torch.uint8, device=DEV)) for fill in (0, 255, 127)]
    for one in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got[0], one))
    assert all(torch.isfinite(t).all() for t in got[0])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("B,T,d", [(918, 47, 152), (209, 243, 132), (2695, 47, 72), (1979, 16, 136), (900, 47, 35), (400, 47, 264), (400, 47, 320), (3000, 9, 80)])
def test_sums_of_narrow_rows_repeat_bit_for_bit(B, T, d, dtype):
    """Rows whose ring is smaller than what the workers leave at its place in the end."""
    x, dy, gain, _ = _rows(B, T, d, DT[dtype], d)
    mean, rstd = _stats(x, "layer")
    first = pe.pe_norm_backward(x, dy, gain, mean, rstd, "square")
    _check_backward(first, x, dy, gain, mean, rstd, list(range(0, B * T + 1, T)), "square", "layer")
    wrong = 0
    for _ in range(100):
        again = pe.pe_norm_backward(x, dy, gain, mean, rstd, "square")
        wrong += not all(torch.equal(a, b) for a, b in zip(first, again))
    assert wrong == 0


# three slots of the forward ring take between 47.5 and 48 KB
BAND = [("bf16", 121), ("bf16", 249), ("fp32", 249), ("bf16", 505), ("fp32", 505), ("bf16", 1018), ("fp32", 1018), ("bf16", 2024), ("bf16", 2040), ("bf16", 2042), ("fp32", 2042)]


def first_forward_calls():
    for dtype, d in BAND:
        for kind in ("layer", "rms"):
            x, _, gain, bias = _rows(1, (1 << 22) // d + 5, d, DT[dtype], d)
            y, mean, rstd = pe.pe_norm_forward(x, gain, bias, kind=kind, eps=EPS)
            ry, rm, rr, y_off, m_off, r_off = forward(x.double(), gain, bias, kind, EPS)
            assert_within("y", y, ry, y_off, half_step(DT[dtype]))
            assert_within("rstd", rstd, rr, r_off)
            if mean is not None:
                assert_within("mean", mean, rm, m_off)


def test_shared_memory_just_below_48_kilobytes():
    """In a process of its own, since a kernel that has been allowed more keeps that."""
    import os
    import subprocess
    import sys
    tests = os.path.dirname(os.path.abspath(__file__))
    code = f"import sys; sys.path[:0] = [{os.path.dirname(tests)!r}, {tests!r}]; import test_gpu_norm_wide as t; t.first_forward_calls()"
    alone = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert alone.returncode == 0, alone.stderr[-2000:]
