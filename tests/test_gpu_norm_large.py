"""Tensors of more than 2^31 elements, and calls that overlap on two streams."""
import pytest
import torch

import paper_2510_00236_b200 as pe
from norm_reference import U, assert_within, backward, forward, half_step
from test_gpu_norm import DEV, EPS, _check_backward, _rows, _stats

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [1024, 1023])
def test_offsets_past_31_bits(d):
    B, T = 3, (1 << 31) // (3 * 1024) + 1500
    g = torch.Generator(device=DEV)
    g.manual_seed(d)
    x = torch.empty(B, T, d, dtype=torch.bfloat16, device=DEV).normal_(generator=g)
    dy = torch.empty(B, T, d, dtype=torch.bfloat16, device=DEV).normal_(generator=g)
    assert x.numel() > 1 << 31
    gain = 1 + 0.1 * torch.randn(d, generator=g, device=DEV)
    y, mean, rstd = pe.pe_norm_forward(x, gain, None, eps=EPS)
    dx, gain_sum, gain_sq, bias_sum, bias_sq = pe.pe_norm_backward(x, dy, gain, mean, rstd, "square")
    assert pe.pe_get_async_status(DEV) == (0, 0)
    # the first and the last rows of every example
    for b in range(B):
        for part in (slice(0, 64), slice(T - 64, T)):
            xs, ds = x[b, part], dy[b, part]
            ry, rm, rr, y_off, m_off, r_off = forward(xs.double(), gain, None, "layer", EPS)
            assert_within("y", y[b, part], ry, y_off, half_step(torch.bfloat16))
            assert_within("mean", mean[b, part], rm, m_off)
            assert_within("rstd", rstd[b, part], rr, r_off)
            rdx, dx_off, _ = backward(xs.double(), ds.double(), gain, mean[b, part], rstd[b, part], [0, 64], "square", "layer")
            assert_within("dx", dx[b, part], rdx, dx_off, half_step(torch.bfloat16))
    # sums: over T rows of terms of about one, each worker's part (a 296th or less of them) added up in turn and then joined
    depth = 3 * T // 148 + 300
    G, H, Gm, Hm = (torch.zeros(B, d, dtype=torch.float64, device=DEV) for _ in range(4))
    for b in range(B):
        for at in range(0, T, 1 << 16):
            e = dy[b, at:at + (1 << 16)].double()
            h = (x[b, at:at + (1 << 16)].double() - mean[b, at:at + (1 << 16), None].double()) * rstd[b, at:at + (1 << 16), None].double()
            G[b] += (e * h).sum(0)
            H[b] += e.sum(0)
            Gm[b] += (e * h).abs().sum(0)
            Hm[b] += e.abs().sum(0)
    for got, got_sq, S, M in ((gain_sum, gain_sq, G, Gm), (bias_sum, bias_sq, H, Hm)):
        off = U * (depth + 4) * M
        assert_within("sum", got, S.sum(0), off.sum(0) + 4 * U * S.abs().sum(0))
        assert_within("square", got_sq, (S * S).sum(0), (2 * S.abs() * off + off * off).sum(0) + 6 * U * (S * S).sum(0))


def test_two_calls_at_once_on_two_streams():
    cases = [(40, 33, 1024, torch.bfloat16), (300, 3, 777, torch.float32)]
    inputs, want = [], []
    for B, T, d, dt in cases:
        x, dy, gain, _ = _rows(B, T, d, dt, d)
        mean, rstd = _stats(x, "layer")
        inputs.append((x, dy, gain, mean, rstd))
        want.append(pe.pe_norm_backward(x, dy, gain, mean, rstd, "square"))
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in cases], [[], []]
    for _ in range(5):
        for k, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[k].append(pe.pe_norm_backward(*inputs[k], "square"))
    torch.cuda.synchronize()
    for k in range(2):
        for one in got[k]:
            assert all(torch.equal(a, b) for a, b in zip(one, want[k]))


def test_rows_of_more_slices_than_a_grid_is_high():
    """65537 slices of 2048 features."""
    B, T, d = 2, 1, 65536 * 2048 + 8
    g = torch.Generator(device=DEV)
    g.manual_seed(4)
    x, dy = (torch.empty(B, T, d, dtype=torch.bfloat16, device=DEV).normal_(generator=g) for _ in range(2))
    mean, rstd = _stats(x, "layer")
    got = pe.pe_norm_backward(x, dy, None, mean, rstd, "square")
    assert pe.pe_get_async_status(DEV) == (0, 0)
    _check_backward(got, x, dy, None, mean, rstd, [0, 1, 2], "square", "layer")


def test_the_widest_row_forward():
    """2^31 - 1025 features, the widest that are taken: a thread's last step ends just below 2^31.  Sums are over 2^21 terms of a thread, added one after the other, then 37 more."""
    d, part = (1 << 31) - 1025, 1 << 27
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    x = torch.empty(1, d, dtype=torch.bfloat16, device=DEV).normal_(generator=g)
    y, mean, rstd = pe.pe_norm_forward(x, eps=EPS)
    pieces = [slice(at, min(d, at + part)) for at in range(0, d, part)]
    mu = sum(float(x[0, p].double().sum()) for p in pieces) / d
    size = sum(float(x[0, p].double().abs().sum()) for p in pieces) / d
    var = sum(float((x[0, p].double() - mu).square().sum()) for p in pieces) / d
    k = (1 << 21) + 40
    mu_off = U * k * size
    r = (var + EPS) ** -0.5
    r_off = r * (0.5 * (U * k * var + mu_off ** 2) / (var + EPS) + 4 * U)
    assert abs(float(mean) - mu) <= mu_off and abs(float(rstd) - r) <= r_off
    for p in pieces:
        want = (x[0, p].double() - mu) * r
        off = mu_off * r + want.abs() * (r_off / r + 3 * U)
        assert_within("y", y[0, p], want, off, half_step(torch.bfloat16))
