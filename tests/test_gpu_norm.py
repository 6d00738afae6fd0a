"""Normalisation layers on the GPU against 64 bits: outputs, statistics over examples, masks, layouts, streams and graphs."""
import pytest
import torch

import paper_2510_00236_b200 as pe
from norm_reference import assert_within, backward, forward, half_step

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 1e-5
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
# one feature to rows wider than any block; odd widths; one-token and one-example batches; examples that end inside and between blocks' rows
SHAPES = [(1, 1, 1), (3, 1, 7), (2, 5, 8), (8, 16, 64), (5, 7, 33), (4, 9, 100), (300, 1, 24), (7, 130, 256), (3, 50, 1000), (2, 33, 1001), (64, 3, 520),
          (1, 700, 768), (6, 40, 2048), (700, 2, 1536), (3, 20, 4096), (2, 9, 4104), (2, 5, 8192), (2, 3, 9001), (1, 3, 16400), (4000, 5, 40)]


def _rows(B, T, d, dtype, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    x = torch.randn(B, T, d, generator=g, device=DEV) * torch.exp(0.5 * torch.randn(d, generator=g, device=DEV)) + 0.5 * torch.randn(B, T, 1, generator=g, device=DEV)
    dy = torch.randn(B, T, d, generator=g, device=DEV)
    gain, bias = 1 + 0.2 * torch.randn(d, generator=g, device=DEV), torch.randn(d, generator=g, device=DEV)
    return x.to(dtype), dy.to(dtype), gain, bias


def _stats(x, kind):
    """mean and rstd of every row, as the forward pass would hand them on."""
    _, mean, rstd, *_ = forward(x.double(), None, None, kind, EPS)
    return (mean.float() if kind == "layer" else None), rstd.float()


def _check_backward(got, x, dy, gain, mean, rstd, ends, phi, kind, rows=slice(None)):
    d = x.shape[-1]
    flat = lambda t: None if t is None else t.reshape(-1, d) if t.dim() > 1 and t.shape[-1] == d and t.numel() > rstd.numel() else t.reshape(-1)
    dx, dx_off, sums = backward(x.reshape(-1, d).double(), dy.reshape(-1, d).double(), gain, flat(mean), rstd.reshape(-1), ends, phi, kind)
    assert_within("dx", got[0].reshape(-1, d)[rows], dx[rows], dx_off[rows], half_step(x.dtype))
    for k, (total, total_off, stat, stat_off) in enumerate(sums):
        if got[1 + 2 * k] is not None:
            assert_within(f"sum {k}", got[1 + 2 * k], total, total_off)
        if got[2 + 2 * k] is not None:
            assert_within(f"stat {k}", got[2 + 2 * k], stat, stat_off)


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("B,T,d", SHAPES + [(1, 2, 70001), (1, 2, 70000)])
def test_forward(B, T, d, dtype, kind):
    x, _, gain, bias = _rows(B, T, d, DT[dtype], d)
    for gn, bs in ((gain, bias), (gain, None), (None, bias), (None, None)):
        y, mean, rstd = pe.pe_norm_forward(x, gn, bs, kind=kind, eps=EPS)
        ry, rm, rr, y_off, m_off, r_off = forward(x.double(), gn, bs, kind, EPS)
        assert_within("y", y, ry, y_off, half_step(DT[dtype]))
        assert_within("rstd", rstd, rr, r_off)
        assert (mean is None) == (kind == "rms")
        if mean is not None:
            assert_within("mean", mean, rm, m_off)


@pytest.mark.parametrize("phi", ["identity", "square", "sign"])
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("B,T,d", SHAPES)
def test_backward(B, T, d, dtype, kind, phi):
    x, dy, gain, _ = _rows(B, T, d, DT[dtype], 7 * d + B)
    mean, rstd = _stats(x, kind)
    got = pe.pe_norm_backward(x, dy, gain, mean, rstd, phi, kind=kind)
    assert (got[3] is None) == (kind == "rms")
    _check_backward(got, x, dy, gain, mean, rstd, list(range(0, B * T + 1, T)), phi, kind)


@pytest.mark.parametrize("B,T,d", [(5, 7, 33), (6, 40, 512), (2, 9, 4104)])
def test_backward_of_chosen_outputs_and_without_gain(B, T, d):
    x, dy, gain, _ = _rows(B, T, d, torch.bfloat16, 3)
    mean, rstd = _stats(x, "layer")
    ends = list(range(0, B * T + 1, T))
    stat = torch.full((d,), 7.0, device=DEV)
    got = pe.pe_norm_backward(x, dy, None, mean, rstd, "square", gain_stat=stat)
    assert got[1] is None and got[3] is None and got[4] is None
    _check_backward(got, x, dy, None, mean, rstd, ends, "square", "layer")
    bias_sum = torch.empty(d, device=DEV)
    m0, r = _stats(x, "rms")
    got = pe.pe_norm_backward(x, dy, gain, None, r, "sign", kind="rms", bias_sum=bias_sum)      # a root-mean-square form with a bias
    assert got[1] is None
    _check_backward(got, x, dy, gain, None, r, ends, "sign", "rms")


def test_accumulation_over_micro_batches():
    B, T, d = 6, 11, 320
    x, dy, gain, _ = _rows(B, T, d, torch.float32, 5)
    mean, rstd = _stats(x, "layer")
    whole = pe.pe_norm_backward(x, dy, gain, mean, rstd, "square")
    sums = [torch.zeros(d, device=DEV) for _ in range(4)]
    for a, b in ((0, 2), (2, 2), (2, 6)):
        pe.pe_norm_backward(x[a:b], dy[a:b], gain, mean[a:b], rstd[a:b], "square", gain_sum=sums[0], gain_stat=sums[1], bias_sum=sums[2], bias_stat=sums[3],
                            accumulate=True)
    _check_backward((whole[0], *sums), x, dy, gain, mean, rstd, list(range(0, B * T + 1, T)), "square", "layer")


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("phi", ["square", "sign"])
@pytest.mark.parametrize("lens,first,behind,d", [([3], 0, 0, 64), ([0, 0, 5, 0], 0, 4, 40), ([1] * 50, 2, 3, 256), ([700, 1, 0, 64, 333, 2], 5, 9, 512),
                                                 ([17, 40, 0, 1, 90], 1, 1, 1001), ([9, 0, 30], 0, 2, 4608), ([0, 0], 3, 2, 64), ([40] * 300, 0, 1, 128)])
def test_packed_batches(lens, first, behind, d, phi, kind):
    ends = [first]
    for n in lens:
        ends.append(ends[-1] + n)
    rows = ends[-1] + behind
    x, dy, gain, _ = _rows(rows, 1, d, torch.bfloat16, rows + d)
    x, dy = x.view(rows, d), dy.view(rows, d)
    outside = torch.ones(rows, dtype=torch.bool, device=DEV)
    outside[ends[0]:ends[-1]] = False
    mean, rstd = _stats(x, kind)
    # nothing outside the sequences is read
    x[outside] = float("nan")
    dy[outside] = float("inf")
    rstd[outside] = float("nan")
    dx = torch.full_like(x, 7.0)
    offs = torch.tensor(ends, dtype=torch.int32, device=DEV)
    got = pe.pe_norm_backward_ragged(x, dy, gain, mean, rstd, offs, phi, kind=kind, dx=dx)
    assert torch.all(dx[outside] == 7.0)
    x[outside], dy[outside], rstd[outside] = 0.0, 0.0, 1.0
    _check_backward(got, x, dy, gain, mean, rstd, ends, phi, kind, ~outside)


def test_packed_batch_equals_the_plain_one_bit_for_bit():
    B, T, d = 9, 21, 384
    x, dy, gain, _ = _rows(B, T, d, torch.bfloat16, 9)
    mean, rstd = _stats(x, "layer")
    plain = pe.pe_norm_backward(x, dy, gain, mean, rstd, "square")
    offs = torch.arange(0, B * T + 1, T, dtype=torch.int32, device=DEV)
    packed = pe.pe_norm_backward_ragged(x.view(-1, d), dy.view(-1, d), gain, mean.view(-1), rstd.view(-1), offs, "square")
    again = pe.pe_norm_backward(x, dy, gain, mean, rstd, "square")
    for a, b, c in zip(plain, packed, again):
        assert torch.equal(a.reshape(-1), b.reshape(-1)) and torch.equal(a, c)


@pytest.mark.parametrize("d", [64, 1001, 2048, 4608])
def test_nan_and_infinity_stay_in_their_rows(d):
    B, T = 4, 6
    x, dy, gain, bias = _rows(B, T, d, torch.float32, d)
    mean, rstd = _stats(x, "layer")
    bad = x.clone()
    bad[1, 2, d // 2] = float("nan")
    bad[3, 0, 0] = float("inf")
    y, m, r = pe.pe_norm_forward(bad, gain, bias, eps=EPS)
    good, gm, gr = pe.pe_norm_forward(x, gain, bias, eps=EPS)
    hit = torch.zeros(B, T, dtype=torch.bool, device=DEV)
    hit[1, 2] = hit[3, 0] = True
    assert torch.equal(y[~hit], good[~hit]) and torch.equal(r[~hit], gr[~hit]) and torch.isnan(y[1, 2]).all() and torch.isnan(y[3, 0]).all()
    bad_dy = dy.clone()
    bad_dy[1, 2, d // 2] = float("nan")
    a, b = pe.pe_norm_backward(x, bad_dy, gain, mean, rstd, "square"), pe.pe_norm_backward(x, dy, gain, mean, rstd, "square")
    assert torch.equal(a[0][~hit], b[0][~hit]) and torch.isnan(a[0][1, 2]).all()
    keep = torch.arange(d, device=DEV) != d // 2
    for s, t in zip(a[1:], b[1:]):
        assert torch.equal(s[keep], t[keep]) and torch.isnan(s[d // 2])


def test_constant_rows_and_zero_rows():
    """A row of one value has no deviation: y is the bias, whatever the value's size; with eps = 0 the result is NaN, as the formula says."""
    d = 96
    x = torch.full((3, 1, d), 1000.0, device=DEV)
    x[1] = 0.0
    bias = torch.randn(d, device=DEV)
    y, mean, rstd = pe.pe_norm_forward(x, None, bias, eps=EPS)
    assert torch.equal(y[:, 0], bias.expand(3, d)) and torch.equal(mean.view(-1), torch.tensor([1000.0, 0.0, 1000.0], device=DEV))
    y, *_ = pe.pe_norm_forward(x, None, None, eps=0.0)
    assert torch.isnan(y).all()


def test_empty_batches():
    d = 40
    for B, T in ((0, 4), (4, 0)):
        x = torch.empty(B, T, d, dtype=torch.bfloat16, device=DEV)
        y, mean, rstd = pe.pe_norm_forward(x)
        assert y.shape == x.shape and rstd.shape == (B, T)
        dx, *sums = pe.pe_norm_backward(x, x, None, mean, rstd, "square", dx=torch.empty_like(x))
        assert all(torch.equal(s, torch.zeros(d, device=DEV)) for s in sums)
        kept = torch.full((d,), 3.0, device=DEV)
        pe.pe_norm_backward(x, x, None, mean, rstd, "square", dx=torch.empty_like(x), gain_sum=kept, accumulate=True)
        assert torch.all(kept == 3.0)


def test_unaligned_fp32_rows():
    """fp32 tensors need 4-byte alignment only."""
    B, T, d = 3, 10, 128
    x, dy, gain, bias = _rows(B, T, d, torch.float32, 21)
    def shifted(t):
        store = torch.empty(t.numel() + 1, device=DEV)
        store[1:] = t.reshape(-1)
        return store[1:].view(t.shape)
    mean, rstd = _stats(x, "layer")
    xs, ds, gs = shifted(x), shifted(dy), shifted(gain)
    y, *_ = pe.pe_norm_forward(xs, gs, shifted(bias), eps=EPS)
    ry, _, _, y_off, *_ = forward(x.double(), gain, bias, "layer", EPS)
    assert_within("y", y, ry, y_off, half_step(torch.float32))
    got = pe.pe_norm_backward(xs, ds, gs, shifted(mean), shifted(rstd), "square")
    _check_backward(got, x, dy, gain, mean, rstd, list(range(0, B * T + 1, T)), "square", "layer")


def test_another_stream_and_a_captured_graph():
    B, T, d = 16, 33, 512
    x, dy, gain, bias = _rows(B, T, d, torch.bfloat16, 33)
    mean, rstd = _stats(x, "layer")
    want = (pe.pe_norm_forward(x, gain, bias)[0], *pe.pe_norm_backward(x, dy, gain, mean, rstd, "square"))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = (pe.pe_norm_forward(x, gain, bias)[0], *pe.pe_norm_backward(x, dy, gain, mean, rstd, "square"))
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    xin, din = torch.zeros_like(x), torch.zeros_like(dy)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = pe.pe_norm_forward(xin, gain, bias)[0]
        outs = pe.pe_norm_backward(xin, din, gain, mean, rstd, "square")
    for _ in range(2):
        xin.copy_(x)
        din.copy_(dy)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((y, *outs), want))


def test_refusals_that_need_a_gpu():
    x, dy, gain, _ = _rows(4, 8, 64, torch.bfloat16, 1)
    mean, rstd = _stats(x, "layer")
    need = pe.pe_norm_backward_workspace_bytes(32, 64)
    assert need > 0
    dx = torch.full_like(x, 5.0)
    for ws in (torch.empty(need - 1, dtype=torch.uint8, device=DEV), torch.empty(need + 8, dtype=torch.uint8, device=DEV)[8:]):
        with pytest.raises(pe.PestatsError) as e:
            pe.pe_norm_backward(x, dy, gain, mean, rstd, "square", dx=dx, workspace=ws)
        assert e.value.status in (9, 3)
    torch.cuda.synchronize()
    assert torch.all(dx == 5.0)
    assert pe.pe_get_async_status(DEV) == (0, 0)


def test_gradients_against_differences():
    """dx and the sums of the gains' and biases' gradients against differences of the 64-bit loss sum(dy * y)."""
    B, T, d = 3, 4, 24
    x, dy, gain, bias = _rows(B, T, d, torch.float32, 77)
    for kind in ("layer", "rms"):
        y, mean, rstd = pe.pe_norm_forward(x, gain, bias, kind=kind, eps=EPS)
        dx, gsum, _, *_ = pe.pe_norm_backward(x, dy, gain, mean, rstd, "square", kind=kind)
        loss = lambda xx, gg: float((forward(xx, gg, bias, kind, EPS)[0] * dy.double()).sum())
        step = 1e-6      # differences are off by step^2 and by 2^-52 / step of the loss: both below 1e-7 of the gradients here
        for at in ((0, 0, 0), (1, 2, 5), (2, 3, d - 1)):
            up, down = x.double(), x.double()
            up[at] += step
            down[at] -= step
            diff = (loss(up, gain.double()) - loss(down, gain.double())) / (2 * step)
            assert abs(diff - float(dx[at])) <= 1e-4 * float(dx.abs().max())
        for j in (0, d - 1):
            up, down = gain.double(), gain.double()
            up[j] += step
            down[j] -= step
            diff = (loss(x.double(), up) - loss(x.double(), down)) / (2 * step)
            assert abs(diff - float(gsum[j])) <= 1e-4 * float(gsum.abs().max())
