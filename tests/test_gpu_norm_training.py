"""The new operators as a training step uses them, beside the statistics of the linear layers: a pre-norm MLP whose backward pass goes through
pe_norm_backward, per-example statistics of both linear layers and of the norm's gain and bias, muon_step on the matrices and microadam_step on gain and bias."""
import pytest
import torch
import torch.nn.functional as F

import paper_2510_00236_b200 as pe
from parity_util import FROB_TOL

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16 = torch.bfloat16
EPS = 1e-5


def _rel(a, b):
    return float((a.detach().double() - b.detach().double()).norm() / b.detach().double().norm())


def test_training_step_of_a_pre_norm_mlp():
    """Against autograd in 64 bits, example by example, on the same bf16 values."""
    torch.manual_seed(5)
    B, T, d, h = 6, 40, 264, 520
    x = torch.randn(B, T, d, device=DEV).to(BF16)
    target = torch.randn(B, T, d, device=DEV)
    up, down = torch.randn(h, d, device=DEV) * d ** -0.5, torch.randn(d, h, device=DEV) * h ** -0.5
    gain, bias = 1 + 0.1 * torch.randn(d, device=DEV), 0.1 * torch.randn(d, device=DEV)
    up_lp, down_lp = up.to(BF16), down.to(BF16)
    # forward: y = x + down gelu(up norm(x)); loss sum_b (1/T) sum (y - target)^2 / 2
    n, mean, rstd = pe.pe_norm_forward(x, gain, bias, eps=EPS)
    a = n @ up_lp.T
    g = F.gelu(a.float()).to(BF16)
    dy = (((x.float() + (g @ down_lp.T).float()) - target) / T).to(BF16)
    # backward
    dg = dy @ down_lp
    a64 = a.double().requires_grad_()
    (da,) = torch.autograd.grad(F.gelu(a64), a64, dg.double())
    da = da.to(BF16)
    dn = da @ up_lp
    dx, gain_sum, gain_sq, bias_sum, bias_sq = pe.pe_norm_backward(x, dn, gain, mean, rstd, "square")
    up_mean, up_sq = pe.pe_linear_stats(n, da, "square")
    down_mean, down_sq = pe.pe_linear_stats(g, dy, "square")
    assert pe.pe_get_async_status(DEV) == (0, 0)
    # the same by autograd in 64 bits from the tensors that each operator was given
    x64 = x.double().requires_grad_()
    gain64, bias64 = gain.double().requires_grad_(), bias.double().requires_grad_()
    n64 = F.layer_norm(x64, (d,), gain64, bias64, EPS)
    per_gain, per_bias = [], []
    for b in range(B):
        gg, gb = torch.autograd.grad(n64[b], (gain64, bias64), dn[b].double(), retain_graph=True)
        per_gain.append(gg)
        per_bias.append(gb)
    (dx64,) = torch.autograd.grad(n64, x64, dn.double())
    assert _rel(n, n64) <= 2.0 ** -8 and _rel(dx, dx64) <= 2.0 ** -8 + 1e-5
    for got, want in ((gain_sum, sum(per_gain)), (gain_sq, sum(v * v for v in per_gain)), (bias_sum, sum(per_bias)), (bias_sq, sum(v * v for v in per_bias))):
        assert _rel(got, want) <= 1e-5
    G = torch.einsum("btf,btd->bfd", da.double(), n.double())
    assert _rel(up_mean, G.sum(0)) <= FROB_TOL and _rel(up_sq, (G * G).sum(0)) <= FROB_TOL
    # updates: the matrices by their orthogonalised momentum, gain and bias by MicroAdam on the examples' squares
    for w, w_lp, s in ((up, up_lp, up_mean), (down, down_lp, down_mean)):
        before, mom = w.clone(), torch.zeros_like(w)
        pe.muon_step(w, mom, s, B, lr=0.02, beta=0.95, theta_lp=w_lp)
        step = (before - w).double() / (0.02 * max(1.0, w.shape[0] / w.shape[1]) ** 0.5)
        sv = torch.linalg.svdvals(step)
        assert 0.3 < float(sv.max()) < 1.25 and torch.equal(w_lp, w.to(BF16))
        assert float((step * s.double()).sum()) > 0          # a step down the mean gradient
    for p, s, q in ((gain, gain_sum, gain_sq), (bias, bias_sum, bias_sq)):
        before, m1, v1 = p.clone(), torch.zeros_like(p), torch.zeros_like(p)
        pe.microadam_step(p, m1, v1, s, q, B, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1)
        want = before.double() - 1e-3 * (s.double() / B) / ((q.double() / B).sqrt() + 1e-8)
        assert _rel(p, want) <= 1e-6


def test_norms_of_a_decoder_under_rms():
    """The root-mean-square norms of a small decoder (64 sequences of 256 tokens, d_model 512), with the statistics accumulated over two micro-batches."""
    torch.manual_seed(6)
    B, T, d = 64, 256, 512
    x, dy = torch.randn(B, T, d, device=DEV).to(BF16), (torch.randn(B, T, d, device=DEV) / T ** 0.5).to(BF16)
    gain = torch.ones(d, device=DEV)
    _, mean, rstd = pe.pe_norm_forward(x, gain, kind="rms", eps=1e-6)
    assert mean is None
    sums = [torch.zeros(d, device=DEV) for _ in range(2)]
    for at in (0, 32):
        part = slice(at, at + 32)
        pe.pe_norm_backward(x[part], dy[part], gain, None, rstd[part], "square", kind="rms", gain_sum=sums[0], gain_stat=sums[1], accumulate=True)
    G = (dy.double() * x.double() * (x.double().square().mean(-1, keepdim=True) + 1e-6) ** -0.5).sum(1)
    assert _rel(sums[0], G.sum(0)) <= 1e-5 and _rel(sums[1], (G * G).sum(0)) <= 1e-5
