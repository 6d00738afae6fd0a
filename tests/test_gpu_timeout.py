"""The give-up path of the tensor-core kernels: every wait on an on-chip barrier has a cycle budget; when one
runs out the kernel skips its outputs, exits normally and latches PE_ERR_TIMEOUT with the identity of the wait.
The budget is lowered to one cycle here, so that the first wait that does not succeed at once gives up (no
kernel is broken and nothing hangs: all waits still end, just unsuccessfully); afterwards the default budget
is restored and the same call must be correct."""
import numpy as np
import pytest
import torch

import oracle
import paper_2510_00236_b200 as pe
from paper_2510_00236_b200 import inputs
from parity_util import FROB_TOL, rel_frob

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
PE_ERR_TIMEOUT = 8


@pytest.fixture()
def short_waits():
    pe.pe_set_path(pe.PATH_TENSOR)
    pe.pe_set_wait_limit_cycles(1, DEV)
    yield
    pe.pe_set_wait_limit_cycles(0, DEV)
    pe.pe_set_path(pe.PATH_AUTO)


def test_waits_that_run_out_are_reported_and_the_library_stays_usable(short_waits):
    li = inputs.gaussian_layer(8, 512, 256, 512, seed=31, device=DEV, with_weights=True)
    B, T, d_in, d_out = li.shape
    sentinel = 7.0
    mean = torch.full((d_out, d_in), sentinel, device=DEV)
    stat = torch.full((d_out, d_in), sentinel, device=DEV)
    pe.pe_linear_stats(li.X, li.dY, "square", mean, stat)               # returns PE_OK: the give-up happens on the device
    status, detail = pe.pe_get_async_status(DEV)
    assert status == PE_ERR_TIMEOUT and 1 <= detail <= 4, (status, detail)
    assert pe.pe_get_async_status(DEV) == (0, 0)                        # reading the status clears it

    tok = torch.full((d_out, d_in), sentinel, device=DEV)
    pe.pe_token_sqstats(li.X, li.dY, tok)                               # the one-kernel per-token statistic
    status, detail = pe.pe_get_async_status(DEV)
    assert status == PE_ERR_TIMEOUT and detail > 0, (status, detail)

    # the fused statistics + update call must leave the parameters alone when it gives up
    W = li.W.clone()
    th, mm, vv = W.clone(), torch.zeros_like(W), torch.zeros_like(W)
    ws = torch.zeros(pe.pe_linear_fused_workspace_bytes(d_in, d_out), dtype=torch.uint8, device=DEV)
    pe.pe_linear_microadam_step(li.X, li.dY, th, mm, vv, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1, out_mean=mean, out_stat=stat,
                                workspace=ws)
    status, detail = pe.pe_get_async_status(DEV)
    assert status == PE_ERR_TIMEOUT, (status, detail)
    assert torch.equal(th, W) and float(mm.abs().max()) == 0.0 and float(vv.abs().max()) == 0.0

    # default budget back: the same calls are correct
    pe.pe_set_wait_limit_cycles(0, DEV)
    st = oracle.linear_stats(inputs.to_numpy_bits(li.X), inputs.to_numpy_bits(li.dY))
    tok_ref = oracle.token_sqstats(inputs.to_numpy_bits(li.X), inputs.to_numpy_bits(li.dY))
    pe.pe_linear_stats(li.X, li.dY, "square", mean, stat)
    pe.pe_token_sqstats(li.X, li.dY, tok)
    assert pe.pe_get_async_status(DEV) == (0, 0)
    assert rel_frob(mean.cpu().numpy(), st.sum_g) <= FROB_TOL and rel_frob(stat.cpu().numpy(), st.sum_g2) <= FROB_TOL
    assert rel_frob(tok.cpu().numpy(), tok_ref) <= FROB_TOL
    pe.pe_linear_microadam_step(li.X, li.dY, th, mm, vv, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1, workspace=ws)
    assert pe.pe_get_async_status(DEV) == (0, 0)
    W0 = W.cpu().numpy().astype(np.float64)
    th_ref, _, _ = oracle.microadam_step(W0, np.zeros_like(W0), np.zeros_like(W0), st.sum_g, st.sum_g2, B, lr=1e-3, beta1=0.9, beta2=0.999,
                                         eps=1e-8, step=1)
    assert np.linalg.norm((th.cpu().numpy() - W0) - (th_ref - W0)) <= FROB_TOL * np.linalg.norm(th_ref - W0)


# whole rows through the forward ring, aligned and of an odd width; slices in clusters; rows wider than that; a single block
NORM_ROWS = [(64, 1024, 2048, torch.bfloat16), (64, 512, 1001, torch.float32), (16, 512, 8192, torch.bfloat16), (8, 128, 40000, torch.bfloat16), (1, 40, 64, torch.float32),
             (64, 2048, 40, torch.bfloat16)]


def _norm_rows(B, T, d, dtype):
    g = torch.Generator(device=DEV)
    g.manual_seed(d)
    x, dy = (torch.randn(B, T, d, generator=g, device=DEV).to(dtype) for _ in range(2))
    return x, dy, 1 + 0.1 * torch.randn(d, generator=g, device=DEV)


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("B,T,d,dtype", NORM_ROWS)
def test_normalisation_layers_whose_waits_run_out_write_nothing_wrong(B, T, d, dtype, kind):
    """Every value is either right or as it was; the sums, all of them or none; and the same calls are right afterwards."""
    x, dy, gain = _norm_rows(B, T, d, dtype)
    y, mean, rstd = pe.pe_norm_forward(x, gain, kind=kind)
    sums = dict(zip(("gain_sum", "gain_stat", "bias_sum", "bias_stat"), torch.arange(4 * d, device=DEV, dtype=torch.float32).view(4, d).unbind()))
    full = {k: v.clone() for k, v in sums.items()}
    dx = pe.pe_norm_backward(x, dy, gain, mean, rstd, "square", kind=kind, accumulate=True, **full)[0]
    assert pe.pe_get_async_status(DEV) == (0, 0)
    ran_out = 0
    for _ in range(4):
        got_y, got_r, got_dx = torch.full_like(x, -77.0), torch.full_like(rstd, -77.0), torch.full_like(x, -77.0)
        got_m = None if mean is None else torch.full_like(mean, -77.0)
        got = {k: v.clone() for k, v in sums.items()}
        pe.pe_set_wait_limit_cycles(1, DEV)
        try:
            pe.pe_norm_forward(x, gain, kind=kind, out=got_y, mean=got_m, rstd=got_r)
            forward = pe.pe_get_async_status(DEV)
            pe.pe_norm_backward(x, dy, gain, mean, rstd, "square", kind=kind, accumulate=True, dx=got_dx, **got)
            backward = pe.pe_get_async_status(DEV)
        finally:
            pe.pe_set_wait_limit_cycles(0, DEV)
        assert forward[0] in (0, PE_ERR_TIMEOUT) and backward[0] in (0, PE_ERR_TIMEOUT)
        for have, want, status in ((got_y, y, forward), (got_r, rstd, forward), (got_m, mean, forward), (got_dx, dx, backward)):
            if have is not None:
                assert torch.all((have == want) | ((have == -77.0) & (status[0] != 0)))
        for k in sums:
            assert torch.equal(got[k], sums[k] if backward[0] else full[k]), k
        ran_out += backward[0] != 0
    if (B, T, d) == (64, 1024, 2048):
        assert ran_out      # (memory is slower than the kernel)
    again = {k: v.clone() for k, v in sums.items()}
    assert torch.equal(pe.pe_norm_backward(x, dy, gain, mean, rstd, "square", kind=kind, accumulate=True, **again)[0], dx)
    assert all(torch.equal(again[k], full[k]) for k in sums) and torch.equal(pe.pe_norm_forward(x, gain, kind=kind)[0], y)
    assert pe.pe_get_async_status(DEV) == (0, 0)


@pytest.mark.parametrize("count,rows,cols", [(1, 40, 72), (1, 300, 500), (2, 320, 4000)])
def test_a_status_of_an_earlier_call_does_not_stop_the_orthogonalised_update(count, rows, cols):
    g = torch.Generator(device=DEV)
    g.manual_seed(rows)
    G, theta0 = (torch.randn(count, rows, cols, generator=g, device=DEV) for _ in range(2))
    want = pe.pe_orthogonalize(G)
    stepped, moved = theta0.clone(), torch.zeros_like(G)
    pe.muon_step(stepped, moved, G, 4, lr=0.1, beta=0.9)
    assert pe.pe_get_async_status(DEV) == (0, 0)
    li = inputs.gaussian_layer(8, 512, 256, 512, seed=31, device=DEV)
    pe.pe_set_path(pe.PATH_TENSOR)
    pe.pe_set_wait_limit_cycles(1, DEV)
    try:
        pe.pe_linear_stats(li.X, li.dY, "square")      # gives up; nobody has asked for the status yet
    finally:
        pe.pe_set_wait_limit_cycles(0, DEV)
        pe.pe_set_path(pe.PATH_AUTO)
    theta, m = theta0.clone(), torch.zeros_like(G)
    pe.muon_step(theta, m, G, 4, lr=0.1, beta=0.9)
    got = pe.pe_orthogonalize(G)
    status, detail = pe.pe_get_async_status(DEV)
    assert status == PE_ERR_TIMEOUT and 1 <= detail <= 4, (status, detail)
    assert torch.equal(theta, stepped) and torch.equal(m, moved) and torch.equal(got, want)
