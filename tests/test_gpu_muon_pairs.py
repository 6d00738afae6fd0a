"""Long matrices, which take two steps at a time, and products that are cut along the contraction index; waits that run out."""
import pytest
import torch

import paper_2510_00236_b200 as pe
from test_gpu_muon import DEV, U, _noise, _rel, exact, tolerance

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("spread", [0.0, 0.3])
@pytest.mark.parametrize("count,rows,cols", [(1, 256, 4096), (1, 5000, 300), (2, 257, 3001), (1, 600, 2500), (3, 2048, 512), (1, 1000, 8000)])
def test_long_matrices(count, rows, cols, spread):
    G = _noise(count, rows, cols, rows + cols, spread)
    got = pe.pe_orthogonalize(G)
    assert pe.pe_get_async_status(DEV) == (0, 0)
    for k in range(count):
        # two steps at a time: five more products of A's size, each off as the others are, and A's errors enter by the square of the slope once per pair of
        # steps (3.4^2 in place of 3.4): no more than four times the bound of single steps
        assert _rel(got[k], exact(G[k])) <= 4 * tolerance(G[k]), k
    assert torch.equal(pe.pe_orthogonalize(G), got)


@pytest.mark.parametrize("steps", [1, 2, 3, 4, 6])
def test_odd_and_even_numbers_of_steps(steps):
    G = _noise(1, 300, 4100, steps)
    assert _rel(pe.pe_orthogonalize(G, steps=steps)[0], exact(G[0], steps)) <= 4 * tolerance(G[0], steps)


def test_long_matrices_that_are_zero_or_not_finite():
    G = _noise(4, 320, 4000, 3)
    clean = pe.pe_orthogonalize(G.clone())
    G[0] = 0.0
    G[2, 319, 3999] = float("inf")
    got = pe.pe_orthogonalize(G)
    assert torch.all(got[0] == 0) and torch.isnan(got[2]).all() and torch.equal(got[1], clean[1]) and torch.equal(got[3], clean[3])


@pytest.mark.parametrize("count,rows,cols", [(1, 4000, 320), (2, 257, 3001)])
def test_muon_step_on_long_matrices(count, rows, cols):
    theta, m, sum_g = _noise(count, rows, cols, 1), _noise(count, rows, cols, 2), _noise(count, rows, cols, 3)
    start, m0 = theta.double(), m.double()
    lp = torch.empty_like(theta, dtype=torch.bfloat16)
    pe.muon_step(theta, m, sum_g, 4, lr=0.03, beta=0.95, update_scale=1.0, theta_lp=lp)
    m_ref = 0.95 * m0 + 0.05 * sum_g.double() / 4
    assert float(((m.double() - m_ref).abs() - 6 * U * (m0.abs() + sum_g.abs())).max()) <= 0
    for k in range(count):
        direction = 0.05 * sum_g[k].double() / 4 + 0.95 * m_ref[k]
        o = exact(direction)
        assert float((theta[k].double() - (start[k] - 0.03 * o)).norm()) <= 0.03 * 8 * tolerance(direction) * float(o.norm()) + 4 * U * float(start[k].norm())
    assert torch.equal(lp, theta.to(torch.bfloat16))


def test_two_graphs_with_workspaces_of_their_own():
    shapes = ((1, 300, 4100), (2, 200, 330))
    held = [torch.zeros(s, device=DEV) for s in shapes]
    graphs, outs = [], []
    for h in held:
        g = torch.cuda.CUDAGraph()
        ws = torch.empty(pe.pe_orthogonalize_workspace_bytes(*h.shape), dtype=torch.uint8, device=DEV)
        out = torch.empty_like(h)
        pe.pe_orthogonalize(h, out=out, workspace=ws)
        with torch.cuda.graph(g):
            pe.pe_orthogonalize(h, out=out, workspace=ws)
        graphs.append((g, ws))
        outs.append(out)
    for k, h in enumerate(held):
        h.copy_(_noise(*h.shape, 30 + k))
    streams = [torch.cuda.Stream() for _ in held]
    torch.cuda.synchronize()
    for _ in range(3):
        for (g, _), s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for h, out in zip(held, outs):
        assert torch.equal(out, pe.pe_orthogonalize(h))


def test_waits_that_run_out_leave_parameters_alone():
    """The budget of every wait is lowered to a cycle: the kernels give up and say so; afterwards the same calls are right."""
    theta, m, sum_g = _noise(1, 512, 1024, 1)[0], _noise(1, 512, 1024, 2)[0], _noise(1, 512, 1024, 3)[0]
    start, m0 = theta.clone(), m.clone()
    # more rows than L2 holds: memory is slower than the kernels, so some of their many waits find nothing yet
    x = torch.randn(64, 1024, 2048, device=DEV, dtype=torch.bfloat16)
    dy = torch.randn_like(x)
    gain = torch.ones(2048, device=DEV)
    y, mean, rstd = pe.pe_norm_forward(x, gain)
    want = pe.pe_norm_backward(x, dy, gain, mean, rstd, "square")
    pe.pe_set_wait_limit_cycles(1, DEV)
    try:
        pe.muon_step(theta, m, sum_g, 4, lr=0.1, beta=0.9)
        status, detail = pe.pe_get_async_status(DEV)
        assert status == 8 and 101 <= detail <= 105, (status, detail)
        assert torch.equal(theta, start)
        pe.pe_norm_backward(x, dy, gain, mean, rstd, "square")
        status, detail = pe.pe_get_async_status(DEV)
        assert status == 8 and detail == 201, (status, detail)
        pe.pe_norm_forward(x, gain)
        assert pe.pe_get_async_status(DEV)[0] == 8
    finally:
        pe.pe_set_wait_limit_cycles(0, DEV)
    assert pe.pe_get_async_status(DEV) == (0, 0)
    m.copy_(m0)
    pe.muon_step(theta, m, sum_g, 4, lr=0.1, beta=0.9)
    assert pe.pe_get_async_status(DEV) == (0, 0) and not torch.equal(theta, start)
    again = pe.pe_norm_backward(x, dy, gain, mean, rstd, "square")
    assert all(torch.equal(a, b) for a, b in zip(want, again)) and torch.equal(pe.pe_norm_forward(x, gain)[0], y)
