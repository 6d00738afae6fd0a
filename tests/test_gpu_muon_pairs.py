"""Long matrices, which take two steps at a time, and products that are cut along the contraction index; waits that run out."""
import pytest
import torch

import paper_2510_00236_b200 as pe
from test_gpu_muon import A, B_, C, DEV, U, _noise, _rel, exact, tolerance

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


# tiles of every width for every product, X X^T in slices for every width, one step and two at a time (test_muon_checks.py looks the plans over)
PRECISE = [(1, 300, 300), (1, 512, 2048), (1, 256, 4096), (1, 2048, 2048), (1, 1537, 1601), (2, 1100, 1100), (1, 8192, 2048), (1, 512, 32768), (12, 600, 600), (12, 601, 1999),
           (1, 1000, 8000), (1, 2049, 3000), (80, 130, 300), (1, 65, 129), (12, 449, 272), (2, 655, 2586), (12, 322, 1069), (20, 590, 326), (2, 962, 2231), (1, 1427, 2202),
           (1, 3078, 514), (40, 129, 129), (40, 143, 74)]


def _halves(v):
    """Operands of 11 bits, scaled as the kernels scale theirs."""
    return (v * 4096.0).half().double() / 4096.0


def sensitivity(G, steps=5):
    """What the iteration makes of operands rounded to 11 bits, relative to the result and to the rounding of 2^-11 (about 3 for noise, 60 where few directions dominate)."""
    X = G.double() / torch.linalg.vector_norm(G.double())
    X = X.T if X.shape[0] > X.shape[1] else X
    Y = X
    eye = torch.eye(X.shape[0], dtype=X.dtype, device=X.device)
    for _ in range(steps):
        S = X @ X.T
        X = (A * eye + B_ * S + C * (S @ S)) @ X
        y = _halves(Y)
        S = y @ y.T
        s = _halves(S)
        Y = _halves(A * eye + B_ * s + C * (s @ s)) @ y
    return float((X - Y).norm() / X.norm()) * 2.0 ** 11


def precision(G, paired, steps=5):
    """Relative error of the Frobenius norm of what the kernels' arithmetic may cost.  Two halves leave 2^-22 of an operand where one leaves 2^-11, at the same places: the
    sensitivity times 2^-22; lo lo, which is left out, is as much at most.  The tensor cores add by truncation, an accumulator takes 64 values in four
    instructions (the cross terms before are 2^-11 of them): 2.5 * 2^-23 of a sum at most, and as much again for the terms within an instruction.  Off by a relative
    e on one side, as the diagonals of A and A A are, whose terms have one sign, a step is off by (|b| s^3 + 3 |c| s^5) e, 12 e at s = 1, where the rounding of
    operands costs about 1.5 of its unit: 12 * 2.5 / 1.5 = 20 sensitivities.  Together 22, say 24; with two steps at a time, five more products, twice that."""
    return (48 if paired else 24) * sensitivity(G, steps) * 2.0 ** -22


@pytest.mark.parametrize("spread", [0.0, 0.3])
@pytest.mark.parametrize("count,rows,cols", PRECISE)
def test_operands_of_22_bits(count, rows, cols, spread):
    """The bounds of the other tests leave room for operands of 11 bits; these are for the arithmetic as it is."""
    G = _noise(count, rows, cols, rows + 3 * cols, spread)
    paired = pe.pe_plan_query(pe.PLAN_ORTHOGONALIZE, 0, count, 1, cols, rows, 148)[3] == 2
    got = pe.pe_orthogonalize(G)
    assert pe.pe_get_async_status(DEV) == (0, 0)
    for k in sorted({0, count // 2, count - 1}):
        assert _rel(got[k], exact(G[k])) <= precision(G[k], paired), k
    if count > 1:      # every matrix by itself, in tiles of another width perhaps
        for k in range(count):
            assert _rel(got[k], pe.pe_orthogonalize(G[k]).double()) <= 2 * precision(G[k], True), k


@pytest.mark.parametrize("count,rows,cols", [(1, 2048, 2048), (1, 8192, 2048), (12, 601, 1999), (1, 512, 2048)])
def test_muon_step_with_operands_of_22_bits(count, rows, cols):
    theta, m, sum_g = torch.zeros(count, rows, cols, device=DEV), _noise(count, rows, cols, 7) * 0.1, _noise(count, rows, cols, 8)
    m0 = m.double()
    paired = pe.pe_plan_query(pe.PLAN_ORTHOGONALIZE, 0, count, 1, cols, rows, 148)[3] == 2
    pe.muon_step(theta, m, sum_g, 4, lr=1.0, beta=0.9, update_scale=1.0)
    for k in range(count):
        g = sum_g[k].double() / 4
        direction = 0.1 * g + 0.9 * (0.9 * m0[k] + 0.1 * g)
        # the direction is rounded to fp32 a few times on its way: 6 * 2^-24 of each value, one more and a half of the operands' units
        assert _rel(-theta[k], exact(direction)) <= 1.1 * precision(direction, paired), k


@pytest.mark.parametrize("count,rows,cols", [(1, 300, 4100), (12, 601, 1999), (1, 158, 1204), (2, 1001, 999)])
def test_what_the_workspace_holds_before_does_not_matter(count, rows, cols):
    G = _noise(count, rows, cols, 9)
    need = pe.pe_orthogonalize_workspace_bytes(count, rows, cols)
    got = [pe.pe_orthogonalize(G, workspace=torch.full((need,), fill, dtype=torch.uint8, device=DEV)) for fill in (0, 255, 127)]
    assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2]) and torch.isfinite(got[0]).all()
