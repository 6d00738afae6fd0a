"""Orthogonalised matrices and the optimizer step around them, against the polynomial in 64 bits."""
import pytest
import torch

import paper_2510_00236_b200 as pe

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
A, B_, C = 3.4445, -4.7750, 2.0315
U = 2.0 ** -24


def exact(G, steps=5):
    """One matrix in 64 bits: the odd polynomial by way of X X^T X."""
    X = G.double()
    norm = torch.linalg.vector_norm(X)
    if float(norm) == 0.0:
        return X
    X = X / norm
    for _ in range(steps):
        S = X.T @ X if X.shape[0] > X.shape[1] else X @ X.T
        cube = X @ S if X.shape[0] > X.shape[1] else S @ X
        fifth = cube @ S if X.shape[0] > X.shape[1] else S @ cube
        X = A * X + B_ * cube + C * fifth
    return X


def tolerance(G, steps=5):
    """Relative error of the Frobenius norm that the arithmetic may cost.  Each step forms its products from operands off by at most 2^-22 each, in sums of
    fp32 (about 2^-22 together with their order, relative to the spectral norms, which are at most 1.21, 1.45 and 3.45): with a factor
    |a| + 3 |b| s^2 + 5 |c| s^4 <= 15 for what enters through A and Q, a step adds at most 15 * 4 * 2^-22 of ||X||_F.  What came before is multiplied by the
    slope: at most 3.4445 a step where singular values are still small, and at most 1.6 in the range [0.68, 1.21] that they end up in; so that
    the relative error grows where a few directions have arrived and most of the norm has not.  Taken from the exact iteration: ||X_k||_F per step."""
    X = G.double()
    X = X / torch.linalg.vector_norm(X)
    X = X.T if X.shape[0] > X.shape[1] else X
    off = 4 * 2.0 ** -22
    for _ in range(steps):
        s = torch.linalg.svdvals(X) if min(X.shape) > 1 else torch.linalg.vector_norm(X).view(1)
        new = (A * s + B_ * s ** 3 + C * s ** 5)
        # slopes per direction: an error of norm `off` is spread over directions and is multiplied by no more than the largest slope
        slope = max(float((A + 3 * B_ * s ** 2 + 5 * C * s ** 4).abs().max()), float((new / s.clamp_min(1e-300)).abs().max()))
        off = off * slope + 15 * 4 * 2.0 ** -22 * float(s.norm())
        X = torch.diag(new)
    return off / float(new.norm())


def _noise(count, rows, cols, seed, spread=0.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    G = torch.randn(count, rows, cols, generator=g, device=DEV)
    if spread:
        r = max(1, min(rows, cols) // 16)
        G = G + spread * torch.randn(count, rows, r, generator=g, device=DEV) @ torch.randn(count, r, cols, generator=g, device=DEV)
    return G


def _rel(got, want):
    return float((got.double() - want).norm() / want.norm())


SHAPES = [(1, 1, 1), (2, 1, 9), (3, 7, 1), (1, 8, 8), (1, 64, 64), (3, 33, 65), (2, 64, 300), (1, 130, 129), (2, 257, 96), (1, 256, 256), (1, 300, 300), (1, 128, 2000),
          (5, 100, 12), (1, 512, 512), (2, 512, 1025), (1, 1030, 520), (1, 16, 5000), (1, 777, 1311)]


@pytest.mark.parametrize("spread", [0.0, 0.3])
@pytest.mark.parametrize("count,rows,cols", SHAPES)
def test_orthogonalize_fp32(count, rows, cols, spread):
    G = _noise(count, rows, cols, rows * 7 + cols, spread) * 1e-3
    got = pe.pe_orthogonalize(G)
    assert pe.pe_get_async_status(DEV) == (0, 0)
    for k in range(count):
        assert _rel(got[k], exact(G[k])) <= tolerance(G[k]), k


@pytest.mark.parametrize("count,rows,cols", [(1, 64, 64), (2, 33, 65), (3, 257, 96), (1, 300, 700), (1, 1, 5)])
def test_orthogonalize_bf16(count, rows, cols):
    G = _noise(count, rows, cols, rows + cols).to(torch.bfloat16)
    got = pe.pe_orthogonalize(G, out=G.clone())
    inplace = G.clone()
    assert pe.pe_orthogonalize(inplace, out=inplace) is inplace and torch.equal(inplace, got)
    for k in range(count):
        want = exact(G[k])
        # one rounding to bf16: at most half a step of each value
        assert _rel(got[k], want) <= tolerance(G[k]) + 2.0 ** -8, k


@pytest.mark.parametrize("steps", [1, 2, 3, 8])
def test_number_of_steps(steps):
    G = _noise(1, 96, 200, steps)
    assert _rel(pe.pe_orthogonalize(G, steps=steps)[0], exact(G[0], steps)) <= tolerance(G[0], steps)


@pytest.mark.parametrize("scale", [1e-30, 1e-42, 1e30, 3e36])
def test_any_scale_of_the_input(scale):
    G = _noise(1, 70, 90, 4) * scale
    assert _rel(pe.pe_orthogonalize(G)[0], exact(G[0])) <= tolerance(G[0])


def test_singular_values_end_near_one():
    G = _noise(1, 128, 512, 11)
    s = torch.linalg.svdvals(pe.pe_orthogonalize(G)[0].double())
    assert 0.6 < float(s.min()) and float(s.max()) < 1.25


def test_zero_matrices_and_non_finite_ones_stay_apart():
    G = _noise(5, 80, 144, 12)
    clean = pe.pe_orthogonalize(G.clone())
    G[1] = 0.0
    G[2, 3, 4] = float("nan")
    G[4, 0, 0] = float("inf")
    got = pe.pe_orthogonalize(G)
    assert torch.equal(got[0], clean[0]) and torch.equal(got[3], clean[3])
    assert torch.all(got[1] == 0) and torch.isnan(got[2]).all() and torch.isnan(got[4]).all()


def test_two_dimensional_and_repeated_calls_agree_bit_for_bit():
    G = _noise(2, 300, 520, 13)
    both = pe.pe_orthogonalize(G)
    assert torch.equal(pe.pe_orthogonalize(G[1].clone()), both[1]) and torch.equal(pe.pe_orthogonalize(G), both)
    # a transposed matrix gives the transposed result: the same iteration
    assert torch.equal(pe.pe_orthogonalize(G[0].T.contiguous()), both[0].T)


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("count,rows,cols", [(1, 64, 64), (2, 33, 65), (3, 96, 40), (1, 520, 300), (1, 300, 1030), (1, 1, 3)])
def test_muon_step(count, rows, cols, nesterov):
    theta, m, sum_g = _noise(count, rows, cols, 1), _noise(count, rows, cols, 2) * 0.1, _noise(count, rows, cols, 3) * 5
    theta0, m0 = theta.double(), m.double()
    lp = torch.empty_like(theta, dtype=torch.bfloat16)
    kw = dict(lr=0.05, beta=0.9, weight_decay=1e-3, grad_scale=2.0)
    pe.muon_step(theta, m, sum_g, 16, nesterov=nesterov, theta_lp=lp, **kw)
    g = 2.0 * sum_g.double() / 16
    m_ref = 0.9 * m0 + 0.1 * g
    assert float(((m.double() - m_ref).abs() - 6 * U * (m0.abs() + g.abs())).max()) <= 0
    upd = 0.1 * g + 0.9 * m_ref if nesterov else m_ref
    scale = max(1.0, rows / cols) ** 0.5
    for k in range(count):
        o = exact(upd[k])
        want = theta0[k] - 0.05 * scale * o - 1e-3 * theta0[k]
        # the direction's own fp32 rounding (6 u of each value) goes through the same slopes as the operands' 2^-22
        assert float((theta[k].double() - want).norm()) <= 0.05 * scale * 2 * tolerance(upd[k]) * float(o.norm()) + 4 * U * float(theta0[k].norm())
    assert torch.equal(lp, theta.to(torch.bfloat16))


def test_muon_step_without_copy_and_with_own_scale():
    theta, m, sum_g = _noise(1, 40, 72, 5)[0], torch.zeros(40, 72, device=DEV), _noise(1, 40, 72, 6)[0]
    start = theta.double()
    pe.muon_step(theta, m, sum_g, 1, lr=0.1, beta=0.5, update_scale=0.25, nesterov=False)
    o = exact(sum_g)
    assert float((theta.double() - (start - 0.025 * o)).norm()) <= 0.025 * 2 * tolerance(sum_g) * float(o.norm()) + 4 * U * float(start.norm())


def test_no_matrices():
    empty = torch.empty(0, 4, 5, device=DEV)
    assert pe.pe_orthogonalize(empty).shape == (0, 4, 5)
    pe.muon_step(empty, empty.clone(), empty.clone(), 4, lr=0.1, beta=0.9)


def test_another_stream_and_a_captured_graph():
    G = _noise(2, 200, 330, 21)
    want = pe.pe_orthogonalize(G)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = pe.pe_orthogonalize(G)
    side.synchronize()
    assert torch.equal(got, want)
    held = torch.zeros_like(G)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = pe.pe_orthogonalize(held)
    for _ in range(2):
        held.copy_(G)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_workspace_is_checked():
    G, out = _noise(1, 64, 64, 1), torch.full((1, 64, 64), 5.0, device=DEV)
    need = pe.pe_orthogonalize_workspace_bytes(1, 64, 64)
    for ws in (torch.empty(need - 1, dtype=torch.uint8, device=DEV), torch.empty(need + 8, dtype=torch.uint8, device=DEV)[8:]):
        with pytest.raises(pe.PestatsError) as e:
            pe.pe_orthogonalize(G, out=out, workspace=ws)
        assert e.value.status in (9, 3)
    torch.cuda.synchronize()
    assert torch.all(out == 5.0)
    # what the workspace holds before the call does not matter
    a = pe.pe_orthogonalize(G, workspace=torch.full((need,), 255, dtype=torch.uint8, device=DEV))
    assert torch.equal(a, pe.pe_orthogonalize(G))
