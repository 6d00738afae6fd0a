"""Normalisation layers in 64 bits, with bounds on what fp32 sums may be off by.

u = 2^-24 is half an fp32 step.  A sum of terms that are each off by at most k u of their magnitude, taken with no more than n
additions one after the other, is off by at most (n + k) u sum |terms| (first order; the tests add a tenth for the rest).
"""
import torch

U = 2.0 ** -24


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def row_adds(d):
    """Additions that a row's sum goes through: a thread's own (64 features, more for rows beyond 65536 or scalar ones beyond 8192), the exchanges, the warps."""
    return 64 + 5 + 32 + d // 1024


def forward(x, gain, bias, kind, eps):
    """x in 64 bits [..., d].  Returns y, mean, rstd and elementwise bounds on the fp32 error of each (before y's rounding)."""
    d = x.shape[-1]
    k = row_adds(d)
    mean = x.mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(x[..., :1])
    mean_off = U * (k + 2) * x.abs().mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(mean)
    c = x - mean
    var = c.square().mean(-1, keepdim=True)
    # a deviation is off by the mean's error and its own rounding
    c_off = mean_off + U * c.abs()
    var_off = (2 * c.abs() * c_off + c_off.square()).mean(-1, keepdim=True) + U * (k + 3) * var
    rstd = (var + eps) ** -0.5
    rstd_off = rstd * (0.5 * var_off / (var + eps) + 3 * U) + rstd * (var_off / (var + eps)) ** 2
    g = torch.ones(d, dtype=x.dtype, device=x.device) if gain is None else gain.double()
    b = torch.zeros(d, dtype=x.dtype, device=x.device) if bias is None else bias.double()
    y = c * rstd * g + b
    y_off = g.abs() * (c_off * rstd + c.abs() * rstd_off + c_off * rstd_off) + 3 * U * ((c * rstd * g).abs() + b.abs())
    return y, mean.squeeze(-1), rstd.squeeze(-1), y_off, mean_off.squeeze(-1), rstd_off.squeeze(-1)


def phi_of(phi, g):
    return g.square() if phi == "square" else torch.sign(g) if phi == "sign" else g


def backward(x, dy, gain, mean, rstd, ends, phi, kind):
    """x, dy in 64 bits [rows, d], mean / rstd the fp32 values that the kernel gets, ends: row offsets of the examples.
    Returns dx, its bound, and for gain and bias (sum, its bound, stat, its bound)."""
    d = x.shape[1]
    k = row_adds(d)
    r = rstd.double()[:, None]
    mu = mean.double()[:, None] if kind == "layer" else torch.zeros_like(r)
    h = (x - mu) * r
    h_off = 2 * U * h.abs()
    g = torch.ones(d, dtype=x.dtype, device=x.device) if gain is None else gain.double()
    w = dy * g
    m1, m2 = (w * h).mean(1, keepdim=True), w.mean(1, keepdim=True)
    m1_off, m2_off = U * (k + 6) * (w * h).abs().mean(1, keepdim=True), U * (k + 3) * w.abs().mean(1, keepdim=True)
    if kind != "layer":
        m2, m2_off = torch.zeros_like(m2), torch.zeros_like(m2)
    dx = r * (w - h * m1 - m2)
    dx_off = r * (U * w.abs() + h.abs() * m1_off + h_off * m1.abs() + m2_off + 3 * U * (w.abs() + (h * m1).abs() + m2.abs())) + 2 * U * dx.abs()
    rows = x.shape[0]
    # additions of a feature's sum: a worker's rows (at least 148 workers, or at most 16 rows each), then the joins of groups, blocks and warps
    depth = min(rows + 8, rows // 148 + 16 + 256 + 40)
    out = []
    for term, k_term in ((dy * h, 4), (dy, 0)):
        sums = torch.stack([term[a:b].sum(0) for a, b in zip(ends[:-1], ends[1:])])
        mags = torch.stack([term[a:b].abs().sum(0) for a, b in zip(ends[:-1], ends[1:])])
        off = U * (depth + k_term) * mags
        total, total_off = sums.sum(0), off.sum(0) + U * (depth + 2) * sums.abs().sum(0)
        stat = phi_of(phi, sums).sum(0)
        if phi == "square":
            stat_off = (2 * sums.abs() * off + off.square()).sum(0) + U * (depth + 3) * stat
        elif phi == "sign":
            stat_off = 2.0 * (sums.abs() <= 1.1 * off).double().sum(0)      # a sum within its error of zero may have either sign
        else:
            stat_off = total_off
        out.append((total, total_off, stat, stat_off))
    return dx, dx_off, out


def assert_within(name, got, want, off, rounding=0.0):
    """|got - want| within a tenth more than off, and a rounding relative to the value; NaN where wanted."""
    got, want = got.double(), want.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want)), name
    worst = ((got - want).abs() - 1.1 * off - rounding * (1 + 1e-6) * (want.abs() + 1.1 * off)).nan_to_num(nan=0.0).max() if got.numel() else torch.zeros(())
    assert float(worst) <= 1e-45, (name, float(worst))
