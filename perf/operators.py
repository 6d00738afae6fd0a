"""Normalisation layers with per-example statistics, and the orthogonalised update, as cases to be timed.

A training step that takes per-example statistics of its linear layers also runs normalisation layers between them and
updates matrices.  ``forward`` and ``backward`` are a normalisation layer (mean and variance, or root mean square alone)
over rows [B, T, d]; the backward pass gives dx and, for the gain and the bias, the sum over the examples b of their
gradients G_b and of phi(G_b), phi the identity or the square.  ``ragged`` is the same for a packed batch.
``orthogonalise`` replaces matrices by a polynomial of their singular values (five quintic Newton-Schulz steps),
``muon`` is the optimizer step around that: momentum, orthogonalised update, parameters.

``run`` computes a case in plain torch operations where ``own`` is false and through the package's public calls where it is
true.  phi = sign is left to the tests: a gradient next to zero may take either sign within rounding.
"""
import math

import torch

own = False

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
EPS = 1e-5
NS_A, NS_B, NS_C = 3.4445, -4.7750, 2.0315      # the quintic a s + b s^3 + c s^5 of a singular value s
STEPS = 5
MUON = dict(lr=0.02, beta=0.95, weight_decay=1e-4)


def listed():
    return [
        # A small fp32 layer: the smallest calls of a training step, where latency counts.
        dict(name="forward_small", kind="forward", norm="layer", dtype="fp32", B=8, T=16, d=64),
        dict(name="backward_small", kind="backward", norm="layer", dtype="fp32", phi="square", B=8, T=16, d=64),
        # The pre-RMSNorm of a 6-layer decoder (d_model 512, 64 sequences of 256 tokens).
        dict(name="forward_decoder", kind="forward", norm="rms", dtype="bf16", B=64, T=256, d=512),
        dict(name="backward_decoder", kind="backward", norm="rms", dtype="bf16", phi="square", B=64, T=256, d=512),
        # The layer norm before the large layer: the largest activations of a single GPU's step.
        dict(name="forward_large", kind="forward", norm="layer", dtype="bf16", B=256, T=1024, d=2048),
        dict(name="backward_large", kind="backward", norm="layer", dtype="bf16", phi="square", B=256, T=1024, d=2048),
        # Many short examples of an odd width, fp32: an example's sum ends after a few rows.
        dict(name="backward_short_odd", kind="backward", norm="layer", dtype="fp32", phi="square", B=4096, T=3, d=1001),
        # A packed batch of unequal sequence lengths (instruction tuning).
        dict(name="backward_ragged", kind="ragged", norm="layer", dtype="bf16", phi="square", B=64, T=700, d=1024),
        # One small fp32 matrix, and the up-projections of a 6-layer decoder stacked in one call.
        dict(name="orthogonalise_small", kind="orthogonalise", dtype="fp32", count=1, rows=64, cols=64),
        dict(name="orthogonalise_stack", kind="orthogonalise", dtype="bf16", count=6, rows=2048, cols=512),
        # The optimizer step of one MLP matrix of that decoder, and of the large layer.
        dict(name="muon_mlp", kind="muon", nesterov=True, count=1, rows=512, cols=2048),
        dict(name="muon_large", kind="muon", nesterov=True, count=1, rows=8192, cols=2048),
    ]


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["forward", "backward", "backward", "ragged", "orthogonalise", "muon"])
    if kind in ("forward", "backward", "ragged"):
        most = 256 * 1024 * 2048 // 4        # elements; fp32 moves twice the bytes, and no case is dearer than the listed ones
        while True:
            B, T, d = _log_uniform(rng, 1, 4096), _log_uniform(rng, 1, 4096), _log_uniform(rng, 16, 16384)      # of a few features little is left of dx but rounding
            if rng.random() < 0.5:
                d = max(64, d // 64 * 64)
            if 1000 <= B * T * d <= most:
                break
        case = dict(kind=kind, norm=rng.choice(["layer", "rms"]), dtype="bf16" if kind == "ragged" else rng.choice(["bf16", "bf16", "fp32"]), B=B, T=T, d=d)
        if kind != "forward":
            case["phi"] = rng.choice(["square", "square", "identity"])
        return case
    while True:
        count, rows, cols = rng.choice([1, 1, 2, 3, 6, 12]), _log_uniform(rng, 1, 8192), _log_uniform(rng, 1, 8192)
        if rng.random() < 0.5:
            rows, cols = max(64, rows // 64 * 64), max(64, cols // 64 * 64)
        n, m = min(rows, cols), max(rows, cols)
        if count * (3.0 * n * n * m + n ** 3) <= 3.0 * 2048 ** 2 * 8192 + 2048 ** 3 and count * n * m <= 3e7:
            break
    case = dict(kind=kind, count=count, rows=rows, cols=cols)
    if kind == "muon":
        case["nesterov"] = rng.random() < 0.7
    else:
        case["dtype"] = rng.choice(["bf16", "fp32"])
    return case


# ------------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) & 0x7fffffffffff)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _offsets(case, seed):
    """A packed batch of B * T tokens in all, cut at random places: most sequences short, a few long, an empty one among them."""
    g = torch.Generator()
    g.manual_seed(seed)
    B, total = case["B"], case["B"] * case["T"]
    offs = torch.zeros(B + 1, dtype=torch.int32)
    offs[1:B] = torch.sort(torch.randint(0, total + 1, (B - 1,), generator=g))[0]
    offs[B] = total
    if B > 2:
        offs[B // 2] = offs[B // 2 + 1]
    return offs


def _matrices(g, count, rows, cols):
    """What momentum looks like: a few directions that stand out of noise, in some scale."""
    r = max(1, min(rows, cols) // 16)
    u, v = _randn(g, count, rows, r), _randn(g, count, r, cols)
    return (_randn(g, count, rows, cols) + (u / r ** 0.5) @ v) * 1e-2


def prepare(case, seed):
    g = _gen(seed)
    s = dict(case)
    kind = case["kind"]
    if kind in ("forward", "backward", "ragged"):
        dt, B, T, d = DTYPES[case["dtype"]], case["B"], case["T"], case["d"]
        if kind == "ragged":
            offs = _offsets(case, seed)
            s["seq_offsets"] = offs.to(DEV)
            lead = (B * T + 5,)        # a few rows behind the last sequence
        else:
            lead = (B, T)
        # the residual stream: features of unequal scale, tokens of unequal size with an offset of their own
        feature = torch.exp(0.5 * _randn(g, d))
        x = _randn(g, *lead, d).mul_(feature).add_(0.3 * _randn(g, *lead, 1)).to(dt)
        s["x"] = x
        s["gain"] = 1 + 0.1 * _randn(g, d)
        s["bias"] = 0.1 * _randn(g, d) if case["norm"] == "layer" else None
        if kind != "forward":
            dy = _randn(g, *lead, d).mul_(T ** -0.5)
            scale = torch.where(torch.rand(*lead[:1], *([1] * (dy.dim() - 1)), generator=g, device=DEV) < 0.1, 5.0, 1.0)
            s["dy"] = dy.mul_(scale).to(dt)
            rows = x.view(-1, d)
            mean, rstd = torch.zeros(rows.shape[0], device=DEV), torch.empty(rows.shape[0], device=DEV)
            for at in range(0, rows.shape[0], 1 << 16):      # what the forward pass kept of every row
                part = rows[at:at + (1 << 16)].float()
                if case["norm"] == "layer":
                    mean[at:at + (1 << 16)] = part.mean(1)
                    part = part - part.mean(1, keepdim=True)
                rstd[at:at + (1 << 16)] = torch.rsqrt(part.square().mean(1) + EPS)
            s["mean"], s["rstd"] = (mean.view(lead) if case["norm"] == "layer" else None), rstd.view(lead)
            s["dx"] = torch.zeros_like(x)
        return s
    count, rows, cols = case["count"], case["rows"], case["cols"]
    G = _matrices(g, count, rows, cols)
    if kind == "orthogonalise":
        s["G"] = G.to(DTYPES[case["dtype"]])
        return s
    s["sum_g"], s["B"] = G * 64.0, 64
    s["m"] = 0.3 * G + 2e-3 * _randn(g, count, rows, cols)
    s["theta"] = _randn(g, count, rows, cols).mul_(cols ** -0.5)
    s["theta_lp"] = s["theta"].to(torch.bfloat16)
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    return (_own if own else _plain)(s)


def _own(s):
    import paper_2510_00236_b200 as pe
    kind = s["kind"]
    if kind == "forward":
        y, mean, rstd = pe.pe_norm_forward(s["x"], s["gain"], s["bias"], kind=s["norm"], eps=EPS)
        return {"y": y, "mean": mean, "rstd": rstd}
    if kind in ("backward", "ragged"):
        args = (s["x"], s["dy"], s["gain"], s["mean"], s["rstd"])
        if kind == "ragged":
            got = pe.pe_norm_backward_ragged(*args, s["seq_offsets"], s["phi"], kind=s["norm"], dx=s["dx"])
        else:
            got = pe.pe_norm_backward(*args, s["phi"], kind=s["norm"], dx=s["dx"])
        return dict(zip(("dx", "gain_sum", "gain_stat", "bias_sum", "bias_stat"), got))
    if kind == "orthogonalise":
        return {"out": pe.pe_orthogonalize(s["G"], steps=STEPS)}
    pe.muon_step(s["theta"], s["m"], s["sum_g"], s["B"], steps=STEPS, nesterov=s["nesterov"], theta_lp=s["theta_lp"], **MUON)
    return {"theta": s["theta"], "theta_lp": s["theta_lp"], "m": s["m"]}


def _plain(s):
    kind = s["kind"]
    if kind == "forward":
        x = s["x"].float()
        mean = x.mean(-1) if s["norm"] == "layer" else None
        if mean is not None:
            x = x - mean.unsqueeze(-1)
        rstd = torch.rsqrt(x.square().mean(-1) + EPS)
        y = x * rstd.unsqueeze(-1) * s["gain"]
        if s["bias"] is not None:
            y = y + s["bias"]
        return {"y": y.to(s["x"].dtype), "mean": mean, "rstd": rstd}
    if kind in ("backward", "ragged"):
        x, dy = s["x"].float(), s["dy"].float()
        if s["mean"] is not None:
            x = x - s["mean"].unsqueeze(-1)
        rstd = s["rstd"].unsqueeze(-1)
        xhat = x * rstd
        w = dy * s["gain"]
        dx = w - xhat * (w * xhat).mean(-1, keepdim=True)
        if s["mean"] is not None:
            dx = dx - w.mean(-1, keepdim=True)
        dx = (dx * rstd).to(s["dx"].dtype)
        contribution = dy * xhat
        if kind == "backward":
            s["dx"].copy_(dx)
            G, H = contribution.sum(1), dy.sum(1)
        else:
            offs = s["seq_offsets"].long()
            row = torch.arange(x.shape[0], device=x.device)
            example = torch.searchsorted(offs[1:], row, right=True)        # rows behind the last sequence: example B
            s["dx"].copy_(torch.where((example < s["B"]).unsqueeze(-1), dx, s["dx"]))
            G = x.new_zeros((s["B"] + 1, x.shape[1])).index_add_(0, example, contribution)[:s["B"]]
            H = x.new_zeros((s["B"] + 1, x.shape[1])).index_add_(0, example, dy)[:s["B"]]
        square = s["phi"] == "square"
        out = {"dx": s["dx"], "gain_sum": G.sum(0), "gain_stat": (G.square() if square else G).sum(0), "bias_sum": None, "bias_stat": None}
        if s["norm"] == "layer":
            out["bias_sum"], out["bias_stat"] = H.sum(0), (H.square() if square else H).sum(0)
        return out
    if kind == "orthogonalise":
        return {"out": _newton_schulz(s["G"].float()).to(s["G"].dtype)}
    grad = s["sum_g"] / s["B"]
    beta = MUON["beta"]
    s["m"].mul_(beta).add_(grad, alpha=1 - beta)
    update = _newton_schulz(s["m"] * beta + grad * (1 - beta) if s["nesterov"] else s["m"])
    scale = max(1.0, s["rows"] / s["cols"]) ** 0.5
    s["theta"].copy_(s["theta"] - MUON["lr"] * scale * update - MUON["weight_decay"] * s["theta"])
    s["theta_lp"].copy_(s["theta"])
    return {"theta": s["theta"], "theta_lp": s["theta_lp"], "m": s["m"]}


def _newton_schulz(G):
    """[count, rows, cols] in 32 bits: X = G / ||G||_F, then five times X <- a X + (b A + c A A) X with A = X X^T of the shorter side."""
    X = G / G.double().square().sum((1, 2), keepdim=True).sqrt().clamp_min(torch.finfo(torch.float64).tiny).float()
    tall = X.shape[1] > X.shape[2]
    if tall:
        X = X.transpose(1, 2)
    for _ in range(STEPS):
        A = X @ X.transpose(1, 2)
        X = NS_A * X + (NS_B * A + NS_C * (A @ A)) @ X
    return X.transpose(1, 2) if tall else X


# ------------------------------------------------------------------------------------------------ floors and definitions
def work(case):
    kind = case["kind"]
    if kind in ("forward", "backward", "ragged"):
        es = 2 if case["dtype"] == "bf16" else 4
        rows, d = case["B"] * case["T"], case["d"]
        kept = rows * (8 if case["norm"] == "layer" else 4)      # mean and rstd of every row
        if kind == "forward":
            return {"bytes": 2 * es * rows * d + kept + 8 * d, "flops": 8 * rows * d}
        return {"bytes": 3 * es * rows * d + kept + 20 * d, "flops": 14 * rows * d}
    count, rows, cols = case["count"], case["rows"], case["cols"]
    n, m = min(rows, cols), max(rows, cols)
    # X X^T and A A are symmetric: half of their products
    flops = count * STEPS * (3.0 * n * n * m + float(n) ** 3)
    if kind == "orthogonalise":
        return {"bytes": count * rows * cols * (4 if case["dtype"] == "bf16" else 8), "flops": flops}
    return {"bytes": count * rows * cols * (4 * 5 + 2), "flops": flops}


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "forward":
        return _exact_forward(s)
    if kind in ("backward", "ragged"):
        return _exact_backward(s)
    if kind == "orthogonalise":
        return {"out": torch.stack([_exact_polynomial(G.double()) for G in s["G"]])}
    grad = s["sum_g"].double() / s["B"]
    beta = MUON["beta"]
    m = beta * s["m"].double() + (1 - beta) * grad
    direction = (1 - beta) * grad + beta * m if s["nesterov"] else m
    scale = math.sqrt(max(1.0, case["rows"] / case["cols"]))
    theta = s["theta"].double()
    theta = theta - MUON["lr"] * scale * torch.stack([_exact_polynomial(D) for D in direction]) - MUON["weight_decay"] * theta
    return {"theta": theta, "theta_lp": theta, "m": m}


def _exact_polynomial(X):
    """The quintic applied five times to the singular values of one matrix in 64 bits, with odd powers X, X X^T X, X X^T X X^T X."""
    norm = torch.linalg.vector_norm(X)
    if float(norm) == 0.0:
        return X
    X = X / norm
    for _ in range(STEPS):
        cube = X @ (X.T @ X) if X.shape[0] > X.shape[1] else (X @ X.T) @ X
        fifth = cube @ (X.T @ X) if X.shape[0] > X.shape[1] else (X @ X.T) @ cube
        X = NS_A * X + NS_B * cube + NS_C * fifth
    return X


def _exact_forward(s):
    y, means, rstds = [], [], []
    for x in s["x"]:                 # one example after the other: 64-bit copies of a large batch do not fit beside three states
        var, mu = torch.var_mean(x.double(), dim=-1, correction=0)
        if s["norm"] == "rms":
            var, mu = var + mu * mu, torch.zeros_like(mu)
        r = 1.0 / torch.sqrt(var + EPS)
        out = (x.double() - mu[..., None]) * r[..., None] * s["gain"].double()
        y.append((out if s["bias"] is None else out + s["bias"].double()).to(torch.float32 if s["x"].dtype == torch.bfloat16 else torch.float64))
        means.append(mu)
        rstds.append(r)
    return {"y": torch.stack(y), "mean": torch.stack(means) if s["norm"] == "layer" else None, "rstd": torch.stack(rstds)}


def _exact_backward(s):
    d, square = s["d"], s["phi"] == "square"
    sums = torch.zeros(4, d, dtype=torch.float64, device=DEV)
    x, dy, rstd = (s[k].view(-1, *s[k].shape[s["x"].dim() - 1:]) for k in ("x", "dy", "rstd"))
    mean = s["mean"].view(-1) if s["mean"] is not None else torch.zeros_like(rstd)
    dx = torch.zeros(x.shape, dtype=torch.float32 if x.dtype == torch.bfloat16 else torch.float64, device=DEV)
    ends = s["seq_offsets"].tolist() if s["kind"] == "ragged" else list(range(0, s["B"] * s["T"] + 1, s["T"]))
    gain = s["gain"].double()
    for a, b in zip(ends[:-1], ends[1:]):
        if a == b:
            continue
        r = rstd[a:b, None].double()
        h = (x[a:b].double() - mean[a:b, None].double()) * r
        e = dy[a:b].double()
        t = e * gain
        back = t - h * ((t * h).sum(1, keepdim=True) / d) - (t.sum(1, keepdim=True) / d if s["norm"] == "layer" else 0.0)
        dx[a:b] = back * r
        for k, one in enumerate(((e * h).sum(0), e.sum(0))):
            sums[2 * k] += one
            sums[2 * k + 1] += one ** 2 if square else one
    out = {"dx": dx.view(s["x"].shape), "gain_sum": sums[0], "gain_stat": sums[1], "bias_sum": None, "bias_stat": None}
    if s["norm"] == "layer":
        out["bias_sum"], out["bias_stat"] = sums[2], sums[3]
    return out
