"""The sensitivity map's operators in 64 bits, from their definitions, and inputs for their tests.

Bounds of errors are derived from u = 2^-24, the rounding of one fp32 operation: a sum of values v in runs of `steps` additions is off by at
most steps * u * sum |v|; a result rounded to a type with eps is off by eps / 2 of itself, or half of the type's smallest step."""
import torch

U = 2.0 ** -24
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SMALLEST = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}


def rounding(ref: torch.Tensor, dtype) -> torch.Tensor:
    return ref.abs() * (torch.finfo(dtype).eps / 2) + SMALLEST[dtype] / 2


def close(got: torch.Tensor, ref: torch.Tensor, tol, what: str) -> None:
    """Every element within its bound; infinities and NaN in the same places."""
    got, ref = got.double(), ref.double()
    assert got.shape == ref.shape, what
    fine = torch.isfinite(ref)
    assert torch.equal(torch.isnan(got), torch.isnan(ref)), what + ": NaN"
    assert torch.equal(got[~fine & ~torch.isnan(ref)], ref[~fine & ~torch.isnan(ref)]), what + ": infinities"
    tol = torch.as_tensor(tol, dtype=torch.float64, device=ref.device).expand_as(ref)
    off = (got - ref).abs()[fine] - tol[fine]
    assert off.numel() == 0 or float(off.max()) <= 0.0, "%s: over its bound by %g" % (what, float(off.max()))


def strided(t: torch.Tensor, pad: int, shift: int) -> torch.Tensor:
    """The same matrix with rows `pad` elements apart that begin `shift` elements after an aligned address."""
    rows, cols = t.shape
    room = torch.full((rows * (cols + pad) + shift + 8,), float("nan"), dtype=t.dtype, device=t.device)
    view = room[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    view.copy_(t)
    return view


# ---------------------------------------------------------------- log probabilities

def log_probs(z, y, top):
    z = z.double()
    rows, V = z.shape
    none = (z == float("-inf")).all(1)
    m = z.amax(1)
    m = torch.where(m == float("-inf"), torch.zeros_like(m), m)
    ln = torch.log(torch.exp(z - m[:, None]).sum(1))
    lse = m + ln
    lse = torch.where((z == float("inf")).any(1), torch.full_like(lse, float("nan")), lse)
    lp = z - m[:, None] - ln[:, None]
    p = torch.exp(lp)
    entropy = torch.where(p > 0, -p * lp, torch.zeros_like(p)).sum(1)
    entropy = torch.where(torch.isnan(lse), lse, entropy)
    entropy = torch.where(none, torch.zeros_like(entropy), entropy)
    at = z.gather(1, y.clamp(0, V - 1)[:, None])[:, 0]
    logp = torch.where(none, torch.full_like(lse, float("-inf")), at - m - ln)
    logp = torch.where(y < 0, torch.zeros_like(logp), logp)
    logp = torch.where(y >= V, torch.full_like(logp, float("nan")), logp)
    rank = torch.where(torch.isnan(z), torch.full_like(z, float("-inf")), z)
    ids = torch.sort(rank, dim=1, descending=True, stable=True).indices[:, :top]
    top_logp = torch.where(none[:, None], torch.full((rows, top), float("-inf"), dtype=z.dtype, device=z.device), rank.gather(1, ids) - m[:, None] - ln[:, None])
    return logp, lse, entropy, top_logp, ids


def log_probs_tolerance(z, lse, entropy):
    """Per row: (of lse and logp, of the entropy).  A thread adds up to `steps` terms at most 1 in a row; a term e^t, t <= 0, is off by
    4 u of itself and by 4 u |t| e^t <= 2 u; the subtraction of the maximum and the logarithm add u of what they give."""
    steps = 32 * (z.shape[1] // 8192 + 1) + 16
    t = (steps + 8) * U
    size = torch.nan_to_num(z.double().abs(), nan=0.0, posinf=0.0, neginf=0.0).amax(1) + torch.nan_to_num(lse.abs(), nan=0.0, posinf=0.0, neginf=0.0)
    import math
    spread = math.log(z.shape[1]) + 1.0                # sum p |t| <= ln V - H + ... <= ln V + 1
    return t + 4 * U * size, 3 * t * (1.0 + spread)


def log_probs_grad(z, y, lse, dlogp, entropy, dentropy, ids, dtop):
    z, lse = z.double(), lse.double()[:, None]
    rows, V = z.shape
    lp = z - lse
    p = torch.exp(lp)
    g = torch.where(y < 0, torch.zeros_like(dlogp), dlogp).double()
    still = (lse[:, 0] == float("-inf"))
    G = g.clone()
    if ids is not None:
        G = G + dtop.double().sum(1)
    factor = G[:, None].expand_as(p)
    if dentropy is not None:
        factor = factor + dentropy.double()[:, None] * (torch.where(p > 0, lp, torch.zeros_like(lp)) + entropy.double()[:, None])
    else:
        if ids is None:
            still = still | (y < 0)
    d = -p * factor
    hit = torch.zeros_like(d)
    hit.scatter_add_(1, y.clamp(0, V - 1)[:, None], g[:, None])
    if ids is not None:
        hit.scatter_add_(1, ids, dtop.double())
    d = d + hit
    lpf = torch.where(p > 0, lp, torch.zeros_like(lp)).abs()
    big = G.abs()[:, None] if dentropy is None else G.abs()[:, None] + dentropy.double().abs()[:, None] * (lpf + entropy.double().abs()[:, None])
    tol = p * (8 + 8 * lpf) * U * big + 4 * U * hit.abs() + 8 * U * p * big
    d = torch.where(still[:, None], torch.zeros_like(d), d)
    tol = torch.where(still[:, None], torch.zeros_like(tol), tol)
    return d, tol


# ---------------------------------------------------------------- layer norm

def norm(x, weight, bias, eps):
    x = x.double()
    mean = x.mean(1)
    rstd = 1.0 / torch.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    n = (x - mean[:, None]) * rstd[:, None]
    w = 1.0 if weight is None else weight.double()
    b = 0.0 if bias is None else bias.double()
    y = n * w + b
    # sums run over at most width / 32 + 16 additions
    steps = x.shape[1] / 32 + 16
    tm = steps * U * x.abs().mean(1) + U * mean.abs()
    d2 = ((x - mean[:, None]) ** 2).mean(1)
    # the mean's error enters the deviations, each of which is rounded as well
    tr_rel = (steps + 8) * U + (2 * tm * (x - mean[:, None]).abs().mean(1) + tm ** 2 + 2 * U * (x.abs() * (x - mean[:, None]).abs()).mean(1)) / (d2 + eps)
    ty = (n.abs() * (tr_rel[:, None] + 8 * U) + rstd[:, None] * (tm[:, None] + U * x.abs())) * (w if weight is None else w.abs()) + 2 * U * y.abs()
    ty = ty + (0.0 if bias is None else U * b.abs())
    return (y, ty), (mean, tm), (rstd, rstd * tr_rel)


def sums(v, cuts):
    """(sum, sum of magnitudes) over rows, or over samples of magnitudes of their sums."""
    if cuts is None:
        return v.sum(0), v.abs().sum(0)
    s = torch.zeros_like(v[0] if v.shape[0] else v.sum(0))
    a = s.clone()
    for lo, hi in zip(cuts, cuts[1:]):
        s = s + v[lo:hi].sum(0).abs()
        a = a + v[lo:hi].abs().sum(0)
    return s, a


def norm_grad(dy, x, mean, rstd, weight, cuts):
    dtype, rows = x.dtype, x.shape[0]
    x, dy, mean, rstd = x.double(), dy.double(), mean.double()[:, None], rstd.double()[:, None]
    n = (x - mean) * rstd
    w = torch.ones_like(x[:1]) if weight is None else weight.double()[None]
    a = dy * w
    dx = rstd * (a - a.mean(1, keepdim=True) - n * (a * n).mean(1, keepdim=True))
    steps = x.shape[1] / 32 + 24
    nt = 4 * U * (n.abs() + rstd * mean.abs())                   # of n: the difference and the product are rounded
    ta = steps * U * a.abs().mean(1, keepdim=True)
    tan = steps * U * (a * n).abs().mean(1, keepdim=True) + (a.abs() * nt).mean(1, keepdim=True)
    san = (a * n).mean(1, keepdim=True).abs()
    tol = rstd * (4 * U * (a.abs() + a.mean(1, keepdim=True).abs() + n.abs() * san) + ta + n.abs() * tan + nt * san) + 4 * U * dx.abs()
    dw, aw = sums(dy * n, cuts)
    db, ab = sums(dy, cuts)
    _, an = sums(dy * nt, cuts)
    long = rows + 64                                             # no run of additions is longer
    return (dx, tol + rounding(dx, dtype)), (dw, long * U * aw + an), (db, long * U * ab)


# ---------------------------------------------------------------- linear layers

def linear(x, dy, cuts):
    x, dy = x.double(), dy.double()
    if cuts is None:
        w, b = dy.abs().T @ x.abs(), dy.abs().sum(0)
        aw, ab = w, b
        rows = x.shape[0]
    else:
        w = torch.zeros(dy.shape[1], x.shape[1], dtype=torch.float64, device=x.device)
        b = torch.zeros(dy.shape[1], dtype=torch.float64, device=x.device)
        aw, ab = w.clone(), b.clone()
        rows = 0
        for lo, hi in zip(cuts, cuts[1:]):
            w += (dy[lo:hi].T @ x[lo:hi]).abs()
            b += dy[lo:hi].sum(0).abs()
            aw += dy[lo:hi].abs().T @ x[lo:hi].abs()
            ab += dy[lo:hi].abs().sum(0)
            rows = max(rows, hi - lo)
        rows += len(cuts)
    # additions that may cut off instead of rounding: 2 u for each; fp32 inputs go as three pieces each, less 2^-22 of a product
    t = 2 * (rows + 16) * U + 2.0 ** -22
    return (w, t * aw), (b, t * ab)
