"""Plain forms of the 8-bit, norm and log probability operators in 64 bits (torch, on the
tensors' own device), the oracle of their tests: written from the definitions in
include/zo_ops.h, without the library; and how far a kernel's result may be off.

U is half a step of binary32 relative to a value; HALF the same of each type."""
import torch

U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
# half a step among the numbers below the normal ones
TINY = {torch.float32: 2.0 ** -150, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}


def quantize(x):
    """x float64 [rows, cols] of binary32 values: codes float64, scales float32 [rows]."""
    most = x.abs().amax(1) if x.shape[1] else torch.zeros(len(x), dtype=x.dtype, device=x.device)
    bad = ~torch.isfinite(x).all(1)
    # 64 bits hold a / 127 to 2^-53, and it is never that near to a border of binary32
    scale = (torch.where(bad, 0.0, most) / torch.full_like(most, 127.0)).float()
    s = scale.double()[:, None]
    q = torch.where(s > 0, x / torch.where(s > 0, s, 1.0), 0.0)
    codes = torch.where(bad[:, None], 0.0, q.round().clamp(-127, 127))
    return codes, torch.where(bad, torch.nan, scale)


def product(a, sa, b, sb, dtype):
    """The exact sums times the scales, binary32 step by step, rounded to dtype."""
    sums = (a @ b.t().contiguous()).float()          # below 2^31: exact in 64 bits, one rounding
    return (sums * sa[:, None] * sb[None]).to(dtype)


def norm(h, w, eps):
    """h, w float64: (rstd, out)."""
    rstd = 1.0 / torch.sqrt(h.square().mean(1) + eps)
    return rstd, h * rstd[:, None] * w


def rstd_off(cols):
    """Relative error of rstd: a sum of at most 32 fused terms a thread and then 6 + 16 joins,
    half of it after the square root; the mean, eps, the root and the inverse a step each."""
    return (0.5 * (min(cols, 32) + 22 + 2) + 2) * U


def norm_grad(dy, h, w, rstd, dh=None):
    """float64: dx, dw, and the bounds of their errors before the rounding to a type."""
    cols, r = h.shape[1], rstd[:, None]
    n, g = h * r, dy * w
    mean = (g * n).mean(1, keepdim=True)
    dx = r * (g - n * mean) + (dh if dh is not None else 0.0)
    dw = (dy * n).sum(0)
    # n and g are off by U each; a dot product of up to 32 fused terms a thread and 22 joins
    mean_off = (min(cols, 32) + 22 + 4) * U * (g * n).abs().mean(1, keepdim=True)
    dx_off = r * (4 * U * g.abs() + 4 * U * (n * mean).abs() + n.abs() * mean_off) + U * dx.abs()
    # every row may be a link of the chain, and the blocks' sums join in 64 steps
    dw_off = (min(len(h), 64 + len(h) // 16) + 66) * U * (dy * n).abs().sum(0)
    return dx, dw, dx_off, dw_off


def score(z, tokens, tau):
    """z float64 [rows, vocab]: logp [rows], stats [rows, 3], log probabilities."""
    bad = (z.isnan() | (z == torch.inf)).any(1)
    m = torch.where(bad, torch.nan, z.masked_fill(z.isnan(), -torch.inf).amax(1))
    empty = m == -torch.inf
    d = (z - torch.where(empty, 0.0, m)[:, None]) / tau
    s = d.exp().sum(1)
    log_s = torch.where(empty, -torch.inf, s.log())
    logp = torch.where(z == -torch.inf, -torch.inf, d - torch.where(empty, 0.0, log_s)[:, None])
    logp = torch.where(bad[:, None], torch.nan, logp)
    p = logp.exp()
    entropy = -torch.where(p > 0, p * logp.masked_fill(logp == -torch.inf, 0.0), 0.0).sum(1)
    stats = torch.stack([m, torch.where(bad, torch.nan, log_s),
                         torch.where(bad, torch.nan, entropy)], 1)
    got = torch.zeros(len(z), dtype=torch.float64, device=z.device)
    if tokens is not None:
        has = (tokens >= 0) & (tokens < z.shape[1])
        at = torch.where(has, tokens, 0).long()[:, None]
        got = torch.where(has, logp.gather(1, at)[:, 0], 0.0)
    return got, stats, logp


def score_off(z, tau):
    """Bounds of the absolute errors of log S, of the entropy and of a log probability
    (less its own 4 U |d|).  A term 2^t is off by U (3 |t| ln 2 + 4): the difference, the
    factor and their product round t by U each, the exponential by a step; a thread adds at
    most 129 of them (the longest row of one read), then come 6 + 16 joins.  The logarithm
    and the divisions take a few steps more."""
    got = score(z, None, tau)
    stats, logp = got[1], got[2]
    p = logp.exp().nan_to_num(0.0)
    d = (logp + stats[:, 1:2]).nan_to_num(0.0, neginf=0.0, posinf=0.0)
    chain = (129 + 22 + 4) * U
    mean_d = (p * d.abs()).sum(1)
    sum_off = chain + 3 * U * mean_d
    log_off = sum_off + 4 * U * stats[:, 1].abs().nan_to_num(0.0, posinf=0.0)
    u_off = chain * mean_d + 4 * U * (p * d * d).sum(1) + sum_off * mean_d
    return log_off + 8 * U, log_off + u_off + 8 * U * (1 + mean_d)


def score_grad(z, tokens, tau, stats, dlogp, dentropy):
    """float64 (stats are those of z, exact): dz and the bound of its error before the
    rounding to a type, the stats being rounded to binary32."""
    rows, vocab = z.shape
    zero = torch.zeros(rows, dtype=torch.float64, device=z.device)
    has = zero.bool() if tokens is None else (tokens >= 0) & (tokens < vocab)
    a = torch.where(has, zero if dlogp is None else dlogp.double(), 0.0)[:, None]
    b = (zero if dentropy is None else dentropy.double())[:, None]
    m, log_s, h = stats.double().unbind(1)
    empty = m == -torch.inf
    d = (z - torch.where(empty, 0.0, m)[:, None]) / tau
    lp = torch.where(z == -torch.inf, -torch.inf, d - torch.where(empty, 0.0, log_s)[:, None])
    p = torch.where(empty[:, None], 0.0, lp.exp())
    finite = lp.masked_fill(lp == -torch.inf, 0.0)
    inner = a + b * (finite + h[:, None])
    dz = -p * inner
    if tokens is not None:
        at = torch.where(has, tokens, 0).long()[:, None]
        one = torch.where(has & ~empty, 1.0, 0.0).double()[:, None]
        dz.scatter_add_(1, at, a * one)
    dz = torch.where((a == 0) & (b == 0), 0.0, dz) / tau
    # log p is off by U times the steps of its parts; the rest are factors
    dist = d.abs().nan_to_num(0.0, posinf=0.0) + log_s.abs().nan_to_num(0.0, posinf=0.0)[:, None]
    lp_off = U * (6 * dist + 4)
    scale = (a.abs() + b.abs() * (finite.abs() + h[:, None].abs())) / tau
    off = p * (scale * (lp_off + 10 * U) + b.abs() / tau * (lp_off + 2 * U * h[:, None].abs()))
    off = off + 2.0 ** -126 * scale + 8 * U * dz.abs()
    if tokens is not None:      # 1 - p from log p: off by as much as log p, at most by p
        off.scatter_add_(1, at, (a.abs() / tau * (p * lp_off).gather(1, at) * 2).double())
    return dz, off
