"""The log probabilities of confident rows in 64 bits, S - 1 kept apart from the 1 of the largest
logit's own term, and how far the kernel's results may be off, from the operations it makes.

U is half a step of binary32 relative to a value; distances below are in octaves,
T = (m - z) log2(e) / tau."""
import math

import torch

U = 2.0 ** -24
LN2 = math.log(2.0)


def _terms(z, tau):
    """Of z float64 [rows, vocab] without NaN or +infinity: m, T, and the terms 2^-T without one
    of the largest logit's."""
    m, at = z.max(1)
    T = (m[:, None] - z) / tau / LN2
    e = torch.exp2(-T)
    return m, T, e.scatter(1, at[:, None], 0.0)


def score(z, tokens, tau):
    """logp [rows] and stats [rows, 3] (float64)."""
    m, T, e = _terms(z, tau)
    rest = e.sum(1)
    log_s = torch.log1p(rest)
    mean = torch.where(e > 0, e * T, 0.0).sum(1) / (1.0 + rest)
    logp = -(T.gather(1, tokens.long()[:, None])[:, 0] * LN2) - log_s
    return logp, torch.stack([m, log_s, log_s + LN2 * mean], 1)


def off(z, tau, vec, apart, count=None):
    """Bounds of the absolute errors of log S and of the entropy, a vector of the row having `vec`
    logits.  A lane has one vector of 1024 and one more logit, so n terms, all about logits that
    are at least as large; its sums move to a larger one with each of its vectors at most, once for
    the last logit and once to the row's largest.  T is off by 5 U of itself (difference, factor
    2 U, product, and what is of second order), so a term by 5 ln 2 U T, below 3.5 U T, and by a
    step, 2 U, of the exponential; each move by a step and a product more, 3 U; sums of positive
    terms by U for each of n terms and 6 + 16 joins; terms below 2^-126 may be 0.  `apart`: whether
    the 1 of the largest logit is left out where S < 2 (its lane's other terms are then added by 64
    threads and 6 joins, in the place of its moves), else it is a term as the others.  `count`:
    the roundings of a sum where they are fewer than that."""
    vocab = z.shape[1]
    if count is None:
        turns = -(-vocab // (1024 * vec))
        count = vec * turns + 1 + 22 + 3 * (turns + 2)
    _, T, e = _terms(z, tau)
    rel = U * (3.5 * T + 2 + count)
    rest = e.sum(1)
    S = 1.0 + rest
    none = vocab * 2.0 ** -126
    s_off = torch.where(e > 0, e * rel, 0.0).sum(1) + none
    if apart:
        s_off = s_off + torch.where(S > 1.9, count * U, 0.0)    # near 2 either way
    else:
        s_off = s_off + count * U
    u = torch.where(e > 0, e * T, 0.0).sum(1)
    u_off = torch.where(e > 0, e * T * (rel + 6 * U), 0.0).sum(1) + 256 * none
    # the logarithm is off by two steps
    log_off = s_off / S + 4 * U * torch.log1p(rest)
    h = torch.log1p(rest) + LN2 * u / S
    h_off = log_off + LN2 * (u_off / S + u / S * (s_off / S + 4 * U)) + 2 * U * h
    return log_off, h_off
