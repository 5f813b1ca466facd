"""Limits, row by row, on how far the kernels of the logits may be from the 64-bit
oracle, from the numbers that take part in a row: a logit whose exponential is
nothing beside the row's others adds no error, however large it is.

E is a binary32 operation's relative error, 2^-24; each count of them below is the
operations of the kernel rounded up to a power of two or so.
"""
import numpy as np

import operators_ref as ref

E = 2.0 ** -24
HALF_ULP = {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}
FLT_MAX = float(np.finfo(np.float32).max)
FAR = 2.0 ** 15 * np.log(2.0)       # what is further below the largest is as good as excluded


def _largest(s):
    return s.max(initial=-np.inf)


def _exponents(s, distance, bases=0.0):
    """Errors of the natural logarithms s of exponentials of -distance: the factor and the
    fused product off by 2 E of the distance, exp and the sum below it by a few units (a
    rounded base is common to a sum's terms and at most 64 from what it stands for); by E
    of the bases where one sum's is changed for another's."""
    with np.errstate(invalid="ignore"):
        off = E * (8 * np.abs(distance) + 8 * np.abs(s) + 4 * bases + 256)
    return np.where(np.isfinite(off), off, 0.0)


def _sum(vocab):
    """Relative error of a sum of vocab positive terms: a thread's run of them (at most a
    256th), then a tree."""
    return E * (vocab / 256 + 64)


def _over_mass(q, err):
    """sum of q err, nothing where there is no mass."""
    return float(np.where(q > 0, q * err, 0.0).sum())


def _slots(cols, vocab):
    """Column -> slot: used slots, of equal columns the first."""
    slots = {}
    for j, c in enumerate(cols):
        if 0 <= c < vocab:
            slots.setdefault(int(c), j)
    return slots


def _softmax(s):
    """Probabilities and their logarithms; none of -infinity alone."""
    m = _largest(s)
    if m == -np.inf:
        return np.zeros(s.shape), np.full(s.shape, -np.inf)
    logs = s - m - np.log(np.exp(s - m).sum())
    return np.exp(logs), logs


def _loss_of(p, logp, logq):
    """sum of p (logp - logq): nothing where p is 0, infinite where only q is."""
    with np.errstate(invalid="ignore"):
        part = np.where(p > 0, p * (logp - logq), 0.0)
    return float(part.sum())


def distill(z, vals, cols, dtype, *, tau=1.0, lse=None, labels=None, kd=1.0, ce=0.0, weight=None):
    """(loss, dz, limit of loss, limits of dz) by the definition in zo_ops.h, float64."""
    vocab = z.shape[1]
    loss, lim_loss = np.zeros(len(z)), np.zeros(len(z))
    dz, lim_dz = np.zeros(z.shape), np.zeros(z.shape)
    for t in range(len(z)):
        w = 1.0 if weight is None else float(weight[t])
        if w == 0.0:
            continue
        m = _largest(z[t]) if np.isfinite(_largest(z[t])) else 0.0
        # from the row's largest: no sum of a large number and a logarithm loses its digits
        x = z[t] - m
        slots = _slots(cols[t], vocab)
        at = np.array(list(slots), int)
        u = np.array([vals[t, j] for j in slots.values()], np.float64)
        out = np.ones(vocab, bool)
        out[at] = False
        q, logq = _softmax(x / tau)
        # a distance that passes binary32 excludes
        logq = np.where(-x / tau > FLT_MAX * (1 + E), -np.inf, logq)
        logq = np.where(-x > FLT_MAX * (1 + E), -np.inf, logq)
        # the bases are products of the two largest logits, S's and the others'; where those
        # are 2^31 or more, differences are formed first and no product is rounded
        base = max((abs(_largest(z[t, g])) for g in (at, out)
                    if np.isfinite(_largest(z[t, g]))), default=0.0)
        bases = 0.0 if base * 1.45 / min(tau, 1.0) >= 2.0 ** 31 else 2 * base / tau
        eq = _exponents(logq, x / tau, np.where(out, bases, 0.0)) + _sum(vocab)
        err_q = _over_mass(q, eq)
        kl, d, err, grad = 0.0, np.zeros(vocab), 0.0, np.zeros(vocab)
        if kd != 0 and (lse is not None or (len(at) and u.max() > -np.inf)):
            u0 = 0.0 if lse is not None else u.max()
            if lse is None:
                p, logp = _softmax(u / tau)
            else:
                logp = u / tau - float(lse[t])
                p = np.exp(logp)
            p = np.where(p < 2.0 ** -150, 0.0, p)     # as binary32 has it
            kl = _loss_of(p, logp, logq[at])
            d = q.copy()
            d[at] -= p
            with np.errstate(invalid="ignore"):
                ep = E * (4 * np.abs(u - u0) / tau + 2 * np.abs(logp) + 8)
            ep = np.where(p > 0, ep, 0.0)
            err_p = _over_mass(p, ep) + E * (len(at) / 64 + 16)
            if lse is None:
                ep = np.where(p > 0, ep + err_p, 0.0)
            term = np.where((p > 0) & np.isfinite(logq[at]), np.abs(logp - logq[at]), 0.0)
            # p log(p / q) - p + q: the factor, the logarithm, and the two that are added
            err = _over_mass(p, ep * (term + 2) + eq[at] + 8 * E * term) + 2 * err_q + 2 * err_p
            grad[at] = q[at] * eq[at] + p * ep
            grad[out] = q[out] * eq[out]
            if lse is not None:
                pr = max(0.0, 1.0 - p.sum())
                m_out = _largest(x[out])              # below the row's largest, or -infinity
                rest = z[t, out] - (_largest(z[t, out]) if m_out > -np.inf else 0.0)
                r, logr = _softmax(rest / tau)
                if -m_out / tau > FAR and pr < 2.0 ** -16:
                    pr = 0.0
                if pr > 0:
                    far = -np.inf
                    if m_out > -np.inf and -m_out / min(tau, 1.0) <= FLT_MAX * (1 + E):
                        i = np.argmax(x[out])
                        far = logq[out][i] - logr[i]
                    kl += pr * (np.log(pr) - far)
                    d[out] -= pr * r
                    # pr log(pr / qr): its slope over what pr may be, and the logarithm
                    if far > -np.inf:
                        er = float(_exponents(far, m_out / tau, bases)) + 2 * _sum(vocab)
                        err += pr * (er + 8 * E * abs(far))
                if m_out > -np.inf and -m_out / tau <= FAR or pr > 0:
                    far = max(-m_out / tau, 0.0) if m_out > -np.inf else 0.0
                    err += err_p * (far + np.log(vocab) + abs(np.log(err_p)) + 2)
                    of = _exponents(logr, rest / tau)
                    grad[out] += r * (err_p + pr * (of + _sum(vocab)))
        row, g = kd * tau * tau * kl, kd * tau * d
        lim, grad = kd * tau * tau * err, kd * tau * grad
        if ce != 0 and labels is not None and 0 <= labels[t] < vocab:
            y = labels[t]
            soft, logs = _softmax(x)
            logs = np.where(-x > FLT_MAX * (1 + E), -np.inf, logs)
            e1 = _exponents(logs, x, np.where(out, bases * tau, 0.0)) + _sum(vocab)
            row -= ce * logs[y]
            g += ce * soft
            g[y] -= ce
            grad += ce * soft * 2 * e1                # at tau = 2 a square of the other
            if logs[y] > -np.inf:
                lim += ce * (2 * e1[y] + 8 * E * abs(logs[y]))
        loss[t], dz[t] = w * row, w * g
        if abs(loss[t]) > FLT_MAX * (1 + E):
            loss[t] = np.copysign(np.inf, loss[t])
        lim_loss[t] = abs(w) * lim + (16 * E * abs(loss[t]) if np.isfinite(loss[t]) else 0.0)
        lim_loss[t] += abs(w) * 2.0 ** -120           # below the normal numbers
        grad = abs(w) * grad + 16 * E * np.abs(dz[t])
        lim_dz[t] = grad + HALF_ULP[dtype] * (np.abs(dz[t]) + grad)
        lim_dz[t] += abs(w) * (kd * tau + ce) * 2.0 ** -120
        # below the normal numbers of the type
        lim_dz[t] += 2.0 ** -25 if dtype == "float16" else 2.0 ** -120
    return loss, dz, lim_loss, lim_dz


def lse(z, tau):
    """Limits of the rows' log-sum-exp of z / tau: the largest over tau rounded, and the
    logarithm of a sum of terms of at most 1."""
    m = np.where(np.isfinite(z.max(1)), z.max(1), 0.0)
    with np.errstate(over="ignore"):
        return E * (4 * np.abs(m) / tau + 8 * np.log(z.shape[1]) + 256) + _sum(z.shape[1])


def _nearby_teacher(r, z, top, tau):
    """Slots of a teacher near the student z: logits, columns, log-sum-exp."""
    u = np.where(np.isfinite(z), z, -np.inf) + r.normal(size=z.shape)
    cols = np.argsort(-u, axis=1, kind="stable")[:, :top].astype(np.int32)
    return (np.take_along_axis(u, cols, 1).astype(np.float32), cols,
            ref.log_sum_exp(u / tau).astype(np.float32))


def far_rest_rows(vocab, tau, masks, labels):
    """Rows that hold all outside S at a mask, each mask with each of several masses that
    the teacher has there (0: none but its rounding)."""
    r = np.random.default_rng(vocab)
    masses = [0.01, 1e-6, 0.0]
    n, top = len(masks) * len(masses), 4
    z = np.repeat(masks, len(masses))[:, None] * np.ones((n, vocab))
    cols = np.stack([r.permutation(vocab)[:top] for _ in range(n)]).astype(np.int32)
    near = r.normal(size=(n, top)).astype(np.float16).astype(np.float64)
    np.put_along_axis(z, cols, near, 1)
    vals = (near + 0.3 * r.normal(size=(n, top))).astype(np.float32)
    inside = ref.log_sum_exp(vals.astype(np.float64) / tau)
    lse = inside - np.log1p(-np.tile(masses, len(masks)))
    y = cols[:, 1].copy()
    y[::2] = (cols[::2, 1] + 1) % vocab             # many of them outside S
    return z, vals, cols, lse.astype(np.float32), y if labels else None


def masked_rows(vocab, tau, lowest):
    """Unused slots, repeated and out-of-range columns, a masked student and teacher
    (-infinity and the type's lowest value), a row that leaves the student nothing, rows
    of weight 0 that hold NaN."""
    r = np.random.default_rng(vocab + 5)
    rows, top = 10, 6
    z = (r.normal(size=(rows, vocab)) * 3).astype(np.float16).astype(np.float64)
    vals, cols, lse = _nearby_teacher(r, z, top, tau)
    cols[0] = [-1, vocab, 2 ** 31 - 1, -2 ** 31, -5, vocab + 7]
    cols[1] = [5, 5, 9, 5, 9, 11]
    vals[1] -= 6.0
    vals[2, 3:] = -np.inf
    z[3, cols[3, 0]] = -np.inf
    out = np.ones(vocab, bool)
    out[cols[4]] = False
    z[4, out] = -np.inf
    lse[4] = ref.log_sum_exp(vals[4][None].astype(np.float64) / tau)[0] - 1e-3
    z[5, ::2] = lowest
    vals[5] = np.where(cols[5] % 2 == 1, vals[5], -1e30)
    z[6] = -np.inf
    z[7] = np.nan
    z[9] = lowest
    z[9, cols[9]] = [0.0, 1.0, -2.0, 0.5, lowest, -np.inf]
    vals[9, 4:] = -np.inf
    lse[9] = ref.log_sum_exp(vals[9][None].astype(np.float64) / tau)[0]
    weight = np.ones(rows, np.float32)
    weight[7], weight[8] = 0.0, -2.5
    labels = np.array([3, -1, vocab, 7, -1, 1, -1, 0, 2, cols[9, 0]], np.int32)
    return z, vals, cols, lse, labels, weight


def extreme_rows(vocab, tau):
    """Binary32 rows whose largest logits lie near the ends of the type, where a product
    with log2(e) / tau overflows."""
    r = np.random.default_rng(vocab + 9)
    top = 5
    big = float(np.float32(3e38))
    step = big - float(np.nextafter(np.float32(big), np.float32(0)))
    z = (r.normal(size=(8, vocab)) * 3).astype(np.float16).astype(np.float64)
    cols = np.stack([r.permutation(vocab)[:top] for _ in range(8)]).astype(np.int32)
    z[0] = -FLT_MAX                                  # masked altogether
    z[1, cols[1]] = big                              # S far above the rest
    z[2, (cols[2, 0] + 1) % vocab] = FLT_MAX         # the rest far above S
    z[3] = -big                                      # equal but for a few one unit below
    z[3, ::3] = -big - step
    z[4] = big
    z[4, cols[4, :2]] = -big                         # differences beyond the type
    z[5, cols[5]] = big
    z[5, cols[5, 1]] = np.float32(big - step)
    z[6] = -FLT_MAX                                  # S alone is not
    z[6, cols[6]] = [1.0, 2.0, 0.0, -1.0, -np.inf]
    z[7] = 2.0 ** 126
    z[7, 1::2] = -np.inf
    vals = r.normal(size=(8, top)).astype(np.float32)
    lse = ref.log_sum_exp(vals.astype(np.float64) / tau) + 0.2
    labels = cols[:, 2].copy()
    labels[3] = 1
    labels[4] = (cols[4, 0] + 1) % vocab
    return z, vals, cols, lse.astype(np.float32), labels


def large_rows(vocab, tau):
    """Binary32 rows all of whose logits are so large that a unit in the last place of
    z log2(e) / tau is more than an exponent may be off by, with products that are finite."""
    r = np.random.default_rng(vocab + 11)
    top = 5
    z = np.empty((7, vocab))
    cols = np.stack([r.permutation(vocab)[:top] for _ in range(7)]).astype(np.int32)
    z[0] = np.float32(-1e30)
    z[1] = -1e10 - 1024.0 * r.integers(0, 2, vocab)
    z[2] = np.float32(1e12)
    z[2, ::2] = 0.0
    z[3] = 2.0 ** 33                                 # S below the rest
    z[3, cols[3]] = 2.0 ** 33 - 1024.0
    z[4] = np.float32(-3.7e12)                       # S above the rest, both far out
    z[4, cols[4]] = np.float32(-2.9e12)
    z[5] = -2.0 ** 31
    z[6] = 7e9
    z[6, 1::3] = -np.inf
    vals = r.normal(size=(7, top)).astype(np.float32)
    lse = ref.log_sum_exp(vals.astype(np.float64) / tau) + 0.2
    return z, vals, cols, lse.astype(np.float32), cols[:, 2].copy()
