"""Plain forms of the operators in 64 bits (numpy), the oracle of their tests:
written from the definitions in include/zo_ops.h, without the library."""
import numpy as np

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6])


def quantize(x):
    """x float64 [rows, cols] -> codes [rows, cols], scale bytes [rows, ceil(cols / 32)]."""
    rows, cols = x.shape
    nb = -(-cols // 32)
    b = np.zeros((rows, nb * 32))
    b[:, :cols] = x
    b = b.reshape(rows, nb, 32)
    most = np.abs(b).max(-1)
    bad = ~np.isfinite(b).all(-1)
    fine = np.where(bad | (most == 0), 1.0, most)
    e = np.floor(np.log2(fine)).astype(int)
    e = np.where(np.ldexp(1.0, e) > fine, e - 1, e)          # log2 may round up
    e = np.where(np.ldexp(1.0, e + 1) <= fine, e + 1, e)
    byte = np.where(most == 0, 0, np.clip(e - 2 + 127, 0, 254))
    with np.errstate(invalid="ignore"):
        y = np.abs(b) / np.ldexp(1.0, byte - 127)[..., None]
    # nearest of the eight magnitudes, ties to the even code, above 6 to 6
    mags = GRID[:8]
    code = np.zeros(b.shape, int)
    for i in range(7):
        mid = (mags[i] + mags[i + 1]) / 2
        with np.errstate(invalid="ignore"):
            code = np.where((y > mid) | ((y == mid) & (i % 2 == 1)), i + 1, code)
    code = code + 8 * np.signbit(b)
    code = np.where(bad[..., None], 0, code)
    byte = np.where(bad, 255, byte)
    return code.reshape(rows, -1)[:, :cols], byte


def layout(code, byte, rows, cols):
    """Where an mx4 matrix keeps them: (codes bytes, scales bytes, masks of the
    bytes that are defined)."""
    rp, kt = -(-rows // 64) * 64, -(-cols // 128)
    codes = np.zeros(rp * kt * 64, np.uint8)
    scales = np.zeros(rp * kt * 4, np.uint8)
    dc, ds = np.zeros(codes.size, bool), np.zeros(scales.size, bool)
    r, c = np.meshgrid(np.arange(rows), np.arange(kt * 128), indexing="ij")
    full = np.zeros((rows, kt * 128), np.uint8)
    full[:, :cols] = code
    k = c % 128
    at = ((r // 16 * kt + c // 128) * 64 + k // 32 * 16 + r % 16) * 16 + k % 32 // 2
    np.add.at(codes, at, (full << (4 * (c % 2))).astype(np.uint8))
    dc[at] = True
    sb = np.zeros((rows, kt * 4), np.uint8)
    sb[:, :byte.shape[1]] = byte
    r, g = np.meshgrid(np.arange(rows), np.arange(kt * 4), indexing="ij")
    at = ((r // 64 * kt + g // 4) * 64 + g % 4 * 16 + r % 16) * 4 + r % 64 // 16
    scales[at] = sb
    ds[at] = True
    return codes, scales, dc, ds


def values(code, byte):
    """float64 values of codes and scale bytes."""
    b = np.repeat(byte, 32, axis=1)[:, :code.shape[1]]
    v = GRID[code] * np.ldexp(1.0, b - 127)
    return np.where(b == 255, np.nan, v)


def rounded(x):
    return values(*quantize(x))


def top_logits(z, top, tau):
    """z float64 [rows, vocab]: values, columns, lse."""
    key = np.where(np.isnan(z), np.inf, z) + 0.0
    # NaN before +infinity, then by value, then by column
    order = np.lexsort((np.broadcast_to(np.arange(z.shape[1]), z.shape), -key, ~np.isnan(z)))
    at = order[:, :top]
    return np.take_along_axis(z, at, 1), at.astype(np.int32), log_sum_exp(z / tau)


def log_sum_exp(s):
    m = s.max(1, initial=-np.inf)
    out = np.full(s.shape[0], -np.inf)
    for i in range(s.shape[0]):
        if np.isnan(s[i]).any():
            out[i] = np.nan
        elif np.isinf(m[i]):
            out[i] = m[i]
        else:
            out[i] = m[i] + np.log(np.exp(s[i] - m[i]).sum())
    return out


def distill(z, vals, cols, *, tau=1.0, lse=None, labels=None, kd=1.0, ce=0.0, weight=None):
    """float64 arrays; per row by the definition.  Returns (loss, dz)."""
    rows, vocab = z.shape
    loss, dz = np.zeros(rows), np.zeros(z.shape)
    for t in range(rows):
        w = 1.0 if weight is None else float(weight[t])
        if w == 0.0:
            continue
        s = z[t] / tau
        total = log_sum_exp(s[None])[0]
        q = np.zeros(vocab) if total == -np.inf else np.exp(s - total)
        slots = {}
        for j, c in enumerate(cols[t]):
            if 0 <= c < vocab and int(c) not in slots:
                slots[int(c)] = j
        at = np.array(list(slots), int)
        u = np.array([vals[t, j] for j in slots.values()]) / tau
        inside = np.zeros(vocab, bool)
        inside[at] = True
        d, kl = np.zeros(vocab), 0.0
        part = kd != 0 and (lse is not None or (len(at) > 0 and u.max() > -np.inf))
        if part:
            if lse is None:
                p = np.exp(u - log_sum_exp(u[None])[0])
            else:
                p = np.exp(u - lse[t])
            d = q.copy()
            d[at] -= p
            logq = s[at] - total if total != -np.inf else np.full(len(at), -np.inf)
            kl = sum(pi * (np.log(pi) - lq) if pi > 0 else 0.0 for pi, lq in zip(p, logq))
            if lse is not None:
                pr = max(0.0, 1.0 - p.sum())
                rest = log_sum_exp(s[None, ~inside])[0] if (~inside).any() else -np.inf
                if rest == -np.inf and pr < 2.0 ** -16:     # the rounding of L
                    pr = 0.0
                if pr > 0:
                    kl += pr * (np.log(pr) - (rest - total)) if rest != -np.inf else np.inf
                if rest != -np.inf:
                    d[~inside] -= pr * np.exp(s[~inside] - rest)
        row = kd * tau * tau * kl if part else 0.0
        g = kd * tau * d
        if ce != 0 and labels is not None and 0 <= labels[t] < vocab:
            one = log_sum_exp(z[t][None])[0]
            row += ce * (one - z[t, labels[t]]) if z[t, labels[t]] != -np.inf else np.inf
            g = g + ce * (np.exp(z[t] - one) if one != -np.inf else 0.0)
            g[labels[t]] -= ce
        loss[t], dz[t] = w * row, w * g
    return loss, dz
