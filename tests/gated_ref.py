"""The gated recurrence in 64 bits, step by step from its definition, and how far results
in 32 bits may be from it (numpy; test infrastructure only).

With U = 2^-24, a rounding to nearest: m = c softplus(lam) sigmoid(r) is formed by some
ten roundings and hardware functions of 2 U each, 16 U; so a = e^-m is off by (16 m + 4) U
of itself.  Products of a over several steps round once more each, and joining a chunk's
parts a few times more: 4 U a step.  sqrt(1 - a^2), a series cut at 2^-19 for bf16 inputs,
and the sigmoids, whose exponents are rounded (|r|, |i| <= 8 here: 8 U), make u off by 64 U
of itself.  These go into the recurrence of the absolute values, term by term."""
import numpy as np

U = 2.0 ** -24


def sigmoid(v):
    return np.where(v > 0, 1.0, np.exp(np.minimum(v, 0))) / (1 + np.exp(-np.abs(v)))


def scan(x, r, i, lam, c, h0=None, spans=None, dh=None, dh_last=None):
    """x, r, i (B, L, D) -> (results, bounds), dicts of h, h_last and, with dh, dx, dr, di,
    dlam, dh0; spans: [(row, first, end)] of the sequences."""
    B, L, D = x.shape
    spans = spans or [(b, 0, L) for b in range(B)]
    n = len(spans)
    softplus = np.maximum(lam, 0) + np.log1p(np.exp(-np.abs(lam)))
    k = c * softplus
    sr, si = sigmoid(r), sigmoid(i)
    rest_r, rest_i = sigmoid(-r), sigmoid(-i)
    m = k * sr
    a = np.exp(-m)
    b = np.sqrt(-np.expm1(-2 * m))
    u = b * si * x
    ea = (16 * m + 8) * U  # a's own error and the products'
    out = {"h": np.zeros((B, L, D)), "h_last": np.zeros((n, D))}
    off = {"h": np.zeros((B, L, D)), "h_last": np.zeros((n, D))}
    size = np.zeros((B, L, D))
    if dh is not None:
        for name, shape in (("dx", x.shape), ("dr", x.shape), ("di", x.shape), ("dlam", (D,)), ("dh0", (n, D))):
            out[name], off[name] = np.zeros(shape), np.zeros(shape)
        with np.errstate(divide="ignore", invalid="ignore"):
            q = np.where(b > 0, m / b, 0.0) * a * a
        slope = np.where(lam < -30, 1.0, sigmoid(lam) / np.maximum(softplus, 1e-300))
    for s, (row, t0, t1) in enumerate(spans):
        h = h0[s].copy() if h0 is not None else np.zeros(D)
        M, E = np.abs(h), np.zeros(D)  # the size of the terms, the error
        prev = np.zeros((t1 - t0, 3, D))
        for t in range(t0, t1):
            prev[t - t0] = h, M, E
            f = a[row, t]
            h = f * h + u[row, t]
            E = f * (E + ea[row, t] * M) + 64 * U * np.abs(u[row, t])
            M = f * M + np.abs(u[row, t])
            E = E + 2 * U * M
            out["h"][row, t], off["h"][row, t], size[row, t] = h, E, M
        out["h_last"][s], off["h_last"][s] = h, E
        if dh is None:
            continue
        g = dh_last[s].copy() if dh_last is not None else np.zeros(D)
        G, F = np.abs(g), np.zeros(D)
        total = np.zeros(D)
        for t in range(t1 - 1, t0 - 1, -1):
            at = row, t
            g, G = g + dh[at], G + np.abs(dh[at])
            F = F + 2 * U * G
            hp, Mp, Ep = prev[t - t0]
            bs = b[at] * si[at]
            out["dx"][at], off["dx"][at] = g * bs, bs * (F + 64 * U * G)
            z = np.abs(x[at]) * rest_i[at]
            out["di"][at], off["di"][at] = g * bs * x[at] * rest_i[at], bs * z * (F + 96 * U * G)
            e = g * (q[at] * si[at] * x[at] - m[at] * a[at] * hp)
            T = q[at] * si[at] * np.abs(x[at]) + m[at] * a[at] * Mp
            err = F * T + G * (96 * U * T + 16 * m[at] * U * T + m[at] * a[at] * Ep)
            out["dr"][at], off["dr"][at] = e * rest_r[at], rest_r[at] * (err + 16 * U * G * T)
            out["dlam"] += e * slope
            off["dlam"] += err * slope
            total += G * T * slope
            F = a[at] * (F + ea[at] * G)
            g, G = g * a[at], G * a[at]
        out["dh0"][s], off["dh0"][s] = g, F + 2 * U * G
        # each of its sums adds at most some 300 times in a row (steps, parts, rows of parts)
        off["dlam"] += 300 * U * total
    return out, off
