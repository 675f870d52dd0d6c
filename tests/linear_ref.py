"""Plain 64-bit forms of linear attention and the block norms, step by step from
their definitions (numpy; test infrastructure only)."""
import numpy as np


def heads(x, r):
    return np.repeat(x, r, axis=-2)


def attn(q, k, v, g, scale, h0=None, spans=None, do=None, dh=None):
    """q, k (B, L, Hk, K), v (B, L, H, V), g (B, L, H) -> a dict of o, h_last and,
    with do, every gradient.  spans: [(row, first, end)] of the sequences."""
    B, L, Hk, K = q.shape
    H, V = v.shape[2:]
    r = H // Hk
    spans = spans or [(b, 0, L) for b in range(B)]
    N = len(spans)
    out = {"o": np.zeros((B, L, H, V)), "h_last": np.zeros((N, H, K, V))}
    if do is not None:
        out.update(dq=np.zeros(q.shape), dk=np.zeros(k.shape), dv=np.zeros(v.shape),
                   dg=np.zeros((B, L, H)), dh0=np.zeros((N, H, K, V)))
    with np.errstate(invalid="ignore", over="ignore"):
        a = np.exp(g)
        for n, (b, i, j) in enumerate(spans):
            S = h0[n].copy() if h0 is not None else np.zeros((H, K, V))
            seen = [S]
            for t in range(i, j):
                S = a[b, t][:, None, None] * S + heads(k[b, t], r)[:, :, None] * v[b, t][:, None, :]
                out["o"][b, t] = scale * (heads(q[b, t], r)[:, :, None] * S).sum(1)
                seen.append(S)
            out["h_last"][n] = S
            if do is None:
                continue
            dS = dh[n].copy() if dh is not None else np.zeros((H, K, V))
            for t in range(j - 1, i - 1, -1):
                S, prev, d = seen[t + 1 - i], seen[t - i], do[b, t]
                dS = dS + scale * heads(q[b, t], r)[:, :, None] * d[:, None, :]
                share = lambda x: x.reshape(Hk, r, K).sum(1)  # noqa: E731
                out["dq"][b, t] = share(scale * (S * d[:, None, :]).sum(2))
                out["dk"][b, t] = share((dS * v[b, t][:, None, :]).sum(2))
                out["dv"][b, t] = (dS * heads(k[b, t], r)[:, :, None]).sum(1)
                dS = dS * a[b, t][:, None, None]
                out["dg"][b, t] = (dS * prev).sum((1, 2))
            out["dh0"][n] = dS
    return out


def magnitudes(q, k, v, g, scale, h0=None, spans=None, do=None, dh=None, interval=256):
    """The same of absolute values: what each result's terms add up to.  dg's is that
    of the sums it is formed from: of q . dq and k . dk over up to ``interval`` steps."""
    ab = lambda x: None if x is None else np.abs(x)  # noqa: E731
    m = attn(ab(q), ab(k), ab(v), g, abs(scale), ab(h0), spans, ab(do), ab(dh))
    if do is not None:
        # a step's q . dq of one head is at most its do . o, k . dk its v . dv
        each = (np.abs(do) * m["o"]).sum(-1) + (np.abs(v) * m["dv"]).sum(-1)
        B, L = g.shape[:2]
        for b, i, j in spans or [(b, 0, L) for b in range(B)]:
            for t0 in range(i, j, interval):
                t1 = min(j, t0 + interval)
                m["dg"][b, t0:t1] += each[b, t0:t1].sum(0)
    return m


def norm(u, width, eps):
    """(u over its groups' root mean square, the gradient's way back)."""
    v = u.reshape(u.shape[0], -1, width)
    inv = 1.0 / np.sqrt((v * v).sum(-1, keepdims=True) / width + eps)
    y = v * inv

    def back(d):
        d = d.reshape(v.shape)
        return (inv * (d - y * (d * y).sum(-1, keepdims=True) / width)).reshape(u.shape)
    return y.reshape(u.shape), back


def _over(x, width):
    """Each value's group's largest magnitude."""
    v = np.abs(x).reshape(x.shape[0], -1, width)
    return np.broadcast_to(v.max(-1, keepdims=True), v.shape).reshape(x.shape)


def gated(x, z, w, group, after, eps, dy=None):
    """Results and, as t_<name>, the size of the terms that each is formed from (the
    norm's gradient is a difference: w dy of the group over its root mean square)."""
    if z is None:
        gate, slope, steep = np.ones_like(x), np.zeros_like(x), np.zeros_like(x)
    else:
        sg = 1.0 / (1.0 + np.exp(-z))
        gate, slope = z * sg, sg * (1.0 + z * (1.0 - sg))
        steep = sg * (1.0 + np.abs(z) * (1.0 - sg))
    u = x if after else x * gate
    n, back = norm(u, group, eps)
    y = n * w * (gate if after else 1.0)
    out = {"y": y, "t_y": np.abs(y)}
    if dy is None:
        return out
    inv = 1.0 / np.sqrt(np.repeat((u * u).reshape(u.shape[0], -1, group).mean(-1), group, -1) + eps)
    dn = dy * w * (gate if after else 1.0)
    size = inv * _over(dn, group)
    du = back(dn)
    if after:
        out.update(dx=du, dz=dy * n * w * slope, dweight=(dy * n * gate).sum(0), t_dx=size,
                   t_dz=np.abs(dy * n * w) * steep)
    else:
        out.update(dx=du * gate, dz=du * x * slope, dweight=(dy * n).sum(0),
                   t_dx=size * np.abs(gate), t_dz=size * np.abs(x) * steep)
    out["t_dweight"] = np.abs(dy * n * (gate if after else 1.0)).sum(0)
    return out


def residual(R, w, eps, dy=None, dres=None, x=None, s=None):
    """From the stored stream R: y and, with dy, the gradients (t_<name> as in gated)."""
    D = R.shape[-1]
    n, back = norm(R, D, eps)
    out = {"y": n * w, "t_y": np.abs(n * w)}
    if dy is not None:
        d0 = 0.0 if dres is None else dres
        dR = back(dy * w) + d0
        inv = 1.0 / np.sqrt((R * R).mean(-1, keepdims=True) + eps)
        size = inv * _over(dy * w, D) + np.abs(d0)
        sc = 1.0 if s is None else s
        out.update(dresidual=dR, dx=dR * sc, dweight=(dy * n).sum(0), t_dresidual=size,
                   t_dx=size * np.abs(sc), t_dweight=np.abs(dy * n).sum(0))
        if s is not None:
            out.update(dres_scale=(x * dR).sum(0), t_dres_scale=(np.abs(x) * size).sum(0))
    return out
