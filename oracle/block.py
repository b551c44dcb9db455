"""What lies around the linear layers of a Transformer block, as plain full-matrix arithmetic in fp64 (oracle; tests only).

Norms (Section 3.2 names LayerNorm; the root-mean-square form leaves the mean out):
``N(t) = (t - mean) * rstd * gamma + beta`` over a row, ``rstd = 1 / sqrt(mean((t - mean)^2) + eps)``.
The residual stream and its norms: ``v = Npost(u)``, ``r = x + scale * gate * v``, ``n = Npre(r)``.

Every ``*_bound`` returns, beside a value, the sum of the magnitudes of the terms it is made of: an fp32 evaluation in which no
term passes through more than ``k`` roundings is within ``k * 2^-24`` times that, to first order.
"""
import numpy as np

KINDS = ("none", "rms", "layer")


def statistics(t, kind, eps):
    """(mean, rstd) of every row, as columns."""
    mean = t.mean(axis=1, keepdims=True) if kind == "layer" else np.zeros((t.shape[0], 1))
    return mean, 1.0 / np.sqrt(((t - mean) ** 2).mean(axis=1, keepdims=True) + eps)


def _vec(v, default):
    return default if v is None else np.asarray(v, dtype=np.float64)


def norm_forward(x, u, post, pre, post_eps, pre_eps, scale, p):
    """x, u [rows, cols] (u may be None); p: dict of post_gamma, post_beta, gate, pre_gamma, pre_beta (or None).
    Returns a dict: r, n (None without Npre), stats [rows, 4]."""
    rows = x.shape[0]
    stats = np.zeros((rows, 4))
    r = x
    if u is not None:
        v = u
        if post != "none":
            mean, rstd = statistics(u, post, post_eps)
            stats[:, 0:1], stats[:, 1:2] = mean, rstd
            v = (u - mean) * rstd * _vec(p.get("post_gamma"), 1.0) + _vec(p.get("post_beta"), 0.0)
        r = x + scale * _vec(p.get("gate"), 1.0) * v
    n = None
    if pre != "none":
        mean, rstd = statistics(r, pre, pre_eps)
        stats[:, 2:3], stats[:, 3:4] = mean, rstd
        n = (r - mean) * rstd * _vec(p.get("pre_gamma"), 1.0) + _vec(p.get("pre_beta"), 0.0)
    return {"r": r, "n": n, "stats": stats}


def norm_forward_bound(x, u, post, pre, post_eps, pre_eps, scale, p, k):
    """Absolute errors of r, n and stats of an fp32 evaluation with chains of at most k roundings."""
    e = k * 2.0 ** -24
    out = norm_forward(x, u, post, pre, post_eps, pre_eps, scale, p)
    rows = x.shape[0]
    stats = np.zeros((rows, 4))
    err_r = np.zeros_like(x)
    if u is not None:
        mag = np.abs(u)
        if post != "none":
            mean, rstd = out["stats"][:, 0:1], out["stats"][:, 1:2]
            stats[:, 0:1] = e * np.abs(u).mean(axis=1, keepdims=True) * (post == "layer")
            stats[:, 1:2] = rstd * (e + rstd * stats[:, 0:1])
            # (u - mean) rstd: the rounding of the difference, the mean's error, rstd's relative error
            mag = (np.abs(u) + np.abs(u).mean(axis=1, keepdims=True)) * rstd * np.abs(_vec(p.get("post_gamma"), 1.0)) * 2 + \
                np.abs(_vec(p.get("post_beta"), 0.0))
        err_r = e * (np.abs(x) + np.abs(scale * _vec(p.get("gate"), 1.0)) * mag)
    err_n = None
    if pre != "none":
        r, mean, rstd = out["r"], out["stats"][:, 2:3], out["stats"][:, 3:4]
        err_mean = (err_r.mean(axis=1, keepdims=True) + e * np.abs(r).mean(axis=1, keepdims=True)) * (pre == "layer")
        dev = np.sqrt(((err_r + err_mean) ** 2).mean(axis=1, keepdims=True))     # of the deviations, in the mean square
        rel = e + rstd * dev
        stats[:, 2:3], stats[:, 3:4] = err_mean, rstd * rel
        hat = np.abs(r - mean) * rstd
        g = np.abs(_vec(p.get("pre_gamma"), 1.0))
        err_n = g * (rstd * (err_r + err_mean) + hat * rel) + 4 * 2.0 ** -24 * (g * hat + np.abs(_vec(p.get("pre_beta"), 0.0)))
    return {"r": err_r, "n": err_n, "stats": stats}


def _through(t, hat, rstd, kind):
    g = t - hat * (t * hat).mean(axis=1, keepdims=True)
    if kind == "layer":
        g = g - t.mean(axis=1, keepdims=True)
    return rstd * g


def norm_backward(dr, dn, r, u, stats, post, pre, scale, p):
    """Gradients from dr (or None) and dn (None without Npre), with the forward pass's statistics."""
    shape = (dr if dr is not None else dn).shape
    g = np.zeros(shape) if dr is None else dr
    out = {}
    if pre != "none":
        hat = (r - stats[:, 2:3]) * stats[:, 3:4]
        out["pre_gamma"], out["pre_beta"] = (dn * hat).sum(axis=0), dn.sum(axis=0)
        g = g + _through(dn * _vec(p.get("pre_gamma"), 1.0), hat, stats[:, 3:4], pre)
    out["dx"] = g
    if u is None:
        return out
    hat, v = None, u
    if post != "none":
        hat = (u - stats[:, 0:1]) * stats[:, 1:2]
        v = hat * _vec(p.get("post_gamma"), 1.0) + _vec(p.get("post_beta"), 0.0)
    out["gate"] = (scale * g * v).sum(axis=0)
    g = scale * g * _vec(p.get("gate"), 1.0)
    if post != "none":
        out["post_gamma"], out["post_beta"] = (g * hat).sum(axis=0), g.sum(axis=0)
        g = _through(g * _vec(p.get("post_gamma"), 1.0), hat, stats[:, 1:2], post)
    out["du"] = g
    return out


def _through_magnitude(t, hat, rstd, kind):
    return rstd * (t + hat * (t * hat).mean(axis=1, keepdims=True) + (t.mean(axis=1, keepdims=True) if kind == "layer" else 0.0))


def norm_backward_bound(dr, dn, r, u, stats, post, pre, scale, p, k, k_rows):
    """Absolute errors of norm_backward's results in fp32: chains of at most k roundings along a row, k_rows more along a
    column's sum.  (Magnitudes pass through every step; a value that goes through two norms pays for both.)"""
    e, ec = k * 2.0 ** -24, (2 * k + k_rows) * 2.0 ** -24
    a = np.abs
    shape = (dr if dr is not None else dn).shape
    g = np.zeros(shape) if dr is None else a(dr)
    out = {}
    if pre != "none":
        hat = (a(r) + a(stats[:, 2:3])) * stats[:, 3:4]
        out["pre_gamma"], out["pre_beta"] = ec * (a(dn) * hat).sum(axis=0), ec * a(dn).sum(axis=0)
        g = g + _through_magnitude(a(dn * _vec(p.get("pre_gamma"), 1.0)), hat, stats[:, 3:4], pre)
    out["dx"] = e * g
    if u is None:
        return out
    hat, v = None, a(u)
    if post != "none":
        hat = (a(u) + a(stats[:, 0:1])) * stats[:, 1:2]
        v = hat * a(_vec(p.get("post_gamma"), 1.0)) + a(_vec(p.get("post_beta"), 0.0))
    out["gate"] = ec * (abs(scale) * g * v).sum(axis=0)
    g = abs(scale) * g * a(_vec(p.get("gate"), 1.0))
    if post != "none":
        out["post_gamma"], out["post_beta"] = ec * (g * hat).sum(axis=0), ec * g.sum(axis=0)
        g = _through_magnitude(g * a(_vec(p.get("post_gamma"), 1.0)), hat, stats[:, 1:2], post)
    out["du"] = 2 * e * g
    return out


def gradient_norm(grads):
    return float(np.sqrt(sum(float((np.asarray(g, dtype=np.float64) ** 2).sum()) for g in grads)))


def clip_factor(norm, max_norm, scale=1.0):
    norm = scale * norm
    with np.errstate(over="ignore"):
        finite = np.isfinite(np.float32(norm))      # (as the norm is stored)
    return scale * min(1.0, max_norm / norm) if finite and norm > 0 else scale
