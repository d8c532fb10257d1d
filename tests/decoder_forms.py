"""Plain forms in 64 bits of the norms of queries and keys with the rotation by position, of the drawing of tokens and of the global
gradient norm, written from their definitions, and bounds of what 32-bit arithmetic may add, from the roundings of each step."""
import math

import numpy as np

U = 2.0 ** -24          # half a step of fp32, relative
ONE = 2.0 ** 40


# ------------------------------------------------------------------------- queries and keys: norm and rotation
def pair_columns(rot, pairs):
    i = np.arange(rot // 2)
    return (2 * i, 2 * i + 1) if pairs else (i, i + rot // 2)


def turn(v, angle, rot, pairs):
    """v [tokens][heads][d], angle [tokens][rot / 2]"""
    out = np.array(v, np.float64)
    if rot:
        a, b = pair_columns(rot, pairs)
        c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
        out[..., a], out[..., b] = v[..., a] * c - v[..., b] * s, v[..., b] * c + v[..., a] * s
    return out


def partners(v, rot, pairs):
    """|v| plus, where a column turns, its partner's: what its terms amount to"""
    out = np.abs(np.array(v, np.float64))
    if rot:
        a, b = pair_columns(rot, pairs)
        out[..., a] = out[..., b] = np.abs(v[..., a]) + np.abs(v[..., b])
    return out


def qk_forward(x, gamma, angle, rot, pairs, eps, norm=True):
    """(y, bound of what fp32 arithmetic adds): the sum of d squares and the root are off by d / 2 + 8 half steps, two products follow; an
    angle by a rounding of its part of a turn (pi U), sine and cosine by four half steps, their products and sum by three."""
    x = np.asarray(x, np.float64)
    d = x.shape[-1]
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps) if norm else 1.0
    n = x * r * (1.0 if gamma is None else np.asarray(gamma, np.float64))
    own = (d / 2 + 10) * U if norm else 0.0
    return turn(n, angle, rot, pairs), partners(n, rot, pairs) * (own + (12 * U if rot else 0.0))


def qk_backward(dy, x, gamma, angle, rot, pairs, eps, norm=True):
    """(dx, dgamma, bound of dx, sum of |terms| of dgamma)"""
    dy = np.asarray(dy, np.float64)
    g = turn(dy, -angle if rot else angle, rot, pairs)
    G = partners(dy, rot, pairs)        # turned back, a pair's two stay within this
    if not norm:
        return g, None, G * 12 * U, None
    x = np.asarray(x, np.float64)
    d = x.shape[-1]
    gamma = np.ones(d) if gamma is None else np.asarray(gamma, np.float64)
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    dx = r * g * gamma - x * r ** 3 * (g * gamma * x).mean(-1, keepdims=True)
    amount = r * G * np.abs(gamma) + np.abs(x) * r ** 3 * (G * np.abs(gamma * x)).mean(-1, keepdims=True)
    # g is off by 12 half steps of G, r three times by d / 2 + 8, the mean's products and sum by d / 2 + 4, six products and a sum
    return dx, (g * x * r).sum((0, 1)), amount * (12 + 3 * (d / 2 + 8) + d / 2 + 12) * U, (G * np.abs(x) * r).sum((0, 1))


# ----------------------------------------------------------------------------------------------- drawing a token
def sample_row(z, temperature, top_p, min_p, top_k, u):
    """(token, logprob, kept) of one row; z and the rule's numbers as they are stored, in 64 bits from here on."""
    z = np.asarray(z, np.float64)
    T, p, mp, u = (float(v) for v in (temperature, top_p, min_p, u))
    if np.isnan(z).any() or not z.max() < math.inf or z.max() == -math.inf or not (0 <= T < math.inf) or p != p or mp != mp:
        return -1, math.nan, 0
    m = z.max()
    if T == 0:
        return int(np.argmax(z)), 0.0, 1
    with np.errstate(over="ignore"):
        e = (z - m) / T
        w = np.rint(ONE * np.exp(e)).astype(np.int64)
    order = np.argsort(-z, kind="stable")
    stays = order[:top_k] if top_k else order
    if p < 1:
        upto = np.cumsum(w[stays])
        need = max(1, math.ceil(p * float(int(upto[-1]))))
        stays = stays[:int(np.searchsorted(upto, need)) + 1]
    least = min(mp, 1.0) * ONE
    stays = np.sort(stays[(w[stays].astype(np.float64) >= least) & (w[stays] > 0)])
    upto = np.cumsum(w[stays])
    total = int(upto[-1])
    target = min(int(math.floor((min(u, 1.0) if u > 0 else 0.0) * float(total))), total - 1)
    token = int(stays[np.searchsorted(upto, target, side="right")])
    return token, e[token] - math.log(total / ONE), len(stays)


# -------------------------------------------------------------------------------------------- the gradients' norm
def grad_norm(parts, max_norm, scale):
    """(norm, factor, norms of each)"""
    scale, max_norm = float(np.float32(scale)), float(np.float32(max_norm))
    each = [float(np.square(np.asarray(p, np.float64)).sum()) for p in parts]
    norm = scale * math.sqrt(math.fsum(each)) if all(map(math.isfinite, each)) else (math.nan if any(v != v for v in each) else math.inf)
    factor = scale * (1.0 if norm <= max_norm else max_norm / norm)
    return norm, factor, [scale * math.sqrt(v) for v in each]
