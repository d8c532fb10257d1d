"""Plain forms in 64 bits of the recurrence, the log probabilities and the AdamW step, written from their definitions, and
bounds of what 32-bit arithmetic may add, from the roundings of each step."""
import numpy as np

U = 2.0 ** -24          # half a step of fp32, relative


# ------------------------------------------------------------------------------------- gated linear recurrence
def starts_of(tokens, sequences, starts=None):
    return list(starts) if starts is not None else [j * (tokens // sequences) for j in range(sequences + 1)]


def scan_forward(f, x, starts, h0=None):
    """(h, states before every token, last states)"""
    f, x = np.asarray(f, np.float64), np.asarray(x, np.float64)
    n, c = len(starts) - 1, f.shape[1]
    with np.errstate(over="ignore"):
        b = 1.0 / (1.0 + np.exp(f))
    h, before, last = np.zeros_like(x), np.zeros_like(x), np.zeros((n, c))
    for j in range(n):
        now = np.zeros(c) if h0 is None else np.asarray(h0[j], np.float64)
        for t in range(starts[j], starts[j + 1]):
            before[t] = now
            now = now + b[t] * (x[t] - now)
            h[t] = now
        last[j] = now
    return h, before, last


def scan_backward(f, x, starts, dh, h0=None, dh_last=None):
    """(dgate, dx, dh0, D), D being the whole gradient of every state"""
    f, x, dh = (np.asarray(a, np.float64) for a in (f, x, dh))
    n, c = len(starts) - 1, f.shape[1]
    with np.errstate(over="ignore"):
        b = 1.0 / (1.0 + np.exp(f))
    _, before, _ = scan_forward(f, x, starts, h0)
    D, first = np.zeros_like(x), np.zeros((n, c))
    for j in range(n):
        g = np.zeros(c) if dh_last is None else np.asarray(dh_last[j], np.float64)
        for t in range(starts[j + 1] - 1, starts[j] - 1, -1):
            D[t] = dh[t] + g
            g = (1.0 - b[t]) * D[t]
        first[j] = g
    return D * (before - x) * b * (1.0 - b), D * b, first, D


def scan_bounds(f, x, starts, h0=None, dh=None, dh_last=None):
    """Bounds of the error of fp32 arithmetic: of h, dgate, dx, dh0 and the last states.  b is off by (|f| + 8) U of itself (the
    exponential's argument, the exponential, the sum and the reciprocal); a step adds that share of b |x - h| and one rounding of
    the difference and of the result, and a decay that is carried as a product adds a rounding of the carried state.  States are
    means of inputs, so X, the largest of them so far, bounds them.  Twice the sum of all that, propagated like the state."""
    f, x = np.asarray(f, np.float64), np.asarray(x, np.float64)
    n, c = len(starts) - 1, f.shape[1]
    with np.errstate(over="ignore"):
        b = 1.0 / (1.0 + np.exp(f))
    db = b * (np.minimum(np.abs(f), 90) + 8) * U
    _, before, _ = scan_forward(f, x, starts, h0)
    eh, ebefore, elast = np.zeros_like(x), np.zeros_like(x), np.zeros((n, c))
    for j in range(n):
        X = np.zeros(c) if h0 is None else np.abs(h0[j])
        e = np.zeros(c)
        for t in range(starts[j], starts[j + 1]):
            X = np.maximum(X, np.abs(x[t]))
            ebefore[t] = e
            e = (1.0 - b[t]) * e + db[t] * 2 * X + 3 * U * X
            eh[t] = e
        elast[j] = e
    out = dict(h=2 * eh, h_last=2 * elast)
    if dh is not None:
        dh = np.asarray(dh, np.float64)
        dgate, dx, first, D = scan_backward(f, x, starts, dh, h0, dh_last)
        eD, efirst = np.zeros_like(x), np.zeros((n, c))
        for j in range(n):
            e = np.zeros(c)
            most = np.zeros(c) if dh_last is None else np.abs(dh_last[j])
            for t in range(starts[j + 1] - 1, starts[j] - 1, -1):
                most = np.maximum(most, np.abs(D[t]))
                e = e + 2 * U * most
                eD[t] = e
                e = (1.0 - b[t]) * e + (db[t] + 2 * U) * most
            efirst[j] = e
        ba, gap = b * (1.0 - b), np.abs(before - x)
        out["dx"] = 2 * (b * eD + (db + U * b) * np.abs(D))
        # b - b^2 is off by what b is, and by a rounding of b^2 that cancellation leaves where b is near one
        eba = db + 2 * U * b
        out["dgate"] = 2 * (ba * gap * eD + np.abs(D) * ba * (2 * ebefore + U * (np.abs(before) + np.abs(x))) + np.abs(D) * gap * (eba + 3 * U * ba))
        out["dh0"] = 2 * efirst
    return out


def scan_shares(f):
    """(a, b), the shares of the old state and of the input: each by itself, so that the smaller one keeps all its bits"""
    f = np.asarray(f, np.float64)
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-f)), 1.0 / (1.0 + np.exp(f))


def scan_by_shares(f, x, starts, h0=None, dh=None, dh_last=None):
    """(results, bounds), each a dict of h, h_last and, with dh, dgate, dx and dh0: the recurrence as h_t = a_t h_{t-1} + b_t x_t, and
    what fp32 arithmetic may add where no bit is lost to cancellation.
    M_t = a_t M_{t-1} + b_t |x_t| is what the terms of h_t amount to: it falls where a gate lets go of the state.  The smaller share is
    off by d U of itself, d = 1.25 |f| + 8 (the exponential's argument and its constant, the exponential, the sum, the reciprocal and the
    product), and by 2^-125 where the exponential has no more bits; the larger by less.  A step adds d U M_t, half a step of the difference of
    input and state, which the smaller share weighs, of the result, and of the carried product: 4 U M_t.  Back it is the same with N, what the
    terms of D amount to.  Twice the sum of it all, propagated like the state."""
    a, b = scan_shares(f)
    f, x = np.asarray(f, np.float64), np.asarray(x, np.float64)
    n, c = len(starts) - 1, f.shape[1]
    d = (1.25 * np.abs(f) + 8) * U
    tiny = 2.0 ** -125
    zero = lambda: np.zeros_like(x)
    h, before, ebefore, mbefore, eh = zero(), zero(), zero(), zero(), zero()
    last, elast = np.zeros((n, c)), np.zeros((n, c))
    for j in range(n):
        now = np.zeros(c) if h0 is None else np.asarray(h0[j], np.float64)
        M, e = np.abs(now), np.zeros(c)
        for t in range(starts[j], starts[j + 1]):
            before[t], ebefore[t], mbefore[t] = now, e, M
            most = M + np.abs(x[t])
            now = a[t] * now + b[t] * x[t]
            M = a[t] * M + b[t] * np.abs(x[t])
            e = a[t] * e + (d[t] + 4 * U) * M + tiny * most
            h[t], eh[t] = now, e
        last[j], elast[j] = now, e
    results, bounds = dict(h=h, h_last=last), dict(h=2 * eh, h_last=2 * elast)
    if dh is None:
        return results, bounds
    dh = np.asarray(dh, np.float64)
    D, N, eD = zero(), zero(), zero()
    first, efirst = np.zeros((n, c)), np.zeros((n, c))
    for j in range(n):
        g = np.zeros(c) if dh_last is None else np.asarray(dh_last[j], np.float64)
        G, e = np.abs(g), np.zeros(c)
        for t in range(starts[j + 1] - 1, starts[j] - 1, -1):
            D[t], N[t] = dh[t] + g, np.abs(dh[t]) + G
            eD[t] = e + 2 * U * N[t]
            g, G = a[t] * D[t], a[t] * N[t]
            e = a[t] * eD[t] + (d[t] + 2 * U) * G + tiny * N[t]
        first[j], efirst[j] = g, e
    ab, gap = a * b, mbefore + np.abs(x)
    results.update(dgate=D * (before - x) * ab, dx=D * b, dh0=first)
    # a b is off by both, and by the roundings of a square and a difference; the gap by that of the state and its own
    bounds.update(dx=2 * (b * eD + (d + 2 * U) * b * N + tiny * N), dh0=2 * efirst,
                  dgate=2 * (ab * (gap * eD + N * (ebefore + U * gap) + N * gap * (2 * d + 5 * U)) + tiny * N * gap))
    return results, bounds


# ------------------------------------------------------------------------------------------ log probabilities
def logprob_forward(z, tokens, scale, top=0):
    """dict of logprob, entropy, stats, top_id, top_logprob, and q, p"""
    z = np.asarray(z, np.float64)
    rows, cols = z.shape
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        m = z.max(1)
        empty = m == -np.inf
        d = np.where(empty[:, None], 0.0 if cols == 0 else -np.inf, z - np.where(empty, 0, m)[:, None])
        e = np.exp(scale * d)
        s = np.where(empty, 1.0, e.sum(1))
        q = scale * d - np.log(s)[:, None]
        p = e / s[:, None]
        H = np.log(s) - scale * np.where(e > 0, d * e, 0.0).sum(1) / s
    named = (tokens >= 0) & (tokens < cols)
    logprob = np.where(named, q[np.arange(rows), np.where(named, tokens, 0)], 0.0)
    order = np.argsort(-z, axis=1, kind="stable")[:, :top].astype(np.int64)
    return dict(logprob=logprob, entropy=np.where(empty, 0.0, H), stats=np.stack([m, np.log(s)], 1), top_id=order,
                top_logprob=np.take_along_axis(q, order, 1), q=q, p=p, empty=empty)


def logprob_backward(z, tokens, scale, dlogprob=None, dentropy=None):
    r = logprob_forward(z, tokens, scale)
    q, p, rows, cols = r["q"], r["p"], *np.asarray(z).shape
    named = (tokens >= 0) & (tokens < cols)
    d = np.zeros((rows, cols))
    if dlogprob is not None:
        dl = np.where(named, dlogprob, 0.0)
        d -= p * dl[:, None]
        d[np.arange(rows)[named], tokens[named]] += dl[named]
    if dentropy is not None:
        with np.errstate(invalid="ignore"):
            d -= dentropy[:, None] * np.where(p > 0, p * (q + r["entropy"][:, None]), 0.0)
    return np.where(r["empty"][:, None], 0.0, d * scale)


def logprob_bounds(z, scale):
    """Bounds of the error of ln s and of q for fp32: an exponential is off by 4 U of itself for each unit of its argument and 4 U
    beside, a lane adds up to cols / 64 of them, and 16 joins follow; a logarithm's result and the two of q's subtraction."""
    r = logprob_forward(z, np.zeros(len(z), np.int64), scale)
    arg = np.where(r["p"] > 0, np.abs(r["q"] + r["stats"][:, 1:]), 0.0)
    mean = (r["p"] * arg).sum(1)
    ls = U * (4 * mean + z.shape[1] / 64 + 24 + 2 * np.abs(r["stats"][:, 1]))
    q = ls[:, None] + U * (4 * arg + 2 * np.abs(np.where(r["p"] > 0, r["q"], 0.0)))
    # sum of p |c d|: each product off by what its exponential is, the sum by its order, s by ls
    entropy = ls + mean * (U * (z.shape[1] / 64 + 32) + ls) + 4 * U * (r["p"] * arg * arg).sum(1) + 2 * U * np.abs(r["entropy"])
    return dict(ls=ls, q=q, entropy=entropy, p=r["p"], forward=r)


# ------------------------------------------------------------------------------------------------------ AdamW
def f32(v):
    return float(np.float32(v))


def hash_bits(n, tensor, seed):
    key = (seed * 0x9E3779B1 + (tensor + 1) * 0x7F4A7C15) % (1 << 32)
    word = np.uint64(0xFFFFFFFF)
    x = (np.arange(n, dtype=np.uint64) + np.uint64(key)) & word
    x = ((x ^ (x >> np.uint64(16))) * np.uint64(0x45C3A2AD)) & word
    x = ((x ^ (x >> np.uint64(15))) * np.uint64(0x2D51F9B5)) & word
    x = x ^ (x >> np.uint64(16))
    return ((x & np.uint64(0xFFFF)).astype(np.float64) + 0.5) / 65536, ((x >> np.uint64(16)).astype(np.float64) + 0.5) / 65536


def by_block(scale, n):
    return np.repeat(np.asarray(scale, np.float64), 64)[:n]


def adamw(w, m, v, g, decay, lr, beta1, beta2, eps, grad_scale, step):
    """(w, m, v) after a step, all in 64 bits"""
    b1, b2 = f32(beta1), f32(beta2)
    w, m, v, g = (np.asarray(a, np.float64) for a in (w, m, v, g))
    g = g * f32(grad_scale)
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    up = m / (1 - b1 ** step) / (np.sqrt(v / (1 - b2 ** step)) + f32(eps))
    return w - f32(lr) * f32(decay) * w - f32(lr) * up, m, v


def quantised(m, v, tensor, seed):
    """(codes of m, scales, codes of v, scales)"""
    n = m.size
    blocks = lambda a: np.concatenate([a, np.zeros(-n % 64)]).reshape(-1, 64)
    sm = np.abs(blocks(m)).astype(np.float32).max(1) * np.float32(1 / 127)
    sv = blocks(v).astype(np.float32).max(1) * np.float32(1 / 65025)
    um, uv = hash_bits(n, tensor, seed)
    bm, bv = by_block(sm, n), by_block(sv, n)
    y = np.divide(m, bm, out=np.zeros(n), where=bm > 0)
    z = np.divide(v, bv, out=np.zeros(n), where=bv > 0)
    cm = np.clip(np.floor(y + um), -127, 127)
    q = np.minimum(np.floor(np.sqrt(z)), 255)
    cv = np.minimum(q + (z - q * q > uv * (2 * q + 1)), 255)
    return cm.astype(np.int8), sm, np.where(z > 0, np.maximum(cv, 1), cv).astype(np.uint8), sv
