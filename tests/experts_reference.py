"""Plain forms in double of the operators of a layer of routed experts, with the magnitudes their error bounds are stated in."""
import numpy as np

import layer_reference as ref


def scores(logits, kind):
    """Rows of double logits (-inf: masked, no NaN, +inf already the largest number) -> scores."""
    x = np.asarray(logits, np.float64)
    with np.errstate(over="ignore", invalid="ignore"):
        if kind == 1:
            return 1.0 / (1.0 + np.exp(-x))
        top = np.where(np.isfinite(x), x, -np.inf).max(1, keepdims=True)
        e = np.where(np.isfinite(x), np.exp(x - np.where(np.isfinite(top), top, 0.0)), 0.0)
        s = e.sum(1, keepdims=True)
        return e / np.where(s > 0, s, 1.0)


def route(logits, k, kind=0, bias=None, groups=1, kept=1, top=1, renormalise=True, scale=1.0):
    """Token by token, expert by expert.  Returns experts, weights, start, tokens, place (numpy)."""
    x = np.asarray(logits, np.float64).copy()
    x[np.isnan(x)] = -np.inf
    x[x == np.inf] = np.finfo(np.float32).max
    T, E = x.shape
    s = scores(x, kind)
    # without a bias or a sum the order is the logits' own
    c = x.copy() if bias is None and (groups == 1 or top == 1) else s + (0.0 if bias is None else np.asarray(bias, np.float64))
    c[x == -np.inf] = -np.inf
    c[np.isnan(c)] = -np.inf
    experts, weights = np.full((T, k), -1, np.int32), np.zeros((T, k))
    size = E // groups
    for t in range(T):
        free = [e for e in range(E) if c[t, e] > -np.inf]
        if groups > 1:
            value = []
            for g in range(groups):
                mine = sorted((c[t, e] for e in free if e // size == g), reverse=True)[:top]
                value.append(float(np.sum(mine)) if mine else -np.inf)
            best = sorted(range(groups), key=lambda g: (-value[g], g))[:kept]
            best = {g for g in best if value[g] > -np.inf}
            free = [e for e in free if e // size in best]
        pick = sorted(free, key=lambda e: (-c[t, e], e))[:k]
        experts[t, :len(pick)] = pick
        if pick and renormalise:
            # ratios of scores, whatever their size
            y = x[t, pick]
            with np.errstate(over="ignore"):
                low = y if kind == 0 else np.minimum(y, 0.0) - np.log1p(np.exp(-np.abs(y)))
                p = np.exp(low - low.max())
            weights[t, :len(pick)] = scale * p / p.sum()
        elif pick:
            weights[t, :len(pick)] = scale * s[t, pick]
    rows = sorted((int(experts[t, j]), t, j) for t in range(T) for j in range(k) if experts[t, j] >= 0)
    start = np.searchsorted([r[0] for r in rows], np.arange(E + 1)).astype(np.int32)
    place = np.full((T, k), -1, np.int32)
    for i, (_, t, j) in enumerate(rows):
        place[t, j] = i
    return experts, weights, start, np.array([r[1] for r in rows], np.int32), place


def codes_of(v, lo, hi):
    with np.errstate(invalid="ignore"):
        return np.where(v > hi, 1, np.where(v < lo, -1, 0)).astype(np.int8)


def pack(codes):
    rows, n = codes.shape
    nb = (n + 127) // 128
    c = np.zeros((rows, nb * 128), np.int8)
    c[:, :n] = codes
    c = c.reshape(rows, nb, 128)
    planes = [np.packbits((c != 0), axis=2, bitorder="little"), np.packbits((c > 0), axis=2, bitorder="little")]
    return np.concatenate(planes, 2).reshape(rows, nb * 32)


def experts(x, tokens, start, w, a_scale, a_offset, w_scale, w_offset, bias=None, kind=0, gated=False):
    """x [T,K], w [E,N,K] codes; scales per input row, and [E,N].  Returns (values, magnitudes, rows that an expert has) of [R, F]."""
    E, N, K = w.shape
    F = N // 2 if gated else N
    R = len(tokens)
    out, mag, live = np.full((R, F), np.nan), np.full((R, F), np.nan), np.zeros(R, bool)
    for e in range(E):
        r = np.arange(start[e], start[e + 1])
        if not len(r):
            continue
        m = tokens[r]
        y, g = ref.linear(x[m], w[e], a_scale[m], a_offset[m], w_scale[e], w_offset[e], None if bias is None else bias[e])
        z = ref.act(y[:, :F], kind)
        # (an activation's slope is below 1.13)
        out[r] = z * y[:, F:] if gated else z
        mag[r] = 1.13 * g[:, :F] * np.abs(y[:, F:]) + np.abs(z) * g[:, F:] if gated else 1.13 * g
        live[r] = True
    return out, mag, live


def block_norm(branch, residual=None, place=None, weights=None, post=None, gate=None, gate_kind=0, scale=None, pre=None, eps=1e-6):
    """All double.  Returns h, n and their magnitudes: what the terms add up to, times how the norms pass an error on."""
    W = (branch if branch is not None else residual).shape[1]
    T = place.shape[0] if place is not None else (branch if branch is not None else residual).shape[0]
    h, mag = np.zeros((T, W)), np.zeros((T, W))
    if branch is not None:
        y, my = branch, np.abs(branch)
        if place is not None:
            w = np.ones(place.shape) if weights is None else weights
            y, my = np.zeros((T, W)), np.zeros((T, W))
            for j in range(place.shape[1]):
                term = np.where(place[:, j, None] >= 0, w[:, j, None] * branch[np.maximum(place[:, j], 0)], 0.0)
                y, my = y + term, my + np.abs(term)
        f = np.ones((T, W))
        if post is not None:
            root = np.sqrt((y * y).mean(1, keepdims=True) + eps)
            # an error of the root: that of its sum, which the terms' errors add to by their vector's length
            my = my + np.abs(y) * (1.0 + np.sqrt((my * my).sum(1, keepdims=True) / np.maximum((y * y).sum(1, keepdims=True), 1e-300)))
            f = f / root * post
        if gate is not None:
            with np.errstate(over="ignore"):
                s = 1.0 / (1.0 + np.exp(-gate))
            f = f * (gate if gate_kind == 0 else s if gate_kind == 1 else gate * s)
        if scale is not None:
            f = f * scale
        h, mag = f * y, np.abs(f) * my
    if residual is not None:
        h, mag = h + residual, mag + np.abs(residual)
    n, mn = h, mag
    if pre is not None:
        root = np.sqrt((h * h).mean(1, keepdims=True) + eps)
        n = h / root * pre
        mn = np.abs(pre) / root * mag + np.abs(n) * (1.0 + np.sqrt((mag * mag).sum(1, keepdims=True) / np.maximum((h * h).sum(1, keepdims=True), 1e-300)))
    return h, mag, n, mn
