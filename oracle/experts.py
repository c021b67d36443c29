"""Mixture-of-experts operators -- oracle side (numpy, fp64): routing, the plan of slots, the experts' MXFP4 products, the combination of
their rows, 8-bit checkpoints and the gated activation.

TEST INFRASTRUCTURE ONLY (see oracle/__init__.py).  Written from the definitions in include/metis.h, one token, expert or block at a time where
that is clearer than fast.
"""
import numpy as np

from . import mx as omx


# ---- routing ----------------------------------------------------------------------------------------------------------------------

def _score(x, scores):
    """Scores of one row; an expert without a finite or +inf logit has none (0)."""
    live = x > -np.inf                             # False for NaN
    if scores == "sigmoid":
        with np.errstate(over="ignore"):
            return np.where(live, 1.0 / (1.0 + np.exp(-np.where(live, x, 0.0))), 0.0)
    if not live.any():
        return np.zeros_like(x)
    e = np.where(live, np.exp(np.where(live, x, 0.0) - x[live].max()), 0.0)
    return e / e.sum()


def selection_keys(x, bias, scores):
    """What the selection compares, [E]; -inf where the expert is not available."""
    live = x > -np.inf
    base = _score(x, scores) if scores == "sigmoid" else x
    key = np.where(live, base, -np.inf) + (0.0 if bias is None else bias)
    return np.where(live & (key > -np.inf), key, -np.inf)


def group_scores(key, groups, scores):
    out = []
    for g in key.reshape(groups, -1):
        top = np.sort(g)[::-1][:2]
        out.append(top[0] + top[1] if scores == "sigmoid" and len(top) > 1 and top[1] > -np.inf else top[0])
    return np.array(out)


def route(logits, k, bias=None, valid=None, scores="softmax", groups=1, top_groups=1, renorm=True, scale=1.0):
    """idx [T, k] (-1 where there is none) and weights [T, k]."""
    x = np.asarray(logits, dtype=np.float64)
    T, E = x.shape
    idx, w = np.full((T, k), -1, dtype=np.int64), np.zeros((T, k))
    for t in range(T):
        if valid is not None and not valid[t]:
            continue
        key = selection_keys(x[t], bias, scores)
        if top_groups < groups:
            order = np.argsort(-group_scores(key, groups, scores), kind="stable")
            keep = np.zeros(groups, dtype=bool)
            keep[order[:top_groups]] = True
            key = np.where(np.repeat(keep, E // groups), key, -np.inf)
        order = np.argsort(-key, kind="stable")[:k]
        order = order[key[order] > -np.inf]
        idx[t, :len(order)] = order
        w[t, :len(order)] = scale * chosen_weights(x[t], order, scores, renorm)
    return idx, w


def chosen_weights(x, order, scores, renorm):
    if len(order) == 0:
        return np.zeros(0)
    if scores == "softmax" and renorm:
        e = np.exp(x[order] - x[order].max())
        return e / e.sum()
    p = _score(x, scores)[order]
    if renorm:
        return p / p.sum() if p.sum() > 0 else np.zeros_like(p)
    return p


def route_grads(logits, idx, dweights, scores="softmax", renorm=True, scale=1.0):
    x = np.asarray(logits, dtype=np.float64)
    out = np.zeros_like(x)
    for t in range(x.shape[0]):
        js = [j for j, e in enumerate(idx[t]) if 0 <= e < x.shape[1] and x[t, e] > -np.inf]
        if not js:
            continue
        e, v = np.asarray(idx[t])[js], scale * np.asarray(dweights[t], dtype=np.float64)[js]
        p = _score(x[t], scores)
        if scores == "sigmoid":
            d, z = v, p[e].sum()
            if renorm:
                d = (v - (v * p[e]).sum() / z) / z if z > 0 else np.zeros_like(v)
            np.add.at(out[t], e, d * p[e] * (1 - p[e]))
        elif renorm:
            q = chosen_weights(x[t], e, scores, True)
            np.add.at(out[t], e, q * (v - (v * q).sum()))
        else:
            g = np.zeros(x.shape[1])
            np.add.at(g, e, v)
            out[t] = p * (g - (v * p[e]).sum())
    return out


def plan(idx, experts):
    """offsets [E + 1], token [T * k], slot [T, k]."""
    T, k = idx.shape
    token, slot, offsets = np.full(T * k, -1), np.full((T, k), -1), [0]
    n = 0
    for e in range(experts):
        for t, j in zip(*np.nonzero(idx == e)):   # row-major: the order of the choices
            token[n], slot[t, j] = t, n
            n += 1
        offsets.append(n)
    return np.array(offsets), token, slot


# ---- the experts' products -----------------------------------------------------------------------------------------------------------

def experts_product(x, w, offsets, token, gather):
    """C [S, N] of x [T or S, K] (quantized here) and w = (codes, scales) of [E * N, K]; unused slots hold zeros."""
    E, S = len(offsets) - 1, len(token)
    xq = omx.dequantize_mx(*omx.quantize_mx(x))
    wv = omx.dequantize_mx(*w)
    N = wv.shape[0] // E
    C = np.zeros((S, N))
    for e in range(E):
        s = np.arange(offsets[e], offsets[e + 1])
        C[s] = xq[token[s] if gather else s] @ wv[e * N:(e + 1) * N].T
    return C


def experts_wgrad(g, x, offsets, token, gather):
    """dW [E * N, K] of g [S, N] and x [T or S, K], both quantized along the slots of each expert, in blocks of 32 from its first."""
    E, N, K = len(offsets) - 1, g.shape[1], x.shape[1]
    out = np.zeros((E * N, K))
    for e in range(E):
        s = np.arange(offsets[e], offsets[e + 1])
        if len(s) == 0:
            continue
        pad = -len(s) % 32
        ge = np.concatenate([np.asarray(g, dtype=np.float64)[s], np.zeros((pad, N))]).T
        xe = np.concatenate([np.asarray(x, dtype=np.float64)[token[s] if gather else s], np.zeros((pad, K))]).T
        out[e * N:(e + 1) * N] = omx.mx_gemm_nt(omx.quantize_mx(ge), omx.quantize_mx(xe))
    return out


def combine(rows, slot, weights=None):
    T, k = slot.shape
    y = np.zeros((T, rows.shape[1]))
    for j in range(k):
        there = slot[:, j] >= 0
        w = 1.0 if weights is None else np.asarray(weights, dtype=np.float64)[there, j, None]
        y[there] += w * np.asarray(rows, dtype=np.float64)[slot[there, j]]
    return y


def combine_grads(dy, rows, slot, weights):
    """drows [S, D] (zeros in unused slots), dweights [T, k]."""
    dy, rows = np.asarray(dy, dtype=np.float64), np.asarray(rows, dtype=np.float64)
    drows, dw = np.zeros_like(rows), np.zeros(slot.shape)
    for t, j in zip(*np.nonzero(slot >= 0)):
        s = slot[t, j]
        drows[s] = float(weights[t, j]) * dy[t]
        dw[t, j] = dy[t] @ rows[s]
    return drows, dw


# ---- 8-bit checkpoints and the gated activation -----------------------------------------------------------------------------------------

def e4m3_values():
    """The 127 non-negative finite E4M3 values in the order of their codes 0x00 .. 0x7E."""
    code = np.arange(127)
    e, m = code >> 3, code & 7
    return np.where(e == 0, m * 2.0 ** -9, (1 + m / 8) * 2.0 ** (e - 7.0))


def quantize_mx8(x):
    """codes [rows, cols] (E4M3 bits) and scales [rows, cols / 32] (E8M0): the smallest power of two 2^t, t >= -127, with
    amax <= 448 * 2^t; nearest E4M3 value of e / 2^t, ties to the even code.  A block with an infinity or a NaN: scale byte 255, codes 0x7F;
    a block of zeros: scale byte 0."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    b = x.reshape(rows, -1, 32)
    bad = ~np.isfinite(b).all(axis=2)
    amax = np.abs(np.where(np.isfinite(b), b, 0.0)).max(axis=2)
    m, e = np.frexp(amax)
    t = np.where(amax > 0, np.clip(np.where(m <= 0.875, e - 9, e - 8), -127, 127), -127)
    y = np.abs(np.where(bad[..., None], 0.0, b)) / np.exp2(t.astype(np.float64))[..., None]
    grid = e4m3_values()
    mid = (grid[1:] + grid[:-1]) / 2
    code = np.searchsorted(mid, y, side="left")    # y on a midpoint: the lower code, ...
    tie = (code < len(mid)) & (y == mid[np.minimum(code, len(mid) - 1)])
    code = np.where(tie & (code % 2 == 1), code + 1, code)       # ... or the even one
    code = code | (np.signbit(b).astype(np.int64) << 7)
    code = np.where(bad[..., None], 0x7F, code)
    return code.reshape(rows, cols).astype(np.uint8), np.where(bad, 255, t + 127).astype(np.uint8)


def dequantize_mx8(codes, scales):
    c = np.asarray(codes).astype(np.int64)
    v = np.append(e4m3_values(), np.nan)[c & 127] * np.where(c & 128, -1.0, 1.0)
    s = np.asarray(scales).astype(np.float64)
    scale = np.where(s == 255, np.nan, np.exp2(s - 127))
    return (v.reshape(c.shape[0], -1, 32) * scale[..., None]).reshape(c.shape)


def swiglu(gu):
    g, u = np.split(np.asarray(gu, dtype=np.float64), 2, axis=1)
    with np.errstate(over="ignore"):
        return g / (1 + np.exp(-g)) * u


def swiglu_grads(gu, dact):
    """d(gate), d(up) side by side, [S, 2 F]."""
    g, u = np.split(np.asarray(gu, dtype=np.float64), 2, axis=1)
    with np.errstate(over="ignore"):
        p = 1 / (1 + np.exp(-g))
    d = np.asarray(dact, dtype=np.float64)
    return np.concatenate([d * u * p * (1 + g * (1 - p)), d * g * p], axis=1)
