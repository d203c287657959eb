"""CPU statements in 64 bits of score routing and the MXFP4 format.

Test infrastructure only: plain numpy from the definitions, one row or block at a time where that is clearest, and
nothing shared with the CUDA path.  MXFP4 follows the OCP Microscaling Formats (MX) specification v1.0.
"""
import numpy as np

SOFTMAX, SIGMOID = 0, 1
GROUP_MAX, GROUP_SUM2 = 0, 1


# ---------------------------------------------------------------------------------------------
# Score routing
# ---------------------------------------------------------------------------------------------
def _sigmoid(z):
    out = np.empty_like(z)
    pos = z >= 0
    out[pos] = 1.0 / (1.0 + np.exp(-z[pos]))
    e = np.exp(z[~pos])
    out[~pos] = e / (1.0 + e)
    return out


def scores_of_row(z, score):
    """Scores of one row; logits of -inf and NaN are switched off (score 0), +inf takes its limit."""
    z = np.asarray(z, dtype=np.float64)
    on = z > -np.inf
    s = np.zeros_like(z)
    if not on.any():
        return s
    if score == SIGMOID:
        s[on] = _sigmoid(z[on])
    else:
        m = z[on].max()
        with np.errstate(invalid="ignore"):
            e = np.where(z[on] == m, 1.0, np.exp(z[on] - m))
        s[on] = e / e.sum()
    return s


def route(z, k, score, bias=None, n_group=1, topk_group=1, group_score=GROUP_MAX, renorm=True, scale=1.0, valid=None):
    """topk_idx [T,k], gates [T,k], scores [T,E], counts [E]."""
    z = np.asarray(z, dtype=np.float64)
    T, E = z.shape
    idx = np.full((T, k), -1, dtype=np.int32)
    gates = np.zeros((T, k))
    scores = np.zeros((T, E))
    size = E // n_group
    for t in range(T):
        if valid is not None and not valid[t]:
            continue
        s = scores[t] = scores_of_row(z[t], score)
        on = z[t] > -np.inf
        with np.errstate(invalid="ignore"):
            key = np.where(on, z[t] if bias is None else s + bias, -np.inf)
        key[~(key > -np.inf)] = -np.inf
        if n_group > 1:
            gkey = np.where(on, s, -np.inf) if bias is None and group_score == GROUP_SUM2 else key
            value = np.full(n_group, -np.inf)
            for g in range(n_group):
                best = sorted((v for v in gkey[g * size:(g + 1) * size] if v > -np.inf), reverse=True)
                if best:
                    value[g] = sum(best[:2]) if group_score == GROUP_SUM2 else best[0]
            stay = sorted(range(n_group), key=lambda g: (-value[g], g))[:topk_group]
            for g in range(n_group):
                if g not in stay:
                    key[g * size:(g + 1) * size] = -np.inf
        chosen = [e for e in sorted(range(E), key=lambda e: (-key[e], e)) if key[e] > -np.inf][:k]
        if not chosen:
            continue
        w = s[chosen]
        if renorm:
            w = chosen_weights(z[t][chosen], score)
        idx[t, :len(chosen)] = chosen
        gates[t, :len(chosen)] = scale * w
    counts = np.bincount(idx[idx >= 0].ravel(), minlength=E).astype(np.int32)
    return idx, gates, scores, counts


def chosen_weights(zs, score):
    """Renormalised weights of the chosen logits, s_j / sum s, formed without underflow."""
    if score == SIGMOID:
        log_s = -np.logaddexp(0.0, -zs)
    else:
        m = zs.max()
        log_s = np.where(zs == m, 0.0, zs - m) if np.isinf(m) else zs
    e = np.exp(log_s - log_s.max())
    return e / e.sum()


def route_backward(z, idx, dgates, score, renorm=True, scale=1.0):
    """d sum(gates * dgates) / d z through the chosen weights."""
    z = np.asarray(z, dtype=np.float64)
    dgates = np.asarray(dgates, dtype=np.float64)
    T, E = z.shape
    dz = np.zeros((T, E))
    for t in range(T):
        slots = [j for j in range(idx.shape[1]) if 0 <= idx[t, j] < E]
        if not slots:
            continue
        sel = idx[t, slots]
        dw = scale * dgates[t, slots]
        s = scores_of_row(z[t], score)
        if renorm:
            p = chosen_weights(z[t][sel], score)
            v = p * (dw - (p * dw).sum())
            if score == SIGMOID:
                v = v * _sigmoid(-z[t][sel])
            np.add.at(dz[t], sel, v)
        elif score == SIGMOID:
            np.add.at(dz[t], sel, dw * s[sel] * _sigmoid(-z[t][sel]))
        else:
            ds = np.zeros(E)
            np.add.at(ds, sel, dw)
            dz[t] = s * (ds - (s * ds).sum())
    return dz


# ---------------------------------------------------------------------------------------------
# MXFP4
# ---------------------------------------------------------------------------------------------
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])    # values of the codes 0..7; bit 3 is the sign
BLOCK = 32


def mx4_quantize(x):
    """codes uint8 [..., K] (one per element) and scale bytes uint8 [..., K/32] of x.
    Scale 2^(floor(log2 max|x|) - 2) as a byte with bias 127 (not below byte 0); elements to the nearest e2m1 value,
    ties to the even code, at most 6 in size; a block that holds an infinity or NaN has the scale byte 255 (NaN)."""
    x = np.asarray(x, dtype=np.float64)
    v = x.reshape(x.shape[:-1] + (-1, BLOCK))
    finite = np.isfinite(v).all(-1)
    v = np.where(finite[..., None], v, 0.0)
    amax = np.abs(v).max(-1)
    exp = np.where(amax > 0, np.frexp(amax)[1] - 1 - 2, -127)
    exp = np.maximum(exp, -127)
    p = np.abs(v) / np.exp2(exp.astype(np.float64))[..., None]
    dist = np.abs(p[..., None] - E2M1)
    best = dist.min(-1, keepdims=True)
    near = dist == best                                       # one code, or two neighbours at a tie
    code = np.argmax(near, -1)
    tie = near.sum(-1) == 2
    code = np.where(tie & (code % 2 == 1), code + 1, code)
    code = code + np.where(np.signbit(v), 8, 0)
    scale = np.where(finite, exp + 127, 255).astype(np.uint8)
    code = np.where(finite[..., None], code, 0).astype(np.uint8)
    return code.reshape(x.shape), scale


def mx4_values(codes, scales):
    sign = np.where(codes & 8, -1.0, 1.0)
    v = (sign * E2M1[codes & 7]).reshape(codes.shape[:-1] + (-1, BLOCK))
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    return (v * s[..., None]).reshape(codes.shape)


def mx4_round(x):
    return mx4_values(*mx4_quantize(x))


def mx4_pack(codes):
    """Two codes per byte along the last index, the even element in the low half."""
    return (codes[..., 0::2] | (codes[..., 1::2] << 4)).astype(np.uint8)


def mx4_tile_scales(scales, fill=0):
    """[rows, K/32] scale bytes in the stored order [ceil(rows/128)][ceil(K/128)][512]: byte
    (r % 32) * 16 + (r / 32 % 4) * 4 + j of a tile is block 4c + j of row r."""
    rows, nb = scales.shape
    tr, tc = (rows + 127) // 128, (nb + 3) // 4
    out = np.full((tr, tc, 512), fill, dtype=np.uint8)
    for r in range(rows):
        for b in range(nb):
            out[r // 128, b // 4, (r % 32) * 16 + (r % 128 // 32) * 4 + b % 4] = scales[r, b]
    return out
