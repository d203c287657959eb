"""CPU statements in 64 bits of the FP8 format, the norm in front of the sublayer and the FP8 expert layer.

Test infrastructure only: plain numpy from the definitions, nothing shared with the CUDA path.  The elements are those of the
OCP 8-bit floating point specification's e4m3.
"""
import numpy as np

BLOCK = 128


def _e4m3():
    """Values of the codes 0..126: exponent field 0 holds multiples of 2^-9, field e multiples of 2^(e - 10) from 2^(e - 7)."""
    v = []
    for code in range(127):
        e, m = code >> 3, code & 7
        v.append(m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10))
    return np.array(v)


E4M3 = _e4m3()


def _nearest(p):
    """Codes of magnitudes p <= 448: the nearest value, the even code of two that are as near."""
    hi = np.clip(np.searchsorted(E4M3, p), 0, 126)
    lo = np.maximum(hi - 1, 0)
    below, above = p - E4M3[lo], E4M3[hi] - p
    take_hi = (above < below) | ((above == below) & (hi % 2 == 0))
    return np.where(take_hi, hi, lo)


def quantize(x, rows=1):
    """codes uint8 [R, K] and scale bytes uint8 [R, ceil(K/128)] of x [R, K], a scale for every `rows` x 128 elements: the
    smallest 2^e, e >= -127, with max|x| / 2^e <= 448, as a byte with bias 127; 255 where the block holds an infinity or NaN."""
    x = np.asarray(x, dtype=np.float64)
    R, K = x.shape
    codes, scales = np.zeros((R, K), np.uint8), np.zeros((R, -(-K // BLOCK)), np.uint8)
    for r in range(0, R, rows):
        for b in range(scales.shape[1]):
            at = np.s_[r:r + rows, b * BLOCK:(b + 1) * BLOCK]
            v = x[at]
            if not np.isfinite(v).all():
                scales[r:r + rows, b] = 255
                continue
            amax = np.abs(v).max()
            e = -127
            if amax > 0:
                e = max(-127, int(np.floor(np.log2(amax))) - 10)
                while amax / 2.0 ** e > 448:
                    e += 1
            codes[at] = _nearest(np.abs(v) / 2.0 ** e) + np.where(np.signbit(v), 128, 0)
            scales[r:r + rows, b] = e + 127
    return codes, scales


def values(codes, scales):
    v = np.where(codes & 128, -1.0, 1.0) * E4M3[codes & 127]
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    return v * s.repeat(BLOCK, 1)[:, :v.shape[1]]


def round_rows(x, rows=1):
    return values(*quantize(x, rows))


def stored_codes(codes):
    """Codes with the zeros that fill a row to a multiple of 32 bytes."""
    return np.pad(codes, ((0, 0), (0, -codes.shape[1] % 32)))


def stored_scales(scales, fill):
    """[R, blocks] scale bytes in the stored order [ceil(R/128)][ceil(blocks/4)][512]: byte
    (r % 32) * 16 + (r / 32 % 4) * 4 + j of a tile is block 4c + j of row r; `fill` where there is none."""
    R, nb = scales.shape
    out = np.full((-(-R // 128), -(-nb // 4), 512), fill, dtype=np.uint8)
    for r in range(R):
        for b in range(nb):
            out[r // 128, b // 4, (r % 32) * 16 + (r % 128 // 32) * 4 + b % 4] = scales[r, b]
    return out


# ---------------------------------------------------------------------------------------------
# Norm
# ---------------------------------------------------------------------------------------------
def rms_norm(h, w, eps):
    h = np.asarray(h, dtype=np.float64)
    return h / np.sqrt((h * h).mean(1, keepdims=True) + eps) * w


def rms_norm_backward(h, w, dy, eps, dh=None):
    """dx [T, d] and dw [d]."""
    h, dy = np.asarray(h, dtype=np.float64), np.asarray(dy, dtype=np.float64)
    s = 1.0 / np.sqrt((h * h).mean(1, keepdims=True) + eps)
    g = dy * w
    dx = s * g - h * s ** 3 * (g * h).mean(1, keepdims=True)
    return (dx if dh is None else dx + dh), (dy * h * s).sum(0)
