"""Plain 64-bit forms of dropout and of the products in 8-bit floating point, from their definitions (include/rn50_hip.h:
dropout_fwd, dropout_bwd, quant_blocks_f8, matmul_f8, fc_f8_fwd, fc_f8_bwd)."""
import numpy as np

from .net import philox4x32_10

E4M3, E5M2 = "e4m3", "e5m2"
_DIGITS = {E4M3: 3, E5M2: 2}
_BIAS = {E4M3: 7, E5M2: 15}
LARGEST = {E4M3: 448.0, E5M2: 57344.0}


# -------------------------------------------------------------------- dropout
def threshold(p):
    return int(np.rint(np.float64(np.float32(p)) * 65536.0))


def factor(p):
    t = threshold(p)
    return np.float32(65536.0 / (65536.0 - t)) if t < 65536 else np.float32(0)


def kept(rows, cols, p, seed, call=0, step=0):
    """The mask, bool [rows, cols]."""
    per = (cols + 7) // 8
    b = np.arange(rows * per, dtype=np.uint64)
    c = (call + step) % 2 ** 64
    ctr = np.empty((rows * per, 4), np.uint32)
    ctr[:, 0] = b & np.uint64(0xFFFFFFFF)
    ctr[:, 1] = (b >> np.uint64(32)) | np.uint64(1 << 31)
    ctr[:, 2], ctr[:, 3] = c & 0xFFFFFFFF, c >> 32
    words = philox4x32_10(ctr, (seed & 0xFFFFFFFF, seed >> 32)).astype(np.uint32)
    halves = np.stack([words & np.uint32(0xFFFF), words >> np.uint32(16)], -1)  # [block, word, half]
    return halves.reshape(rows, per * 8)[:, :cols] >= threshold(p)


def dropout(x, p, seed, call=0, step=0, residual=None):
    """In 64 bits, with the factor as the float that the definition has."""
    keep = kept(x.shape[0], x.shape[1], p, seed, call, step)
    y = np.where(keep, np.asarray(x, np.float64) * np.float64(factor(p)), 0.0)
    return y if residual is None else y + np.asarray(residual, np.float64)


# ----------------------------------------------------------------- 8-bit numbers
def values(fmt):
    """What the 256 codes of a format stand for."""
    digits, bias = _DIGITS[fmt], _BIAS[fmt]
    out = np.empty(256)
    for c in range(256):
        e, m = (c & 127) >> digits, c & ((1 << digits) - 1)
        v = np.ldexp(m, 1 - bias - digits) if e == 0 else np.ldexp(m + (1 << digits), e - bias - digits)
        if fmt == E4M3 and (c & 127) == 127:
            v = np.nan
        if fmt == E5M2 and e == 31:
            v = np.inf if m == 0 else np.nan
        out[c] = -v if c & 128 else v
    return out


def encode(x, fmt):
    """Codes of numbers up to the largest one: to nearest, a tie to the even code."""
    codes = values(fmt)[:128]
    codes = codes[codes <= LARGEST[fmt]]  # ascending from 0
    v = np.abs(np.asarray(x, np.float64))
    hi = np.clip(np.searchsorted(codes, v), 0, len(codes) - 1)
    lo = np.maximum(hi - 1, 0)
    up, down = codes[hi] - v, v - codes[lo]
    c = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return (c | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def row_bytes(K):
    return (K + 127) // 128 * 128


def quant(x, fmt=E4M3):
    """q uint8 codes [M, row_bytes(K)] and scale uint8 [ceil(K/512), M, 4]; x: single-precision numbers."""
    x = np.asarray(x, np.float64)
    M, K = x.shape
    B = row_bytes(K) // 128
    pad = np.zeros((M, B * 128))
    pad[:, :K] = x
    pad = pad.reshape(M, B, 128)
    with np.errstate(all="ignore"):
        a = np.maximum(np.abs(pad).max(2), 2.0 ** -100)
    finite = np.isfinite(pad).all(2)
    a = np.where(finite, a, LARGEST[fmt])
    e = np.frexp(a / LARGEST[fmt])[1]  # a / F = f 2^e, 1/2 <= f < 1 (the division's rounding: put right below)
    e = np.where(a <= np.ldexp(LARGEST[fmt], e - 1), e - 1, e)
    e = np.where(a > np.ldexp(LARGEST[fmt], e), e + 1, e)
    q = encode(np.where(finite[:, :, None], np.ldexp(pad, -e[:, :, None]), 0.0), fmt)
    q = np.where(finite[:, :, None], q, np.uint8(0x7F)).reshape(M, B * 128)
    q[:, K:] = 0
    scale = np.zeros((M, (K + 511) // 512 * 4), np.uint8)
    scale[:, :B] = np.where(finite, e, 0) + 127
    return q, np.ascontiguousarray(scale.reshape(M, -1, 4).transpose(1, 0, 2))


def stands_for(q, scale, fmt=E4M3):
    """The numbers of a quantized matrix, [M, row bytes]."""
    M, Kp = q.shape
    e = scale.transpose(1, 0, 2).reshape(M, -1)[:, :Kp // 128].astype(np.int64) - 127
    return np.ldexp(values(fmt)[q].reshape(M, Kp // 128, 128), e[:, :, None]).reshape(M, Kp)


def matmul(a, w, bias=None):
    """(y, the sum of the terms' magnitudes) of matrices of numbers (as stands_for gives them)."""
    y, size = a @ w.T, np.abs(a) @ np.abs(w).T
    return (y, size) if bias is None else (y + bias, size + np.abs(bias))


def fc_fwd(x, w, w_scale, bias=None, drop=None):
    """(y, magnitude, xt, xt_scale): x single-precision numbers, w and w_scale as quant leaves them, drop: (p, seed, call, step)."""
    x = np.asarray(x, np.float32)
    if drop is not None:
        x = np.where(kept(*x.shape, *drop), x * factor(drop[0]), np.float32(0))  # (rounded to float, as it is quantized)
    y, size = matmul(stands_for(*quant(x)), stands_for(w, w_scale), bias)
    return (y, size) + quant(np.ascontiguousarray(x.T))


def fc_bwd(dy, wt, wt_scale, xt, xt_scale, fmt=E4M3, drop=None):
    """((dx, magnitude), (dW, magnitude), (db, magnitude))."""
    dy = np.asarray(dy, np.float32)
    dx, sx = matmul(stands_for(*quant(dy, fmt), fmt), stands_for(wt, wt_scale))
    if drop is not None:
        dx, sx = dropout(dx, *drop), dropout(sx, *drop)
    dw = matmul(stands_for(*quant(np.ascontiguousarray(dy.T), fmt), fmt), stands_for(xt, xt_scale))
    d = dy.astype(np.float64)
    return (dx, sx), dw, (d.sum(0), np.abs(d).sum(0))
