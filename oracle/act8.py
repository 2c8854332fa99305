"""Activations in 8 bits, root-mean-square norm and the weight gradient of an inner product in numpy, 64 bits, channels on axis 1 of [n, c] (rows) or
[n, c, pixels] (maps).  TEST INFRASTRUCTURE ONLY."""
import numpy as np

TOP = {"e4m3": 448.0, "i8": 127.0}
NAN = {"e4m3": 0x7F, "i8": 0x80}
# the largest magnitude that a code can stand for: in fp16, and in fp32 and bf16
LIMIT = {("e4m3", "f16"): 61440.0, ("i8", "f16"): 65024.0, ("e4m3", "f32"): 1.875 * 2.0 ** 127, ("i8", "f32"): 127 * 2.0 ** 120}


def e4m3_table():
    """What the 256 codes stand for."""
    byte = np.arange(256)
    sign, exponent, mantissa = np.where(byte > 127, -1.0, 1.0), (byte >> 3) & 15, byte & 7
    v = np.where(exponent > 0, (1 + mantissa / 8) * 2.0 ** (exponent - 7.0), mantissa * 2.0 ** -9)
    v[(byte & 0x7F) == 0x7F] = np.nan
    return sign * v


def _blocks(x):
    """Lines in blocks of 32, zeros behind the last element."""
    length = x.shape[-1]
    b = np.zeros(x.shape[:-1] + (-(-length // 32) * 32,))
    b[..., :length] = x
    return b.reshape(x.shape[:-1] + (-1, 32))


def pack(x, code, kind):
    """codes and scales (uint8) of x along its last axis; kind: the tensor's type."""
    x = np.asarray(x, np.float64)
    limit = LIMIT[code, "f16" if kind == "f16" else "f32"]
    b = _blocks(np.where(np.isfinite(x), np.clip(x, -limit, limit), 0.0))
    largest = np.abs(b).max(-1)
    k = np.full(largest.shape, -117)
    some = largest > 0
    k[some] = np.maximum(np.ceil(np.log2(largest[some] / TOP[code])).astype(int) - 1, -117)       # the logarithm may be one off
    for _ in range(3):
        k = np.where(largest > TOP[code] * 2.0 ** k, k + 1, k)
    u = b / 2.0 ** k[..., None]
    if code == "e4m3":
        table = e4m3_table()[:127]
        a = np.abs(u)
        hi = np.clip(np.searchsorted(table, a), 0, 126)
        lo = np.maximum(hi - 1, 0)
        down, up = a - table[lo], table[hi] - a
        q = np.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi) + np.where(np.signbit(u), 128, 0)
    else:
        q = np.rint(u).astype(int) & 0xFF
    q = q.reshape(x.shape[:-1] + (-1,))[..., :x.shape[-1]]
    return np.where(np.isfinite(x), q, NAN[code]).astype(np.uint8), (k + 127).astype(np.uint8)


def unpack(codes, scales, code):
    codes = np.asarray(codes)
    v = e4m3_table()[codes] if code == "e4m3" else np.where(codes == 128, np.nan, codes.astype(np.int8).astype(np.float64))
    return v * np.repeat(2.0 ** (scales.astype(np.float64) - 127), 32, axis=-1)[..., :codes.shape[-1]]


def _along(p, like):
    return np.asarray(p, np.float64).reshape((1, -1) + (1,) * (like.ndim - 2))


def rms_norm(s, gamma, eps=1e-5):
    """y, rstd (without axis 1)."""
    s = np.asarray(s, np.float64)
    rstd = 1.0 / np.sqrt((s * s).mean(axis=1, keepdims=True) + eps)
    y = s * rstd
    return (y if gamma is None else y * _along(gamma, s)), rstd[:, 0]


def rms_norm_bwd(dy, s, rstd, gamma):
    """ds, dgamma."""
    dy, s, r = np.asarray(dy, np.float64), np.asarray(s, np.float64), np.expand_dims(np.asarray(rstd, np.float64), 1)
    h = s * r
    g = dy if gamma is None else dy * _along(gamma, s)
    ds = r * (g - h * (g * h).mean(axis=1, keepdims=True))
    return ds, (dy * h).sum(axis=(0,) + tuple(range(2, s.ndim)))


def weight_gradient(dy, x):
    """dw [c_out, c], db."""
    dy, x = np.asarray(dy, np.float64), np.asarray(x, np.float64)
    a, b = np.moveaxis(dy, 1, 0).reshape(dy.shape[1], -1), np.moveaxis(x, 1, 0).reshape(x.shape[1], -1)
    return a @ b.T, a.sum(1)
