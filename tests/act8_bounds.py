"""Bounds of the arithmetic of activations in 8 bits, root-mean-square norm and the weight gradient against the 64-bit oracle, element by element.

u = 2^-24 is half a step of fp32.  A sum of terms |a| has an error of at most D u sum|a|, D = the longest chain of additions that an element passes
through: less than 320 + C/64 over the channels of a position, 320 + Q/64 over Q positions, 128 + Q/8 in a product over Q positions (at most three terms
each; a matrix instruction takes 16 positions or more in one step).  Other operations: u of their result each; sqrt and divisions 2 u.
"""
import numpy as np

from norm_bounds import HALF, TINY, U, close, rounded, to64  # noqa: F401
from oracle import act8 as OA


def _along(p, like):
    p = np.ones(like.shape[1]) if p is None else np.asarray(p, np.float64)
    return p.reshape((1, -1) + (1,) * (like.ndim - 2))


def norm_bounds(s, s_err, gamma, eps):
    """Reference y and rstd of s (known to s_err), and the bounds of their fp32 forms."""
    depth = 320 + s.shape[1] / 64
    y, rstd = OA.rms_norm(s, gamma, eps)
    r = np.expand_dims(rstd, 1)
    square = np.abs(s) + s_err
    e_mean = ((2 * np.abs(s) * s_err + s_err ** 2) + (depth + 2) * U * square ** 2).mean(axis=1, keepdims=True) + 3 * U / r ** 2
    rel = 0.5 * e_mean * r ** 2 * (1 + 2 * e_mean * r ** 2) + 4 * U
    g = np.abs(_along(gamma, s))
    e_y = (s_err * r * (1 + rel) + np.abs(s) * r * (rel + 3 * U)) * (1 + 4 * U) * g + 2.0 ** -148
    return y, rstd, e_y, rel[:, 0] * rstd


def bwd_bounds(dy, s, rstd, gamma, dsum):
    """Reference dx and dgamma, and the bounds of their fp32 forms."""
    c, q = s.shape[1], s.shape[0] * int(np.prod(s.shape[2:], dtype=np.int64))
    depth, depth_q = 320 + c / 64, 320 + q / 64
    ds, dg = OA.rms_norm_bwd(dy, s, rstd, gamma)
    r = np.expand_dims(np.abs(np.asarray(rstd, np.float64)), 1)
    h, g = np.abs(s) * r, np.abs(dy * _along(gamma, s))
    mgh = (g * h).mean(axis=1, keepdims=True)
    e_mgh = (depth + 6) * U * mgh
    e_t = r * (2 * U * g + h * e_mgh + 3 * U * h * (mgh + e_mgh) + 3 * U * (g + h * mgh)) * (1 + 4 * U) + 2.0 ** -148
    if dsum is not None:
        ds = ds + dsum
        e_t = e_t + U * (np.abs(ds) + e_t)
    others = (0,) + tuple(range(2, s.ndim))
    return ds, dg, e_t, (depth_q + 4) * U * (np.abs(dy) * h).sum(axis=others)


def product_bounds(dy, x):
    """Reference dw and db, and the bounds of theirs."""
    q = x.shape[0] * int(np.prod(x.shape[2:], dtype=np.int64))
    dw, db = OA.weight_gradient(dy, x)
    aw, ab = OA.weight_gradient(np.abs(dy), np.abs(x))
    return dw, db, (128 + q / 8) * U * aw, (320 + q / 8) * U * ab


def held(codes, scales, code, kind, ref, err, what):
    """Are these the codes and scales of values that are ref, known to err?"""
    codes, scales = codes.cpu().numpy(), scales.cpu().numpy().astype(int)
    limit = OA.LIMIT[code, "f16" if kind == "f16" else "f32"]
    ref, err = np.clip(ref, -limit, limit), np.broadcast_to(err, ref.shape)
    least = OA.pack(np.maximum(np.abs(ref) - err, 0), code, kind)[1]
    most = OA.pack(np.abs(ref) + err, code, kind)[1]
    assert ((least <= scales) & (scales <= most)).all(), what + ": another scale"
    k = np.repeat(scales - 127.0, 32, axis=-1)[..., :ref.shape[-1]]
    step = 2.0 ** (k - 1) if code == "i8" else np.maximum(2.0 ** (k - 10), (np.abs(ref) + err) * 2.0 ** -4)
    close(OA.unpack(codes, scales, code), ref, step + err, what)
