"""Bounds of dropout's and layer norm's arithmetic against the 64-bit oracle, element by element.

u = 2^-24 is half a step of fp32, ut that of the stored type (plus half its smallest subnormal).  A sum of terms |a| in any of the orders the kernels
take has an error of at most D u sum|a|, D = the longest chain of additions that an element passes through: less than 80 + C/64 over the channels of
a position (a thread's own, then trees) and 64 + Q/64 over Q positions.  Other operations: u of their result each; sqrt and the divisions
within one unit, 2 u.
"""
import numpy as np
import torch

from oracle import norm as ON

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
U = 2.0 ** -24
HALF = {"f32": U, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -24}      # half the smallest subnormal and a margin of two


def to64(t):
    return t.detach().double().cpu().numpy()


def close(got, ref, bound, what):
    got, ref = to64(got) if isinstance(got, torch.Tensor) else got, np.asarray(ref)
    assert got.shape == ref.shape, what
    bad = ~(np.abs(got - ref) <= bound)
    bad &= ~(np.isnan(got) & np.isnan(ref)) & ~(got == ref)
    if bad.any():
        i = tuple(int(k) for k in np.argwhere(bad)[0])
        raise AssertionError("%s: %d of %d beyond the bound, first at %s: %r instead of %r, bound %r" % (
            what, bad.sum(), bad.size, i, got[i], ref[i], np.broadcast_to(bound, ref.shape)[i]))


def rounded(ref, kind, err):
    """bound of a stored value whose fp32 form is off by err"""
    return err + HALF[kind] * (np.abs(ref) + err) + TINY[kind]


def place(values, kind, pad=0, order="dense"):
    """A GPU tensor of these values: dense, with `pad` elements of NaN behind every line, or channels last in memory."""
    t = torch.from_numpy(np.ascontiguousarray(values)).to(TYPES[kind]).cuda()
    if order == "last":
        return t.movedim(1, -1).contiguous().movedim(-1, 1)
    if pad:
        wide = torch.full(t.shape[:-1] + (t.shape[-1] + pad,), float("nan"), dtype=t.dtype, device="cuda")
        wide[..., :t.shape[-1]] = t
        t = wide[..., :t.shape[-1]]
    return t


def inputs(shape, kind, seed, spread=1.0):
    rng = np.random.default_rng(seed)
    c = shape[1]
    along = (1, c) + (1,) * (len(shape) - 2)
    x = rng.normal(size=shape) * np.exp(0.5 * rng.normal(size=along)) + spread * rng.normal(size=along)
    return x, 2 * rng.normal(size=shape), 1 + 0.2 * rng.normal(size=c).astype(np.float32), 0.2 * rng.normal(size=c).astype(np.float32), \
        0.01 * rng.normal(size=shape), 0.01 * rng.normal(size=shape)


def norm_bounds(s, s_err, gamma, beta, eps, kind):
    """Reference y, mean, rstd of s (known to s_err) and the bounds of all three."""
    c = s.shape[1]
    depth = 80 + c / 64
    y, mean, rstd = ON.layer_norm(s, gamma, beta, eps)
    m, r = mean[:, None], rstd[:, None]
    e_mean = (depth * U * np.abs(s) + s_err).mean(axis=1, keepdims=True) + 2 * U * np.abs(m)
    d = np.abs(s - m)
    e_d = s_err + e_mean + U * d
    e_var = (2 * d * e_d + e_d ** 2 + depth * U * d * d).mean(axis=1, keepdims=True) + 4 * U / r ** 2
    rel = 0.5 * e_var * r ** 2 * (1 + e_var * r ** 2) + 4 * U
    along = (1, c) + (1,) * (s.ndim - 2)
    g = np.ones(along) if gamma is None else np.abs(np.asarray(gamma, np.float64)).reshape(along)
    b = np.zeros(along) if beta is None else np.abs(np.asarray(beta, np.float64)).reshape(along)
    e_y = (e_d * r + d * r * (rel + 2 * U)) * (1 + rel) * g * (1 + U) + 2 * U * (d * r * g + b)
    return y, mean, rstd, rounded(y, kind, e_y), e_mean[:, 0], rel[:, 0] * rstd


def bwd_bounds(dy, s, mean, rstd, gamma, dsum, kind):
    c, q = s.shape[1], s.shape[0] * int(np.prod(s.shape[2:], dtype=np.int64))
    depth, depth_q = 80 + c / 64, 64 + q / 64
    ds, dg, db = ON.layer_norm_bwd(dy, s, mean, rstd, gamma)
    m, r = mean[:, None], rstd[:, None]
    along = (1, c) + (1,) * (s.ndim - 2)
    w = np.ones(along) if gamma is None else np.asarray(gamma, np.float64).reshape(along)
    h, g = np.abs((s - m) * r), np.abs(dy * w)
    e_h = U * (2 * np.abs(s - m) * r) + U * h
    e_g = U * g
    mg = g.mean(axis=1, keepdims=True)
    e_mg = (depth + 3) * U * mg
    mgh, e_mgh = (g * h).mean(axis=1, keepdims=True), ((depth + 4) * U * g * h + g * e_h).mean(axis=1, keepdims=True)
    inner = g + mg + h * mgh
    e_t = np.abs(r) * (e_g + e_mg + h * e_mgh + e_h * (mgh + e_mgh) + 4 * U * inner) + U * np.abs(r) * inner
    t = ds
    if dsum is not None:
        t = ds + dsum
        e_t = e_t + U * (np.abs(t) + e_t)
    others = (0,) + tuple(range(2, s.ndim))
    e_dg = ((depth_q + 2) * U * np.abs(dy) * h + np.abs(dy) * e_h).sum(axis=others)
    e_db = depth_q * U * np.abs(dy).sum(axis=others)
    return t, dg, db, e_t, e_dg, e_db
