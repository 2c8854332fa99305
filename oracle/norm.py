"""Dropout and layer norm in numpy, 64 bits, channels on axis 1 of [n, c, ...].  TEST INFRASTRUCTURE ONLY."""
import numpy as np


def philox4x32(counter, key, rounds=10):
    """Philox4x32 (Salmon, Moraes, Dror, Shaw, SC 2011): counter [4, ...] and key (k0, k1) of 32-bit words."""
    w = [np.asarray(x, dtype=np.uint64) for x in counter]
    k0, k1 = int(key[0]), int(key[1])
    low, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    for _ in range(rounds):
        a, b = w[0] * np.uint64(0xD2511F53), w[2] * np.uint64(0xCD9E8D57)
        w = [(b >> half) ^ w[1] ^ np.uint64(k0), b & low, (a >> half) ^ w[3] ^ np.uint64(k1), a & low]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return np.stack(w)


def threshold(p):
    return int(np.floor(p * 65536 + 0.5))


def keep_mask(positions, channels, p, seed, offset):
    """[positions, channels]: which elements dropout keeps; positions: how many, or an array of position numbers."""
    q = np.asarray(positions, dtype=np.uint64).reshape(-1) if np.ndim(positions) else np.arange(positions, dtype=np.uint64)
    groups = (channels + 7) // 8
    shape = (len(q), groups)
    ctr = [np.broadcast_to((q & np.uint64(0xFFFFFFFF))[:, None], shape),
           np.arange(groups, dtype=np.uint64)[None, :] + ((q >> np.uint64(32)) * np.uint64(1 << 24))[:, None],
           np.full(shape, offset & 0xFFFFFFFF, np.uint64), np.full(shape, offset >> 32, np.uint64)]
    w = philox4x32(ctr, (seed & 0xFFFFFFFF, seed >> 32)).astype(np.uint32)          # [4, positions, groups]
    u = np.stack([w & np.uint32(0xFFFF), w >> np.uint32(16)], axis=-1)              # [4, positions, groups, 2]
    u = u.transpose(1, 2, 0, 3).reshape(len(q), groups * 8)[:, :channels]
    return u >= threshold(p)


def dropout(x, p, seed, offset):
    """x [n, c, ...]; position = image * plane + pixel."""
    x = np.asarray(x, dtype=np.float64)
    n, c = x.shape[:2]
    plane = int(np.prod(x.shape[2:], dtype=np.int64))
    t = threshold(p)
    keep = keep_mask(n * plane, c, p, seed, offset).reshape((n, plane, c)).transpose(0, 2, 1).reshape(x.shape)
    scale = 0.0 if t >= 65536 else 65536.0 / (65536 - t)
    with np.errstate(invalid="ignore"):
        return np.where(keep, x * scale, 0.0)


def layer_norm(s, gamma, beta, eps=1e-5):
    """Norm over axis 1.  Returns y, mean, rstd (without axis 1)."""
    s = np.asarray(s, dtype=np.float64)
    along = (1, -1) + (1,) * (s.ndim - 2)
    mean = s.mean(axis=1, keepdims=True)
    rstd = 1.0 / np.sqrt(((s - mean) ** 2).mean(axis=1, keepdims=True) + eps)
    y = (s - mean) * rstd
    if gamma is not None:
        y = y * np.asarray(gamma, dtype=np.float64).reshape(along)
    if beta is not None:
        y = y + np.asarray(beta, dtype=np.float64).reshape(along)
    return y, mean[:, 0], rstd[:, 0]


def layer_norm_bwd(dy, s, mean, rstd, gamma):
    """ds, dgamma, dbeta."""
    dy, s = np.asarray(dy, dtype=np.float64), np.asarray(s, dtype=np.float64)
    along = (1, -1) + (1,) * (s.ndim - 2)
    h = (s - np.expand_dims(mean, 1)) * np.expand_dims(rstd, 1)
    g = dy if gamma is None else dy * np.asarray(gamma, dtype=np.float64).reshape(along)
    ds = np.expand_dims(rstd, 1) * (g - g.mean(axis=1, keepdims=True) - h * (g * h).mean(axis=1, keepdims=True))
    others = (0,) + tuple(range(2, s.ndim))
    return ds, (dy * h).sum(axis=others), dy.sum(axis=others)
