"""GPU: an infinite gradient makes what the formulas make of it: its channel's sums, and the results of its position; nothing else."""
import numpy as np
import pytest
import torch

from norm_bounds import bwd_bounds, close, inputs, place, rounded, to64
from oracle import norm as ON

pytestmark = [pytest.mark.gpu, pytest.mark.filterwarnings("ignore:invalid value encountered")]          # (infinite less infinite)


def check(shape, kind, order, channel, pixel, adds):
    from paper_1509_03371_amd import binding as B
    x, _, gamma, beta, dy, dsum = inputs(shape, kind, 61)
    x, dsum = place(x, kind, 0, order), place(dsum, kind, 0, order)
    gd = torch.from_numpy(gamma).cuda()
    _, s, mean, rstd = B.layer_norm(x, gd, axis=1)
    clean = place(dy, kind, 0, order)
    at = (shape[0] - 1, channel, pixel)
    clean[at] = 0
    hot = clean.clone()
    hot[at] = float("inf")
    kw = dict(dsum=dsum, p=0.3, seed=5) if adds else {}
    dx, dres, dg, db = B.layer_norm_backward(hot, s, mean, rstd, gd, axis=1, **kw)
    t, rg, rb, et, eg, eb = bwd_bounds(to64(clean), to64(s), to64(mean), to64(rstd), gamma, to64(dsum) if adds else None, kind)
    with np.errstate(invalid="ignore"):
        hit = (slice(shape[0] - 1, shape[0]), slice(None), slice(pixel, pixel + 1))
        part, _, _ = ON.layer_norm_bwd(to64(hot)[hit], to64(s)[hit], to64(mean)[hit[0], hit[2]], to64(rstd)[hit[0], hit[2]], gamma)
    t[hit] = part + (to64(dsum)[hit] if adds else 0)
    assert not np.isfinite(t[hit]).any() and np.isneginf(t[hit]).any()
    close(dres, t, rounded(t, kind, et), "gradient of the sum")
    if adds:
        keep = ON.dropout(np.ones(shape), 0.3, 5, 0) != 0
        got = to64(dx)
        assert np.array_equal(got[hit], np.where(keep[hit], t[hit], 0), equal_nan=True)
    h = (to64(s)[at] - to64(mean)[at[0], pixel]) * to64(rstd)[at[0], pixel]
    rg[channel], rb[channel] = np.sign(h) * np.inf, np.inf
    close(dg, rg, eg, "dgamma")
    close(db, rb, eb, "dbeta")


# planes whose last tile is not full (lanes behind its end hold pixels of others), whatever takes them: registers of 64, 32, 16, 8 and 4 pixel lanes, one
# launch with roles, octets in turn, planes of fewer than four pixels
MAPS = [(1, 24, 70001), (2, 48, 40003), (1, 104, 20002), (1, 304, 9001), (1, 800, 5003), (1, 1600, 2001), (1, 24, 901), (2, 2056, 1303), (700, 24, 3)]


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("adds", [False, True])
@pytest.mark.parametrize("shape", MAPS, ids=str)
def test_at_a_pixel_that_two_lanes_hold(shape, kind, adds):
    for back in (1, 2, 4):
        check(shape, kind, "dense", 3, max(0, shape[2] - back), adds)


# the last octet is not whole, or a wave has lanes without one
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("adds", [False, True])
@pytest.mark.parametrize("shape", [(1, 20, 70001), (2, 40, 40003), (1, 99, 20002), (1, 301, 9001), (1, 776, 5003), (1, 1601, 2001), (1, 20, 901), (1, 40, 901), (2, 2049, 1303),
                                   (700, 20, 3), (700, 24, 2)], ids=str)
def test_in_the_last_channels(shape, kind, adds):
    c = shape[1]
    for channel in {c - 1, (c - 1) // 8 * 8}:
        check(shape, kind, "dense", channel, 0, adds)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("adds", [False, True])
@pytest.mark.parametrize("shape", [(1, 20, 3001), (1, 777, 901), (1, 1000, 37), (2, 5, 700), (1, 20001, 30)], ids=str)
def test_rows(shape, kind, adds):
    check(shape, kind, "last", shape[1] - 1, shape[2] - 1, adds)
