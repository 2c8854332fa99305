"""GPU: rows and maps so far apart that 32 bits do not span them, against the 64-bit oracle at the bounds of dense ones."""
import numpy as np
import pytest
import torch

from norm_bounds import TYPES, U, bwd_bounds, close, inputs, norm_bounds, place, rounded, to64
from oracle import norm as ON

pytestmark = pytest.mark.gpu


def check(shape, stride, kind, p, seed):
    from paper_1509_03371_amd import binding as B
    lines = shape[0] if len(shape) == 2 else shape[0] * shape[1]
    # NaN in between: what is read there, or counted, shows
    store = torch.full((stride * (lines - 1) + 24 * (shape[-1] + 3),), float("nan"), dtype=TYPES[kind], device="cuda")
    used = [0]

    def far(values):
        strides = (stride, 1) if len(shape) == 2 else (stride * shape[1], stride, 1)
        v = store.as_strided(shape, strides, used[0])
        used[0] += shape[-1] + 3                # (odd: lines begin anywhere)
        v.copy_(values)
        return v

    def empty():
        return far(torch.zeros(shape, dtype=TYPES[kind], device="cuda"))

    x, r, gamma, beta, dy, dsum = inputs(shape, kind, seed)
    x, r, dy, dsum = (far(place(a, kind)) for a in (x, r, dy, dsum))
    gd, bd = torch.from_numpy(gamma).cuda(), torch.from_numpy(beta).cuda()
    kw = dict(axis=1, p=p, seed=3, offset=8)
    y, s, mean, rstd = B.layer_norm(x, gd, bd, 1e-3, residual=r, out=empty(), sum_out=empty(), **kw)
    dropped = ON.dropout(to64(x), p, 3, 8)
    rs = to64(r) + dropped
    es = U * (2 * np.abs(dropped) + np.abs(rs)) * (1 + 4 * U)
    close(s, rs, rounded(rs, kind, es), "s")
    ry, rm, rr, by, bm, brs = norm_bounds(rs, es, gamma, beta, 1e-3, kind)
    close(y, ry, by, "y")
    close(mean, rm, bm, "mean")
    close(rstd, rr, brs, "rstd")
    t, rg, rb, et, eg, eb = bwd_bounds(to64(dy), to64(s), to64(mean), to64(rstd), gamma, to64(dsum), kind)
    rdx = ON.dropout(t, p, 3, 8)
    scale = 65536.0 / (65536 - ON.threshold(p))
    given = [to64(v) for v in (dy, s, dsum)]
    for place_of_result in (None, dy, dsum):                   # a buffer of its own, in place
        dx, dres, dg, db = B.layer_norm_backward(dy, s, mean, rstd, gd, dsum=dsum, dx=empty() if place_of_result is None else place_of_result,
                                                 dresidual=empty() if p else None, **kw)
        close(dg, rg, eg, "dgamma")
        close(db, rb, eb, "dbeta")
        close(dres, t, rounded(t, kind, et), "dresidual")
        close(dx, rdx, (rdx != 0) * rounded(rdx, kind, et * scale + 2 * U * np.abs(rdx)), "dx")
        for v, was in zip((dy, s, dsum), given):
            v.copy_(torch.from_numpy(was))
    none = B.layer_norm_backward(dy, s, mean, rstd, gd, dsum=dsum, dx=empty(), dresidual=empty() if p else None, parameters=False, **kw)
    close(none[1], t, rounded(t, kind, et), "without the sums")
    out = empty()
    assert np.array_equal(to64(B.dropout(x, 0.4, 9, axis=1, out=out)), to64(B.dropout(x.contiguous(), 0.4, 9, axis=1)))


# rows of one launch and of two, of fewer than eight channels, longer than registers
@pytest.mark.parametrize("shape,stride", [((70, 40), 1 << 24), ((70, 5), 1 << 24), ((67, 1), 1 << 24), ((65, 8), 1 << 24), ((257, 9), 1 << 24), ((130, 264), 1 << 24), ((9, 777), 1 << 27),
                                          ((600, 130), 1 << 24), ((3, 600), 1 << 31), ((2, 20003), 1 << 31)], ids=str)
@pytest.mark.parametrize("p", [0.0, 0.2])
def test_rows(shape, stride, p):
    check(shape, stride, "bf16", p, 77)


@pytest.mark.parametrize("shape,stride", [((60, 333), 1 << 24), ((40, 1001), 1 << 25)], ids=str)
@pytest.mark.parametrize("kind", ["f32", "f16"])
def test_rows_of_other_types(shape, stride, kind):
    check(shape, stride, kind, 0.1, 78)


@pytest.mark.parametrize("shape,stride", [((2, 30, 9), 1 << 27), ((1, 9, 70), 1 << 29), ((1, 5, 2), 1 << 29), ((3, 11, 1), 1 << 27), ((2, 17, 701), 1 << 27)], ids=str)
@pytest.mark.parametrize("p", [0.0, 0.2])
def test_maps(shape, stride, p):
    check(shape, stride, "bf16", p, 79)
