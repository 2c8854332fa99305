"""GPU: root-mean-square norm on the caller's tensors and its gradient, from tensors and from tensors held in 8 bits, against the 64-bit oracle (bounds:
act8_bounds.py)."""
import numpy as np
import pytest
import torch

from act8_bounds import U, bwd_bounds, close, held, norm_bounds, rounded, to64
from norm_bounds import TYPES, inputs, place
from oracle import act8 as OA

pytestmark = pytest.mark.gpu

ROWS = [(1, 1), (3, 2), (5, 7), (1, 8), (300, 9), (2, 48), (64, 63), (65, 64), (1000, 33), (37, 200), (9, 300), (16, 1024), (9, 777), (4, 1025), (33, 2048), (5, 4099), (600, 520),
        (3, 9000), (2, 20011), (1, 40000)]
MAPS = [(1, 1, 1), (2, 1, 77), (1, 3, 5), (3, 8, 1), (2, 9, 64), (1, 48, 1001), (2, 65, 333), (1, 200, 400), (4, 16, 31), (1, 1024, 49), (2, 777, 10), (70, 30, 3), (1, 2049, 33),
        (1, 5000, 3), (1, 64, 5000)]


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shape", ROWS + MAPS, ids=str)
def test_norm(shape, kind):
    from paper_1509_03371_amd import binding as B
    for i, (pad, residual, code) in enumerate([(0, False, None), (5, True, "e4m3"), (0, True, "i8"), (3, False, "i8")]):
        x, r, gamma, _, _, _ = inputs(shape, kind, 40 + i, 0.3)
        x, r = place(x, kind, pad), place(r, kind) if residual else None
        gd, gr = (None, None) if i == 0 else (torch.from_numpy(gamma).cuda(), gamma)
        y8, sum8 = (B.Packed.like(x, code, axis=1), B.Packed.like(x, "e4m3", axis=1)) if code else (None, None)
        y, s, rstd = B.rms_norm(x, gd, 1e-3, axis=1, residual=r, y8=y8, sum8=sum8)
        rs, es = to64(x), 0.0
        if residual:
            rs = rs + to64(r)
            es = U * np.abs(rs)
            close(s, rs, rounded(rs, kind, es), "s")
        else:
            assert s is x
        ry, rr, ey, er = norm_bounds(rs, es, gr, 1e-3)
        close(y, ry, rounded(ry, kind, ey), "y")
        close(rstd, rr, er, "rstd")
        if code:
            flat = shape if y8.order[0] == B.SK_MAPS else shape[:2]         # (one pixel an image: rows)
            held(y8.codes.reshape(flat), y8.scales, code, kind, ry.reshape(flat), np.reshape(ey, flat), "y8")
            held(sum8.codes.reshape(flat), sum8.scales, "e4m3", kind, rs.reshape(flat), np.reshape(es, flat) if residual else 0.0, "sum8")
            # one result alone: the same bits
            alone = B.Packed.like(x, code, axis=1)
            none, no_sum, _ = B.rms_norm(x, gd, 1e-3, axis=1, residual=r, out=False, sum_out=False, y8=alone)
            assert none is None and no_sum is None and torch.equal(alone.codes, y8.codes) and torch.equal(alone.scales, y8.scales)
            if not residual:
                p = B.pack8(x, "e4m3", axis=1)
                assert torch.equal(p.scales, sum8.scales) and torch.equal(p.codes, sum8.codes), "the same tensor in 8 bits"


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shape", ROWS + MAPS, ids=str)
def test_gradient(shape, kind):
    from paper_1509_03371_amd import binding as B
    for i, (pad, code, order) in enumerate([(0, None, "dense"), (5, "e4m3", "dense"), (0, "i8", "dense"), (3, None, "dense"), (0, "e4m3", "last")]):
        x, _, gamma, _, dy, dsum = inputs(shape, kind, 50 + i, 0.3)
        x, dy = place(x, kind, pad, order), place(dy, kind, pad, order)
        dsum = place(dsum, kind, 0, order) if i in (1, 3) else None
        gd, gr = (None, None) if i == 2 else (torch.from_numpy(gamma).cuda(), gamma)
        rstd = torch.from_numpy((1.0 / np.sqrt((to64(x) ** 2).mean(axis=1) + 1e-3)).astype(np.float32)).cuda()
        s = x if code is None else B.pack8(x, code, axis=1)
        rs = to64(x) if code is None else to64(B.unpack8(s))
        dx, dg = B.rms_norm_backward(dy, s, rstd, gd, axis=1, dsum=dsum)
        t, rg, et, eg = bwd_bounds(to64(dy), rs, to64(rstd), gr, None if dsum is None else to64(dsum))
        close(dx, t, rounded(t, kind, et), "dx")
        close(dg, rg, eg, "dgamma")
        only, none = B.rms_norm_backward(dy, s, rstd, gd, axis=1, dsum=dsum, parameters=False)
        assert torch.equal(only, dx) and none is None
        again = B.rms_norm_backward(dy, s, rstd, gd, axis=1, dsum=dsum)
        assert torch.equal(again[0], dx) and torch.equal(again[1], dg), "two equal calls"


@pytest.mark.parametrize("shape", [(7, 33), (3, 20, 6)], ids=str)
def test_gradient_by_differences(shape):
    """The kernels' gradient against differences of the 64-bit norm."""
    from paper_1509_03371_amd import binding as B
    x, _, gamma, _, dy, _ = inputs(shape, "f32", 60)
    dy = dy * 100
    xd, gd, dyd = place(x, "f32"), torch.from_numpy(gamma).cuda(), place(dy, "f32")
    x, dy, g64 = to64(xd), to64(dyd), gamma.astype(np.float64)
    _, _, rstd = B.rms_norm(xd, gd, axis=1)
    dx, dg = (to64(t) for t in B.rms_norm_backward(dyd, xd, rstd, gd, axis=1))
    step = 1e-5
    for grad, arr in ((dx, x), (dg, g64)):
        for i in np.ndindex(arr.shape):
            old = arr[i]
            arr[i] = old + step
            up = (OA.rms_norm(x, g64)[0] * dy).sum()
            arr[i] = old - step
            down = (OA.rms_norm(x, g64)[0] * dy).sum()
            arr[i] = old
            assert abs((up - down) / (2 * step) - grad[i]) <= 1e-4 * (1 + abs(grad[i]))


@pytest.mark.parametrize("shape", [(40, 300), (2, 48, 130)], ids=str)
def test_in_place(shape):
    from paper_1509_03371_amd import binding as B
    for kind in TYPES:
        x, r, gamma, _, dy, dsum = (torch.from_numpy(np.asarray(a)).to(TYPES[kind]).cuda() for a in inputs(shape, kind, 70))
        gamma = gamma.float()
        y8 = B.Packed.like(x, "i8", axis=1)
        y, s, rstd = B.rms_norm(x, gamma, axis=1, residual=r, y8=y8)
        dx, dg = B.rms_norm_backward(dy, s, rstd, gamma, axis=1, dsum=dsum)
        for first, second in ((0, 1), (1, 0)):
            both, again8 = [x.clone(), r.clone()], B.Packed.like(x, "i8", axis=1)
            B.rms_norm(both[0], gamma, axis=1, residual=both[1], out=both[first], sum_out=both[second], y8=again8)
            assert torch.equal(both[first], y) and torch.equal(both[second], s) and torch.equal(again8.codes, y8.codes) and torch.equal(again8.scales, y8.scales)
        for place_ in range(3):
            three = [dy.clone(), s.clone(), dsum.clone()]
            got, dgamma = B.rms_norm_backward(three[0], three[1], rstd, gamma, axis=1, dsum=three[2], dx=three[place_])
            assert torch.equal(got, dx) and torch.equal(dgamma, dg)


@pytest.mark.parametrize("shape", [(9, 700), (2, 40, 65)], ids=str)
def test_positions_that_are_no_numbers_stay_alone(shape):
    from paper_1509_03371_amd import binding as B
    for bad in (float("nan"), float("inf")):
        x, _, gamma, _, dy, _ = inputs(shape, "f32", 80)
        xd, gd, dyd = place(x, "f32"), torch.from_numpy(gamma).cuda(), place(dy, "f32")
        y, _, rstd = B.rms_norm(xd, gd, axis=1)
        dx, _ = B.rms_norm_backward(dyd, xd, rstd, gd, axis=1)
        where = (1, 7) if len(shape) == 2 else (1, 7, 33)
        position = (1, slice(None)) if len(shape) == 2 else (1, slice(None), 33)
        other = torch.ones(shape, dtype=torch.bool, device="cuda")
        other[position] = False
        xb = xd.clone()
        xb[where] = bad
        y8 = B.Packed.like(xb, "e4m3", axis=1)
        yb, _, rb = B.rms_norm(xb, gd, axis=1, y8=y8)
        assert torch.equal(yb[other], y[other]) and not torch.isfinite(yb[where])
        v = B.unpack8(y8, dtype=torch.float32)
        assert torch.equal(torch.isnan(v), ~torch.isfinite(yb))
        dyb = dyd.clone()
        dyb[where] = bad
        dxb, dgb = B.rms_norm_backward(dyb, xd, rstd, gd, axis=1)
        assert torch.equal(dxb[other], dx[other]) and not torch.isfinite(dxb[where])
        assert (~torch.isfinite(dgb)).sum() == 1 and not torch.isfinite(dgb[7])


def test_nothing_to_do():
    from paper_1509_03371_amd import binding as B
    for shape in ((0, 5), (3, 5, 0)):
        x = torch.empty(shape, device="cuda")
        gamma = torch.ones(5, device="cuda")
        y, _, rstd = B.rms_norm(x, gamma, axis=1)
        dx, dg = B.rms_norm_backward(x, x, rstd, gamma, axis=1)
        assert y.shape == shape and dx.shape == shape and torch.equal(dg, torch.zeros(5, device="cuda"))
