"""GPU: root-mean-square norm, tensors in 8 bits and the weight gradient over lines that lie far apart: on both sides of the strides at which the kernels take other
offsets or other lanes, each operand far, against the 64-bit oracle (bounds: act8_bounds.py).  All tensors of a call share one buffer, each in a slot of its own between the
lines of the others, with NaN behind every line."""
import numpy as np
import pytest
import torch

from act8_bounds import bwd_bounds, close, held, norm_bounds, product_bounds, rounded, to64
from norm_bounds import TYPES, inputs
from oracle import act8 as OA

pytestmark = pytest.mark.gpu


class Room:
    """Places for tensors of one size and one set of strides, side by side in the gaps; `fill` around them."""

    def __init__(self, shape, strides, dtype, fill, slots):
        self.shape, self.strides, self.slot, self.used, self.fill = shape, strides, shape[-1] + 3, 0, fill
        self.last = slots * self.slot
        span = sum((n - 1) * st for n, st in zip(shape[:-1], strides[:-1])) + self.last
        self.all = torch.empty(span, dtype=dtype, device="cuda")
        self.lines = self.all.as_strided(shape[:-1] + (self.last,), strides)
        self.lines.fill_(fill)

    def place(self, values=None):
        at = self.used
        self.used += self.slot
        assert self.used <= self.last
        v = self.all.as_strided(self.shape, self.strides, at)
        return v if values is None else v.copy_(torch.as_tensor(values))

    def untouched(self):
        """Nothing behind any line was written."""
        gaps = self.lines.unflatten(-1, (-1, self.slot))[..., self.shape[-1]:]
        return bool((torch.isnan(gaps) if self.fill != self.fill else gaps == self.fill).all())


def run(shape, strides, code_strides, scale_strides, kind, c_out=37):
    from paper_1509_03371_amd import binding as B
    x, r, gamma, _, dy, dsum = inputs(shape, kind, 31, 0.3)
    blocks = shape[:-1] + (-(-shape[-1] // 32),)
    room = Room(shape, strides, TYPES[kind], float("nan"), 8)
    codes, scales = (Room(s, st, torch.uint8, 0xFF, 3) for s, st in ((shape, code_strides), (blocks, scale_strides)))
    xd, rd, dyd, dsd = (room.place(t) for t in (x, r, dy, dsum))
    y8, sum8 = (B.Packed(codes.place(), scales.place(), code, axis=1) for code in ("e4m3", "i8"))
    gd = torch.from_numpy(gamma).cuda()
    y, s, rstd = B.rms_norm(xd, gd, axis=1, residual=rd, out=room.place(), sum_out=room.place(), y8=y8, sum8=sum8)
    rs = to64(xd) + to64(rd)
    es = 2.0 ** -24 * np.abs(rs)
    close(s, rs, rounded(rs, kind, es), "s")
    ry, rr, ey, er = norm_bounds(rs, es, gamma, 1e-5)
    close(y, ry, rounded(ry, kind, ey), "y")
    close(rstd, rr, er, "rstd")
    held(y8.codes, y8.scales, "e4m3", kind, ry, ey, "y8")
    held(sum8.codes, sum8.scales, "i8", kind, rs, es, "sum8")
    # gradients of what is far and of what is dense, to a place that is far
    dense = B.Packed(sum8.codes.clone(memory_format=torch.contiguous_format), sum8.scales.clone(memory_format=torch.contiguous_format), "i8", axis=1)
    v = OA.unpack(sum8.codes.cpu().numpy(), sum8.scales.cpu().numpy(), "i8")
    out = room.place()
    for source, values in ((s, to64(s)), (sum8, v), (dense, v)):
        dx, dg = B.rms_norm_backward(dyd, source, rstd, gd, axis=1, dsum=dsd, dx=out)
        t, rg, et, eg = bwd_bounds(to64(dyd), values, to64(rstd), gamma, to64(dsd))
        close(dx, t, rounded(t, kind, et), "dx")
        close(dg, rg, eg, "dgamma")
    # dense gradients of what is held far
    dx, dg = B.rms_norm_backward(dyd.contiguous(), sum8, rstd, gd, axis=1)
    t, rg, et, eg = bwd_bounds(to64(dyd), v, to64(rstd), gamma, None)
    close(dx, t, rounded(t, kind, et), "dx")
    close(dg, rg, eg, "dgamma")
    # in place
    t, _, et, _ = bwd_bounds(to64(dyd), v, to64(rstd), gamma, to64(dsd))
    B.rms_norm_backward(dyd, sum8, rstd, gd, axis=1, dsum=dsd, dx=dsd)
    close(dsd, t, rounded(t, kind, et), "dx in dsum's place")
    # there and back, to the bit
    p = B.pack8(xd, axis=1, out=y8)
    c64, s64 = OA.pack(to64(xd), "e4m3", kind)
    assert torch.equal(p.scales.cpu(), torch.from_numpy(s64)) and np.array_equal(OA.unpack(p.codes.cpu().numpy(), s64, "e4m3"), OA.unpack(c64, s64, "e4m3"))
    assert np.array_equal(to64(B.unpack8(p, out=out)), to64(torch.from_numpy(OA.unpack(c64, s64, "e4m3")).to(TYPES[kind])))
    # the weight gradient of what is far
    dz = torch.from_numpy(0.01 * np.random.default_rng(32).normal(size=shape[:1] + (c_out,) + shape[2:])).to(TYPES[kind]).cuda()
    dw, db = B.weight_gradient8(dz, p)
    rw, rb, ew, eb = product_bounds(to64(dz), OA.unpack(c64, s64, "e4m3"))
    close(dw, rw, ew, "dw")
    close(db, rb, eb, "db")
    if c_out == shape[1]:                              # ... from gradients that are far too
        again = B.weight_gradient8(room.place(dz), p)
        assert torch.equal(again[0], dw) and torch.equal(again[1], db)
    assert room.untouched() and codes.untouched() and scales.untouched()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n,stride", [(67, (1 << 24) - 1), (67, 1 << 24), (3, (1 << 31) + 9)], ids=str)
@pytest.mark.parametrize("c", [5, 48, 200])
def test_rows(c, n, stride, kind):
    """Several rows a wave: 32 bits span those of a wave up to 2^24 elements."""
    run((n, c), (stride, 1), (stride, 1), (stride, 1), kind, c)


@pytest.mark.parametrize("c", [5, 48, 200])
def test_many_rows(c):
    """More rows than one launch takes the parameters' sums of: the copies of other lanes' shares."""
    if c < 8:                                          # (2048 near rows are one workgroup's; far codes alone make all rows far)
        run((2100, c), (200, 1), (1 << 24, 1), (64, 1), "bf16", c)
    else:
        run((530, c), (1 << 24, 1), (1 << 24, 1), (64, 1), "bf16", c)


@pytest.mark.parametrize("only", ["codes", "scales", "tensors"])
@pytest.mark.parametrize("shape", [(20, 48), (3, 11, 70)], ids=str)
def test_one_kind_of_operand_far(shape, only):
    near = (1000, 1) if len(shape) == 2 else (40000, 1000, 1)
    far = (1 << 25, 1) if len(shape) == 2 else ((1 << 31) + 700, 1 << 27, 1)
    run(shape, *(far if only == what else near for what in ("tensors", "codes", "scales")), "bf16")


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("strides", [((1 << 31) + 8, 700, 1), (1 << 31, ((1 << 29) - 1) // 19, 1), (1 << 31, (1 << 29) // 19 + 1, 1), (700, 1 << 26, 1)], ids=str)
def test_maps(strides, kind):
    """Images far apart; maps just within what 32 bits of bytes span and just beyond; the maps of all images side by side, far from the next."""
    run((3, 11, 70), strides, strides, strides, kind, 11)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("positions", [(701,), (3, 230), (150,)], ids=str)
def test_large_tiles_added_to(positions, kind):
    """accumulate where the tiles are the largest, with and without copies."""
    from paper_1509_03371_amd import binding as B
    c, c_out = (2050, 2101) if positions != (150,) else (3000, 2900)
    shape = lambda n: positions[:1] + (n,) + positions[1:]  # noqa: E731
    gen = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(shape(c), generator=gen, device="cuda").to(TYPES[kind])
    dy = (0.01 * torch.randn(shape(c_out), generator=gen, device="cuda")).to(TYPES[kind])
    p = B.pack8(x, "i8", axis=1)
    dw, db = B.weight_gradient8(dy, p)
    rw, rb, ew, eb = product_bounds(to64(dy), to64(B.unpack8(p)))
    close(dw, rw, ew, "dw")
    close(db, rb, eb, "db")
    w0, b0 = torch.randn(dw.shape, generator=gen, device="cuda"), torch.randn(db.shape, generator=gen, device="cuda")
    w1, b1 = B.weight_gradient8(dy, p, accumulate=True, dw=w0.clone(), db=b0.clone())
    assert torch.equal(w1, w0 + dw) and torch.equal(b1, b0 + db)
