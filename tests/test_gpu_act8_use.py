"""GPU: root-mean-square norm, tensors in 8 bits and the weight gradient as a training step uses them together: on other streams, captured and replayed, over strides and
lengths that 32 bits do not span."""
import numpy as np
import pytest
import torch

from act8_bounds import bwd_bounds, close, held, norm_bounds, product_bounds, rounded, to64
from norm_bounds import TYPES, inputs, place
from oracle import act8 as OA

pytestmark = pytest.mark.gpu


class Step:
    """residual + norm, whose result in 8 bits an inner product reads; backwards from the held tensors alone."""

    def __init__(self, shape, c_out, kind, seed):
        from paper_1509_03371_amd import binding as B
        x, r, gamma, _, dy, _ = inputs(shape, kind, seed, 0.3)
        rng = np.random.default_rng(seed)
        self.x, self.r, self.dy = (place(t, kind) for t in (x, r, dy))
        self.dz = place(0.01 * rng.normal(size=shape[:1] + (c_out,) + shape[2:]), kind)
        self.gamma = torch.from_numpy(gamma).cuda()
        self.y8, self.sum8 = B.Packed.like(self.x, "e4m3", axis=1), B.Packed.like(self.x, "i8", axis=1)

    def run(self, stream=None):
        from paper_1509_03371_amd import binding as B
        _, s, rstd = B.rms_norm(self.x, self.gamma, axis=1, residual=self.r, out=False, y8=self.y8, sum8=self.sum8, stream=stream)
        dw, db = B.weight_gradient8(self.dz, self.y8, stream=stream)
        dx, dgamma = B.rms_norm_backward(self.dy, self.sum8, rstd, self.gamma, axis=1, dsum=self.x, stream=stream)
        return [s, rstd, dw, db, dx, dgamma, B.unpack8(self.y8, stream=stream), B.unpack8(self.sum8, stream=stream)]


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shape", [(700, 200), (2, 72, 1001)], ids=str)
def test_together(shape, kind):
    step = Step(shape, 50, kind, 1)
    s, rstd, dw, db, dx, dgamma, y8, s8 = step.run()
    rs = to64(step.x) + to64(step.r)
    es = 2.0 ** -24 * np.abs(rs)
    gamma = step.gamma.cpu().numpy()
    close(s, rs, rounded(rs, kind, es), "s")
    ry, rr, ey, er = norm_bounds(rs, es, gamma, 1e-5)
    close(rstd, rr, er, "rstd")
    held(step.y8.codes, step.y8.scales, "e4m3", kind, ry, ey, "y8")
    held(step.sum8.codes, step.sum8.scales, "i8", kind, rs, es, "sum8")
    rw, rb, ew, eb = product_bounds(to64(step.dz), to64(y8))
    close(dw, rw, ew, "dw")
    close(db, rb, eb, "db")
    t, rg, et, eg = bwd_bounds(to64(step.dy), to64(s8), to64(rstd), gamma, to64(step.x))
    close(dx, t, rounded(t, kind, et), "dx")
    close(dgamma, rg, eg, "dgamma")


@pytest.mark.parametrize("shape", [(700, 200), (40, 96), (2, 72, 1001), (1, 20, 50)], ids=str)
def test_streams_and_graphs(shape):
    """Eager on the default stream, on another one, on one that is passed, and as a graph whose inputs change between replays."""
    steps = [Step(shape, 50, "bf16", k) for k in range(3)]
    want = [[t.clone() for t in s.run()] for s in steps]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = steps[1].run()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want[1]))
    got = steps[1].run(stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want[1]))
    one, two = Step(shape, 50, "bf16", 0), Step(shape, 50, "bf16", 2)
    graphs, outs = [], []
    for s in (one, two):                             # two graphs that live side by side
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(s.run())
        graphs.append(g)
    for k in (0, 1, 2, 1, 0):
        for name in ("x", "r", "dy", "dz", "gamma"):
            getattr(one, name).copy_(getattr(steps[k], name))
        graphs[0].replay()
        graphs[1].replay()
        eager = steps[k].run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs[0], want[k])), k
        assert all(torch.equal(a, b) for a, b in zip(outs[1], want[2]))
        assert all(torch.equal(a, b) for a, b in zip(eager, want[k]))


@pytest.mark.parametrize("layout", ["rows", "maps"])
def test_far_strides(layout):
    """Rows, or maps, further apart than 32 bits of bytes span: the results of the same tensors side by side."""
    from paper_1509_03371_amd import binding as B
    shape = (3, 700) if layout == "rows" else (1, 11, 70)
    far = ((1 << 31) + 8, 1) if layout == "rows" else (11 << 30, (1 << 30) + 4, 1)
    step = Step(shape, 20, "bf16", 5)
    want = step.run()
    room = (shape[0] - 1) * far[0] + sum((n - 1) * st for n, st in zip(shape[1:], far[1:])) + 1

    def move(t, fill=True):
        v = torch.empty(room, dtype=t.dtype, device="cuda").as_strided(shape, far)
        return v.copy_(t) if fill else v

    x, r, dy = move(step.x), move(step.r), move(step.dy)
    y8 = B.Packed(move(step.y8.codes, False), step.y8.scales.clone(), "e4m3", 1)
    sum8 = B.Packed(step.sum8.codes.clone(), step.sum8.scales.clone(), "i8", 1)
    s = move(step.x, False)
    _, _, rstd = B.rms_norm(x, step.gamma, axis=1, residual=r, out=False, sum_out=s, y8=y8, sum8=sum8)
    assert torch.equal(s, want[0]) and torch.allclose(rstd, want[1], rtol=1e-6, atol=0)
    assert torch.equal(B.unpack8(B.pack8(x, axis=1, out=y8), out=move(step.x, False)).float(), B.unpack8(B.pack8(step.x, axis=1)).float())
    B.rms_norm(x, step.gamma, axis=1, residual=r, out=False, sum_out=False, y8=y8)
    dw, db = B.weight_gradient8(step.dz, y8)
    rw, rb, ew, eb = product_bounds(to64(step.dz), OA.unpack(y8.codes.cpu().numpy(), y8.scales.cpu().numpy(), "e4m3"))
    close(dw, rw, ew, "dw")
    close(db, rb, eb, "db")
    dx, dgamma = B.rms_norm_backward(dy, sum8, rstd, step.gamma, axis=1, dsum=x, dx=s)
    t, rg, et, eg = bwd_bounds(to64(dy), to64(B.unpack8(sum8)), to64(rstd), step.gamma.cpu().numpy(), to64(x))
    close(dx, t, rounded(t, "bf16", et), "dx")
    close(dgamma, rg, eg, "dgamma")


def test_more_than_32_bits_of_elements():
    from paper_1509_03371_amd import binding as B
    n = (1 << 32) + 1000
    x = torch.zeros(1, 1, n, dtype=torch.bfloat16, device="cuda")
    start = (1 << 32) - 96
    part = torch.randn(n - start, device="cuda").to(torch.bfloat16)
    x[0, 0, start:] = part
    for code in OA.TOP:
        p = B.pack8(x, code, axis=1)
        codes, scales = OA.pack(to64(part), code, "bf16")
        assert np.array_equal(p.scales[0, 0, start // 32:].cpu().numpy(), scales) and not p.codes[0, 0, :start].any()
        back = B.unpack8(p)
        assert np.array_equal(to64(back[0, 0, start:]), OA.unpack(codes, scales, code)) and not back[0, 0, :start].any()


@pytest.mark.parametrize("kind", sorted(TYPES))
def test_many_small_planes(kind):
    """Images of a few pixels: more of them than workgroups."""
    from paper_1509_03371_amd import binding as B
    for shape in ((5000, 20, 3), (3000, 40, 4), (700, 100, 6)):
        x, _, gamma, _, dy, _ = inputs(shape, kind, 9, 0.3)
        x, dy, gd = place(x, kind), place(dy, kind), torch.from_numpy(gamma).cuda()
        y8 = B.Packed.like(x, "e4m3", axis=1)
        y, _, rstd = B.rms_norm(x, gd, axis=1, y8=y8)
        ry, rr, ey, er = norm_bounds(to64(x), 0.0, gamma, 1e-5)
        close(y, ry, rounded(ry, kind, ey), "y")
        close(rstd, rr, er, "rstd")
        held(y8.codes, y8.scales, "e4m3", kind, ry, ey, "y8")
        dx, dgamma = B.rms_norm_backward(dy, x, rstd, gd, axis=1)
        t, rg, et, eg = bwd_bounds(to64(dy), to64(x), to64(rstd), gamma, None)
        close(dx, t, rounded(t, kind, et), "dx")
        close(dgamma, rg, eg, "dgamma")


def test_inputs_without_strides_of_their_own():
    """Broadcast inputs: the same row, or pixel line, for all."""
    from paper_1509_03371_amd import binding as B
    for shape, narrow in (((300, 90), (1, 90)), ((3, 40, 77), (1, 40, 77))):
        step = Step(shape, 50, "bf16", 11)
        r = step.r[:1].clone()
        y, s, rstd = B.rms_norm(step.x, step.gamma, axis=1, residual=r.expand(shape))
        same = B.rms_norm(step.x, step.gamma, axis=1, residual=r.expand(shape).contiguous())
        assert r.shape == narrow and all(torch.equal(a, b) for a, b in zip((y, s, rstd), same))
        dy = step.dz[:1].clone()
        wide = (shape[0],) + tuple(dy.shape[1:])
        got, same = B.weight_gradient8(dy.expand(wide), B.pack8(step.x, axis=1)), B.weight_gradient8(dy.expand(wide).contiguous(), B.pack8(step.x, axis=1))
        assert torch.equal(got[0], same[0]) and torch.equal(got[1], same[1])
        assert torch.equal(B.unpack8(B.pack8(r.expand(shape), axis=1)), B.unpack8(B.pack8(r, axis=1)).expand(shape))


def test_graph_of_large_tiles():
    from paper_1509_03371_amd import binding as B
    x, dy = torch.randn(701, 2050, device="cuda").half(), 0.01 * torch.randn(701, 2101, device="cuda").half()
    p = B.pack8(x, "i8")
    want = [t.clone() for t in B.weight_gradient8(dy, p)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = B.weight_gradient8(dy, p)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        got[0].zero_()


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("more", [1, 2, 3])
def test_planes_that_end_behind_a_tiles_first_pixels(more, kind):
    """The last tile of a plane holds one to three pixels: its first lane reads from the tile in front of it."""
    from paper_1509_03371_amd import binding as B
    for c, tile in ((9, 256), (48, 128), (100, 64), (200, 32), (600, 32), (1100, 32)):
        shape = (2, c, 2 * tile + more)
        x, r, gamma, _, dy, _ = inputs(shape, kind, 13, 0.3)
        x, r, dy, gd = place(x, kind), place(r, kind), place(dy, kind), torch.from_numpy(gamma).cuda()
        sum8 = B.Packed.like(x, "i8", axis=1)
        y, s, rstd = B.rms_norm(x, gd, axis=1, residual=r, sum8=sum8)
        rs = to64(x) + to64(r)
        es = 2.0 ** -24 * np.abs(rs)
        ry, rr, ey, er = norm_bounds(rs, es, gamma, 1e-5)
        close(y, ry, rounded(ry, kind, ey), "y")
        close(rstd, rr, er, "rstd")
        held(sum8.codes, sum8.scales, "i8", kind, rs, es, "sum8")
        for source in (s, sum8):
            dx, dgamma = B.rms_norm_backward(dy, source, rstd, gd, axis=1, dsum=r)
            t, rg, et, eg = bwd_bounds(to64(dy), to64(s if source is s else B.unpack8(sum8)), to64(rstd), gamma, to64(r))
            close(dx, t, rounded(t, kind, et), "dx")
            close(dgamma, rg, eg, "dgamma")
