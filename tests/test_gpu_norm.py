"""GPU: dropout and layer norm on the caller's tensors, against the 64-bit oracle (bounds: norm_bounds.py)."""
import numpy as np
import pytest
import torch

from norm_bounds import TYPES, U, bwd_bounds, close, inputs, norm_bounds, place, rounded, to64
from oracle import norm as ON

pytestmark = pytest.mark.gpu

ROWS = [(1, 1), (3, 2), (5, 7), (1, 8), (300, 9), (2, 48), (64, 63), (65, 64), (1000, 33), (37, 200), (16, 1024), (9, 777), (4, 1025), (33, 2048), (5, 4099), (3, 9000),
        (2, 20011), (1, 40000)]
MAPS = [(1, 1, 1), (2, 1, 77), (1, 3, 5), (3, 8, 1), (2, 9, 64), (1, 48, 1001), (2, 65, 333), (1, 200, 400), (4, 16, 31), (1, 1024, 49), (2, 777, 10), (1, 2049, 33),
        (1, 5000, 3), (1, 64, 5000)]


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shape", ROWS + MAPS, ids=str)
def test_dropout(shape, kind):
    from paper_1509_03371_amd import binding as B
    for i, (p, pad) in enumerate([(0.5, 0), (0.1, 3), (0.9, 8)]):
        x = place(inputs(shape, kind, 10 + i)[0], kind, pad)
        seed, offset = 0x9E3779B97F4A7C15 + i, (i << 33) + 5
        got = B.dropout(x, p, seed, offset, axis=1)
        ref = ON.dropout(to64(x), p, seed, offset)
        assert np.array_equal(to64(got) == 0, ref == 0), "another mask"
        close(got, ref, rounded(ref, kind, 2 * U * np.abs(ref)), "y")
        grad = B.dropout(got, p, seed, offset, axis=1)          # the mask once more
        assert np.array_equal(to64(grad) == 0, to64(got) == 0)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shape", ROWS + MAPS, ids=str)
def test_layer_norm_and_gradient(shape, kind):
    from paper_1509_03371_amd import binding as B
    for i, (pad, order) in enumerate([(0, "dense"), (5, "dense"), (0, "last")]):
        x, _, gamma, beta, dy, _ = inputs(shape, kind, 20 + i)
        x, dy = place(x, kind, pad, order), place(dy, kind, pad, order)
        gd, bd = (None, None) if i == 1 else (torch.from_numpy(gamma).cuda(), torch.from_numpy(beta).cuda())
        gr, br = (None, None) if i == 1 else (gamma, beta)
        y, s, mean, rstd = B.layer_norm(x, gd, bd, axis=1)
        assert s is x
        ry, rm, rr, by, bm, brs = norm_bounds(to64(x), 0.0, gr, br, 1e-5, kind)
        close(y, ry, by, "y")
        close(mean, rm, bm, "mean")
        close(rstd, rr, brs, "rstd")
        dx, dres, dg, db = B.layer_norm_backward(dy, x, mean, rstd, gd, axis=1)
        assert dres is dx
        t, rg, rb, et, eg, eb = bwd_bounds(to64(dy), to64(x), to64(mean), to64(rstd), gr, None, kind)
        close(dx, t, rounded(t, kind, et), "dx")
        close(dg, rg, eg, "dgamma")
        close(db, rb, eb, "dbeta")


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shape", ROWS + MAPS, ids=str)
def test_dropout_residual_norm_and_gradient(shape, kind):
    from paper_1509_03371_amd import binding as B
    for i, (p, pad) in enumerate([(0.1, 0), (0.6, 7), (0.0, 0)]):
        x, r, gamma, beta, dy, dsum = inputs(shape, kind, 30 + i)
        x, r, dy, dsum = (place(a, kind, q) for a, q in ((x, pad), (r, 0), (dy, 0), (dsum, pad)))
        gd, bd = torch.from_numpy(gamma).cuda(), torch.from_numpy(beta).cuda()
        seed, offset = 77 + (i << 40), 3 + i
        y, s, mean, rstd = B.layer_norm(x, gd, bd, 1e-3, axis=1, residual=r, p=p, seed=seed, offset=offset)
        dropped = ON.dropout(to64(x), p, seed, offset)
        rs = to64(r) + dropped
        es = U * (2 * np.abs(dropped) + np.abs(rs)) * (1 + 4 * U)
        close(s, rs, rounded(rs, kind, es), "s")
        ry, rm, rr, by, bm, brs = norm_bounds(rs, es, gamma, beta, 1e-3, kind)
        close(y, ry, by, "y")
        close(mean, rm, bm, "mean")
        close(rstd, rr, brs, "rstd")
        dx, dres, dg, db = B.layer_norm_backward(dy, s, mean, rstd, gd, axis=1, dsum=dsum, p=p, seed=seed, offset=offset)
        t, rg, rb, et, eg, eb = bwd_bounds(to64(dy), to64(s), to64(mean), to64(rstd), gamma, to64(dsum), kind)
        close(dres, t, rounded(t, kind, et), "dresidual")
        rdx = ON.dropout(t, p, seed, offset)
        scale = 65536.0 / (65536 - ON.threshold(p))
        close(dx, rdx, (rdx != 0) * rounded(rdx, kind, et * scale + 2 * U * np.abs(rdx)), "dx")
        close(dg, rg, eg, "dgamma")
        close(db, rb, eb, "dbeta")
        # without what is optional: the same numbers
        only_dx, none, _, _ = B.layer_norm_backward(dy, s, mean, rstd, gd, axis=1, dsum=dsum, p=p, seed=seed, offset=offset, residual=False, parameters=False)
        assert torch.equal(only_dx, dx) and (none is None) == (p > 0)
        again = B.layer_norm_backward(dy, s, mean, rstd, gd, axis=1, dsum=dsum, p=p, seed=seed, offset=offset)
        assert all(torch.equal(a, b) for a, b in zip(again, (dx, dres, dg, db))), "two equal calls"


def test_mask_does_not_depend_on_type_order_or_strides():
    from paper_1509_03371_amd import binding as B
    ones = np.ones((2, 45, 77))
    masks = [to64(B.dropout(place(ones, kind, pad, order), 0.3, 99, 4, axis=1)) != 0
             for kind, pad, order in (("f32", 0, "dense"), ("bf16", 3, "dense"), ("f16", 0, "last"), ("f32", 1, "dense"), ("bf16", 0, "last"))]
    assert all(np.array_equal(m, masks[0]) for m in masks)
    rows = to64(B.dropout(torch.ones(154, 45, device="cuda"), 0.3, 99, 4)) != 0
    assert np.array_equal(rows.reshape(2, 77, 45).transpose(0, 2, 1), masks[0])


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("order", ["dense", "last"])
def test_rates_at_the_ends_and_values_that_are_not_numbers(kind, order):
    from paper_1509_03371_amd import binding as B
    x = place(inputs((2, 19, 70), kind, 1)[0], kind, 0, order)
    x[0, 3, 5], x[1, 7, 8], x[1, 18, 69] = float("inf"), float("nan"), float("-inf")
    assert torch.equal(B.dropout(x, 0.0, 1, axis=1).nan_to_num(), x.nan_to_num())
    assert torch.equal(B.dropout(x, 1e-9, 1, axis=1).nan_to_num(), x.nan_to_num())
    assert (B.dropout(x, 1.0, 1, axis=1) == 0).all()
    for seed in range(6):
        y = to64(B.dropout(x, 0.5, seed, axis=1))
        ref = ON.dropout(to64(x), 0.5, seed, 0)
        assert np.array_equal(y, ref, equal_nan=True)
    y, _, mean, rstd = B.layer_norm(x, axis=1)
    ry, rm, rr, by, _, _ = norm_bounds(np.nan_to_num(to64(x), nan=0, posinf=0, neginf=0), 0.0, None, None, 1e-5, kind)
    hit = np.zeros((2, 70), bool)
    hit[0, 5] = hit[1, 8] = hit[1, 69] = True
    assert np.isnan(to64(y).transpose(0, 2, 1)[hit]).all()
    close(np.where(hit[:, None], 0, to64(y)), np.where(hit[:, None], 0, ry), by, "positions beside them")
    # everything dropped and no residual: what is normalised is zero
    beta = torch.linspace(-1, 1, 19, device="cuda")
    y, s, mean, rstd = B.layer_norm(x, None, beta, axis=1, p=1.0, seed=3)
    assert (s == 0).all() and (mean == 0).all() and torch.equal(y, beta.to(y.dtype)[None, :, None].expand(2, 19, 70))
    dx, dres, dg, _ = B.layer_norm_backward(y, s, mean, rstd, None, axis=1, p=1.0, seed=3)
    assert (dx == 0).all() and (dg == 0).all() and torch.isfinite(dres).all()


@pytest.mark.parametrize("shape", [(50, 1000), (6, 20000), (1, 64, 900), (2, 3000, 7)], ids=str)
def test_far_means_and_equal_channels(shape):
    # a mean of 1000 deviations: sums of squares around zero would lose half the digits
    from paper_1509_03371_amd import binding as B
    x = place(1000.0 + np.random.default_rng(3).normal(size=shape), "f32")
    x[0] = 7.25
    y, _, mean, rstd = B.layer_norm(x, axis=1)
    ry, rm, rr, by, bm, brs = norm_bounds(to64(x), 0.0, None, None, 1e-5, "f32")
    close(y, ry, by, "y")
    close(rstd[1:], rr[1:], brs[1:], "rstd")
    close(mean, rm, bm, "mean")


@pytest.mark.parametrize("shape", [(40, 300), (7, 12000), (5, 20003), (2, 48, 130), (1, 3001, 9), (1, 20, 257), (2, 9, 1026), (1, 700, 33), (3, 64, 515)], ids=str)
def test_in_place(shape):
    from paper_1509_03371_amd import binding as B
    x, r, gamma, beta, dy, dsum = (torch.from_numpy(np.float32(a)).cuda() for a in inputs(shape, "f32", 9))
    kw = dict(axis=1, p=0.3, seed=5, offset=6)
    want = B.dropout(x, 0.3, 5, 6, axis=1)
    t = x.clone()
    assert B.dropout(t, 0.3, 5, 6, axis=1, out=t) is t and torch.equal(t, want)
    want = B.layer_norm(x, gamma, beta, residual=r, **kw)
    for target in ("x", "r"):
        a, b = x.clone(), r.clone()
        y = torch.empty_like(x)
        got = B.layer_norm(a, gamma, beta, residual=b, sum_out=a if target == "x" else b, out=y, **kw)
        assert all(torch.equal(u, v) for u, v in zip(got, want)), target
        a, b = x.clone(), r.clone()
        got = B.layer_norm(a, gamma, beta, residual=b, sum_out=b if target == "x" else a, out=a if target == "x" else b, **kw)
        assert all(torch.equal(u, v) for u, v in zip(got, want)), target
    _, s, mean, rstd = want
    want = B.layer_norm_backward(dy, s, mean, rstd, gamma, dsum=dsum, **kw)
    a, b, c = dy.clone(), s.clone(), dsum.clone()
    got = B.layer_norm_backward(a, b, mean, rstd, gamma, dsum=c, dx=a, dresidual=c, **kw)
    assert all(torch.equal(u, v) for u, v in zip(got, want))
    a, b, c = dy.clone(), s.clone(), dsum.clone()
    got = B.layer_norm_backward(a, b, mean, rstd, gamma, dsum=c, dx=c, dresidual=b, **kw)
    assert all(torch.equal(u, v) for u, v in zip(got, want))


def test_only_its_own_elements_are_written():
    from paper_1509_03371_amd import binding as B
    for shape in ((5, 33), (3, 1031), (2, 9, 41), (1, 130, 65)):
        for kind in ("f32", "bf16"):
            x = place(inputs(shape, kind, 2)[0], kind)
            wide = torch.full(shape[:-1] + (shape[-1] + 11,), 5.0, dtype=x.dtype, device="cuda")
            wide2 = wide.clone()
            inner, inner2 = wide[..., 6:6 + shape[-1]], wide2[..., 3:3 + shape[-1]]
            y, s, _, _ = B.layer_norm(x, axis=1, p=0.2, seed=1, out=inner, sum_out=inner2)
            for w, at in ((wide, 6), (wide2, 3)):
                assert (w[..., :at] == 5).all() and (w[..., at + shape[-1]:] == 5).all()
            want = B.layer_norm(x, axis=1, p=0.2, seed=1)
            assert torch.equal(y, want[0]) and torch.equal(s, want[1])
            wide.fill_(5.0)
            B.dropout(x, 0.2, 1, axis=1, out=inner)
            assert (wide[..., :6] == 5).all() and (wide[..., 6 + shape[-1]:] == 5).all() and torch.equal(inner, B.dropout(x, 0.2, 1, axis=1))


def test_other_orders_and_refusals_of_the_binding():
    from paper_1509_03371_amd import binding as B
    x = torch.randn(6, 100, device="cuda")
    want = B.layer_norm(x)[0]
    assert torch.equal(B.layer_norm(x, axis=1)[0], want)
    y = B.layer_norm(x.t().contiguous().t())[0]                     # positions side by side
    assert torch.allclose(y, want, atol=1e-5)
    assert torch.allclose(B.layer_norm(x.t(), axis=0)[0].t(), want, atol=1e-5)
    vec = B.layer_norm(x[0])
    assert torch.equal(vec[0], want[0]) and vec[2].shape == ()
    ones = torch.ones(1, device="cuda").expand(6, 100)              # a broadcast gradient
    _, s, mean, rstd = B.layer_norm(x)
    got = B.layer_norm_backward(ones, s, mean, rstd, dx=torch.empty_like(x))
    full = B.layer_norm_backward(ones.contiguous(), s, mean, rstd)
    assert all(torch.allclose(a, b, atol=1e-5) for a, b in zip(got, full))
    empty = torch.empty(0, 100, device="cuda")
    out = B.layer_norm_backward(empty, empty, torch.empty(0, device="cuda"), torch.empty(0, device="cuda"))
    assert out[0].shape == (0, 100) and (out[2] == 0).all() and (out[3] == 0).all()
    assert B.dropout(empty, 0.5, 1).shape == (0, 100) and B.layer_norm(empty)[0].shape == (0, 100)
    for bad in (lambda: B.layer_norm(x, torch.ones(99, device="cuda")), lambda: B.layer_norm(x, residual=x[:5]), lambda: B.layer_norm(x, axis=2),
                lambda: B.layer_norm(torch.randn(4, 5, 6, device="cuda").permute(2, 1, 0)[:, ::2], axis=2), lambda: B.dropout(x, 0.5, -1),
                lambda: B.layer_norm_backward(x, s, mean, rstd, dresidual=torch.empty_like(x)),
                lambda: B.layer_norm_backward(x, s, mean[:5], rstd)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: B.layer_norm(x.double()), lambda: B.layer_norm(x, torch.ones(100)), lambda: B.layer_norm(x, residual=x.bfloat16()),
                lambda: B.dropout(x, 0.5, 1, step=torch.zeros(1, device="cuda"))):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: B.dropout(x, 1.5, 1), lambda: B.layer_norm(x, eps=0.0), lambda: B.dropout(x[:, 1:], 0.5, 1, out=x[:, :-1]),
                lambda: B.dropout(x, 0.5, 1, out=x[0].expand(6, 100))):
        with pytest.raises(B.SknetError):
            bad()


def test_on_another_stream():
    from paper_1509_03371_amd import binding as B
    x = torch.randn(3000, 1024, device="cuda")
    dy = torch.randn_like(x)
    want = B.layer_norm(x, p=0.1, seed=3)
    back = B.layer_norm_backward(dy, *want[1:], p=0.1, seed=3)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for stream in (s, s.cuda_stream):
        got = B.layer_norm(x, p=0.1, seed=3, stream=stream)
        grads = B.layer_norm_backward(dy, *got[1:], p=0.1, seed=3, stream=stream)
        s.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and all(torch.equal(a, b) for a, b in zip(grads, back))


def test_recorded_passes_and_the_step_counter():
    # forward and backward as one program uses them, recorded twice (two graphs whose scratch must not meet), replayed with a
    # counter that the program advances
    from paper_1509_03371_amd import binding as B
    dev = torch.device("cuda")
    x, r, dy = (torch.randn(1500, 520, device=dev).bfloat16() for _ in range(3))
    maps, dmaps = (torch.randn(2, 70, 999, device=dev) for _ in range(2))
    gamma, beta = torch.rand(520, device=dev) + 0.5, torch.randn(520, device=dev)
    step = torch.zeros((), dtype=torch.int64, device=dev)

    def one(at=None, offset=0):
        y, s, mean, rstd = B.layer_norm(x, gamma, beta, residual=r, p=0.25, seed=11, offset=offset, step=at)
        grads = B.layer_norm_backward(dy, s, mean, rstd, gamma, dsum=y, p=0.25, seed=11, offset=offset, step=at)
        return (y, s, mean, rstd) + grads

    def two(at=None, offset=0):
        d = B.dropout(maps, 0.5, 12, offset, axis=1, step=at)
        y, s, mean, rstd = B.layer_norm(d, axis=1)
        dx, _, dg, db = B.layer_norm_backward(dmaps, s, mean, rstd, axis=1)
        return d, y, dg, db, B.dropout(dx, 0.5, 12, offset, axis=1, step=at)

    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        one(step), two(step)
        g1, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(g1, stream=stream):
            out1 = one(step)
        with torch.cuda.graph(g2, stream=stream):
            out2 = two(step)
        for rep in range(4):
            step.fill_(1000 + 7 * rep)
            x.copy_(torch.randn_like(x))
            maps.copy_(torch.randn_like(maps))
            want1, want2 = one(None, 1000 + 7 * rep), two(None, 1000 + 7 * rep)
            for t in out1 + out2:
                t.zero_()
            g1.replay()
            g2.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out1 + out2, want1 + want2)), rep


def test_a_block_of_a_network_by_differences():
    # loss = <w, norm(r + dropout(x)) > + <v, s>: the gradients that the calls return against differences of the 64-bit oracle along
    # random directions (central differences of step 1e-4: error of second order, 1e-6 relative at these curvatures)
    from paper_1509_03371_amd import binding as B
    rng = np.random.default_rng(8)
    for shape in ((12, 96), (2, 40, 15)):
        x, r, gamma, beta, w, v = inputs(shape, "f32", 8)
        x, r, w, v = (np.float32(a).astype(np.float64) for a in (x, r, 100 * w, 100 * v))
        dev = [torch.from_numpy(np.float32(a)).cuda() for a in (x, r, gamma, beta, w, v)]
        kw = dict(p=0.2, seed=4, offset=1)
        y, s, mean, rstd = B.layer_norm(dev[0], dev[2], dev[3], axis=1, residual=dev[1], **kw)
        dx, dr, dg, db = B.layer_norm_backward(dev[4], s, mean, rstd, dev[2], axis=1, dsum=dev[5], **kw)

        def loss(x, r, gamma, beta):
            s = r + ON.dropout(x, 0.2, 4, 1)
            return (w * ON.layer_norm(s, gamma, beta)[0]).sum() + (v * s).sum()

        point = [x, r, np.float64(gamma), np.float64(beta)]
        for i, grad in enumerate((dx, dr, dg, db)):
            d = rng.normal(size=point[i].shape)
            lo, hi = list(point), list(point)
            lo[i], hi[i] = point[i] - 1e-4 * d, point[i] + 1e-4 * d
            slope = (loss(*hi) - loss(*lo)) / 2e-4
            mine = (to64(grad) * d).sum()
            assert abs(slope - mine) <= 1e-4 * np.sqrt((to64(grad) ** 2).sum() * (d ** 2).sum()), (shape, i)


@pytest.mark.parametrize("shape,stride", [((70, 40), 1 << 24), ((70, 5), 1 << 24), ((67, 1), 1 << 24), ((65, 8), 1 << 24), ((3, 600), 1 << 31), ((2, 30, 9), 1 << 27), ((1, 9, 70), 1 << 29), ((1, 5, 2), 1 << 29)], ids=str)
def test_strides_that_32_bits_do_not_span(shape, stride):
    from paper_1509_03371_amd import binding as B
    size = stride * (shape[0] if len(shape) == 2 else shape[0] * shape[1])
    store = torch.empty(size, dtype=torch.bfloat16, device="cuda")

    def far(t, shift):
        strides = (stride, 1) if t.dim() == 2 else (stride * t.shape[1], stride, 1)
        v = store.as_strided(t.shape, strides, shift)
        v.copy_(t)
        return v

    x, r, gamma, beta, dy, dsum = inputs(shape, "bf16", 77)
    x, r, dy, dsum = (place(a, "bf16") for a in (x, r, dy, dsum))
    gd, bd = torch.from_numpy(gamma).cuda(), torch.from_numpy(beta).cuda()
    kw = dict(axis=1, p=0.2, seed=3, offset=8)
    want = B.layer_norm(x, gd, bd, residual=r, **kw)
    back = B.layer_norm_backward(dy, want[1], want[2], want[3], gd, dsum=dsum, **kw)
    fx, fr = far(x, 0), far(r, 4096)
    y, s = far(torch.zeros_like(x), 8192), far(torch.zeros_like(x), 12288)
    got = B.layer_norm(fx, gd, bd, residual=fr, out=y, sum_out=s, **kw)
    for g, w, in zip(got, want):        # sums in another order: to rounding
        close(g, to64(w), 2.0 ** -7 * np.abs(to64(w)) + 1e-3, "forward")
    assert np.array_equal(to64(got[1]), to64(want[1]))
    fdy, fds = far(dy, 16384), far(dsum, 20480)
    dx, dr = far(torch.zeros_like(x), 24576), far(torch.zeros_like(x), 28672)
    grads = B.layer_norm_backward(fdy, s, got[2], got[3], gd, dsum=fds, dx=dx, dresidual=dr, **kw)
    for g, w in zip(grads, back):
        close(g, to64(w), 2.0 ** -6 * np.abs(to64(w)) + 1e-3, "backward")
    out = far(torch.zeros_like(x), 32768)
    assert np.array_equal(to64(B.dropout(fx, 0.4, 9, axis=1, out=out)), to64(B.dropout(x, 0.4, 9, axis=1)))


@pytest.mark.parametrize("shape", [((1 << 21) + 3, 1100), (2, 9, (1 << 27) + 5), (3, 17, (1 << 26) + 1)], ids=str)
def test_tensors_of_more_than_32_bits_of_elements(shape):
    from paper_1509_03371_amd import binding as B
    x = torch.zeros(shape, dtype=torch.bfloat16, device="cuda")
    last = 300
    tail = x[-last:] if len(shape) == 2 else x[-1:, :, -last:]
    tail.copy_(torch.randn(tail.shape, device="cuda"))
    c = shape[1]
    positions = np.arange(x.numel() // c - last, x.numel() // c, dtype=np.uint64)
    keep = ON.keep_mask(positions, c, 0.25, 5, 6)
    part = to64(tail) if len(shape) == 2 else to64(tail)[0].T
    y = B.dropout(x, 0.25, 5, 6, axis=1)
    got = to64(y[-last:]) if len(shape) == 2 else to64(y[-1, :, -last:]).T
    ref = np.where(keep, part * (65536.0 / (65536 - ON.threshold(0.25))), 0.0)
    close(got, ref, rounded(ref, "bf16", 2 * U * np.abs(ref)), "dropout")
    out, s, mean, rstd = B.layer_norm(x, axis=1, p=0.25, seed=5, offset=6, out=y)
    got = to64(out[-last:]) if len(shape) == 2 else to64(out[-1, :, -last:]).T
    ry, rm, rr, by, bm, brs = norm_bounds(ref, 2 * U * np.abs(ref), None, None, 1e-5, "bf16")
    close(got, ry, by, "y")
    close(to64(mean).reshape(-1)[-last:], rm, bm, "mean")
    assert (out[:5] == 0).all() if len(shape) == 2 else (out[0, :, :1000] == 0).all()
    dx, _, dg, db = B.layer_norm_backward(x, s, mean, rstd, axis=1, dx=out)
    t, rg, rb, et, eg, eb = bwd_bounds(part, to64(s[-last:]) if len(shape) == 2 else to64(s[-1, :, -last:]).T, to64(mean).reshape(-1)[-last:],
                                       to64(rstd).reshape(-1)[-last:], None, None, "bf16")
    got = to64(dx[-last:]) if len(shape) == 2 else to64(dx[-1, :, -last:]).T
    close(got, t, rounded(t, "bf16", et), "dx")
    # (zeros elsewhere add nothing to the sums, and no rounding)
    close(dg, rg, eg, "dgamma")
    close(db, rb, eb, "dbeta")


@pytest.mark.parametrize("shape", [(5000, 20, 2), (700, 3, 3), (6, 2100, 3), (2, 2100, 70), (1, 40000, 5)], ids=str)
def test_small_planes_and_many_channels(shape):
    from paper_1509_03371_amd import binding as B
    x, r, gamma, beta, dy, dsum = inputs(shape, "f32", 5)
    x, r, dy, dsum = (place(a, "f32") for a in (x, r, dy, dsum))
    gd, bd = torch.from_numpy(gamma).cuda(), torch.from_numpy(beta).cuda()
    kw = dict(axis=1, p=0.3, seed=2, offset=1)
    y, s, mean, rstd = B.layer_norm(x, gd, bd, residual=r, **kw)
    dropped = ON.dropout(to64(x), 0.3, 2, 1)
    rs = to64(r) + dropped
    es = U * (2 * np.abs(dropped) + np.abs(rs)) * (1 + 4 * U)
    ry, rm, rr, by, bm, brs = norm_bounds(rs, es, gamma, beta, 1e-5, "f32")
    close(y, ry, by, "y")
    close(rstd, rr, brs, "rstd")
    dx, dres, dg, db = B.layer_norm_backward(dy, s, mean, rstd, gd, dsum=dsum, **kw)
    t, rg, rb, et, eg, eb = bwd_bounds(to64(dy), to64(s), to64(mean), to64(rstd), gamma, to64(dsum), "f32")
    close(dres, t, rounded(t, "f32", et), "dresidual")
    close(dg, rg, eg, "dgamma")
    close(db, rb, eb, "dbeta")


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shape", [(3000, 1), (40, 1), (1, 1, 900), (3, 1, 5), (2, 1, 70000)], ids=str)
def test_one_channel_has_no_gradient(shape, kind):
    # (s - mean) and (gamma dy - its mean) are zero, not nearly
    from paper_1509_03371_amd import binding as B
    x, _, _, beta, dy, dsum = inputs(shape, kind, 3)
    x, dy, dsum = (place(a, kind) for a in (x, dy, dsum))
    gamma = torch.full((1,), 1.2345678, device="cuda")
    y, s, mean, rstd = B.layer_norm(x, gamma, torch.from_numpy(beta).cuda(), axis=1)
    assert torch.equal(y, torch.from_numpy(beta).cuda().to(y.dtype).expand(y.numel()).reshape(shape))
    dx, _, dg, db = B.layer_norm_backward(dy, x, mean, rstd, gamma, axis=1)
    assert (dx == 0).all() and (dg == 0).all() and (db != 0).all()
    dx, dr, _, _ = B.layer_norm_backward(dy, x, mean, rstd, gamma, axis=1, dsum=dsum, p=0.5, seed=1)
    assert torch.equal(dr, dsum) and torch.equal(dx, B.dropout(dsum, 0.5, 1, axis=1))
