"""CPU: the oracle of dropout and layer norm against published vectors, differences and moments; the refusals of the operators'
C entry points (no call here gets as far as a launch); how the binding sees tensors as rows or maps."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import norm as ON
from paper_1509_03371_amd import binding as B


def test_generator_known_answers():
    # the vectors published with the generator: zeros, ones, and digits of pi
    def words(ctr, key):
        return [int(x) for x in ON.philox4x32(ctr, key)]
    assert words([0] * 4, (0, 0)) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert words([0xFFFFFFFF] * 4, (0xFFFFFFFF, 0xFFFFFFFF)) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert words([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], (0xA4093822, 0x299F31D0)) == [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.9, 1.0])
def test_oracle_mask_keeps_its_share(p):
    keep = ON.keep_mask(4000, 50, p, 0x123456789ABCDEF0, 7)
    n = keep.size
    assert abs(keep.mean() - (1 - p)) <= 5 * np.sqrt(p * (1 - p) / n) + 1e-4 * (0 < p < 1)
    if 0 < p < 1:              # neighbours agree as often as independent draws do
        for a, b in ((keep[:, 1:], keep[:, :-1]), (keep[1:], keep[:-1])):
            both = p * p + (1 - p) ** 2
            assert abs((a == b).mean() - both) <= 5 * np.sqrt(both * (1 - both) / a.size) + 1e-3
        assert not np.array_equal(keep, ON.keep_mask(4000, 50, p, 0x123456789ABCDEF1, 7))
        assert not np.array_equal(keep, ON.keep_mask(4000, 50, p, 0x123456789ABCDEF0, 8))


def test_oracle_mask_of_far_positions():
    far = np.array([5, (1 << 32) + 5, (3 << 32) + 5], dtype=np.uint64)
    m = ON.keep_mask(far, 200, 0.5, 1, 2)
    assert np.array_equal(m[0], ON.keep_mask(6, 200, 0.5, 1, 2)[5])
    assert not np.array_equal(m[0], m[1]) and not np.array_equal(m[1], m[2])


def test_oracle_gradient_by_differences():
    rng = np.random.default_rng(5)
    x, gamma, beta, dy = rng.normal(size=(2, 7, 3)), rng.normal(size=7), rng.normal(size=7), rng.normal(size=(2, 7, 3))
    _, mean, rstd = ON.layer_norm(x, gamma, beta)
    dx, dg, db = ON.layer_norm_bwd(dy, x, mean, rstd, gamma)
    step = 1e-6
    for grad, arr in ((dx, x), (dg, gamma), (db, beta)):
        for i in np.ndindex(arr.shape):
            old = arr[i]
            arr[i] = old + step
            up = (ON.layer_norm(x, gamma, beta)[0] * dy).sum()
            arr[i] = old - step
            down = (ON.layer_norm(x, gamma, beta)[0] * dy).sum()
            arr[i] = old
            assert abs((up - down) / (2 * step) - grad[i]) <= 1e-6 * (1 + abs(grad[i]))


# ---- refusals.  Addresses that nothing may follow: every call here ends before it launches.

def extent(layout=B.SK_ROWS, n=4, c=8, plane=1, dtype=B.SK_F32):
    return B.SkExtent(dtype, layout, n, c, plane)


def view(address=0x10000, stride_n=8, stride_c=0):
    return B.SkView(address, stride_n, stride_c)


def status(fn, *args):
    out = fn(*[C.byref(a) if isinstance(a, C.Structure) else a for a in args])
    assert out != 0, "accepted"
    return B.STATUS_NAMES[out]


X, Y, R, S = view(0x10000), view(0x20000), view(0x30000), view(0x40000)
DROP = B.SkDrop(0.5, 1, 2, None)


def test_dropout_refusals():
    def go(e=extent(), x=X, y=Y, drop=DROP):
        return status(B.lib.sknet_dropout, e, x, y, drop, None)
    assert go(e=None) == go(x=None) == go(y=None) == go(drop=None) == "SK_EINVAL"
    assert go(e=extent(dtype=3)) == go(e=extent(layout=2)) == "SK_EINVAL"
    assert go(e=extent(c=0)) == go(e=extent(n=-1)) == go(e=extent(plane=2)) == "SK_ESHAPE"
    assert go(e=extent(c=(1 << 27) + 1)) == go(e=extent(n=(1 << 40) + 1, c=1)) == go(e=extent(n=1 << 30, c=1 << 20)) == "SK_EUNSUPPORTED"
    assert go(x=view(0)) == go(y=view(0)) == go(x=view(0x10002)) == "SK_EINVAL"
    assert go(x=view(stride_n=-8)) == go(y=view(0x20000, 7)) == go(y=view(0x20000, 0)) == "SK_ESHAPE"
    assert go(x=view(stride_n=1 << 60)) == "SK_EUNSUPPORTED"
    for p in (-0.01, 1.01, float("nan"), float("inf")):
        assert go(drop=B.SkDrop(p, 1, 2, None)) == "SK_EINVAL"
    assert go(drop=B.SkDrop(0.5, 1, 2, 0x1004)) == "SK_EINVAL"
    # y on top of x, shifted or with other strides
    assert go(y=view(0x10000 + 16)) == go(y=view(0x10000, 9)) == go(x=view(stride_n=16), y=view(0x10000 + 28, 16)) == "SK_EINVAL"
    maps = extent(B.SK_MAPS, 2, 3, 10)
    assert status(B.lib.sknet_dropout, maps, view(0x10000, 30, 10), view(0x20000, 30, 9), DROP, None) == "SK_ESHAPE"
    assert status(B.lib.sknet_dropout, maps, view(0x10000, 30, 10), view(0x20000, 29, 10), DROP, None) == "SK_ESHAPE"
    assert status(B.lib.sknet_dropout, maps, view(0x10000, 60, 10), view(0x10000 + 4 * 29, 60, 10), DROP, None) == "SK_EINVAL"
    assert "rate" in B.lib.sknet_last_error().decode() or "overlaps" in B.lib.sknet_last_error().decode()


def test_layer_norm_refusals():
    def go(e=extent(), x=X, r=R, drop=DROP, eps=1e-5, s=S, y=Y):
        return status(B.lib.sknet_layer_norm, e, x, r, drop, None, None, eps, s, y, None, None, None)
    assert go(e=None) == go(x=None) == go(y=None) == "SK_EINVAL"
    for eps in (0.0, -1e-5, float("nan"), float("inf")):
        assert go(eps=eps) == "SK_EINVAL"
    assert go(r=view(0)) == go(s=view(0)) == go(drop=B.SkDrop(2.0, 1, 2, None)) == "SK_EINVAL"
    assert go(s=view(0x40000, 4)) == go(y=view(0x20000, 4)) == "SK_ESHAPE"
    assert go(y=S) == go(y=view(0x40000 + 8)) == go(s=view(0x30000 + 4)) == go(y=view(0x30000, 12)) == "SK_EINVAL"


def test_layer_norm_backward_refusals():
    good = dict(e=extent(), dy=X, s=S, mean=0x50000, rstd=0x60000, gamma=None, dsum=None, drop=None, dx=Y, dr=None, dg=0x70000, db=0x80000, ws=None, n=0)

    def go(**kw):
        a = dict(good, **kw)
        return status(B.lib.sknet_layer_norm_backward, a["e"], a["dy"], a["s"], a["mean"], a["rstd"], a["gamma"], a["dsum"], a["drop"], a["dx"], a["dr"],
                      a["dg"], a["db"], a["ws"], a["n"], None)
    assert go(e=None) == go(dy=None) == go(s=None) == go(mean=None) == go(rstd=None) == "SK_EINVAL"
    assert go(dx=view(0x20000, 7)) == go(dr=view(0x90000, 0)) == "SK_ESHAPE"
    assert go(dr=Y) == go(dx=view(0x40000 + 4)) == go(dx=view(0x10000 + 4)) == go(dsum=view(0)) == go(dsum=view(0x20000 + 4)) == "SK_EINVAL"
    assert go(drop=B.SkDrop(-1.0, 0, 0, None)) == go(ws=0x10008, n=1 << 30) == "SK_EINVAL"
    need = C.c_uint64()
    big = extent(n=100000, c=64)
    assert B.lib.sknet_layer_norm_workspace(C.byref(big), C.byref(need)) == 0
    assert need.value
    if need.value:
        assert go(e=big, dy=view(0x10000000, 64), s=view(0x20000000, 64), dx=view(0x30000000, 64), ws=0x40000000, n=need.value - 1) == "SK_EINVAL"
    assert status(B.lib.sknet_layer_norm_workspace, extent(c=0), C.byref(need)) == "SK_ESHAPE"
    assert status(B.lib.sknet_layer_norm_workspace, extent(), None) == "SK_EINVAL"


def test_values_that_are_written_lie_apart():
    def forward(gamma=0x50000, beta=0x60000, mean=0x70000, rstd=0x80000):
        return status(B.lib.sknet_layer_norm, extent(), X, None, None, gamma, beta, 1e-5, None, Y, mean, rstd, None)

    def backward(e=extent(), far=1, mean=0x50000, rstd=0x60000, gamma=0x70000, dgamma=0x80000, dbeta=0x90000, ws=None, n=0):
        dy, s, dx = (view(a * far, e.c) for a in (0x10000, 0x20000, 0x30000))
        return status(B.lib.sknet_layer_norm_backward, e, dy, s, mean, rstd, gamma, None, None, dx, None, dgamma, dbeta, ws, n, None)
    # 4 means and 8 gammas: 16 and 32 bytes
    assert forward(mean=0x80000) == forward(rstd=0x70000 + 12) == forward(mean=0x50000 + 28) == forward(rstd=0x60000 - 12) == "SK_EINVAL"
    assert forward(gamma=0x50002) == forward(rstd=0x80001) == "SK_EINVAL"
    assert backward(dgamma=0x90000) == backward(dbeta=0x80000 + 28) == backward(dgamma=0x70000) == backward(dbeta=0x50000 - 28) == "SK_EINVAL"
    assert backward(dgamma=0x60000 + 12) == backward(gamma=0x70002) == backward(dbeta=0x90002) == "SK_EINVAL"
    big, need = extent(n=100000, c=64), C.c_uint64()
    assert B.lib.sknet_layer_norm_workspace(C.byref(big), C.byref(need)) == 0 and need.value > 256
    spread = dict(e=big, far=0x1000, mean=0x60000000, rstd=0x70000000, gamma=0x80000000, dgamma=0x90000000, dbeta=0xa0000000, n=need.value)
    assert backward(ws=0x90000000, **spread) == backward(ws=0x80000000, **spread) == backward(ws=0x60000000, **spread) == "SK_EINVAL"


def test_calls_without_positions_do_nothing():
    for e in (extent(n=0), extent(B.SK_MAPS, 0, 5, 9), extent(B.SK_MAPS, 3, 5, 0)):
        none = view(0)
        assert B.lib.sknet_dropout(C.byref(e), C.byref(none), C.byref(none), C.byref(DROP), None) == 0
        assert B.lib.sknet_layer_norm(C.byref(e), C.byref(none), None, None, None, None, 1e-5, None, C.byref(none), None, None, None) == 0


def test_binding_sees_rows_and_maps():
    def first(t, axis):
        return next(iter(B._orders(t.shape, t.stride(), axis % t.dim()).items()))
    x = torch.zeros(2, 3, 5, 7)
    assert first(x, -1) == ((B.SK_ROWS, 30, 7, 1), (7, 0))
    assert first(x, 1) == ((B.SK_MAPS, 2, 3, 35), (105, 35))
    assert first(x.permute(0, 2, 3, 1).contiguous().permute(0, 3, 1, 2), 1) == ((B.SK_ROWS, 70, 3, 1), (3, 0))   # channels last in memory
    assert first(torch.zeros(4, 10)[:, :6], 1) == ((B.SK_ROWS, 4, 6, 1), (10, 0))
    assert first(torch.zeros(6, 4).t(), 1) == ((B.SK_MAPS, 1, 6, 4), (0, 4))
    assert first(torch.zeros(9), 0) == ((B.SK_ROWS, 1, 9, 1), (0, 0))
    assert first(torch.zeros(0, 9), 1)[0] == (B.SK_ROWS, 0, 9, 1)
    wide = torch.zeros(2, 8, 5, 7)[:, 2:5]
    assert first(wide, 1) == ((B.SK_MAPS, 2, 3, 35), (280, 35))
    gaps = torch.zeros(2, 3, 5, 9)[..., :7]            # rows of pixels with gaps: no plane, but positions one by one where there is one image
    assert not any(k[3] > 1 for k in B._orders(gaps.shape, gaps.stride(), 1))


def test_binding_refuses_what_is_no_gpu_tensor():
    for call in (lambda t: B.dropout(t, 0.5, 1), lambda t: B.layer_norm(t), lambda t: B.layer_norm_backward(t, t, t, t)):
        for t in (torch.zeros(3, 4), np.zeros((3, 4), np.float32), None):
            with pytest.raises(TypeError):
                call(t)


# ---- the layers of a net

def test_net_layers_shapes_and_refusals():
    import sk_synth as S
    layers = [S.conv(8, 4, 1, relu=False), S.norm(relu=True), S.pool(2, 1), S.conv(16, 5, 2), S.dropout(0.5), S.norm(), S.conv(2, 1, 1, relu=False)]
    for dtype in ("f32", "bf16", "f16"):
        net = B.SKNet(layers, 1, 2, dtype=dtype)
        assert net.num_convs() == 3 and net.num_norms() == 2 and [net.norm_size(i) for i in range(2)] == [8, 16]
        plain = B.SKNet([l for l in layers if l["type"] in ("conv", "pool")], 1, 2)
        assert net.context() == plain.context()
        shapes = net.infer_shapes(60, 50)
        assert [s[1:] for i, s in enumerate(shapes) if i not in (2, 5, 6)] == [s[1:] for s in plain.infer_shapes(60, 50)]
        g, b = net.get_norm(1)
        assert (g == 1).all() and (b == 0).all()
        net.set_norm(1, beta=np.arange(16))
        net.set_norm(0, gamma=np.full(8, 2.0))
        assert (net.get_norm(1)[0] == 1).all() and (net.get_norm(1)[1] == np.arange(16)).all() and (net.get_norm(0)[0] == 2).all()
        assert net.get_dropout() == (0, 0)
        net.set_dropout((1 << 64) - 1, 77)
        assert net.get_dropout() == ((1 << 64) - 1, 77)
        for bad in (lambda: net.set_norm(2), lambda: net.get_norm(-1), lambda: net.get_norm_grad(0), lambda: net.set_dropout(1, 1 << 40)):
            with pytest.raises(B.SknetError):
                bad()
        with pytest.raises(ValueError):
            net.set_norm(0, gamma=np.zeros(9))
        net.close()
    for layer in (B.SkLayer(B.SK_LAYERNORM, 0, 2, 1, 1, 0), B.SkLayer(B.SK_DROPOUT, 100, 1, 2, 1, 0), B.SkLayer(B.SK_LAYERNORM, 0, 1, 1, 2, 0),
                  B.SkLayer(B.SK_DROPOUT, 65537, 1, 1, 1, 0), B.SkLayer(B.SK_DROPOUT, -1, 1, 1, 1, 0), B.SkLayer(B.SK_DROPOUT, 5, 1, 1, 1, 1), B.SkLayer(4, 0, 1, 1, 1, 0)):
        arr, out = (B.SkLayer * 2)(B.SkLayer(B.SK_CONV, 2, 1, 1, 1, 0), layer), C.c_void_p()
        assert B.STATUS_NAMES[B.lib.sknet_create(arr, 2, 1, 2, 0, 0, C.byref(out))] in ("SK_EINVAL", "SK_ESHAPE") and not out.value
        assert B.STATUS_NAMES[B.lib.sknet3d_create(arr, 2, 1, 2, C.byref(out))] in ("SK_EINVAL", "SK_ESHAPE")
    for kind in (B.SK_LAYERNORM, B.SK_DROPOUT):            # 2-D nets only
        arr, out = (B.SkLayer * 2)(B.SkLayer(B.SK_CONV, 2, 1, 1, 1, 0), B.SkLayer(kind, 0, 1, 1, 1, 0)), C.c_void_p()
        assert B.STATUS_NAMES[B.lib.sknet3d_create(arr, 2, 1, 2, C.byref(out))] == "SK_EINVAL"
    with pytest.raises(B.SknetError):
        B.SKNet([S.dropout(0.5)], 2, 2)
    with pytest.raises(ValueError):
        B.SKNet([S.conv(2, 1), S.dropout(1.5)], 1, 2)


def test_oracle_net_gradients_by_differences():
    import sk_synth as S
    from oracle import nets as NETS
    layers = [S.conv(5, 2, 1, relu=False), S.norm(relu=True), S.dropout(0.3), S.pool(2, 1), S.norm(), S.conv(6, 1), S.dropout(0.5), S.conv(3, 1, relu=False)]
    ws, bs = S.he_normal_weights(layers, 2, 7, bias_scale=0.1)
    ws, bs = [w.astype(np.float64) for w in ws], [b.astype(np.float64) for b in bs]
    rng = np.random.default_rng(8)
    norms = [(1 + 0.3 * rng.normal(size=5), 0.3 * rng.normal(size=5)), (1 + 0.3 * rng.normal(size=5), 0.3 * rng.normal(size=5))]
    img, lab = rng.random((1, 2, 6, 5)), rng.integers(0, 3, (1, 6, 5)).astype(np.int32)
    drop = (99, 4)

    def loss():
        _, acts, am = NETS.sknet_forward(img, layers, ws, bs, keep=True, norms=norms, drop=drop)
        return acts, am, NETS.L.softmax_loss(acts[-1], lab)[0]

    acts, am, _ = loss()
    grads = []
    _, dws, dbs, _ = NETS.sknet_backward(layers, ws, acts, am, lab, norms=norms, drop=drop, norm_grads=grads)
    for arr, grad in [(ws[0], dws[0]), (ws[1], dws[1]), (bs[0], dbs[0])] + [(norms[i][j], grads[i][j]) for i in range(2) for j in range(2)]:
        for i in list(np.ndindex(arr.shape))[::3]:
            old = arr[i]
            arr[i] = old + 1e-5
            up = loss()[2]
            arr[i] = old - 1e-5
            down = loss()[2]
            arr[i] = old
            assert abs((up - down) / 2e-5 - grad[i]) <= 1e-6
