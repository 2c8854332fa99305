"""GPU: layer norm and dropout as layers of an SK net, every storage type.  Layer by layer against the 64-bit oracle on the maps and error maps that the
pass itself stored (bounds: norm_bounds.py), whole fp32 nets against the oracle at the bound of the other fp32 training tests."""
import numpy as np
import pytest
import torch

import sk_synth as S
from norm_bounds import TYPES, U, bwd_bounds, close, norm_bounds, rounded
from oracle import nets as NETS
from oracle import norm as ON

pytestmark = pytest.mark.gpu
FP32_TOL = 1e-4


def relerr(got, ref):
    return float(np.abs(np.asarray(got, dtype=np.float64) - ref).max() / max(np.abs(ref).max(), 1e-30))


MIXED = [S.conv(12, 4, 1, relu=False), S.norm(relu=True), S.pool(2, 1), S.dropout(0.3), S.conv(24, 4, 2), S.norm(), S.pool(2, 2), S.conv(40, 1), S.dropout(0.5),
         S.norm(relu=True), S.conv(2, 1, 1, relu=False)]
ENDS = [S.dropout(0.1), S.norm(), S.conv(9, 3, 1), S.norm(), S.dropout(0.4), S.norm(relu=True), S.conv(3, 1, 1, relu=False), S.norm(relu=True)]
SINGLE = [S.norm(relu=True), S.conv(70, 1, 1), S.dropout(0.2), S.conv(130, 1), S.norm(), S.conv(4, 1, 1, relu=False)]


def make(layers, c_in, dtype, seed):
    from paper_1509_03371_amd import binding as B
    ws, bs = S.he_normal_weights(layers, c_in, seed, bias_scale=0.1)
    net = B.SKNet(layers, c_in, [l["f_out"] for l in layers if l["type"] == "conv"][-1], dtype=dtype)
    for i, (w, b) in enumerate(zip(ws, bs)):
        net.set_weights(i, w, b)
    rng = np.random.default_rng(seed + 1)
    norms = []
    for i in range(net.num_norms()):
        c = net.norm_size(i)
        norms.append((np.float32(1 + 0.3 * rng.normal(size=c)), np.float32(0.3 * rng.normal(size=c))))
        net.set_norm(i, *norms[-1])
    return net, [w.astype(np.float64) for w in ws], [b.astype(np.float64) for b in bs], norms


def data(n, c, h, w, classes, seed):
    rng = np.random.default_rng(seed)
    lab = rng.integers(0, classes, (n, h, w)).astype(np.int32)
    lab[rng.random((n, h, w)) < 0.2] = -1
    return np.float32(rng.random((n, c, h, w))), lab


WIDE = [S.conv(2056, 1, relu=False), S.norm(relu=True), S.dropout(0.1), S.conv(1100, 1), S.norm(), S.conv(520, 1, relu=False), S.dropout(0.2), S.norm(relu=True),
        S.conv(260, 1), S.norm(), S.conv(2, 1, relu=False)]

NETS_ = [(MIXED, 1, 2, 2, 31, 45), (ENDS, 3, 3, 1, 20, 33), (SINGLE, 2, 4, 2, 9, 30)]
# layer by layer only: among 2056 x 117 samples in front of a ReLU some lie within fp32 rounding of zero, and a whole net's gradients then differ by those
WIDE_ = (WIDE, 3, 2, 1, 9, 13)


@pytest.mark.parametrize("layers,c_in,classes,n,h,w", NETS_, ids=["mixed", "ends", "single"])
def test_fp32_net_against_the_oracle(layers, c_in, classes, n, h, w):
    net, ws, bs, norms = make(layers, c_in, "f32", 41)
    img, lab = data(n, c_in, h, w, classes, 42)
    net.set_dropout(0xABCDEF0123456789, 5)
    net.plan(n, h, w, training=True)
    x, y = torch.from_numpy(img).cuda(), torch.from_numpy(lab).cuda()
    for step in (6, 7):                                   # each pass has masks of its own
        prob = net.forward(x)
        loss = net.backward(y)
        assert net.get_dropout() == (0xABCDEF0123456789, step)
        ref, acts, ams = NETS.sknet_forward(img, layers, ws, bs, keep=True, norms=norms, drop=(0xABCDEF0123456789, step))
        grads = []
        ref_loss, dws, dbs, _ = NETS.sknet_backward(layers, ws, acts, ams, lab, norms=norms, drop=(0xABCDEF0123456789, step), norm_grads=grads)
        assert np.abs(prob.cpu().numpy() - ref).max() <= FP32_TOL
        assert abs(loss.item() - ref_loss) <= FP32_TOL * abs(ref_loss)
        for i in range(net.num_convs()):
            dw, db = net.get_grad(i)
            assert relerr(dw, dws[i]) <= FP32_TOL and np.abs(db - dbs[i]).max() <= FP32_TOL * max(np.abs(dbs[i]).max(), np.abs(dws[i]).max()), i
        for i in range(net.num_norms()):
            for mine, his in zip(net.get_norm_grad(i), grads[i]):
                assert np.abs(mine - his).max() <= FP32_TOL * max(np.abs(g).max() for g in grads[i]), i
    # the static scratch: the same gradients
    want = [net.get_grad(i) for i in range(net.num_convs())] + [net.get_norm_grad(i) for i in range(net.num_norms())]
    net.backward(y, loss=torch.empty(1, device="cuda"), noalloc=True)
    got = [net.get_grad(i) for i in range(net.num_convs())] + [net.get_norm_grad(i) for i in range(net.num_norms())]
    for a, b in zip(got, want):
        assert all(np.abs(u - v).max() <= 1e-5 * max(np.abs(q).max() for q in b) for u, v in zip(a, b))
    # an update, with momentum and decay, and a second one
    before = [net.get_norm(i) for i in range(net.num_norms())]
    vel = [[np.zeros_like(v, dtype=np.float64) for v in pair] for pair in before]
    for _ in range(2):
        grads = [net.get_norm_grad(i) for i in range(net.num_norms())]
        net.sgd_step(0.05, momentum=0.9, weight_decay=0.01)
        for i, pair in enumerate(before):
            now = net.get_norm(i)
            new = []
            for j in range(2):
                vel[i][j] = 0.9 * vel[i][j] + 0.05 * (grads[i][j] + 0.01 * np.float64(pair[j]))
                new.append(pair[j] - vel[i][j])
                assert np.abs(now[j] - new[j]).max() <= 8 * U * (np.abs(new[j]).max() + 1)
            before[i] = now
        net.forward(x)
        net.backward(y)
    net.close()


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("layers,c_in,classes,n,h,w", NETS_ + [WIDE_], ids=["mixed", "ends", "single", "wide"])
def test_layers_on_the_maps_the_pass_stored(layers, c_in, classes, n, h, w, kind):
    net, _, _, norms = make(layers, c_in, kind, 51)
    img, lab = data(n, c_in, h, w, classes, 52)
    x, y = torch.from_numpy(img).cuda(), torch.from_numpy(lab).cuda()
    net.set_dropout(77)
    net.plan(n, h, w, training=True)
    net.forward(x)
    acts = [net.get_activation(i).astype(np.float64) for i in range(-1, len(layers))]
    ni = 0
    order = []
    for li, lay in enumerate(layers):
        if lay["type"] == "dropout":
            ref = ON.dropout(acts[li], lay["p"], 77, li * 2 ** 40 + 1)
            assert np.array_equal(acts[li + 1] == 0, ref == 0)
            close(acts[li + 1], ref, rounded(ref, kind, 2 * U * np.abs(ref)), "dropout %d" % li)
        elif lay["type"] == "norm":
            ref, _, _, bound, _, _ = norm_bounds(acts[li], 0.0, *norms[ni], 1e-5, kind)
            if lay["relu"]:
                ref = np.maximum(ref, 0.0)
            close(acts[li + 1], ref, bound, "norm %d" % li)
            order.append(li)
            ni += 1
    # error maps: what a layer hands down, from what it got
    net.backward(y)
    sums = [net.get_norm_grad(i) for i in range(ni)]
    maps = [net.get_activation_grad(li, y).astype(np.float64) for li in range(len(layers))]
    maps[-1] = torch.from_numpy(maps[-1]).float().to(TYPES[kind]).double().numpy()
    for li, lay in enumerate(layers):
        if lay["type"] not in ("norm", "dropout"):
            continue
        below = li > 0 and layers[li - 1].get("relu", False)
        if lay["type"] == "dropout":
            if li == 0:
                continue
            ref = ON.dropout(maps[li], lay["p"], 77, li * 2 ** 40 + 1)
            bound = rounded(ref, kind, 2 * U * np.abs(ref))
        else:
            i = order.index(li)
            _, mean, rstd = ON.layer_norm(acts[li], None, None)
            # the pass uses its own statistics: off from these by their bounds, which enter as an error of s and of the scale
            _, _, _, _, e_mean, e_rstd = norm_bounds(acts[li], 0.0, None, None, 1e-5, kind)
            t, dg, db, e_t, e_dg, e_db = bwd_bounds(maps[li], acts[li], mean, rstd, norms[i][0], None, kind)
            r, rel = rstd[:, None], (e_rstd / rstd)[:, None]
            e_h = e_mean[:, None] * r + rel * np.abs(acts[li] - mean[:, None]) * r
            g = np.abs(maps[li] * np.float64(norms[i][0]).reshape(1, -1, 1, 1))
            h = np.abs(acts[li] - mean[:, None]) * r
            gh = (g * h).mean(axis=1, keepdims=True)
            e_t = 1.01 * (e_t + rel * np.abs(t) + r * (e_h * gh + h * (g * e_h).mean(axis=1, keepdims=True)))
            for mine, ref, bound in zip(sums[i], (dg, db), (e_dg + 1.01 * (np.abs(maps[li]) * e_h).sum(axis=(0, 2, 3)), e_db)):
                close(mine, ref, bound, "norm %d" % li)
            if li == 0:
                continue
            ref, bound = t, rounded(t, kind, e_t)
        if below:
            ref = np.where(acts[li] > 0, ref, 0.0)
        close(maps[li - 1], ref, bound, "error map below %s %d" % (lay["type"], li))
    net.close()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_inference_leaves_dropout_out(kind):
    from paper_1509_03371_amd import binding as B
    layers = [S.conv(16, 4, 1), S.dropout(0.2), S.pool(2, 1), S.dropout(0.7), S.conv(40, 1), S.dropout(0.5), S.conv(2, 1, 1, relu=False)]
    bare = [l for l in layers if l["type"] != "dropout"]
    img = torch.from_numpy(data(2, 1, 40, 51, 2, 61)[0]).cuda()
    ws, bs = S.he_normal_weights(layers, 1, 62, bias_scale=0.1)
    nets = [B.SKNet(ls, 1, 2, dtype=kind) for ls in (layers, bare)]
    for keep in (True, False):
        prob = []
        for net in nets:
            for i, (w, b) in enumerate(zip(ws, bs)):
                net.set_weights(i, w, b)
            net.plan(2, 40, 51, keep=keep)
            prob.append(net.forward(img))
        assert torch.equal(*prob)
        if keep:
            for i, j in ((0, 0), (1, 0), (2, 1), (3, 1), (4, 2), (5, 2), (6, 3), (-1, -1)):
                assert np.array_equal(nets[0].get_activation(i), nets[1].get_activation(j)), i
    # training and inference plans of one net in turn: parameters and the step survive
    net = nets[0]
    net.set_dropout(9, 100)
    net.plan(2, 40, 51, training=True)
    net.forward(img)
    net.plan(2, 40, 51)
    assert net.get_dropout() == (9, 101) and torch.equal(net.forward(img), prob[0])
    net.plan(2, 40, 51, training=True)
    net.forward(img)
    assert net.get_dropout() == (9, 102)
    for n in nets:
        n.close()


def test_fused_training_head_behind_dropout_and_not_behind_a_relu():
    from paper_1509_03371_amd import binding as B
    layers = S.sknet_layers(width=24, hidden=100, classes=3, stages=1)
    layers = layers[:2] + [S.dropout(0.25)] + layers[2:]
    img, lab = data(2, 1, 30, 37, 3, 71)
    grads = []
    for fused in (False, True):
        net, ws, bs, _ = make(layers, 1, "bf16", 72)
        net.plan(2, 30, 37, training=True, fused_head=fused)
        prob = net.forward(torch.from_numpy(img).cuda())
        loss = net.backward(torch.from_numpy(lab).cuda()).item()
        ref, acts, ams = NETS.sknet_forward(img, layers, ws, bs, keep=True, drop=(0, 1))
        ref_loss, dws, _, _ = NETS.sknet_backward(layers, ws, acts, ams, lab, drop=(0, 1))
        # the bounds of the 16-bit training tests
        assert np.abs(prob.cpu().numpy() - ref).max() <= 2e-2 and abs(loss - ref_loss) <= 2e-2 * ref_loss
        for i in range(net.num_convs()):
            assert relerr(net.get_grad(i)[0], dws[i]) <= 5e-2, (fused, i)
        net.close()
    relu = layers[:2] + [S.norm(relu=True)] + layers[3:]
    net = B.SKNet(relu, 1, 3, dtype="bf16")
    with pytest.raises(B.SknetError) as e:
        net.plan(2, 30, 37, training=True, fused_head=True)
    assert e.value.status_name == "SK_EUNSUPPORTED"
    net.plan(2, 30, 37, training=True)
    net.close()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_recorded_training_steps_move_on(kind):
    net, _, _, _ = make(MIXED, 1, kind, 81)
    img, lab = data(1, 1, 30, 40, 2, 82)
    x, y = torch.from_numpy(img).cuda(), torch.from_numpy(lab).cuda()
    prob, loss = torch.empty(1, 2, 30, 40, device="cuda"), torch.empty(1, device="cuda")
    net.set_dropout(3)
    net.plan(1, 30, 40, training=True)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            net.forward(x, prob, torch.cuda.current_stream())
            net.backward(y, loss, torch.cuda.current_stream())
        seen = []
        for rep in range(3):
            g.replay()
            torch.cuda.synchronize()
            seen.append((prob.clone(), loss.clone(), net.get_norm_grad(1), net.get_dropout()[1]))
            prob.zero_()
    assert [s[3] for s in seen] == [1, 2, 3] and not torch.equal(seen[0][0], seen[1][0])
    net.set_dropout(3)
    for p, l, grad, _ in seen:                              # the same steps, launched one by one
        assert torch.equal(net.forward(x), p) and torch.equal(net.backward(y), l)
        assert all(np.array_equal(a, b) for a, b in zip(net.get_norm_grad(1), grad))
    net.close()


def test_many_layers_update_one_by_one():
    # more tensors than one launch updates
    layers = []
    for i in range(12):
        layers += [S.conv(8, 1, 1, relu=False), S.norm(relu=True)]
    layers.append(S.conv(2, 1, 1, relu=False))
    net, _, _, _ = make(layers, 1, "f32", 91)
    img, lab = data(1, 1, 12, 17, 2, 92)
    net.plan(1, 12, 17, training=True)
    net.forward(torch.from_numpy(img).cuda())
    net.backward(torch.from_numpy(lab).cuda())
    before = [net.get_norm(i) for i in range(12)]
    grads = [net.get_norm_grad(i) for i in range(12)]
    net.sgd_step(0.1)
    for i in range(12):
        for old, g, new in zip(before[i], grads[i], net.get_norm(i)):
            assert np.abs(new - (old - 0.1 * np.float64(g))).max() <= 4 * U * (np.abs(old).max() + np.abs(g).max())
    net.close()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_step_names_and_times(kind):
    net, _, _, _ = make(MIXED, 1, kind, 95)
    img, lab = data(1, 1, 30, 40, 2, 96)
    net.plan(1, 30, 40, training=True)
    net.forward(torch.from_numpy(img).cuda())
    names = [net.step_name(i) for i in range(net.num_steps())]
    assert "norm1" in names and "dropout3" in names and "conv10_k1_d1_o2" in names
    assert all(net.time_step(i, 2) >= 0 for i in range(len(names)))
    y = torch.from_numpy(lab).cuda()
    assert all(net.time_backward_step(y, i, 1, 2) >= 0 for i in (1, 3, 5, 8, 9))
    from paper_1509_03371_amd import binding as B
    for i in (1, 3):
        with pytest.raises(B.SknetError):                   # part 0 is a convolution's
            net.time_backward_step(y, i, 0, 2)
    assert net.get_dropout()[1] == 1                        # timing a step is no pass
    net.close()
