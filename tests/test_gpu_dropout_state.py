"""GPU: seed and step of a net's dropout layers, set between the passes."""
import numpy as np
import pytest
import torch

from test_gpu_norm_net import MIXED, data, make

pytestmark = pytest.mark.gpu


def gradients(net):
    return [v for i in range(net.num_convs()) for v in net.get_grad(i)] + [v for i in range(net.num_norms()) for v in net.get_norm_grad(i)]


def same(a, b):
    return all(np.array_equal(u, v) for u, v in zip(a, b))


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("seed,step", [(99, 500), (3, 500), (99, 10)])
def test_a_backward_pass_makes_the_masks_of_the_pass_before_it(kind, seed, step):
    net, _, _, _ = make(MIXED, 1, kind, 81)
    img, lab = data(1, 1, 30, 40, 2, 82)
    x, y = torch.from_numpy(img).cuda(), torch.from_numpy(lab).cuda()
    loss = torch.empty(1, device="cuda")
    net.set_dropout(3, 10)
    net.plan(1, 30, 40, training=True)
    net.forward(x)
    net.backward(y)
    want = gradients(net)
    net.backward(y, loss=loss, noalloc=True)
    bare = gradients(net)
    maps = [net.get_activation_grad(i, y) for i in range(len(MIXED))]
    net.set_dropout(seed, step)
    assert net.get_dropout() == (seed, step)
    net.backward(y)
    assert same(gradients(net), want)
    net.backward(y, loss=loss, noalloc=True)
    assert same(gradients(net), bare)
    assert same([net.get_activation_grad(i, y) for i in range(len(MIXED))], maps)
    # what was set counts from the next pass on
    prob = net.forward(x)
    net.backward(y)
    after = gradients(net)
    assert net.get_dropout() == (seed, step + 1) and not same(after, want)
    other, _, _, _ = make(MIXED, 1, kind, 81)
    other.set_dropout(seed, step)
    other.plan(1, 30, 40, training=True)
    assert torch.equal(other.forward(x), prob)
    other.backward(y)
    assert same(gradients(other), after)
    net.close()
    other.close()


def test_a_recorded_forward_pass_keeps_its_seed():
    # the step is read when the pass runs, the seed is the recording's; the backward pass behind a replay goes by the pass recorded
    net, _, _, _ = make(MIXED, 1, "f32", 81)
    img, lab = data(1, 1, 30, 40, 2, 82)
    x, y = torch.from_numpy(img).cuda(), torch.from_numpy(lab).cuda()
    prob = torch.empty(1, 2, 30, 40, device="cuda")
    net.set_dropout(3)
    net.plan(1, 30, 40, training=True)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            net.forward(x, prob, torch.cuda.current_stream())
        seen = []
        for step in (7, 7, 20):
            net.set_dropout(1000, step)
            g.replay()
            net.backward(y, stream=stream)
            torch.cuda.synchronize()
            seen.append((prob.clone(), gradients(net)))
            assert net.get_dropout() == (1000, step + 1)
            prob.zero_()
    for step, (p, grads) in zip((7, 7, 20), seen):
        net.set_dropout(3, step)
        assert torch.equal(net.forward(x), p)
        net.backward(y)
        assert same(gradients(net), grads)
    net.close()
