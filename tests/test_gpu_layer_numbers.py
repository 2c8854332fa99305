"""GPU: layers are named by their number among all of a net's, dropout layers that an inference plan leaves out among them."""
import pytest
import torch

import sk_synth as S

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_fused_layers_are_named_by_the_callers_number(dtype):
    from paper_1509_03371_amd import binding as B
    layers = [S.dropout(0.1), S.conv(48, 4, 1), S.pool(2, 1), S.dropout(0.2), S.conv(48, 4, 2), S.pool(2, 2), S.conv(200, 1), S.dropout(0.5), S.conv(2, 1, 1, relu=False)]
    net = B.SKNet(layers, 1, 2, dtype=dtype)
    for i, (w, b) in enumerate(zip(*S.he_normal_weights(layers, 1, 5))):
        net.set_weights(i, w, b)
    net.plan(1, 64, 70)
    net.forward(torch.rand(1, 1, 64, 70, device="cuda"))
    refused = 0
    for i in range(len(layers)):
        try:
            net.get_activation(i)
        except B.SknetError as e:
            if "fuses layer" not in str(e):
                continue
            named = int(str(e).split("fuses layer ")[1].split()[0])
            # a dropout layer stands for the one in front of it
            assert named == i or (layers[i]["type"] == "dropout" and named == i - 1), (i, str(e))
            refused += 1
    assert refused
    net.close()


def test_times_of_a_layer_norm_are_those_of_its_input_gradient():
    from paper_1509_03371_amd import binding as B
    layers = [S.conv(9, 3, 1, relu=False), S.norm(relu=True), S.dropout(0.2), S.conv(2, 1, 1, relu=False)]
    net = B.SKNet(layers, 1, 2)
    for i, (w, b) in enumerate(zip(*S.he_normal_weights(layers, 1, 5))):
        net.set_weights(i, w, b)
    net.plan(1, 20, 30, training=True)
    net.forward(torch.rand(1, 1, 20, 30, device="cuda"))
    labels = torch.zeros(1, 20, 30, dtype=torch.int32, device="cuda")
    for i in (1, 2):
        with pytest.raises(B.SknetError) as e:
            net.time_backward_step(labels, i, 0, 2)
        assert e.value.status_name == "SK_EINVAL" and "convolution" in str(e.value) and "weights" not in str(e.value)
        assert net.time_backward_step(labels, i, 1, 2) >= 0
    net.close()
