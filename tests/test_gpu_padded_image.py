"""GPU: the padded image of a pass, read back: from every plan that makes one; the others say that they do not."""
import numpy as np
import pytest
import torch

import sk_synth as S
from oracle import layers as OL

pytestmark = pytest.mark.gpu

NET = [S.conv(48, 4, 1), S.pool(2, 1), S.conv(16, 4, 2), S.conv(2, 1, 1, relu=False)]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("layers,index", [(NET, -1), ([S.dropout(0.5)] + NET, 0), ([S.dropout(0.5)] + NET, -1)], ids=["image", "dropout first", "image before dropout"])
def test_padded_image_is_read_or_refused(dtype, layers, index):
    from paper_1509_03371_amd import binding as B
    ws, bs = S.he_normal_weights(layers, 1, 5, bias_scale=0.1)
    v = sum((l["k"] - 1) * l["d"] for l in layers)
    net = B.SKNet(layers, 1, 2, dtype=dtype)
    for i, (w, b) in enumerate(zip(ws, bs)):
        net.set_weights(i, w, b)
    read = []
    # (an image of its own for each plan: a buffer of the size of one that was freed may hold what that held)
    for seed, keep in ((6, True), (7, False), (8, True)):
        img = S.uniform_image(2, 1, 61, 70, seed)
        want = torch.from_numpy(OL.mirror_pad(img, (v + 1) // 2, (v + 1) // 2, v // 2, v // 2, 0).astype(np.float32))
        want = want.to({"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[dtype]).float().numpy()
        net.plan(2, 61, 70, keep=keep)
        net.forward(torch.from_numpy(img).cuda())
        try:
            got = net.get_activation(index)
        except B.SknetError as e:
            assert e.status_name == "SK_ESTATE" and "mode 2" in str(e) and not keep
        else:
            assert np.array_equal(got, want), keep
            read.append(keep)
    assert read.count(True) == 2
    net.close()
