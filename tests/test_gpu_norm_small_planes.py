"""GPU: parameter gradients of planes of one to three pixels, whose positions waves share across images."""
import numpy as np
import pytest
import torch

from norm_bounds import bwd_bounds, close, inputs, place, rounded, to64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shape,step", [((1, 1, 1), 1), ((1, 9, 3), 1), ((3, 70, 1), 2), ((21, 8, 3), 1), ((32, 33, 2), 1), ((43, 7, 3), 1), ((1000, 5, 1), 3), ((2500, 20, 2), 1),
                                        ((30011, 11, 3), 1), ((70003, 40, 2), 1), ((4001, 64, 1), 2), ((5, 3001, 3), 1), ((130, 2049, 2), 1)], ids=str)
def test_gradients_of_small_planes(shape, step, kind):
    # step: the channels' distance in planes, so that planes of one pixel are no rows
    from paper_1509_03371_amd import binding as B
    x, _, gamma, beta, dy, dsum = inputs(shape, kind, 15)
    x, dy, dsum = (place(np.repeat(a, step, axis=1), kind)[:, ::step] for a in (x, dy, dsum))
    gd = torch.from_numpy(gamma).cuda()
    _, s, mean, rstd = B.layer_norm(x, gd, axis=1)
    t, rg, rb, et, eg, eb = bwd_bounds(to64(dy), to64(s), to64(mean), to64(rstd), gamma, to64(dsum), kind)
    out = torch.empty(shape[:1] + (shape[1] * step,) + shape[2:], dtype=x.dtype, device="cuda")[:, ::step]
    dx, dres, dg, db = B.layer_norm_backward(dy, s, mean, rstd, gd, axis=1, dsum=dsum, dx=out)
    close(dres, t, rounded(t, kind, et), "gradient of the sum")
    close(dg, rg, eg, "dgamma")
    close(db, rb, eb, "dbeta")
    again = B.layer_norm_backward(dy, s, mean, rstd, gd, axis=1, dsum=dsum, dx=out)
    assert torch.equal(again[2], dg) and torch.equal(again[3], db)
