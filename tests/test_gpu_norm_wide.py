"""GPU: the parameter gradients of rows of as many channels as the calls take."""
import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("c", [(1 << 27) - 8, (1 << 27) - 3, 1 << 27])
def test_gradients_of_the_most_channels(c):
    from paper_1509_03371_amd import binding as B
    gen = torch.Generator(device="cuda").manual_seed(c)
    s, dy = (torch.empty(2, c, dtype=torch.bfloat16, device="cuda").normal_(generator=gen) for _ in range(2))
    mean, rstd = torch.tensor([0.3, -0.7], device="cuda"), torch.tensor([1.9, 0.6], device="cuda")
    dgamma, dbeta = (torch.full((c,), float("nan"), device="cuda") for _ in range(2))
    B.layer_norm_backward(dy, s, mean, rstd, dgamma=dgamma, dbeta=dbeta)
    for at in range(0, c, 1 << 24):
        part = slice(at, min(c, at + (1 << 24)))
        g, h = dy[:, part].double(), (s[:, part].double() - mean.double()[:, None]) * rstd.double()[:, None]
        # a difference, two products and a sum, in fp32
        assert ((dgamma[part] - (g * h).sum(0)).abs() <= 4 * U * (g * h).abs().sum(0) + 1e-37).all(), at
        assert ((dbeta[part] - g.sum(0)).abs() <= 2 * U * g.abs().sum(0) + 1e-37).all(), at
    # no positions: the gradients are cleared
    none = torch.empty(0, c, dtype=torch.bfloat16, device="cuda")
    B.layer_norm_backward(none, none, mean[:0], rstd[:0], dgamma=dgamma, dbeta=dbeta)
    assert not dgamma.any() and not dbeta.any()
