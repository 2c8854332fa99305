"""GPU: means of many deviations, where sums of squares about zero would lose the variance, in every kernel of rows and maps; with a few positions whose
channels are all equal."""
import numpy as np
import pytest
import torch

from norm_bounds import U, close, norm_bounds, place, rounded, to64
from oracle import norm as ON

pytestmark = pytest.mark.gpu

SHAPES = [(50, 8), (50, 40), (50, 1000), (40, 3000), (6, 20000), (5, 40000), (2, 24, 900), (2, 64, 900), (2, 120, 70), (1, 500, 301), (1, 1000, 130), (1, 2000, 33), (2, 3000, 7),
          (40, 9, 3)]


# the mean in deviations: as far as the type tells values of one deviation apart (bf16 at 64 in steps of 1/2, fp16 at 300 of 1/4)
@pytest.mark.parametrize("kind,mean", [("f32", 1000.0), ("bf16", 64.0), ("f16", 300.0)])
@pytest.mark.parametrize("adds", [False, True])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_far_means(shape, kind, mean, adds):
    from paper_1509_03371_amd import binding as B
    rng = np.random.default_rng(3)
    x = mean + rng.normal(size=shape)
    equal = np.zeros(shape[:1] + shape[2:], bool)
    equal.reshape(-1)[[0, 4, equal.size // 2]] = True
    x = np.where(np.expand_dims(equal, 1), 7.25, x)
    x = place(x, kind)
    gamma = torch.from_numpy(np.float32(1 + 0.2 * rng.normal(size=shape[1]))).cuda()
    if adds:
        r = place(np.where(np.expand_dims(equal, 1), 0.0, rng.normal(size=shape)), kind)
        y, s, m, rstd = B.layer_norm(x, gamma, None, axis=1, residual=r, sum_out=torch.empty_like(x))
        rs = to64(x) + to64(r)
        es = U * np.abs(rs)
        close(s, rs, rounded(rs, kind, es), "s")
    else:
        y, s, m, rstd = B.layer_norm(x, gamma, None, axis=1)
        rs, es = to64(x), 0.0
    ry, rm, rr, by, bm, brs = norm_bounds(rs, es, gamma.cpu().numpy(), None, 1e-5, kind)
    close(m, rm, bm, "mean")
    close(y, ry, by, "y")
    other = ~equal
    assert other.sum() >= 2
    # where the channels differ the bound is far below what a lost variance would be off by
    assert (brs[other] <= 0.05 * rr[other]).all()
    close(to64(rstd)[other], rr[other], brs[other], "rstd")
    # equal channels: at most the mean's rounding is left, so rstd lies between that of the bound and 1 / sqrt(eps)
    close(to64(rstd)[equal], rr[equal], brs[equal], "rstd of equal channels")
