"""GPU: the root-mean-square norm's rstd is rounded once.

Channels are whole numbers of 0 to 3, as many as a power of two, and eps = 1: every partial sum of the squares, in any order, and their mean plus eps are then exact in fp32 (at most
9 * 2^16 + 2^16 < 2^24 units of 1 / c), so that rstd = 1 / sqrt of that number is all that is rounded: to the nearest, half a step of fp32.  2^-16 of that is left for what a
correction of the root in fp32 leaves out (terms of (2^-23)^2)."""
import numpy as np
import pytest
import torch

from norm_bounds import TYPES, to64

pytestmark = pytest.mark.gpu

# every kernel of rows and of maps
SHAPES = [(300, 8), (300, 64), (300, 256), (300, 512), (300, 1024), (300, 2048), (300, 4096), (200, 8192), (150, 16384), (100, 32768), (70, 65536),
          (2, 8, 300), (2, 32, 257), (2, 64, 129), (2, 128, 65), (2, 256, 100), (2, 1024, 70), (2, 2048, 70), (90, 64, 3), (90, 2048, 1)]


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_rounded_once(shape, kind):
    from paper_1509_03371_amd import binding as B
    rng = np.random.default_rng(shape[1])
    share = rng.random(size=(shape[0], 1) + shape[2:])           # of the channels that are not zero: positions have unlike sums
    x = rng.integers(1, 4, size=shape) * (rng.random(shape) < share)
    ref = 1.0 / np.sqrt((x.astype(np.float64) ** 2).mean(axis=1) + 1.0)
    xd = torch.from_numpy(x).to(TYPES[kind]).cuda()
    _, _, rstd = B.rms_norm(xd, None, 1.0, axis=1, out=False, sum_out=False)
    half = np.spacing(ref.astype(np.float32)).astype(np.float64) / 2
    off = np.abs(to64(rstd) - ref) / half
    assert off.max() <= 1 + 2.0 ** -16, "%.3f half steps off, %.1f %% of %d by more than one" % (off.max(), 100 * (off > 1 + 2.0 ** -16).mean(), off.size)


@pytest.mark.parametrize("shape", [(9, 700), (9, 40000), (2, 40, 65), (2, 1100, 65)], ids=str)
def test_ends_of_the_range(shape):
    """Sums of squares that are infinite or no numbers, and the least ones: nothing but eps, itself subnormal."""
    from paper_1509_03371_amd import binding as B
    x = torch.zeros(shape, device="cuda")
    x[1, 3, ...], x[0, 5, ...] = float("inf"), float("nan")
    eps = 2.0 ** -140
    _, _, rstd = B.rms_norm(x, None, eps, axis=1, out=False, sum_out=False)
    assert torch.isnan(rstd[0]).all() and (rstd[1] == 0).all() and (rstd[2:] == 2.0 ** 70).all()
    # four squares of 2^124: the mean's division and rstd are rounded, the first by half its error in the root
    x[0], x[1, :4, ...], x[1, 4:, ...] = 0.0, 2.0 ** 62, 0.0
    _, _, rstd = B.rms_norm(x, None, eps, axis=1, out=False, sum_out=False)
    ref = 1.0 / np.sqrt(2.0 ** 126 / shape[1])
    assert (rstd[0] == 2.0 ** 70).all() and np.abs(to64(rstd[1]) / ref - 1).max() <= 1.6 * 2.0 ** -24


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(5, 60), (5, 40000), (1, 60, 65)], ids=str)
def test_squares_beyond_the_range(shape, kind):
    """Finite values whose squares are not: rstd is 0, and the position alone has no digits."""
    from paper_1509_03371_amd import binding as B
    x = torch.ones(shape, dtype=TYPES[kind], device="cuda")
    where = (2, 7) if len(shape) == 2 else (0, 7, 33)
    x[where] = 2.0 ** 70
    y, _, rstd = B.rms_norm(x, axis=1)
    there = torch.zeros(rstd.shape, dtype=torch.bool, device="cuda")
    there[where[0] if len(shape) == 2 else (0, 33)] = True
    assert (rstd[there] == 0).all() and (rstd[~there] > 0.99).all()
    assert torch.equal((y == 0).all(dim=1), there)
