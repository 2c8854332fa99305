"""GPU: weight gradient of an inner product over inputs held in 8 bits, against the 64-bit oracle (bounds: act8_bounds.py)."""
import numpy as np
import pytest
import torch

from act8_bounds import close, product_bounds, to64
from norm_bounds import TYPES, place

pytestmark = pytest.mark.gpu

# positions (rows, or images and pixels), input channels, output channels
SIZES = [((1,), 1, 1), ((3,), 5, 2), ((31,), 33, 17), ((32,), 32, 16), ((100,), 777, 201), ((257,), 128, 128), ((1000,), 48, 200), ((513,), 129, 257), ((64,), 300, 1000),
         ((5000,), 40, 24), ((4096,), 64, 300), ((40,), 2050, 9),
         ((1, 1), 1, 1), ((2, 3), 5, 2), ((1, 31), 33, 17), ((1, 32), 32, 16), ((1, 100), 777, 201), ((3, 257), 128, 128), ((2, 1000), 48, 200), ((1, 513), 129, 257), ((9, 7), 300, 100),
         ((1, 5000), 40, 24), ((2, 2048), 64, 300), ((70, 1), 20, 30)]


def case(positions, c, c_out, kind, seed, pad=0, order="dense"):
    rng = np.random.default_rng(seed)
    shape = lambda n: positions[:1] + (n,) + positions[1:]  # noqa: E731
    x = np.maximum(rng.normal(size=shape(c)), -0.2) * np.exp(rng.normal(size=(1, c) + (1,) * (len(positions) - 1)))
    dy = 0.01 * rng.normal(size=shape(c_out)) * np.exp(rng.normal(size=(1, c_out) + (1,) * (len(positions) - 1)))
    return place(x, kind, pad, order), place(dy, kind, pad, order)


@pytest.mark.parametrize("code", ["e4m3", "i8"])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("positions,c,c_out", SIZES, ids=str)
def test_weight_gradient(positions, c, c_out, kind, code):
    from paper_1509_03371_amd import binding as B
    for i, (pad, order) in enumerate([(0, "dense"), (3, "dense"), (0, "last")]):
        x, dy = case(positions, c, c_out, kind, 90 + i, pad, order)
        p = B.pack8(x, code, axis=1)
        dw, db = B.weight_gradient8(dy, p)
        rw, rb, ew, eb = product_bounds(to64(dy), to64(B.unpack8(p)))
        close(dw, rw, ew, "dw")
        close(db, rb, eb, "db")
        again, none = B.weight_gradient8(dy, p, bias=False)
        assert none is None and torch.equal(again, dw), "two equal calls"
        w0, b0 = torch.randn(c_out, c, device="cuda"), torch.randn(c_out, device="cuda")
        w1, b1 = w0.clone(), b0.clone()
        B.weight_gradient8(dy, p, accumulate=True, dw=w1, db=b1)
        assert torch.equal(w1, w0 + dw) and torch.equal(b1, b0 + db)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("positions", [(70,), (2, 45)], ids=str)
def test_values_that_are_no_numbers_stay_in_their_channel(positions, kind):
    from paper_1509_03371_amd import binding as B
    for code in ("e4m3", "i8"):
        x, dy = case(positions, 100, 60, kind, 95)
        dw, db = B.weight_gradient8(dy, B.pack8(x, code, axis=1))
        where = (slice(None),) * 1
        xb, dyb = x.clone(), dy.clone()
        xb[1, 7, ...] = float("nan")
        dyb[1, 9, ...] = float("inf")
        wb, bb = B.weight_gradient8(dyb, B.pack8(xb, code, axis=1))
        other = torch.ones(60, 100, dtype=torch.bool, device="cuda")
        other[9], other[:, 7] = False, False
        assert torch.equal(wb[other], dw[other]) and torch.isnan(wb[:, 7]).all()
        assert not torch.isfinite(wb[9]).any() and bb[9] == float("inf") and torch.equal(bb[torch.arange(60) != 9], db[torch.arange(60) != 9]), where


def test_infinite_and_far_gradients():
    """An infinite gradient times positive inputs is infinite, not NaN; the largest and smallest fp32 gradients are whole."""
    from paper_1509_03371_amd import binding as B
    x = torch.ones(40, 33, device="cuda")
    p = B.pack8(x, "i8")
    for kind in TYPES:
        dy = torch.zeros(40, 5, dtype=TYPES[kind], device="cuda")
        dy[3, 1], dy[4, 2], dy[5, 3] = float("inf"), float("-inf"), float("nan")
        dw, db = B.weight_gradient8(dy, p)
        assert (dw[1] == float("inf")).all() and (dw[2] == float("-inf")).all() and torch.isnan(dw[3]).all() and (dw[0] == 0).all() and (dw[4] == 0).all()
        assert db[1] == float("inf") and db[2] == float("-inf") and torch.isnan(db[3])
    dy = torch.zeros(40, 5, device="cuda")
    dy[7, 0], dy[8, 1], dy[9, 2], dy[10, 3] = 3.4e38, -1.00000011920928955, 1e-30, 16777215.0
    dw, _ = B.weight_gradient8(dy, p)
    assert torch.equal(dw[:, 0], torch.stack([dy[7, 0], dy[8, 1], dy[9, 2], dy[10, 3], dy[0, 4]]))


def test_no_positions():
    from paper_1509_03371_amd import binding as B
    for shape, out in (((0, 5), (0, 3)), ((2, 5, 0), (2, 3, 0))):
        p = B.pack8(torch.empty(shape, device="cuda"), axis=1)
        dy = torch.empty(out, device="cuda")
        dw, db = torch.full((3, 5), 2.0, device="cuda"), torch.full((3,), 2.0, device="cuda")
        B.weight_gradient8(dy, p, accumulate=True, dw=dw, db=db)
        assert (dw == 2).all() and (db == 2).all()
        B.weight_gradient8(dy, p, dw=dw, db=db)
        assert (dw == 0).all() and (db == 0).all()


@pytest.mark.parametrize("code", ["e4m3", "i8"])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("positions,c,c_out", [((701,), 2050, 2101), ((3, 230), 2050, 2101), ((150,), 3000, 2900)], ids=str)
def test_many_weights(positions, c, c_out, kind, code):
    """Enough weights for the largest tiles, which end inside the tensors."""
    from paper_1509_03371_amd import binding as B
    x, dy = case(positions, c, c_out, kind, 97, 3 if kind == "f16" else 0)
    p = B.pack8(x, code, axis=1)
    dw, db = B.weight_gradient8(dy, p)
    rw, rb, ew, eb = product_bounds(to64(dy), to64(B.unpack8(p)))
    close(dw, rw, ew, "dw")
    close(db, rb, eb, "db")
    again = B.weight_gradient8(dy, p)
    assert torch.equal(again[0], dw) and torch.equal(again[1], db), "two equal calls"
