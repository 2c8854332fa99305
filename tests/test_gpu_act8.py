"""GPU: tensors into 8 bits and back, against the 64-bit oracle: codes, scales and values to the bit."""
import numpy as np
import pytest
import torch

from norm_bounds import TYPES, place, to64
from oracle import act8 as OA

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1), (3, 2), (5, 31), (4, 32), (7, 33), (300, 9), (64, 64), (65, 100), (33, 1024), (9, 777), (5, 4099), (2, 40001),
          (1, 1, 1), (2, 1, 77), (1, 3, 31), (3, 8, 1), (2, 9, 64), (1, 48, 1001), (2, 65, 333), (1, 200, 400), (4, 16, 33), (1, 1024, 49), (2, 777, 2), (1, 64, 5000)]


def values(shape, seed):
    """Lines whose blocks have unlike magnitudes."""
    rng = np.random.default_rng(seed)
    x = rng.normal(size=shape) * np.exp(rng.normal(size=shape[:-1] + (1,)))
    x *= np.exp2(np.repeat(rng.integers(-8, 8, size=shape[:-1] + (-(-shape[-1] // 32),)), 32, axis=-1)[..., :shape[-1]])
    x[rng.random(shape) < 0.1] = 0.0
    return x


def same(packed, x, kind, lines=lambda t: t):
    codes, scales = OA.pack(to64(lines(x)), packed.code, kind)
    assert np.array_equal(packed.scales.cpu().numpy(), scales), "scales"
    got = lines(packed.codes).cpu().numpy()
    bad = got != codes
    if packed.code == "e4m3":                       # either zero, either NaN
        bad &= ~(((got | codes) & 0x7F) == 0) & ~(((got & codes) & 0x7F) == 0x7F)
    assert not bad.any(), (got[bad][:5], codes[bad][:5])
    return OA.unpack(codes, scales, packed.code)


@pytest.mark.parametrize("code", ["e4m3", "i8"])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_pack_and_unpack(shape, kind, code):
    from paper_1509_03371_amd import binding as B
    for i, pad in enumerate((0, 5)):
        x = place(values(shape, i), kind, pad)
        p = B.pack8(x, code, axis=1)
        rows = len(shape) == 2 or (shape[2] == 1 and (pad == 0 or shape[1] == 1))      # one pixel an image: blocks of channels, if they are side by side
        assert p.order == ((B.SK_ROWS, shape[0], shape[1], 1) if rows else (B.SK_MAPS,) + shape)
        lines = (lambda t: t.reshape(shape[:2])) if rows else (lambda t: t)
        ref = same(p, x, kind, lines).reshape(shape)
        for other in TYPES:
            out = place(np.full(shape, 7.0), other, pad)
            assert B.unpack8(p, out=out) is out
            with np.errstate(over="ignore"):
                assert torch.equal(out.cpu(), torch.from_numpy(ref).to(TYPES[other])), other
            if pad:                                  # what lies between the lines stays
                assert torch.isnan(out._base[..., shape[-1]:]).all()
        assert np.array_equal(to64(B.unpack8(p)), ref)


@pytest.mark.parametrize("code", ["e4m3", "i8"])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_every_16_bit_value(kind, code):
    """Blocks of all values that a type of 16 bits has (fp32: those of bf16), each beside larger and smaller ones."""
    from paper_1509_03371_amd import binding as B
    bits = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16)
    v = bits.view(torch.float16 if kind == "f16" else torch.bfloat16).to(TYPES[kind])
    for x in (v.reshape(-1, 32), v.reshape(32, -1).t().contiguous(), v.reshape(-1, 1), v[torch.randperm(1 << 16, generator=torch.Generator().manual_seed(1))].reshape(-1, 64)):
        x = x.cuda()
        ref = same(B.pack8(x, code), x, kind)
        got = B.unpack8(B.pack8(x, code), dtype=TYPES[kind])
        assert torch.equal(got.cpu().nan_to_num(7.0), torch.from_numpy(ref).to(TYPES[kind]).nan_to_num(7.0))
        finite = torch.isfinite(x)
        assert torch.isfinite(got[finite]).all() and torch.isnan(got[~finite]).all()


@pytest.mark.parametrize("code", ["e4m3", "i8"])
def test_borders_of_scales_and_codes(code):
    """fp32 values on, just under and just over the borders where a block's scale or a code changes."""
    from paper_1509_03371_amd import binding as B
    top = OA.TOP[code]
    x = []
    for k in (-117, -60, -1, 0, 5, 100, 119):
        for edge in (top, top / 2, 1.0):
            v = np.float32(edge * 2.0 ** k)
            x += [[w] + [np.float32(0)] * 31 for w in (np.nextafter(v, np.float32(0)), v, np.nextafter(v, np.float32(np.inf)))]
    codes = OA.e4m3_table()[:127] if code == "e4m3" else np.arange(128.0)
    half = ((codes[1:] + codes[:-1]) / 2).astype(np.float32)
    for w in (np.nextafter(half, np.float32(0)), half, np.nextafter(half, np.float32(500))):
        w = np.concatenate([w, -w])
        x += [[np.float32(top)] + list(part) + [np.float32(0)] * (31 - len(part)) for part in np.array_split(w, 12)]
    x = torch.from_numpy(np.array(x, np.float32)).cuda()
    same(B.pack8(x, code), x, "f32")


@pytest.mark.parametrize("code", ["e4m3", "i8"])
@pytest.mark.parametrize("shape", [(6, 200), (2, 3, 200), (3, 40, 7)], ids=str)
def test_what_is_no_number_stays_alone(shape, code):
    from paper_1509_03371_amd import binding as B
    for kind in TYPES:
        x = place(values(shape, 3), kind)
        x.view(-1)[::7] = float("inf")
        x.view(-1)[3::11] = float("nan")
        x.view(-1)[5::13] = float("-inf")
        x[..., -5:] = float("nan")
        ref = same(B.pack8(x, code, axis=1), x, kind)
        got = B.unpack8(B.pack8(x, code, axis=1), dtype=TYPES[kind])
        assert torch.equal(torch.isnan(got), ~torch.isfinite(x))
        assert np.array_equal(to64(got), to64(torch.from_numpy(ref).to(TYPES[kind])), equal_nan=True)


def test_orders_of_axes():
    """Channels last in memory are rows, channels in front of pixels are maps, whatever the number of axes."""
    from paper_1509_03371_amd import binding as B
    x = torch.from_numpy(values((2, 40, 6, 7), 4)).float().cuda()
    p = B.pack8(x, "i8", axis=1)
    assert p.order == (B.SK_MAPS, 2, 40, 42) and p.scales.shape == (2, 40, 2)
    same(p, x, "f32", lambda t: t.reshape(2, 40, 42))
    last = x.to(memory_format=torch.channels_last)
    q = B.pack8(last, "i8", axis=1)
    assert q.order == (B.SK_ROWS, 84, 40, 1) and q.scales.shape == (84, 2)
    same(q, last, "f32", lambda t: t.permute(0, 2, 3, 1).reshape(84, 40))
    out = B.unpack8(q, dtype=torch.float32)
    assert out.stride() == last.stride()
    one = B.pack8(x[:, :1].contiguous(), "i8", axis=1)
    assert one.order[0] == B.SK_MAPS
    for shape, axis in (((0, 5), 1), ((3, 5, 0), 1), ((0, 4, 9), 1)):
        empty = torch.empty(shape, device="cuda")
        assert B.unpack8(B.pack8(empty, axis=axis)).shape == shape
