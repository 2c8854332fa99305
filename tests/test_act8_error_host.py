"""CPU: how far codes may be off, as the header states it, on the oracle: ordinary blocks, the least scale, values beyond what codes can stand for."""
import numpy as np
import pytest

from oracle import act8 as OA

MOST = {"f16": 65504.0, "f32": float(np.finfo(np.float32).max)}


@pytest.mark.parametrize("code", ["e4m3", "i8"])
@pytest.mark.parametrize("kind", ["f32", "f16"])
def test_half_a_step(code, kind):
    rng = np.random.default_rng(7)
    limit = OA.LIMIT[code, kind]
    low = -140 if kind == "f32" else -24
    largest = np.concatenate([np.exp2(rng.uniform(low, np.log2(limit), 4000)), [limit, np.nextafter(limit, 0), 2.0 ** -120, 2.0 ** -118, 127 * 2.0 ** -117, 448 * 2.0 ** -117, 0.0]])
    x = np.clip(largest[:, None] * np.concatenate([np.ones((len(largest), 1)), rng.uniform(-1, 1, (len(largest), 31)) ** 3], axis=1), -limit, limit)
    codes, scales = OA.pack(x, code, kind)
    k = scales.astype(float) - 127
    off = np.abs(OA.unpack(codes, scales, code) - x)
    most = np.abs(x).max(axis=1, keepdims=True)
    if code == "e4m3":
        assert (off <= np.where(np.abs(x) < 2.0 ** (k - 6), 2.0 ** (k - 10), 2.0 ** -4 * np.abs(x))).all()
    else:
        assert (off <= 2.0 ** (k - 1)).all()
        assert ((2.0 ** (k - 1) < most / 126) | (k == -117)).all()
    if kind == "f32":                                  # the least scale: steps that do not shrink with the block
        assert ((k == -117) & (most > 0) & (off.max(axis=1, keepdims=True) > most / 126)).any()


@pytest.mark.parametrize("code", ["e4m3", "i8"])
@pytest.mark.parametrize("kind", ["f32", "f16"])
def test_limited(code, kind):
    limit = OA.LIMIT[code, kind]
    assert limit < MOST[kind]
    x = np.array([[MOST[kind], -MOST[kind], limit, 1.0] + [0.0] * 28])
    codes, scales = OA.pack(x, code, kind)
    assert np.array_equal(OA.unpack(codes, scales, code)[0, :3], [limit, -limit, limit])
    assert scales[0, 0] <= 247
