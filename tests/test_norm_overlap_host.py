"""CPU: which views of one buffer layer norm takes as apart, against the sets of their elements.  No call gets as far as a launch: the address of the means, which
is checked behind the views, is refused."""
import ctypes as C
import itertools
import random

import numpy as np

from paper_1509_03371_amd import binding as B

BASE = 0x100000


def answer(extent, x, y, s=None):
    """'overlap', 'apart', or 'itself' for an output two of whose elements share a place."""
    status = B.lib.sknet_layer_norm(C.byref(extent), C.byref(x), None, None, None, None, 1e-5, None if s is None else C.byref(s), C.byref(y), 0x90000002, None, None)
    text = B.lib.sknet_last_error().decode()
    assert status, "accepted"
    if "mean is not aligned" in text:
        return "apart"
    if "elements of" in text:
        return "itself"
    assert "overlap" in text, text
    return "overlap"


def places(extent, view, size):
    """Byte addresses of every element's bytes, one row an element."""
    n, c, m = (np.arange(k) for k in (extent.n, extent.c, extent.plane))
    if extent.layout == B.SK_ROWS:
        at = n[:, None] * view.stride_n + c[None, :]
    else:
        at = n[:, None, None] * view.stride_n + c[None, :, None] * view.stride_c + m[None, None, :]
    return (view.data + size * at.reshape(-1)[:, None] + np.arange(size)).reshape(-1)


def expected(extent, a, b, size):
    pa, pb = places(extent, a, size), places(extent, b, size)
    if len(np.unique(pb)) != len(pb):
        return "itself"
    return "overlap" if len(np.intersect1d(pa, pb)) else "apart"


def test_images_whose_distance_is_no_multiple_of_the_maps():
    e = B.SkExtent(B.SK_F32, B.SK_MAPS, 2, 2, 2)
    x, y = B.SkView(BASE, 20, 8), B.SkView(BASE + 4 * 12, 20, 8)          # elements 20 and 21 are in both
    assert expected(e, x, y, 4) == "overlap" and answer(e, x, y) == "overlap"
    other = B.SkView(BASE + 0x10000, 20, 8)
    assert answer(e, other, y, x) == "overlap"                            # two outputs
    drop = B.SkDrop(0.5, 1, 2, None)
    assert B.STATUS_NAMES[B.lib.sknet_dropout(C.byref(e), C.byref(x), C.byref(y), C.byref(drop), None)] == "SK_EINVAL"
    maps_outside = B.SkView(BASE, 8, 20), B.SkView(BASE + 4 * 12, 8, 20)
    assert answer(e, *maps_outside) == "overlap"


def test_equal_strides_against_sets_of_elements():
    seen = {"overlap": 0, "apart": 0}
    for n, c, plane in itertools.product((1, 2, 3), (1, 2, 4), (1, 2, 3)):
        e = B.SkExtent(B.SK_F32, B.SK_MAPS, n, c, plane)
        for sn, sc in itertools.product((1, 2, 3, 5, 8, 13, 20, 24), (1, 2, 3, 4, 7, 8, 17)):
            for off in (-33, -20, -13, -8, -5, -3, -2, -1, 1, 2, 3, 4, 6, 7, 9, 12, 16, 21, 34):
                x, y = B.SkView(BASE, sn, sc), B.SkView(BASE + 4 * off, sn, sc)
                want = expected(e, x, y, 4)
                got = answer(e, x, y)
                if got == "itself" and want != "itself":              # lines of an output that interleave are refused without sharing an element
                    assert sn < (c - 1) * sc + plane and sc < (n - 1) * sn + plane
                    continue
                assert got == want, (n, c, plane, sn, sc, off)
                if want != "itself":
                    seen[want] += 1
    assert min(seen.values()) > 1000
    rows = 0
    for n, c, sn, off in itertools.product((1, 2, 3), (1, 2, 5), (1, 2, 5, 6, 11), range(-30, 31)):
        if off == 0:
            continue
        e = B.SkExtent(B.SK_BF16, B.SK_ROWS, n, c, 1)
        x, y = B.SkView(BASE, sn, 0), B.SkView(BASE + 2 * off, sn, 0)
        want = expected(e, x, y, 2)
        assert answer(e, x, y) == want, (n, c, sn, off)
        rows += want == "apart"
    assert rows > 100


def test_other_strides_never_pass_where_elements_meet():
    # (views of unlike strides whose ranges cross may be refused without sharing an element)
    rng = random.Random(4)
    met = 0
    for _ in range(4000):
        n, c, plane = rng.randint(1, 3), rng.randint(1, 4), rng.randint(1, 4)
        e = B.SkExtent(B.SK_F16, B.SK_MAPS, n, c, plane)
        x = B.SkView(BASE, rng.randint(0, 25), rng.randint(0, 9))
        y = B.SkView(BASE + 2 * rng.randint(-60, 60), rng.randint(0, 25), rng.randint(0, 9))
        same = x.data == y.data and (n == 1 or x.stride_n == y.stride_n) and (c == 1 or x.stride_c == y.stride_c)
        got, want = answer(e, x, y), expected(e, x, y, 2)
        if same and got == "apart":                    # in place, element for element
            continue
        if want == "overlap":
            met += 1
            assert got != "apart", (n, c, plane, x.stride_n, x.stride_c, y.data - BASE, y.stride_n, y.stride_c)
    assert met > 500
