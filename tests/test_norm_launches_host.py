"""CPU: what the host code of layer norm's gradient launches, and what it says of a launch that fails.  A program that has the few runtime calls of a launch
in itself loads the library, which then launches there: each grid is looked at, and one launch after the other is made to fail."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <dlfcn.h>
#include "sknet.h"

struct Dim { uint32_t x, y, z; };
static int launches, failing, last_error, too_large;
static long groups[8];
static Dim grid_, block_;
static size_t lds_;
static void *stream_;
extern "C" {
int __hipPushCallConfiguration(Dim g, Dim b, size_t lds, void *s) { grid_ = g; block_ = b; lds_ = lds; stream_ = s; return 0; }
int __hipPopCallConfiguration(Dim *g, Dim *b, size_t *lds, void **s) { *g = grid_; *b = block_; *lds = lds_; *s = stream_; return 0; }
int hipLaunchKernel(const void *, Dim g, Dim b, void **, size_t lds, void *)
{
    if (launches < 8) groups[launches] = (long)g.x * g.y;
    ++launches;
    const uint32_t most = 0xffffffffu;                  // threads of a grid along an axis
    if ((uint64_t)g.x * b.x > most || (uint64_t)g.y * b.y > 65535u * 1024u || !g.x || !g.y || !b.x || b.x * b.y * b.z > 1024 || lds > 160 * 1024) ++too_large;
    return last_error = launches == failing ? 719 : last_error;
}
int hipGetLastError() { const int e = last_error; last_error = 0; return e; }
const char *hipGetErrorString(int) { return "failed"; }
}

int main(int argc, char **argv)
{
    void *lib = dlopen(argv[1], RTLD_NOW);
    if (!lib) { printf("%s\n", dlerror()); return 2; }
    auto backward = (decltype(&sknet_layer_norm_backward))dlsym(lib, "sknet_layer_norm_backward");
    auto space = (decltype(&sknet_layer_norm_workspace))dlsym(lib, "sknet_layer_norm_workspace");
    const sk_extent e{atoi(argv[2]), atoi(argv[3]), atol(argv[4]), atol(argv[5]), atol(argv[6])};
    const int adds = atoi(argv[7]), in_place = atoi(argv[8]);
    const int64_t sc = e.layout == SK_ROWS ? 0 : e.plane, sn = atol(argv[9]) ? atol(argv[9]) : e.c * e.plane;
    uint64_t need = 0;
    if (space(&e, &need) != SK_OK) return 3;
    auto at = [](int i) { return (void *)((uintptr_t)(i + 1) << 50); };       // addresses that nothing follows
    sk_view v[5];
    for (int i = 0; i < 5; ++i) v[i] = sk_view{at(i), sn, sc};
    const sk_drop drop{0.5, 1, 2, nullptr};
    int made = 0;
    for (failing = 0; failing == 0 || failing <= made; ++failing) {
        launches = last_error = 0;
        const sk_status s = backward(&e, &v[0], &v[1], (float *)at(5), (float *)at(6), (float *)at(7), adds ? &v[2] : nullptr, adds ? &drop : nullptr,
                                     in_place ? &v[0] : &v[3], adds ? &v[4] : nullptr, (float *)at(8), (float *)at(9), need ? at(10) : nullptr, need, nullptr);
        if (!failing) made = launches;
        printf("%s%d:%d", failing ? " " : "", failing, (int)s);
        if (failing) continue;
        for (int i = 0; i < made; ++i) printf("%s%ld", i ? "," : " groups ", groups[i]);
    }
    printf(" launches %d too large %d\n", made, too_large);
    return 0;
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    from paper_1509_03371_amd import binding as B
    d = tmp_path_factory.mktemp("launches")
    (d / "main.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-rdynamic", "-I", os.path.join(ROOT, "include"), str(d / "main.cpp"), "-o", str(d / "main"), "-ldl"], check=True)
    return lambda *a: subprocess.run([str(d / "main"), B.LIB_PATH] + [str(int(x)) for x in a], capture_output=True, text=True, timeout=60)


ROWS, MAPS = 0, 1
#   layout, n, c, plane, stride of rows (0: dense), launches
CALLS = {
    "one workgroup": (ROWS, 8, 7, 1, 0, 1),
    "roles": (ROWS, 100, 300, 1, 0, 1),
    "copies": (ROWS, 100000, 64, 1, 0, 2),
    "long rows": (ROWS, 40, 20000, 1, 0, 3),
    "rows far apart": (ROWS, 5000, 40, 1, 1 << 24, 2),
    "maps with roles": (MAPS, 1, 64, 900, 0, 1),
    "maps with copies": (MAPS, 4, 64, 10000, 0, 2),
    "many maps": (MAPS, 4, 3000, 1000, 0, 3),
    "small planes": (MAPS, 300, 64, 2, 0, 3),
    "the most channels": (ROWS, 2, 1 << 27, 1, 0, 3),
}


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("adds,in_place", [(0, 0), (1, 0), (0, 1)])
def test_a_failed_launch_is_reported(program, name, dtype, adds, in_place):
    layout, n, c, plane, stride, launches = CALLS[name]
    if in_place and "roles" in name:
        launches += 1                                   # the sums first
    r = program(dtype, layout, n, c, plane, adds, in_place, stride)
    assert r.returncode == 0, r.stdout + r.stderr
    words = r.stdout.split()
    assert words[0] == "0:0" and "launches %d " % launches in r.stdout, r.stdout
    assert words[3:3 + launches] == ["%d:5" % (i + 1) for i in range(launches)], r.stdout       # SK_EDEVICE whichever it was


EMPTY = {"no rows, the most channels": (ROWS, 0, 1 << 27, 1, 0, 1), "no pixels": (MAPS, 3, 1 << 27, 0, 0, 1), "many rows": (ROWS, 1 << 36, 8, 1, 0, 2),
         "many rows of wide gaps": (ROWS, 1 << 26, 64, 1, 1 << 20, 2), "many images": (MAPS, 1 << 36, 9, 3, 0, 3), "one long plane": (MAPS, 1, 24, 1 << 36, 0, 2),
         "the most channels of maps": (MAPS, 40, 1 << 27, 3, 0, 3)}


@pytest.mark.parametrize("name", list(CALLS) + list(EMPTY))
@pytest.mark.parametrize("dtype", [0, 1])
def test_grids_fit_a_launch(program, name, dtype):
    # 2^32 - 1 threads along an axis: a workgroup of 256 for each sixteen of 2^28 sums would be one more
    layout, n, c, plane, stride, launches = {**CALLS, **EMPTY}[name]
    r = program(dtype, layout, n, c, plane, 0, 0, stride)
    assert r.returncode == 0 and "launches %d too large 0" % launches in r.stdout, r.stdout


def test_sums_of_small_planes_are_shared_out(program):
    # planes of two pixels of a million images: waves for the card, not sixteen shares of images
    r = program(0, MAPS, 1 << 20, 64, 2, 0, 0, 0)
    assert r.returncode == 0
    assert int(r.stdout.split("groups ")[1].split()[0].split(",")[0]) >= 1024, r.stdout


@pytest.mark.parametrize("c", [40, 300, 6000])
def test_rows_far_apart_take_as_many_workgroups(program, c):
    # few rows, one launch: those with the results, and those with the sums of 64 channels each
    asked = []
    for stride in (0, 1 << 24):
        r = program(0, ROWS, 400, c, 1, 0, 0, stride)
        assert r.returncode == 0 and "launches 1 " in r.stdout, r.stdout
        asked.append(int(r.stdout.split("groups ")[1].split()[0]))
    assert asked[1] >= asked[0] > 1, asked
