"""Grids and workgroups that the 8-bit cache's entry points launch, without a GPU: the
launch configurations that the library hands to the HIP runtime are recorded and the
launches left out (a preloaded library), in a process of its own.  256 CUs, as on
MI355X, without a device.  And the registers that its kernels take."""
import os
import shutil
import subprocess
import sys

import pytest

from paper_2406_18832_amd import build_lib, ot
from tests.test_kernel_resources import kernel_resources

RECORDER = r"""
#include <stddef.h>
#include <stdint.h>
struct dim3 { uint32_t x, y, z; };
extern "C" {
uint64_t ot_test_sizes[4][6], ot_test_launches;
int __hipPushCallConfiguration(dim3 g, dim3 b, size_t, void *) {
  const uint32_t v[6] = {g.x, g.y, g.z, b.x, b.y, b.z};
  for (int i = 0; i < 6; ++i) ot_test_sizes[ot_test_launches & 3][i] = v[i];
  ++ot_test_launches;
  return 1;  // nonzero: the launch is left out
}
int hipGetLastError(void) { return 0; }  // and has not failed, without a device
}
"""

CALLER = r"""
import ctypes, sys
R, L = ctypes.CDLL(sys.argv[1]), ctypes.CDLL(sys.argv[2])
sizes = ((ctypes.c_uint64 * 6) * 4).in_dll(R, "ot_test_sizes")
launches = ctypes.c_uint64.in_dll(R, "ot_test_launches")
vp, i64, ci, f = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_float
p = vp(4096)   # aligned, never read
for line in sys.stdin:
    name, *n = line.split()
    T, B, Hq, H, D, q, window, pages, ws = (i64(int(x)) for x in n)
    ld = i64(Hq.value * D.value)
    launches.value = 0
    if name == "append":
        rc = L.ot_kv8_append(p, ld, p, ld, T, B, H, D, p, p, p, pages, i64(1 << 20), p, p, p, p, None)
    elif name == "read":
        rc = L.ot_kv8_read(p, p, p, p, i64(1 << 20), p, p, p, pages, T, B, H, D, p, p, None)
    else:
        rc = L.ot_attn_kv8(p, ld, T, B, Hq, H, D, p, p, p, pages, i64(1 << 20), p, p, p, p, f(0.1), ci(1),
                           window, q, p, p, p if ws.value else None, None)
    print(rc, launches.value, *(v for i in range(min(launches.value, 4)) for v in sizes[i]), flush=True)
"""


@pytest.fixture(scope="module")
def launch(tmp_path_factory):
    """launch([(call, T, B, Hq, Hkv, D, max_q, window, max_pages, workspace), ...]) ->
    [(status, [(grid, block), ...]), ...]."""
    d = tmp_path_factory.mktemp("launches")
    src, so = d / "recorder.cpp", d / "recorder.so"
    src.write_text(RECORDER)
    subprocess.run([os.environ.get("CXX") or shutil.which("g++") or "c++", "-shared", "-fPIC", "-O1",
                    str(src), "-o", str(so)], check=True)

    def run(calls):
        env = dict(os.environ, LD_PRELOAD=str(so))
        out = subprocess.run([sys.executable, "-c", CALLER, str(so), ot.LIB_PATH], env=env,
                             input="".join(" ".join(map(str, c)) + "\n" for c in calls), text=True,
                             capture_output=True, timeout=300)
        assert out.returncode == 0, out.stderr[-2000:]
        rows = [[int(v) for v in line.split()] for line in out.stdout.splitlines()]
        assert len(rows) == len(calls)
        return [(r[0], [(r[2 + 6 * i:5 + 6 * i], r[5 + 6 * i:8 + 6 * i]) for i in range(r[1])])
                for r in rows]
    return run


def within_limits(launches):
    for grid, block in launches:
        assert all(g >= 1 for g in grid) and grid[1] < 65536 and grid[2] < 65536
        assert all(g * b < 1 << 32 for g, b in zip(grid, block)), (grid, block)
        assert block[0] * block[1] * block[2] <= 1024


# T, B, Hq, Hkv, D, max_q: the most tokens, sequences and heads in many proportions
SIZES = [(T, B, H * G, H, D, q) for T in (1, 100, 65535, 1 << 20, 1 << 24) for B in (1, 64, 65, 8192, 65535)
         for H, G in ((1, 1), (1, 64), (40, 1), (127, 1), (128, 1), (250, 1), (255, 3), (1024, 16))
         for D in (64, 128, 192) for q in sorted({1, min(T, 40), T})]


def test_every_launch_stays_within_its_limits(launch):
    calls = [("attend", *s, 0, 4000, w) for s in SIZES for w in (0, 1)]
    calls += [(name, T, B, H, H, D, 1, 0, 4000, 0) for name in ("append", "read")
              for T, B, Hq, H, D, q in SIZES if q == 1]
    done = 0
    for c, (rc, launches) in zip(calls, launch(calls)):
        assert rc in (ot.OT_OK, ot.OT_ESHAPE), c
        assert bool(launches) == (rc == ot.OT_OK), c
        within_limits(launches)
        done += rc == ot.OT_OK
    assert len(calls) / 2 < done < len(calls)


def test_windows_of_any_size(launch):
    """A window past every position is none."""
    calls = [("attend", 300, 2, 4, 4, 64, 300, w, pages, 1) for pages in (8, 4000)
             for w in (1 << 30, (1 << 31) - 1, 1 << 31, (1 << 63) - 1)]
    got = launch(calls)
    assert all(g[0] == ot.OT_OK for g in got)
    assert got[1:4] == [got[0]] * 3 and got[5:] == [got[4]] * 3
    assert len(got[0][1]) == 1 and len(got[4][1]) == 2  # short tables: no join


def test_few_rows_take_one_launch_where_tables_are_short(launch):
    calls = [("attend", 4, 4, 8, 8, 64, 1, 0, pages, ws) for pages in (16, 17) for ws in (0, 1)]
    assert [len(g[1]) for g in launch(calls)] == [1, 1, 1, 2]


def test_windows_choose_launches(launch):
    """Windows of few pages: no joining, and tiles of 128 rows."""
    calls = [("attend", 4, 4, 8, 8, 64, 1, w, 4000, 1) for w in (1, 800, 2000)]
    assert [len(g[1]) for g in launch(calls)] == [1, 1, 2]
    calls = [("attend", 8192, 1, 40, 40, 112, 8192, w, 4000, ws) for w in (0, 1500, 1499, 5) for ws in (0, 1)]
    assert [g[1][0][1][0] for g in launch(calls)] == [512] * 4 + [256] * 4
    assert all(len(g[1]) == 1 for g in launch(calls))


def test_plans_say_how_tiles_are_shared():
    plan, size = ot.ot_attn_kv8_plan, ot.ot_attn_kv8_workspace_size
    assert plan(64, 1, 8, 8, 128, 64, True) == "tiles 128, 64 parts" and size(64, 1, 8, 8, 128, 64) > 0
    assert plan(64, 1, 8, 8, 128, 64) == "tiles 128"
    for s in ((8192, 1, 72, 72, 128, 8192), (4096, 64, 40, 40, 128, 64), (4096, 1, 64, 64, 160, 4096)):
        # as many tiles as the device takes at a time, several times over
        assert plan(*s, True) == plan(*s) == f"tiles {256 if s[4] == 160 or s[0] == 8192 else 128}"
        assert size(*s) == 0


@pytest.mark.timeout(900)
@pytest.mark.parametrize("src", ["ot_kv8_cache.hip", "ot_kv8_decode.hip", "ot_kv8_tiles.hip"])
def test_kernels_do_not_spill(src, tmp_path):
    res = kernel_resources(os.path.join(build_lib.CSRC, src), tmp_path)
    kernels = {k: v for k, v in res.items() if "kv8" in k}
    assert len(kernels) >= 5
    assert not {k: v for k, v in kernels.items() if v["spill"] is None or v["spill"] > 0}
