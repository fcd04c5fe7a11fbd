"""Grids of the paged cache's calls beyond one launch (no GPU needed): the arithmetic by itself, and what the calls launch, with a stand-in for the runtime's side of a
launch that writes down the grid and starts nothing (addresses are made up and never dereferenced)."""
import json
import os
import shutil
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2510_13797_amd", "csrc")


def _compiler():
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no host compiler")
    return cxx


def test_launches_stay_below_what_one_takes(tmp_path):
    exe = str(tmp_path / "paged_grid_model")
    subprocess.check_call([_compiler(), "-std=c++17", "-O2", "-Wall", "-Werror", "-I", CSRC, "-o", exe, os.path.join(HERE, "paged_grid_model.cpp")])
    cases = [(g, t) for t in (64, 128, 256, 1024) for g in (1, 5, 255, (1 << 21) - 1, 1 << 21, (1 << 21) + 1, (1 << 24) - 1, 1 << 24, 512 * 32769, (1 << 31) - 1)]
    out = subprocess.run([exe], input="".join("%d %d\n" % c for c in cases).encode(), stdout=subprocess.PIPE, timeout=60, check=True).stdout.decode()
    rows = [dict((k, int(v)) for k, v in (x.split("=") for x in l.split())) for l in out.split("\n") if l]
    assert len(rows) == len(cases)
    for (groups, threads), r in zip(cases, rows):
        assert r["all"] == groups and r["joined"] and r["most"] < 1 << 32, (groups, threads, r)
        assert r["launches"] == -(-groups * threads // (1 << 31)), (groups, threads, r)


LAUNCH = r"""
struct Dim3 { unsigned x, y, z; };
static unsigned long long seen[1 << 16][2];
static int n;
extern "C" int __hipPushCallConfiguration(Dim3 grid, Dim3 block, unsigned long, void*) {
  seen[n][0] = (unsigned long long)grid.x * grid.y * grid.z;
  seen[n++][1] = (unsigned long long)block.x * block.y * block.z;
  return 1;
}
extern "C" int launches() { return n; }
extern "C" unsigned long long launched(int i, int what) { return seen[i][what]; }
"""
CALLS = r"""
import ctypes as C, json, sys
stand_in = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)
stand_in.launched.restype = C.c_ulonglong
sys.path.insert(0, sys.argv[2])
from paper_2510_13797_amd import bc
P, got = 0x7F0000100000, []
for call, B, Hq, Hkv, d, rows, max_new, page_rows, table_pages in json.loads(sys.argv[3]):
    at = stand_in.launches()
    shape, pages = bc.bc_shape(B, Hq, Hkv, d, bc.BC_BF16, 1.0), bc.bc_pages(*[P] * 8, 9, page_rows, table_pages, 0)
    if call == "append":
        bc.bc_paged_append(shape, pages, rows, P, max_new, P, (Hq + 2 * Hkv) * d, P, P, d, None, None, 1e-6, None, None, P + 4096, None)
    else:
        bc.bc_paged_attend(shape, pages, rows, P, max_new, P, P, None, P, 1 << 60, None)
    got.append([[stand_in.launched(i, w) for w in (0, 1)] for i in range(at, stand_in.launches())])
print(json.dumps(got))
"""


def test_no_launch_is_larger_than_the_runtime_takes(tmp_path):
    shim = str(tmp_path / "launch.so")
    (tmp_path / "launch.cpp").write_text(LAUNCH)
    subprocess.check_call([_compiler(), "-O1", "-shared", "-fPIC", "-o", shim, str(tmp_path / "launch.cpp")])
    calls = [("append", 512, 1, 1, 128, 512 * 1024, 512 * 1024, 1024, 1),                 # chunks whose longest is not given: each may have all rows
             ("append", 512, 1, 1, 64, 1 << 20, 1 << 20, 1024, 1),
             ("append", 8192, 8, 1, 128, 1 << 21, 1 << 21, 16, 4),
             ("append", 64, 12, 2, 128, 64, 64, 16, 4),
             ("append", 1 << 23, 8, 1, 128, 1 << 23, 1, 16, 4), ("append", 4096, 16384, 2048, 128, 4096, 1, 16, 4),
             ("attend", 4096, 8, 1, 64, 1 << 16, 1 << 16, 16, 4096),
             ("attend", 1024, 8, 1, 128, 1 << 18, 1 << 18, 1024, 1024),
             ("attend", 1 << 23, 8, 1, 128, 1 << 23, 1, 1024, 1 << 20), ("attend", 1 << 23, 8, 1, 128, 1 << 23, 4, 1024, 1 << 20),
             ("attend", 1 << 20, 8, 1, 128, 100, 16, 1024, 1 << 20),
             ("attend", 16, 32, 8, 128, 16, 1, 1024, 30)]
    out = subprocess.run([sys.executable, "-c", CALLS, shim, os.path.dirname(HERE), json.dumps(calls)], stdout=subprocess.PIPE, timeout=300, check=True).stdout.decode()
    launches = json.loads(out.strip().split("\n")[-1])
    assert len(launches) == len(calls)
    for call, these in zip(calls, launches):
        assert these, call
        for groups, threads in these:
            assert groups * threads < 1 << 32, (call, these)
    # all of a call's workgroups are out: of the block kernel a workgroup for 16 rows and one more, of the attention's one for 128 columns
    assert sum(g for g, _ in launches[0]) == 512 * 32769 and sum(g for g, _ in launches[6]) == 4096 * 4096
    assert [len(these) for these in launches][3] == 1 and len(launches[-1]) == 1
