"""What products in 8-bit floating point read of their operands, without a GPU: a workgroup's
buffers are as long as its tiles in every form, up to the longest inputs; and that no product is
refused for a launch that it does not make."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CODE = """
#include "f8_plan.h"
using namespace qlm_f8_host;
extern "C" void form(int n_out, int n_in, int rows, int *got)
{
    const Parts p = parts_of(n_out, n_in, rows);
    const int all[] = {p.n_first, p.first.side, p.first.splits, p.first.per_split, p.rest.side};
    for (int i = 0; i < 5; ++i) got[i] = all[i];
}
extern "C" int fit(int n_out, int n_in, int rows)
{
    const Parts p = parts_of(n_out, n_in, rows);
    return fits(n_out, n_in, p.n_first, p.first) &&
           (p.n_first == rows || fits(n_out, n_in, rows - p.n_first, p.rest));
}
extern "C" int bytes(int left, int own, int blocks, int b0) { return load_bytes(left, own, blocks, b0); }
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("reads")
    (d / "plan.cpp").write_text(CODE)
    lib = str(d / "plan.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-I",
                    os.path.join(ROOT, "paper_2407_00047_amd", "csrc"), "-o", lib,
                    str(d / "plan.cpp")], check=True)
    return ctypes.CDLL(lib)


def test_buffers_are_as_long_as_a_workgroups_tiles(plan):
    seen = set()
    for n_in in (1, 129, 16384, 1 << 20, (1 << 22) - 127, 1 << 23, (1 << 23) + 1, (1 << 24) - 128,
                 (1 << 24) - 127, 1 << 24):
        blocks = -(-n_in // 128)
        for n_out in (16, 300, 1000, 4096, 20001):
            for rows in (100, 256, 257, 512, 700, 1024, 4100):
                got = (ctypes.c_int * 5)()
                plan.form(n_out, n_in, rows, got)
                n_first, side, splits, per, rest = got
                forms = [(side, splits, per, n_first)]
                if n_first < rows:
                    forms.append((rest, 1, blocks, rows - n_first))
                for side, splits, per, m in forms:
                    if not side:
                        continue
                    own = side // 16
                    for have in (-(-m // 16), -(-n_out // 16)):
                        for first in {0, (have - 1) // own * own}:
                            for split in {0, splits - 1}:
                                b0, tiles = split * per, min(have - first, own)
                                # (from the first tile's block b0 to the end of the last tile)
                                want = (tiles * blocks - b0) * 2048
                                assert want < 1 << 31
                                assert plan.bytes(have - first, own, blocks, b0) == want, \
                                    (rows, n_out, n_in, side, have, first, split)
                                seen.add((side, n_in >= 1 << 23))
    assert {(64, True), (64, False), (128, False), (256, False)} <= seen, seen


@pytest.mark.parametrize("rows,n_out,n_in", [(131072, 131072, 128), (131077, 131072, 100),
                                             (65536, 262144, 4096), (1 << 20, 100000, 1000),
                                             (1024, 1 << 24, 64), (1 << 24, 1 << 16, 128),
                                             (640, 1 << 24, 5000), (2000000000, 128, 128)])
def test_many_outputs_are_not_refused(plan, rows, n_out, n_in):
    """2^34 outputs and more, of whose sums none are joined."""
    got = (ctypes.c_int * 5)()
    plan.form(n_out, n_in, rows, got)
    assert got[2] == 1
    assert plan.fit(n_out, n_in, rows)


def test_what_cannot_be_launched_is_refused(plan):
    """Tiles that 32 bits do not count."""
    assert not plan.fit(1 << 24, 128, (1 << 31) - 17)
    assert not plan.fit(1 << 24, 1 << 24, (1 << 31) - 17)
