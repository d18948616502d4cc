"""How products in 8-bit floating point choose their form, without a GPU: the runs of inputs and the
parts of rows cover everything once, offsets fit, and the sizes that the GPU tests take reach
every form."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CODE = """
#include "f8_plan.h"
using namespace qlm_f8_host;
extern "C" void parts(int n_out, int n_in, int rows, int *got)
{
    const Parts p = parts_of(n_out, n_in, rows);
    const int all[] = {p.n_first, p.first.side, p.first.splits, p.first.per_split,
                       p.rest.side, p.rest.splits, p.rest.per_split};
    const int more[] = {p.first.one_more, p.rest.one_more};
    for (int i = 0; i < 2; ++i) got[7 + i] = more[i];
    for (int i = 0; i < 7; ++i) got[i] = all[i];
}
extern "C" void thin(int n_out, int n_in, int rows, int *got)
{
    const Thin t = thin_of((n_out + 15ll) / 16, (rows + 15ll) / 16, (n_in + 127) / 128);
    got[0] = t.outs;
    got[1] = t.rows;
}
"""


@pytest.fixture(scope="module")
def parts(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cpp").write_text(CODE)
    lib = str(d / "plan.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-I",
                    os.path.join(ROOT, "paper_2407_00047_amd", "csrc"), "-o", lib,
                    str(d / "plan.cpp")], check=True)
    lib = ctypes.CDLL(lib)

    def call(rows, n_out, n_in, what=lib.parts, n=7):
        got = (ctypes.c_int * 9)()
        what(n_out, n_in, rows, got)
        return list(got)[:n]

    call.more = lambda *sizes: call(*sizes, n=9)[7:]     # a last tile of rows taken along
    call.thin = lambda *sizes: tuple(call(*sizes, what=lib.thin)[:2])
    return call


def test_everything_is_taken_once(parts):
    for n_out in (1, 15, 16, 100, 129, 1000, 4097, 20001, 1 << 20, 1 << 24):
        for n_in in (1, 128, 129, 640, 5000, 16384, 1 << 17, (1 << 20) + 1, 1 << 23, 1 << 24):
            blocks = -(-n_in // 128)
            for rows in (1, 16, 17, 64, 65, 255, 256, 257, 777, 1024, 4100, 100003, (1 << 31) - 17):
                n_first, *forms = parts(rows, n_out, n_in)
                split = n_first < rows
                assert 0 < n_first <= rows
                # a last tile that is taken along is one behind whole tiles of 256
                for more, r, side in zip(parts.more(rows, n_out, n_in),
                                         (n_first, rows - n_first if split else rows),
                                         (forms[0], forms[3])):
                    assert not more or (side == 256 and r > 256 and -(-r // 16) % 16 == 1)
                # the second part starts with a tile of rows, and has no runs whose sums need room
                assert not split or (n_first % 256 == 0 and forms[1] == 1 and forms[4] == 1)
                for side, splits, per in (forms[:3], forms[3:])[:1 + split]:
                    assert side in (0, 64, 128, 256) and splits >= 1
                    assert (splits - 1) * per < blocks <= splits * per
                    assert splits == 1 or side > 0
                    if side == 0:
                        assert parts.thin(rows, n_out, n_in) in \
                            ((1, 1), (1, 2), (2, 2), (2, 3), (2, 4), (4, 2))
                    # a workgroup's offsets into its tiles
                    assert side == 0 or blocks * 2048 * (side // 16) < 1 << 31


def test_sizes_of_the_gpu_tests_reach_every_form(parts):
    from test_gpu_f8 import FORMS, SIZES
    seen = set()
    for m, n, k in FORMS + SIZES:
        n_first, *forms = parts(m, n, k)
        seen.add((forms[0], forms[1] > 1, n_first < m))
        seen.add(("more", parts.more(m, n, k)[0], forms[1] > 1))
        if n_first < m:
            seen.add(("rest", forms[3]))
        elif forms[0] == 0:
            seen.add(("thin", *parts.thin(m, n, k)))
    want = {(0, False, False), (64, False, False), (64, True, False), (128, False, False),
            (128, True, False), (256, False, False), (256, False, True), (128, False, True),
            (64, False, True), ("rest", 0), ("rest", 64), ("more", 1, False), ("more", 1, True)}
    want |= {("thin", *t) for t in ((1, 1), (1, 2), (2, 2), (2, 3), (2, 4), (4, 2))}
    assert want <= seen, want - seen
