"""How products with 4-bit weights of many rows share the inputs among workgroups,
without a GPU: every step of 128 inputs is taken once, and no read passes a row's end.

A workgroup takes its steps in pairs, k0 and k0 + 1, k0 + 2 and k0 + 3, ..., and reads
both steps of the last pair although its split may end between them.  Rows hold a whole
number of pairs (they are read where they are only then, else padded with zeros)."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

WALK = """
#include "w4_split.h"
extern "C" void split_of(int n_out, int n_in, int rows, int *splits, int *per)
{
    qlm_w4_host::split_of(n_out, n_in, rows, splits, per);
}
// Sizes whose walk goes wrong; the first one's outputs, steps and rows in bad.
extern "C" long walk(int most_out, int most_steps, int most_rows, int *bad)
{
    long wrong = 0;
    for (int n = 1; n <= most_out; n += n % 64 == 1 ? 63 : 1)
        for (int steps = 1; steps <= most_steps; ++steps)
            for (int rows = 1; rows <= most_rows; rows += 64) {
                int splits = 0, per = 0;
                qlm_w4_host::split_of(n, steps * qlm_w4_host::kStep, rows, &splits, &per);
                const int held = (steps + 1) / 2 * 2;
                bool ok = splits >= 1 && per >= 1;
                int next = 0;
                for (int s = 0; s < splits && ok; ++s) {
                    const int k0 = s * per, k1 = k0 + per < steps ? k0 + per : steps;
                    ok = k0 == next && k0 < k1;
                    next = k1;
                    for (int kb = k0; kb < k1; kb += 2)
                        // (past the split's end only zeros may be read)
                        ok = ok && kb + 1 < held && (kb + 1 < k1 || kb + 1 >= steps);
                }
                if (!ok || next != steps) {
                    if (!wrong++) bad[0] = n, bad[1] = steps, bad[2] = rows;
                }
            }
    return wrong;
}
"""


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    d = tmp_path_factory.mktemp("w4_split")
    src, lib = str(d / "walk.cpp"), str(d / "walk.so")
    with open(src, "w") as f:
        f.write(WALK)
    subprocess.run(["g++", "-std=c++17", "-O2", "-shared", "-fPIC", "-I",
                    os.path.join(ROOT, "paper_2407_00047_amd", "csrc"), "-o", lib, src], check=True)
    return ctypes.CDLL(lib)


def test_steps_of_every_split(rule):
    """Outputs to 21000 (the rule knows them by 64s: both ends of each), 256 steps, 1200 rows."""
    rule.walk.restype = ctypes.c_long
    bad = (ctypes.c_int * 3)()
    wrong = rule.walk(21000, 256, 1200, bad)
    assert wrong == 0, "%d sizes; the first: %d outputs, %d steps, %d rows" % (wrong, *bad)


@pytest.mark.parametrize("n,k,rows", [(4096, 11008, 32), (3584, 18944, 8), (6144, 8192, 64),
                                      (83, 2816, 20), (5120, 13824, 128), (20001, 8192, 48)])
def test_splits_of_whole_pairs(rule, n, k, rows):
    splits, per = ctypes.c_int(), ctypes.c_int()
    rule.split_of(n, k, rows, ctypes.byref(splits), ctypes.byref(per))
    assert splits.value == 1 or per.value % 2 == 0
