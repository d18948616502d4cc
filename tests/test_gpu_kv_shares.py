"""Appends on either side of the number of new slots of a block from which a thread holds
neighbouring ones, wherever in a block they begin, over tokens that are held already."""
import pytest

from test_gpu_kv import Setup
from test_gpu_rotated import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available()
    return torch


@pytest.fixture(scope="module")
def qlm():
    from paper_2407_00047_amd import qlm
    return qlm


# (slots held, new ones)
SHARES = [(0, 47), (0, 48), (0, 49), (0, 63), (0, 64), (1, 48), (2, 49), (3, 47), (5, 59), (15, 49),
          (16, 33), (17, 47), (64, 49), (10, 8), (11, 9), (12, 16), (13, 17), (40, 100), (63, 50)]
HELD, COUNTS = ([s[i] for s in SHARES] for i in (0, 1))
LENGTHS = [h + c for h, c in SHARES]


@pytest.mark.parametrize("fmt,dtype", [("e4m3", "bf16"), ("int8", "f16")])
@pytest.mark.parametrize("grow", [1.0, 8.0])
@pytest.mark.parametrize("d,kv", [(64, 3), (48, 1), (128, 2), (80, 2), (256, 1), (144, 1)])
def test_append_shares(torch, qlm, d, kv, grow, fmt, dtype):
    """grow: how far the new tokens pass those held, whose codes are then rescaled."""
    s = Setup(torch, qlm, HELD, kv, d, fmt, seed=d, room=max(COUNTS))
    ora = s.fill(dtype)
    k, kx = s.rows(sum(COUNTS), kv, dtype, 2.0 * grow)
    v, vx = s.rows(sum(COUNTS), kv, dtype, grow)
    qlm.kv_append(s.cache, s.batch(COUNTS, LENGTHS), k, v)
    ora.append(s.table, LENGTHS, COUNTS, kx, vx)
    s.assert_same(ora)


@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("d,pairs", [(64, 32), (128, 64), (80, 10), (256, 128)])
def test_rotated_shares(torch, qlm, d, pairs, neighbours):
    Case(torch, qlm, LENGTHS, COUNTS, 2, 2, d, "int8", "bf16", pairs, neighbours, seed=d).check(qlm)
