"""Appends with the rotation by position of prompts so long that a thread takes four heads' queries
(more than 4096 waves of single ones), on the GPU: every pairing, width, number of heads and way of
giving positions against the definition, and bit for bit the same as in shorter calls."""
import numpy as np
import pytest

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


COUNTS = [2500, 0, 1, 1700]
LENGTHS = [2510, 3, 1, 1810]


def many(heads, d, pairs, neighbours, rows):
    """Whether the call passes the 4096 waves."""
    units = d // 16 if neighbours else -(-pairs // 8) + -(-(d - 2 * pairs) // 16)
    return rows * -(-heads * units // 64) > 4096


@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("heads,d,pairs,axes", [(3, 64, 32, 1), (5, 80, 40, 3), (8, 128, 64, 3),
                                                (3, 80, 10, 1), (5, 128, 33, 4), (8, 64, 20, 1),
                                                (1, 256, 128, 1), (6, 48, 1, 2), (7, 16, 8, 1)])
def test_long_prompts(torch, qlm, heads, d, pairs, axes, in_place, neighbours):
    assert many(heads, d, pairs, neighbours, sum(COUNTS))
    c = Case(torch, qlm, LENGTHS, COUNTS, heads, 1, d, "e4m3", "bf16", pairs, neighbours, axes=axes,
             seed=heads * d + pairs)
    c.check(qlm, out=c.q if in_place else None)


@pytest.mark.parametrize("first", [None, [40, 0, 7, 1000]])
@pytest.mark.parametrize("heads,pairs,neighbours", [(5, 20, False), (4, 32, False), (7, 32, True)])
def test_positions_of_the_cache(torch, qlm, heads, pairs, neighbours, first):
    assert many(heads, 64, pairs, neighbours, sum(COUNTS))
    Case(torch, qlm, LENGTHS, COUNTS, heads, 1, 64, "int8", "f16", pairs, neighbours, given=False,
         first=first, n_positions=4000).check(qlm)


@pytest.mark.parametrize("shift", [0, 1, 4])
@pytest.mark.parametrize("heads,d,pairs,neighbours", [(5, 80, 20, False), (6, 64, 32, False),
                                                      (3, 128, 30, True), (9, 128, 64, True)])
def test_same_as_short_calls(torch, qlm, heads, d, pairs, neighbours, shift):
    """The queries of 4300 rows of one sequence, and the same rows 1000 at a time; starts of any
    alignment, between values that stay."""
    rows, part = 4300, 1000
    assert many(heads, d, pairs, neighbours, rows) and not many(heads, d, pairs, neighbours, part)
    torch.manual_seed(heads)
    angle = torch.rand((5000, pairs), device="cuda") * 6.0
    rotary = qlm.Rotary(angle.cos(), angle.sin(), neighbours)
    cache = qlm.DeviceKvCache.empty(68, 1, d)
    table = torch.arange(68, dtype=torch.int32, device="cuda")[None]
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    k = torch.randn((rows, 1, d), device="cuda").bfloat16()
    wide = torch.randn((rows * heads * d + 16,), device="cuda").bfloat16()
    q = wide[shift:shift + rows * heads * d].view(rows, heads, d)
    room = torch.full((rows * heads * d + 16,), 5.0, device="cuda").bfloat16()
    out = room[shift:shift + rows * heads * d].view(rows, heads, d)
    at = torch.randint(0, 5000, (rows,), device="cuda", dtype=torch.int32)
    qlm.kv_append_rotated(cache, qlm.KvBatch(table, i32(rows), i32(0, rows), rows, rows), k, k, q,
                          rotary, position=at, out=out)
    for r in range(0, rows, part):
        n = min(part, rows - r)
        batch = qlm.KvBatch(table, i32(r + n), i32(0, n), n, n)
        few = qlm.kv_append_rotated(cache, batch, k[r:r + n], k[r:r + n], q[r:r + n], rotary,
                                    position=at[r:r + n].contiguous())
        assert torch.equal(few, out[r:r + n]), r
    beside = torch.cat([room[:shift], room[shift + rows * heads * d:]])
    assert bool((beside == 5.0).all())
    # and against 64 bits: three roundings of single precision, then half a step
    c, s = (t.cpu().numpy()[at.cpu().numpy()][:, None].astype(np.float64)
            for t in (rotary.cos, rotary.sin))
    x = q.double().cpu().numpy()
    i = np.arange(pairs)
    a, b = (2 * i, 2 * i + 1) if neighbours else (i, i + pairs)
    want = x.copy()
    want[..., a], want[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    top = np.abs(x).max(axis=-1, keepdims=True)
    e = np.abs(out.double().cpu().numpy() - want)
    assert (e <= 2.0 ** -8 * np.abs(want) + 6 * 2.0 ** -24 * top + 2.0 ** -25).all()
