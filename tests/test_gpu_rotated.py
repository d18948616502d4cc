"""Appends with the rotation by position on the GPU: keys' codes, scales, positions and
weights value for value against the definition (each product and sum rounded to single
precision), queries bit for bit, and the rotation itself against 64 bits."""
import numpy as np
import pytest

import kv_oracle as ko
from test_gpu_kv import Setup, row_type

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


def tables(torch, n_positions, pairs, seed=0):
    angle = np.outer(np.arange(n_positions), 100.0 ** (-np.arange(pairs) / pairs)) + 0.1 * seed
    cos, sin = (torch.tensor(f(angle).astype(np.float32), device="cuda") for f in (np.cos, np.sin))
    return cos, sin


def turned(x, cos, sin, at, neighbours, kind=np.float32):
    """x [row, head, dim] turned; at [row, pair]: the place in the tables."""
    x = x.astype(kind)
    pairs = cos.shape[1]
    i = np.arange(pairs)
    a, b = (2 * i, 2 * i + 1) if neighbours else (i, i + pairs)
    c, s = cos[at, i].astype(kind)[:, None], sin[at, i].astype(kind)[:, None]
    y = x.copy()
    with np.errstate(invalid="ignore", over="ignore"):
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
    return y


class Case:
    def __init__(self, torch, qlm, lengths, counts, heads, kv, d, fmt, dtype, pairs, neighbours,
                 axes=1, given=True, first=None, n_positions=300, seed=0, low=-5):
        self.torch = torch
        self.s = Setup(torch, qlm, lengths, kv, d, fmt, seed)
        self.lengths, self.counts, self.heads, self.dtype = lengths, counts, heads, dtype
        rows = sum(counts)
        self.cos, self.sin = tables(torch, n_positions, pairs, seed)
        rng = np.random.default_rng(seed + 1)
        axis = rng.integers(-1, axes + 1, pairs).astype(np.int32) if axes > 1 else None
        dev = lambda x: None if x is None else torch.tensor(np.asarray(x, np.int32), device="cuda")  # noqa: E731
        self.rotary = qlm.Rotary(self.cos, self.sin, neighbours, dev(axis))
        # (positions before and behind the tables are the first and the last)
        where = rng.integers(low, n_positions + 5, (axes, rows)).astype(np.int32) if given else None
        self.position, self.first = dev(where), dev(first)
        seq = np.repeat(np.arange(len(counts)), counts)
        place = np.concatenate([np.arange(n) for n in counts] + [np.zeros(0, int)]).astype(int)
        begin = np.array(lengths) - counts if first is None else np.array(first)
        if given:
            on = np.zeros(pairs, int) if axis is None else axis.clip(0, axes - 1)
            at = where[on].T
        else:
            at = np.broadcast_to((begin[seq] + place)[:, None], (rows, pairs))
        self.at = at.clip(0, n_positions - 1).astype(int)
        self.neighbours = neighbours
        self.k, self.kx = self.s.rows(rows, kv, dtype, 2.0)
        self.v, self.vx = self.s.rows(rows, kv, dtype)
        self.q, self.qx = self.s.rows(rows, heads, dtype) if heads else (None, None)
        # the tokens that the sequences hold already: their blocks have scales
        held = [max(0, n - c) for n, c in zip(lengths, counts)]
        k, v = (self.s.rows(sum(held), kv, dtype)[0] for _ in range(2))
        qlm.kv_append(self.s.cache, self.s.batch(held, held), k, v)

    def turn(self, x, kind=np.float32):
        host = lambda t: t.cpu().numpy()  # noqa: E731
        return turned(x, host(self.cos), host(self.sin), self.at, self.neighbours, kind)

    def batch(self, row_start=True, **more):
        return self.s.batch(self.counts, **more) if row_start else self.s.batch(**more)

    def run(self, qlm, row_start=True, out=None, **more):
        batch = self.batch(row_start, **more)
        return qlm.kv_append_rotated(self.s.cache, batch, self.k, self.v, self.q, self.rotary,
                                     position=self.position, first_position=self.first, out=out)

    def check(self, qlm, row_start=True, out=None):
        ora = ko.Cache.read(self.s.cache, self.s.fmt)
        got = self.run(qlm, row_start, out)
        first = None if self.first is None else self.first.cpu().numpy().astype(int)
        ora.append(self.s.table, self.lengths, self.counts, self.turn(self.kx).astype(np.float64),
                   self.vx, first)
        self.s.assert_same(ora)
        if self.heads:
            want = self.torch.from_numpy(self.turn(self.qx)).to(row_type(self.torch, self.dtype))
            same = (got.cpu() == want) | (got.cpu().isnan() & want.isnan())
            assert bool(same.all()), int((~same).sum())
            exact = self.turn(self.qx, np.float64)
            # three roundings of single precision, of numbers up to |a| + |b| <= 2 max; then the
            # type's own half step
            step = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}[self.dtype]
            top = np.abs(self.qx).max(axis=-1, keepdims=True)
            e = np.abs(got.double().cpu().numpy() - exact)
            assert (e <= step * np.abs(exact) + (6 * 2.0 ** -24 * top + 2.0 ** -25)).all()


LENGTHS = [0, 1, 2, 63, 64, 65, 130, 200]
COUNTS = [0, 1, 1, 3, 64, 2, 130, 70]


@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("fmt,dtype", [("e4m3", "bf16"), ("int8", "f16")])
@pytest.mark.parametrize("d,pairs,heads,kv", [(16, 1, 1, 1), (16, 8, 3, 3), (64, 32, 4, 1),
                                              (64, 20, 2, 2), (80, 40, 5, 1), (80, 33, 4, 2),
                                              (128, 64, 8, 2), (128, 32, 1, 1), (256, 128, 2, 1),
                                              (144, 61, 3, 1)])
def test_sizes(torch, qlm, d, pairs, heads, kv, fmt, dtype, neighbours):
    Case(torch, qlm, LENGTHS, COUNTS, heads, kv, d, fmt, dtype, pairs, neighbours,
         seed=d + pairs).check(qlm)


@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("axes", [2, 3, 4])
def test_axes(torch, qlm, axes, neighbours):
    """Several positions a row, and axes before and behind those that there are."""
    Case(torch, qlm, LENGTHS, COUNTS, 4, 2, 64, "e4m3", "bf16", 32, neighbours, axes=axes,
         seed=axes).check(qlm)


@pytest.mark.parametrize("first", [None, [0, 40, 7, 100, 0, 250, 299, 1000]])
@pytest.mark.parametrize("heads", [0, 3])
def test_positions_of_the_cache(torch, qlm, first, heads):
    """Without positions a row has the one that the cache keeps for its slot."""
    Case(torch, qlm, LENGTHS, COUNTS, heads, 3, 32, "int8", "bf16", 16, False, given=False,
         first=first).check(qlm)


@pytest.mark.parametrize("given", [False, True])
def test_one_row_a_sequence(torch, qlm, given):
    """Decode: a row for each sequence, without row_start (a sequence of no slots has a row
    too, which is nowhere written, but turned)."""
    lengths = [1, 0, 64, 65, 100, 128]
    c = Case(torch, qlm, lengths, [1] * 6, 4, 2, 64, "e4m3", "f16", 32, False, given=given)
    c.check(qlm, row_start=False)


@pytest.mark.parametrize("n", [63, 64, 65, 1000, 4097])
def test_many_sequences(torch, qlm, n):
    """Rows are matched with their sequences 64 at a time."""
    counts = [(5 * i % 3) for i in range(n)]
    Case(torch, qlm, [c + i % 7 for i, c in enumerate(counts)], counts, 1, 1, 16, "e4m3", "bf16", 8,
         False, given=False).check(qlm)


@pytest.mark.parametrize("pairs,neighbours", [(32, False), (32, True), (20, False), (5, True)])
def test_in_place(torch, qlm, pairs, neighbours):
    c = Case(torch, qlm, LENGTHS, COUNTS, 6, 2, 64, "e4m3", "bf16", pairs, neighbours)
    c.check(qlm, out=c.q)


def test_rows_of_no_sequence(torch, qlm):
    """Rows behind the last sequence's, and those past max_new, stay as they were."""
    counts = [3, 5, 0, 2]
    c = Case(torch, qlm, [10, 5, 0, 70], counts, 2, 2, 32, "e4m3", "bf16", 16, False)
    pad = torch.ones((4, 2, 32), dtype=torch.bfloat16, device="cuda")
    wide = [torch.cat([x, pad]) for x in (c.k, c.v, c.q)]
    table = torch.cat([c.position, torch.zeros((1, 4), dtype=torch.int32, device="cuda")], 1)
    b = c.batch()
    b = qlm.KvBatch(b.block_table, b.lengths, b.row_start, 14, 4)      # (5 rows: one too many)
    out = torch.full((14, 2, 32), 7.0, dtype=torch.bfloat16, device="cuda")
    qlm.kv_append_rotated(c.s.cache, b, *wide[:2], wide[2], c.rotary, position=table, out=out)
    want = torch.from_numpy(c.turn(c.qx)).bfloat16()
    got = out.cpu()
    assert torch.equal(got[:7], want[:7]) and bool((got[7] == 7.0).all())
    assert torch.equal(got[8:10], want[8:]) and bool((got[10:] == 7.0).all())


def test_values_that_are_not_finite(torch, qlm):
    c = Case(torch, qlm, [70, 5], [70, 5], 2, 1, 32, "e4m3", "bf16", 8, False, seed=3)
    for x, host in ((c.k, c.kx), (c.q, c.qx)):
        for row, dim, value in ((0, 3, np.inf), (1, 20, -np.inf), (2, 11, np.nan), (3, 30, np.nan),
                                (71, 0, 3.3e38), (71, 8, 3.3e38)):
            x[row, 0, dim] = value
            host[row, 0, dim] = float(x[row, 0, dim])
    got = c.run(qlm)
    want = torch.from_numpy(c.turn(c.qx)).bfloat16()
    assert torch.equal(got.cpu().isnan(), want.isnan())
    fine = ~want.isnan()
    assert torch.equal(got.cpu()[fine], want[fine])
    ora = ko.Cache.read(c.s.cache, "e4m3")
    key = c.turn(c.kx).astype(np.float64)[:70, 0]
    held = ora.k[c.s.table[0][0], 0]
    assert (np.isnan(held) == np.isnan(key[:64])).all()
    assert (np.abs(held[np.isinf(key[:64])]) == 448).all()


def test_same_as_append_where_nothing_turns(torch, qlm):
    """cos 1 and sin 0: the codes of qlm_kv_append."""
    a = Case(torch, qlm, LENGTHS, COUNTS, 2, 2, 64, "e4m3", "bf16", 32, False)
    b = Case(torch, qlm, LENGTHS, COUNTS, 2, 2, 64, "e4m3", "bf16", 32, False)
    a.rotary.cos.fill_(1.0)
    a.rotary.sin.zero_()
    q = a.run(qlm)
    qlm.kv_append(b.s.cache, b.batch(), b.k, b.v)
    assert torch.equal(q, a.q)
    for n in ("k_codes", "v_codes", "k_scale", "v_scale"):
        x, y = getattr(a.s.cache, n), getattr(b.s.cache, n)
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)) if "codes" in n else \
            torch.equal(x.nan_to_num(7.0), y.nan_to_num(7.0))


def test_captured_and_replayed(torch, qlm):
    """A captured step replayed between eager work, over positions and rows that change."""
    c = Case(torch, qlm, [100, 65, 3], [1, 1, 1], 4, 2, 64, "e4m3", "bf16", 32, False)
    e = Case(torch, qlm, [100, 65, 3], [1, 1, 1], 4, 2, 64, "e4m3", "bf16", 32, False)
    out = torch.empty_like(c.q)
    batch, other = c.batch(), e.batch()
    args = lambda k, b, o: (qlm.kv_append_rotated(k.s.cache, b, k.k, k.v, k.q, k.rotary,  # noqa: E731
                                                  position=k.position, out=o))
    args(c, batch, out)
    args(e, other, None)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        args(c, batch, out)
    for i in range(4):
        for k in (c, e):
            k.position.add_(7 * i)
            k.k.mul_(1.5)
        graph.replay()
        want = args(e, other, None)
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        for n in ("k_codes", "v_codes"):
            assert torch.equal(getattr(c.s.cache, n).view(torch.uint8),
                               getattr(e.s.cache, n).view(torch.uint8)), (i, n)


def test_on_a_side_stream(torch, qlm):
    c = Case(torch, qlm, [100, 65, 3], [4, 1, 1], 4, 2, 64, "e4m3", "bf16", 32, False)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = qlm.kv_append_rotated(c.s.cache, c.batch(), c.k, c.v, c.q, c.rotary, position=c.position,
                                stream=side)
    side.synchronize()
    assert torch.equal(got.cpu(), torch.from_numpy(c.turn(c.qx)).bfloat16())
