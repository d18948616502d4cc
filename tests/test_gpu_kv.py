"""The 8-bit token cache on the GPU against its definition in 64 bits: codes,
scales, positions and weights value for value; outputs within the error bound
of single-precision sums and half-precision probabilities."""
import numpy as np
import pytest

import kv_oracle as ko

pytestmark = pytest.mark.gpu

BLOCK = 64


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available()
    return torch


@pytest.fixture(scope="module")
def qlm():
    from paper_2407_00047_amd import qlm
    return qlm


def code_type(torch, fmt):
    return torch.float8_e4m3fn if fmt == "e4m3" else torch.int8


def row_type(torch, dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float16


class Setup:
    """A pool with stale contents (not-a-number codes, weights and scales in
    every slot that no token stands in), sequences in blocks drawn at random."""

    def __init__(self, torch, qlm, lengths, kv, d, fmt, seed=0, room=0, spare=3):
        self.rng = rng = np.random.default_rng(seed)
        self.torch, self.qlm, self.fmt, self.kv, self.d = torch, qlm, fmt, kv, d
        self.lengths = list(lengths)
        need = [-(-(n + room) // BLOCK) for n in lengths]
        total = sum(need) + spare
        ids = rng.permutation(total)
        width = max(1, max(need, default=1))
        self.table = np.full((len(lengths), width), -7, np.int32)
        at = 0
        for s, n in enumerate(need):
            self.table[s, :n] = ids[at:at + n]
            at += n
        self.cache = qlm.DeviceKvCache.empty(total, kv, d, code_type(torch, fmt))
        c = self.cache
        stale = 0x7f if fmt == "e4m3" else 0x81
        c.k_codes.view(torch.uint8).fill_(stale)
        c.v_codes.view(torch.uint8).fill_(stale)
        for x in (c.k_scale, c.v_scale, c.weight):
            x.fill_(float("nan"))
        c.position.fill_(-5)
        self.dev_table = torch.from_numpy(self.table).cuda()

    def batch(self, counts=None, lengths=None, **more):
        torch = self.torch
        lengths = self.lengths if lengths is None else lengths
        dl = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        if counts is None:
            return self.qlm.KvBatch(self.dev_table, dl, **more)
        start = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32,
                             device="cuda")
        return self.qlm.KvBatch(self.dev_table, dl, start, int(sum(counts)),
                                max(1, max(counts, default=1)), **more)

    def rows(self, n, heads, dtype, spread=1.0):
        """Rows as a strided view of a larger tensor, and their values."""
        torch = self.torch
        x = self.rng.normal(size=(n, heads, self.d)) * spread
        big = torch.empty((n, heads + 1, self.d + 8), dtype=row_type(torch, dtype), device="cuda")
        view = big[:, :heads, 8:]
        view.copy_(torch.from_numpy(x).cuda())
        return view, view.double().cpu().numpy()

    def fill(self, dtype="bf16"):
        """Every sequence's tokens written by one append; the oracle's cache."""
        counts = self.lengths
        k, kx = self.rows(sum(counts), self.kv, dtype, 2.0)
        v, vx = self.rows(sum(counts), self.kv, dtype)
        ora = ko.Cache.read(self.cache, self.fmt)
        self.qlm.kv_append(self.cache, self.batch(counts), k, v)
        ora.append(self.table, self.lengths, counts, kx, vx)
        return ora

    def seed_weights(self, ora, w):
        """Given weights into the used slots, in both caches."""
        for s, n in enumerate(self.lengths):
            for i in range(n):
                ora.weight[self.table[s][i // BLOCK], :, i % BLOCK] = w[s][:, i]
        self.cache.weight.copy_(self.torch.from_numpy(ora.weight.astype(np.float32)).cuda())

    def assert_same(self, ora, label=""):
        now = ko.Cache.read(self.cache, self.fmt)
        for name in ("ks", "vs", "position", "weight", "k", "v"):
            a, b = getattr(now, name), getattr(ora, name)
            bad = ~((a == b) | (np.isnan(a) & np.isnan(b)))
            assert not bad.any(), (label, name, int(bad.sum()), np.argwhere(bad)[:3].tolist())


def check(got, want, bound, dtype, label=""):
    """Within the bound; not-a-number where the definition says so."""
    got = got.double().cpu().numpy()
    lim = ko.out_bound(want, bound, dtype)
    nan = np.isnan(want)
    assert (np.isnan(got) == nan).all(), (label, int(np.isnan(got).sum()), int(nan.sum()))
    e = np.abs(got - want)
    bad = ~nan & ~(e <= lim)
    assert not bad.any(), (label, int(bad.sum()), float(np.nanmax(e / lim)))


LENGTHS = [0, 1, 2, 15, 63, 64, 65, 127, 130]


# -- append -------------------------------------------------------------------

@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("d,kv,dtype", [(16, 1, "f16"), (64, 3, "bf16"), (80, 2, "f16"),
                                        (128, 2, "bf16"), (256, 1, "f16")])
def test_append_prompts(torch, qlm, fmt, d, kv, dtype):
    s = Setup(torch, qlm, LENGTHS, kv, d, fmt, seed=d)
    s.assert_same(s.fill(dtype))


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_append_tokens_one_by_one(torch, qlm, fmt):
    """Growing scales: every token larger than the last now and then, so that
    the codes held are requantised; through the end of a block."""
    s = Setup(torch, qlm, [3, 60, 64, 0], 2, 48, fmt, seed=5, room=8)
    ora = s.fill()
    lengths = list(s.lengths)
    for step in range(7):
        counts = [1, 1, 1, 1]
        lengths = [n + 1 for n in lengths]
        k, kx = s.rows(4, s.kv, "bf16", 1.5 ** step)
        v, vx = s.rows(4, s.kv, "f16", 0.5 + (step % 3))
        s.qlm.kv_append(s.cache, s.batch(None, lengths), k, v)
        ora.append(s.table, lengths, counts, kx, vx)
        s.assert_same(ora, step)


def test_append_chunks_and_positions(torch, qlm):
    """Chunks that begin and end inside blocks, with positions of their own."""
    s = Setup(torch, qlm, [10, 70, 0, 129], 2, 64, "e4m3", seed=6, room=150)
    ora = s.fill()
    counts = [100, 0, 64, 2]
    lengths = [a + b for a, b in zip(s.lengths, counts)]
    first = [1000, 7, 500, 2 ** 31 - 3]
    k, kx = s.rows(sum(counts), 2, "bf16", 3.0)
    v, vx = s.rows(sum(counts), 2, "bf16", 3.0)
    qlm.kv_append(s.cache, s.batch(counts, lengths), k, v,
                  torch.tensor(first, dtype=torch.int32, device="cuda"))
    ora.append(s.table, lengths, counts, kx, vx, first)
    s.assert_same(ora)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_append_extreme_values(torch, qlm, fmt):
    """Zeros, the largest and least values, infinities and not-a-numbers."""
    s = Setup(torch, qlm, [1, 4, 64, 3, 5], 1, 32, fmt, seed=7)
    x = s.rng.normal(size=(77, 1, 32))
    x[0] = 0.0
    x[1, 0, :4] = [3.3e38, -3.3e38, 1e-38, 0.0]
    x[2, 0, :3] = [np.inf, -np.inf, np.nan]
    x[5:69, 0, 7] = 448.0 * 2.0 ** -3
    x[69:72] = np.nan
    x[72:] *= 1e-36
    t = torch.from_numpy(x).cuda().to(torch.bfloat16)
    ora = ko.Cache.read(s.cache, fmt)
    qlm.kv_append(s.cache, s.batch(s.lengths), t, t)
    h = t.double().cpu().numpy()
    ora.append(s.table, s.lengths, s.lengths, h, h)
    s.assert_same(ora)


def test_append_rows_without_slots(torch, qlm):
    """A length shorter than the new tokens, an unmapped block: nothing else moves."""
    s = Setup(torch, qlm, [40, 80], 1, 16, "int8", seed=8)
    s.table[1, 0] = 10 ** 6
    s.dev_table.copy_(torch.from_numpy(s.table))
    ora = ko.Cache.read(s.cache, "int8")
    k, kx = s.rows(150, 1, "f16")
    qlm.kv_append(s.cache, s.batch([70, 80]), k, k)
    ora.append(s.table, s.lengths, [70, 80], kx, kx)
    s.assert_same(ora)


# -- attention ------------------------------------------------------------------

@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d,kv,g", [(16, 2, 1), (64, 1, 8), (80, 2, 5), (96, 1, 16), (128, 2, 4),
                                    (128, 1, 17), (208, 1, 3), (256, 1, 40)])
def test_attend_one_token(torch, qlm, fmt, dtype, d, kv, g):
    s = Setup(torch, qlm, LENGTHS + [1000], kv, d, fmt, seed=d + g)
    ora = s.fill(dtype)
    n = len(s.lengths)
    q, qx = s.rows(n, kv * g, dtype, 1.5)
    want, bound = ora.attend(s.table, s.lengths, [1] * n, qx, d ** -0.5)
    check(qlm.kv_attention(s.cache, s.batch(), q), want, bound, dtype)


@pytest.mark.parametrize("fmt,dtype,d,kv,g", [
    ("e4m3", "bf16", 128, 2, 4), ("int8", "f16", 64, 1, 8), ("e4m3", "f16", 80, 1, 3),
    ("int8", "bf16", 256, 1, 2), ("e4m3", "bf16", 32, 2, 1), ("int8", "f16", 192, 1, 5)])
@pytest.mark.parametrize("counts", [[0, 1, 2, 3, 1], [5, 16, 7, 0, 9], [33, 64, 70, 140, 1],
                                    [200, 0, 65, 300, 12]])
def test_attend_rows_and_weights(torch, qlm, fmt, dtype, d, kv, g, counts):
    """Several rows a sequence: each sees the slots up to its own; one has more
    rows than slots, so that its first rows see nothing.  Weights begin from
    nothing, then add to what is there."""
    s = Setup(torch, qlm, [0, 130, 66, 340, 12], kv, d, fmt, seed=sum(counts) + d)
    ora = s.fill(dtype)
    q, qx = s.rows(sum(counts), kv * g, dtype, 1.5)
    scale = 0.7 * d ** -0.5
    b = s.batch(counts)
    for decay in (0.0, 0.5):
        want, bound, wb = ora.attend(s.table, s.lengths, counts, qx, scale, decay)
        got = qlm.kv_attention(s.cache, b, q, scale=scale, weight_decay=decay)
        check(got, want, bound, dtype, decay)
        now = s.cache.weight.double().cpu().numpy()
        assert (np.isnan(now) == np.isnan(ora.weight)).all()
        off = np.abs(now - ora.weight) - wb
        assert not (off > 0).any(), (decay, float(np.nanmax(off)))
        ora.weight = now                     # (the next step adds to what is there)
    # without weights the outputs are the same
    assert torch.equal(got, qlm.kv_attention(s.cache, b, q, scale=scale))


@pytest.mark.parametrize("counts", [[1, 0, 70, 1, 3, 1, 0, 1, 2], [200, 1, 1, 1, 1, 1, 1, 1, 1],
                                    [1, 2, 3, 4, 5, 6, 7, 8, 90]])
def test_attend_scores_in_passes(torch, qlm, counts):
    """Prompts beside few rows whose scores, sized for 2^20 slots of 4 heads, are formed for
    four sequences at a time."""
    kv, d, g = 4, 64, 2
    s = Setup(torch, qlm, [300, 65, 130, 1, 64, 700, 90, 2, 128], kv, d, "e4m3", seed=sum(counts))
    ora = s.fill()
    wide = torch.full((9, 1 << 14), -1, dtype=torch.int32, device="cuda")
    wide[:, :s.table.shape[1]] = s.dev_table
    s.dev_table = wide
    b = s.batch(counts)
    q, qx = s.rows(sum(counts), kv * g, "bf16", 1.5)
    for decay in (0.0, 0.5):
        want, bound, wb = ora.attend(s.table, s.lengths, counts, qx, 0.125, decay)
        check(qlm.kv_attention(s.cache, b, q, scale=0.125, weight_decay=decay), want, bound, "bf16",
              decay)
        now = s.cache.weight.double().cpu().numpy()
        assert (np.isnan(now) == np.isnan(ora.weight)).all()
        off = np.abs(now - ora.weight) - wb
        assert not (off > 0).any(), (decay, float(np.nanmax(off)))
        ora.weight = now


@pytest.mark.parametrize("fmt,g,n", [("e4m3", 8, 1), ("int8", 2, 1), ("e4m3", 4, 4)])
def test_attend_long(torch, qlm, fmt, g, n):
    """Long axes, split over workgroups and joined."""
    s = Setup(torch, qlm, [20011, 4100], 1, 64, fmt, seed=g)
    ora = s.fill()
    q, qx = s.rows(2 * n, g, "bf16", 2.0)
    want, bound, wb = ora.attend(s.table, s.lengths, [n, n], qx, 0.125, 0.0)
    got = qlm.kv_attention(s.cache, s.batch([n, n]), q, weight_decay=0.0)
    check(got, want, bound, "bf16")
    off = np.abs(s.cache.weight.double().cpu().numpy() - ora.weight) - wb
    assert not (off > 0).any(), float(np.nanmax(off))


@pytest.mark.parametrize("counts", [[1], [6], [90]])
def test_unseen_not_a_numbers(torch, qlm, counts):
    """A not-a-number value of a late token reaches the rows that see it, and no
    other; a not-a-number key likewise."""
    n = counts[0]
    for which in ("k", "v"):
        s = Setup(torch, qlm, [100], 1, 64, "e4m3", seed=3)
        k, kx = s.rows(100, 1, "bf16")
        v, vx = s.rows(100, 1, "bf16")
        (k if which == "k" else v)[100 - (n + 1) // 2, 0, 5] = float("nan")
        kx, vx = k.double().cpu().numpy(), v.double().cpu().numpy()
        ora = ko.Cache.read(s.cache, "e4m3")
        qlm.kv_append(s.cache, s.batch([100]), k, v)
        ora.append(s.table, [100], [100], kx, vx)
        q, qx = s.rows(n, 4, "bf16")
        want, bound = ora.attend(s.table, [100], counts, qx, 0.125)
        check(qlm.kv_attention(s.cache, s.batch(counts), q), want, bound, "bf16", which)


def test_attend_wide_ranges(torch, qlm):
    """Blocks whose scales lie far apart, queries far from one, sharp scores."""
    for fmt in ("e4m3", "int8"):
        s = Setup(torch, qlm, [300], 1, 64, fmt, seed=11)
        k, _ = s.rows(300, 1, "bf16", 1e-3)
        v, _ = s.rows(300, 1, "bf16")
        v[64:128] *= 1e4
        v[128:192] *= 1e-6
        k[200:] *= 50.0
        ora = ko.Cache.read(s.cache, fmt)
        qlm.kv_append(s.cache, s.batch([300]), k, v)
        ora.append(s.table, [300], [300], k.double().cpu().numpy(), v.double().cpu().numpy())
        for spread in (1e-30, 1.0, 1e3, 1e5):
            q, qx = s.rows(1, 4, "bf16", spread)
            want, bound = ora.attend(s.table, [300], [1], qx, 0.125)
            check(qlm.kv_attention(s.cache, s.batch(), q), want, bound, "bf16", (fmt, spread))


@pytest.mark.parametrize("n", [1, 3, 40, 200])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_attend_large_scores(torch, qlm, fmt, n):
    """Scores far from zero (to 1e12): outputs stay inside the values' range, and every
    row's and head's weights still add up to one."""
    s = Setup(torch, qlm, [1100], 1, 64, fmt, seed=n)
    k, _ = s.rows(1100, 1, "bf16", 30.0)
    v, _ = s.rows(1100, 1, "bf16")
    qlm.kv_append(s.cache, s.batch([1100]), k, v)
    top = float(ko.Cache.read(s.cache, fmt).sequence(s.table[0], 1100, 0)[1].max())
    for spread in (1e2, 1e4, 1e6, 1e10):
        q, _ = s.rows(n, 4, "bf16", spread)
        for scale in (0.125, -0.125):
            out = qlm.kv_attention(s.cache, s.batch([n]), q, scale=scale, weight_decay=0.0)
            assert bool(out.isfinite().all()) and float(out.abs().max()) <= 1.01 * abs(top) + 5
            total = float(s.cache.weight.nan_to_num(0.0).double().sum())
            # (a sum of up to 1100 single-precision terms each)
            assert abs(total - 4 * n) <= 4 * n * 1100 * 2.0 ** -22, (spread, scale, total)


@pytest.mark.parametrize("fmt,dtype", [("e4m3", "bf16"), ("int8", "bf16"), ("e4m3", "f16"),
                                       ("int8", "f16")])
@pytest.mark.parametrize("counts", [[1, 1, 0], [30, 9, 12], [200, 70, 90]])
def test_attend_nothing_to_tell_apart(torch, qlm, fmt, dtype, counts):
    """Queries of zeros or next to them, keys of zeros or next to them, a scale of zero:
    every seen slot has the same part, and the unseen ones none."""
    lengths = [200, 130, 100]
    for keys, spread, scale in ((0.0, 0.0, 0.125), (0.0, 1.0, 0.125), (1.0, 0.0, -0.125),
                                (1e-7, 1e-4, 0.125), (1.0, 1.0, 0.0), (0.0, 1.0, 0.0)):
        s = Setup(torch, qlm, lengths, 2, 64, fmt, seed=sum(counts))
        k, kx = s.rows(sum(lengths), 2, dtype, keys)
        v, vx = s.rows(sum(lengths), 2, dtype)
        ora = ko.Cache.read(s.cache, fmt)
        qlm.kv_append(s.cache, s.batch(lengths), k, v)
        ora.append(s.table, lengths, lengths, kx, vx)
        q, qx = s.rows(sum(counts), 8, dtype, spread)
        label = (keys, spread, scale)
        want, bound, wb = ora.attend(s.table, lengths, counts, qx, scale, 0.0)
        got = qlm.kv_attention(s.cache, s.batch(counts), q, scale=scale, weight_decay=0.0)
        check(got, want, bound, dtype, label)
        now = s.cache.weight.double().cpu().numpy()
        assert (np.isnan(now) == np.isnan(ora.weight)).all(), label
        off = np.abs(now - ora.weight) - wb
        assert not (off > 0).any(), (label, float(np.nanmax(off)))


def test_unmapped_blocks(torch, qlm):
    """A block number outside the pool names no slots: the others are attended."""
    s = Setup(torch, qlm, [300, 64], 1, 64, "e4m3", seed=13)
    ora = s.fill()
    s.table[0, 2], s.table[1, 0] = -1, 10 ** 8
    s.dev_table.copy_(torch.from_numpy(s.table))
    for n in (1, 20):
        q, qx = s.rows(2 * n, 4, "f16")
        want, bound, wb = ora.attend(s.table, s.lengths, [n, n], qx, 0.125, 0.0)
        got = qlm.kv_attention(s.cache, s.batch([n, n]), q, weight_decay=0.0)
        check(got, want, bound, "f16")
        now = s.cache.weight.double().cpu().numpy()
        off = np.abs(now - ora.weight) - wb
        assert not (off > 0).any()


def test_far_blocks(torch, qlm):
    """Blocks whose bytes lie past 2^32 in both pools."""
    kv, d, n_blocks = 8, 128, 70000
    cache = qlm.DeviceKvCache.empty(n_blocks, kv, d, torch.float8_e4m3fn)
    s = Setup(torch, qlm, [70], kv, d, "e4m3", seed=17)
    far = s.table.copy()
    far[0, :2] = [n_blocks - 1, n_blocks - 70]
    table = torch.from_numpy(far).cuda()
    k, kx = s.rows(70, kv, "bf16")
    v, vx = s.rows(70, kv, "bf16")
    q, qx = s.rows(1, kv * 2, "bf16")
    outs = []
    for c, t in ((s.cache, s.dev_table), (cache, table)):
        lens = torch.tensor([70], dtype=torch.int32, device="cuda")
        start = torch.tensor([0, 70], dtype=torch.int32, device="cuda")
        qlm.kv_append(c, qlm.KvBatch(t, lens, start, 70, 70), k, v)
        outs.append(qlm.kv_attention(c, qlm.KvBatch(t, lens), q, weight_decay=0.0))
        qlm.kv_evict(c, qlm.KvBatch(t, lens), 64, 4)
        outs.append(qlm.kv_attention(c, qlm.KvBatch(t, lens.clamp(max=64)), q))
    assert torch.equal(outs[0], outs[2]) and torch.equal(outs[1], outs[3])
    assert not outs[0].isnan().any()


def test_other_stream_and_graph(torch, qlm):
    """The calls run on the stream they are given, and replay in a graph beside
    eager work, every replay as the eager result."""
    s = Setup(torch, qlm, [700, 90], 2, 128, "e4m3", seed=19, room=64)
    s.fill()
    k, _ = s.rows(2, 2, "bf16")
    q, _ = s.rows(2, 8, "bf16")
    b = s.batch(None, [n + 1 for n in s.lengths])
    ws = qlm.kv_attention_workspace(s.cache, b, 8, True)
    out = torch.empty(q.shape, dtype=q.dtype, device="cuda")
    qlm.kv_append(s.cache, b, k, k)
    want = qlm.kv_attention(s.cache, b, q, weight_decay=0.0).clone()
    weight = s.cache.weight.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    qlm.kv_append(s.cache, b, k, k, stream=side)
    qlm.kv_attention(s.cache, b, q, weight_decay=0.0, out=out, ws=ws, stream=side)
    side.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        qlm.kv_append(s.cache, b, k, k)
        qlm.kv_attention(s.cache, b, q, weight_decay=0.0, out=out, ws=ws)
    for _ in range(3):
        out.zero_()
        s.cache.weight.fill_(7.0)
        ws.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        used = ~weight.isnan()
        assert torch.equal(s.cache.weight[used], weight[used])


# -- eviction -------------------------------------------------------------------

@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("d,kv,budget,recent", [(64, 2, 64, 0), (128, 1, 128, 30), (80, 3, 64, 64),
                                                (256, 1, 192, 1), (16, 2, 128, 128)])
def test_evict(torch, qlm, fmt, d, kv, budget, recent):
    s = Setup(torch, qlm, [0, 1, 63, 64, 65, 128, 129, 200, 333, 2050], kv, d, fmt, seed=budget + d)
    ora = s.fill()
    w = [np.exp(2 * s.rng.normal(size=(kv, n))).astype(np.float32) for n in s.lengths]
    s.seed_weights(ora, w)
    got = qlm.kv_evict(s.cache, s.batch(), budget, recent)
    want = ora.evict(s.table, s.lengths, budget, recent)
    assert got.cpu().tolist() == want
    s.assert_same(ora)


def test_evict_ties_and_odd_weights(torch, qlm):
    """Equal weights (the lowest slot stays), zeros of both signs, negatives,
    infinities and not-a-numbers; protected slots stay whatever they weigh."""
    rng = np.random.default_rng(0)
    for trial in range(4):
        s = Setup(torch, qlm, [300, 129, 1500], 2, 32, "e4m3", seed=trial)
        ora = s.fill()
        odd = np.array([0.0, -0.0, 1.0, 1.0, -1.0, np.inf, -np.inf, np.nan, 1e-45, 3e38], np.float32)
        w = [odd[rng.integers(0, len(odd), size=(2, n))] for n in s.lengths]
        if trial == 3:
            w = [np.zeros((2, n), np.float32) for n in s.lengths]
        s.seed_weights(ora, w)
        got = qlm.kv_evict(s.cache, s.batch(), 128, 16)
        assert got.cpu().tolist() == ora.evict(s.table, s.lengths, 128, 16)
        s.assert_same(ora, trial)


def test_evict_in_place_and_again(torch, qlm):
    """Lengths written over the batch's own; the cut sequences go on: tokens
    appended, attended to, cut again."""
    s = Setup(torch, qlm, [150, 90, 64], 2, 64, "int8", seed=23, room=128)
    ora = s.fill()
    w = [np.exp(s.rng.normal(size=(2, n))).astype(np.float32) for n in s.lengths]
    s.seed_weights(ora, w)
    lengths = torch.tensor(s.lengths, dtype=torch.int32, device="cuda")
    now = list(s.lengths)
    for step in range(3):
        b = qlm.KvBatch(s.dev_table, lengths)
        assert qlm.kv_evict(s.cache, b, 64, 8, out=lengths) is lengths
        now = ora.evict(s.table, now, 64, 8)
        assert lengths.cpu().tolist() == now
        s.assert_same(ora, step)
        counts = [30, 1, 5]
        now = [a + c for a, c in zip(now, counts)]
        lengths += torch.tensor(counts, dtype=torch.int32, device="cuda")
        k, kx = s.rows(36, 2, "f16", 2.0)
        first = [1000 * (step + 1)] * 3
        start = torch.tensor([0, 30, 31, 36], dtype=torch.int32, device="cuda")
        b = qlm.KvBatch(s.dev_table, lengths, start, 36, 30)
        qlm.kv_append(s.cache, b, k, k, torch.tensor(first, dtype=torch.int32, device="cuda"))
        ora.append(s.table, now, counts, kx, kx, first)
        q, qx = s.rows(36, 4, "f16")
        want, bound, _ = ora.attend(s.table, now, counts, qx, 0.125, 1.0)
        check(qlm.kv_attention(s.cache, b, q, weight_decay=1.0), want, bound, "f16", step)
        ora.weight = s.cache.weight.double().cpu().numpy()


def test_evict_leaves_unmapped_sequences(torch, qlm):
    s = Setup(torch, qlm, [300, 300], 1, 16, "e4m3", seed=29)
    ora = s.fill()
    s.seed_weights(ora, [np.ones((1, 300), np.float32)] * 2)
    s.table[1, 3] = -1
    s.dev_table.copy_(torch.from_numpy(s.table))
    got = qlm.kv_evict(s.cache, s.batch(), 64, 0)
    assert got.cpu().tolist() == ora.evict(s.table, s.lengths, 64, 0) == [64, 300]
    s.assert_same(ora)


def test_evict_long(torch, qlm):
    s = Setup(torch, qlm, [40001, 777], 1, 16, "int8", seed=31)
    ora = s.fill()
    s.seed_weights(ora, [np.exp(3 * s.rng.normal(size=(1, n))).astype(np.float32)
                         for n in s.lengths])
    got = qlm.kv_evict(s.cache, s.batch(), 2048, 100)
    assert got.cpu().tolist() == ora.evict(s.table, s.lengths, 2048, 100)
    s.assert_same(ora)


def test_empty_batch(torch, qlm):
    s = Setup(torch, qlm, [5], 1, 16, "e4m3")
    none = torch.empty((0,), dtype=torch.int32, device="cuda")
    b = qlm.KvBatch(torch.empty((0, 4), dtype=torch.int32, device="cuda"), none)
    x = torch.empty((0, 1, 16), dtype=torch.float16, device="cuda")
    qlm.kv_append(s.cache, b, x, x)
    assert qlm.kv_attention(s.cache, b, x).shape == (0, 1, 16)
    assert qlm.kv_evict(s.cache, b, 64).numel() == 0
