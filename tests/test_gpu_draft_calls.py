"""Calls of the drafting step's operators as programs make them: views of one tensor of
projections, operands anywhere in memory, two calls at once, captured graphs that share a
workspace, offsets past 32 bits."""
import numpy as np
import pytest

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


def turning(torch, qlm, n_positions, pairs):
    angle = torch.arange(n_positions, device="cuda")[:, None] * 0.1 + torch.arange(
        pairs, device="cuda") * 0.3
    return qlm.Rotary(angle.cos().float(), angle.sin().float())


def batch_of(torch, qlm, table, lengths, counts):
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    return qlm.KvBatch(table, i32(lengths), i32(np.concatenate([[0], np.cumsum(counts)])),
                       int(sum(counts)), max(counts))


def slots(torch, cache):
    """What an append writes, as bytes and numbers that compare."""
    return [cache.k_codes.view(torch.uint8), cache.v_codes.view(torch.uint8), cache.k_scale,
            cache.v_scale, cache.position, cache.weight]


def clear(cache):
    import torch
    for x in slots(torch, cache):
        x.zero_()


@pytest.mark.parametrize("heads,kv,d", [(6, 2, 64), (3, 1, 80), (2, 2, 16)])
def test_views_of_one_projection(torch, qlm, heads, kv, d):
    """Queries, keys and values side by side in one tensor, the queries turned in place: what
    lies beside them stays."""
    torch.manual_seed(1)
    counts, lengths = [3, 1, 70], [10, 64, 70]
    rotary = turning(torch, qlm, 100, d // 2)
    table = torch.arange(6, dtype=torch.int32, device="cuda").view(3, 2)
    batch = batch_of(torch, qlm, table, lengths, counts)
    whole = torch.randn((74, heads + 2 * kv, d), device="cuda").bfloat16()
    kept = whole.clone()
    one, two = (qlm.DeviceKvCache.empty(6, kv, d) for _ in range(2))
    held = [n - c for n, c in zip(lengths, counts)]
    before = batch_of(torch, qlm, table, held, held)
    old = torch.randn((sum(held), kv, d), device="cuda").bfloat16()
    for c in (one, two):
        clear(c)
        qlm.kv_append(c, before, old, old)
    parts = lambda x: (x[:, heads:heads + kv], x[:, heads + kv:], x[:, :heads])  # noqa: E731
    want = qlm.kv_append_rotated(two, batch, *(p.contiguous() for p in parts(kept)), rotary)
    k, v, q = parts(whole)
    got = qlm.kv_append_rotated(one, batch, k, v, q, rotary, out=q)
    assert got is q and torch.equal(got, want) and not torch.equal(got, kept[:, :heads])
    assert torch.equal(whole[:, heads:], kept[:, heads:])
    for a, b in zip(slots(torch, one), slots(torch, two)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("k", [64, 60, 63, 1])
@pytest.mark.parametrize("at", [0, 1, 2, 4, 8, 16])
def test_weights_from_anywhere(torch, qlm, at, k):
    """Codes at any byte, rows of any size: packed as from an aligned copy."""
    torch.manual_seed(at)
    n = 37
    big = torch.randint(0, 255, (at + n * k,), dtype=torch.uint8, device="cuda")
    codes = big[at:].view(n, k)
    scale = torch.rand((1, 1), device="cuda")
    got = qlm.f8_pack(codes.view(torch.float8_e4m3fn), scale).packed
    full = torch.zeros((48, 128), dtype=torch.uint8, device="cuda")
    full[:n, :k] = codes
    want = full.view(3, 16, 8, 16).transpose(1, 2).contiguous().flatten()
    assert torch.equal(got[:3 * 2048], want)
    assert torch.equal(got[3 * 2048:].view(torch.float32), scale.flatten())


def matrices(torch, qlm, m, n, k, seed):
    torch.manual_seed(seed)
    w = (torch.randn((n, k), device="cuda") * 100).clamp(-448, 448).to(torch.float8_e4m3fn)
    w = qlm.f8_pack(w, torch.rand((-(-n // 128), -(-k // 128)), device="cuda") + 0.5)
    return torch.randn((m, k), device="cuda").bfloat16(), w


# (few rows; inputs in runs, joined; tiles of rows in two parts)
SIZES = [(7, 500, 900), (466, 505, 13323), (770, 2100, 1500)]


@pytest.mark.parametrize("m,n,k", SIZES)
def test_products_on_two_streams(torch, qlm, m, n, k):
    """Two products of the same weights at once, each with what its call allocates."""
    x, w = matrices(torch, qlm, m, n, k, 3)
    y = x.flip(0).contiguous()
    want = [qlm.f8_matmul(qlm.f8_rows(z), w) for z in (x, y)]
    sides = [torch.cuda.Stream() for _ in range(2)]
    for s in sides:
        s.wait_stream(torch.cuda.current_stream())
    got = [[], []]
    for _ in range(10):
        for s, z, g in zip(sides, (x, y), got):
            g.append(qlm.f8_matmul(qlm.f8_rows(z, stream=s), w, stream=s))
    torch.cuda.synchronize()
    for g, r in zip(got, want):
        assert all(torch.equal(a, r) for a in g)


@pytest.mark.parametrize("m,n,k", SIZES)
def test_graphs_that_share_a_workspace(torch, qlm, m, n, k):
    """Two captured products and eager ones between them, one workspace, one stream."""
    x, w = matrices(torch, qlm, m, n, k, 4)
    pair = [qlm.f8_rows(x), qlm.f8_rows(x * 3 + 1)]
    ws = qlm.f8_workspace(w, m)
    outs, graphs = [], []
    for r in pair:
        out = qlm.f8_matmul(r, w, ws=ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            qlm.f8_matmul(r, w, out=out, ws=ws)
        outs.append(out)
        graphs.append(g)
    want = [qlm.f8_matmul(r, w) for r in pair]
    for i in (0, 1, 1, 0, 0, 1):
        outs[i].fill_(float("nan"))
        ws.fill_(255)
        graphs[i].replay()
        between = qlm.f8_matmul(pair[1 - i], w, ws=ws)
        torch.cuda.synchronize()
        assert torch.equal(outs[i], want[i]) and torch.equal(between, want[1 - i])


def test_runs_of_inputs_are_reached(torch, qlm):
    w = matrices(torch, qlm, 1, 505, 13323, 0)[1]
    assert qlm.f8_workspace_bytes(w, 466) > 0


def drafted(torch, qlm, seqs, rows, vocab, seed, kind="float32"):
    torch.manual_seed(seed)
    table = torch.zeros((seqs, 1), dtype=torch.int32, device="cuda")
    batch = batch_of(torch, qlm, table, [50] * seqs, [rows] * seqs)
    n = seqs * rows
    dt = getattr(torch, kind)
    target = torch.softmax(2 * torch.randn((n, vocab), device="cuda"), -1).to(dt)
    draft = torch.softmax(2 * torch.randn((n, vocab), device="cuda"), -1).to(dt)
    tokens = torch.randint(0, vocab, (n,), dtype=torch.int32, device="cuda")
    return [batch, tokens, target, draft, torch.rand(n, device="cuda")]


def test_verifications_share_a_workspace(torch, qlm):
    """Two captured verifications and eager ones between them; two on streams of their own."""
    a, b = (drafted(torch, qlm, 2, 4, 70000, s) for s in (1, 2))
    ws = qlm.draft_verify_workspace(a[0], 70000)
    assert ws.numel() > 1
    same = lambda x, y: all(torch.equal(p, q) for p, q in zip(x, y))  # noqa: E731
    want = [qlm.draft_verify(*z) for z in (a, b)]
    got, graphs = [], []
    for z in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got.append(qlm.draft_verify(*z, ws=ws))
        graphs.append(g)
    for i in (0, 1, 1, 0):
        for x in got[i]:
            x.fill_(-9)
        ws.fill_(255)
        graphs[i].replay()
        between = qlm.draft_verify(*(a, b)[1 - i], ws=ws)
        torch.cuda.synchronize()
        assert same(got[i], want[i]) and same(between, want[1 - i])
    sides = [torch.cuda.Stream() for _ in range(2)]
    for s in sides:
        s.wait_stream(torch.cuda.current_stream())
    both = [[qlm.draft_verify(*z, stream=s) for s, z in zip(sides, (a, b))] for _ in range(10)]
    torch.cuda.synchronize()
    assert all(same(p, q) for pair in both for p, q in zip(pair, want))


@pytest.mark.parametrize("draws", [True, False])
def test_rows_past_four_gigabytes(torch, qlm, draws):
    """Rows of probabilities 2^30 numbers apart: the last ones start past 2^32."""
    batch, tokens, target, draft, u = drafted(torch, qlm, 1, 6, 5000, 5, "float16")
    u.zero_()                                         # every draft with any weight is kept
    target[4, int(tokens[5])] = 0.0                   # but the last one
    want = qlm.draft_verify(batch, tokens, target, draft if draws else None, u)
    big = torch.empty(5 * 2 ** 30 + 5000, dtype=torch.float16, device="cuda")
    far = torch.as_strided(big, (6, 5000), (2 ** 30, 1))
    far.copy_(target)
    got = qlm.draft_verify(batch, tokens, far, draft if draws else None, u)
    assert int(want[1]) == 5 and all(torch.equal(a, b) for a, b in zip(got, want))
    if draws:
        far.copy_(draft)
        got = qlm.draft_verify(batch, tokens, target, far, u)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_rows_to_code_past_four_gigabytes(torch, qlm):
    torch.manual_seed(6)
    x = torch.randn((6, 300), device="cuda").bfloat16()
    big = torch.empty(5 * 2 ** 30 + 300, dtype=torch.bfloat16, device="cuda")
    far = torch.as_strided(big, (6, 300), (2 ** 30, 1))
    far.copy_(x)
    got, want = qlm.f8_rows(far), qlm.f8_rows(x)
    assert torch.equal(got.codes.view(torch.uint8), want.codes.view(torch.uint8))
    assert torch.equal(got.scale, want.scale)


def test_outputs_past_four_gigabytes(torch, qlm):
    """70001 rows of 31000 outputs, and codes of 2.3 GB: the same rows in a call of a few.  One
    block of inputs is summed alike in every form."""
    x, w = matrices(torch, qlm, 70001, 31000, 128, 7)
    out = qlm.f8_matmul(qlm.f8_rows(x), w)
    for a, b in ((0, 40), (34000, 34321), (69990, 70001)):
        assert torch.equal(out[a:b], qlm.f8_matmul(qlm.f8_rows(x[a:b].contiguous()), w)), a


def test_codes_past_two_gigabytes(torch, qlm):
    """140001 rows of 16384 inputs: codes of 2.3 GB."""
    torch.manual_seed(8)
    x = torch.randn((140001, 16384), device="cuda", dtype=torch.bfloat16)
    rows = qlm.f8_rows(x)
    tail = qlm.f8_rows(x[139984:].contiguous())       # (17 rows, from a tile's first one on)
    assert torch.equal(rows.codes[8749:].view(torch.uint8), tail.codes.view(torch.uint8))
    w = matrices(torch, qlm, 1, 40, 16384, 9)[1]
    out = qlm.f8_matmul(rows, w, dtype=torch.float32)
    few = qlm.f8_matmul(tail, w, dtype=torch.float32)
    # sums of 128 blocks in another order: 2^-24 each of sums whose sizes stay within the blocks'
    # own, sqrt(128) of the result's scale and more; the blocks themselves are alike
    scale = float(few.abs().max())
    assert float((out[139984:] - few).abs().max()) <= 128 * 2.0 ** -24 * 8 * scale
    assert bool(torch.isfinite(out).all())


def test_cache_past_four_gigabytes(torch, qlm):
    """Blocks whose codes stand past 2^32 bytes: as the first ones."""
    torch.manual_seed(10)
    kv, d, n_blocks = 8, 128, 70000
    cache = qlm.DeviceKvCache.empty(n_blocks, kv, d)
    rotary = turning(torch, qlm, 200, 64)
    k, v, q = (torch.randn((70, h, d), device="cuda").bfloat16() for h in (kv, kv, 16))
    got = []
    for ids in ([0, 1], [n_blocks - 1, n_blocks - 2]):
        at = torch.tensor(ids, device="cuda")
        for x in slots(torch, cache):
            x[at] = 0
        table = at.int().view(1, 2)
        out = qlm.kv_append_rotated(cache, batch_of(torch, qlm, table, [70], [70]), k, v, q, rotary)
        got.append([out] + [x[at] for x in slots(torch, cache)])
    assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("kind", ["float8_e4m3fn", "int8"])
@pytest.mark.parametrize("kv,d", [(3, 16), (2, 64), (1, 80), (2, 128), (1, 144), (1, 256)])
def test_tokens_that_grow(torch, qlm, kv, d, kind):
    """Tokens one by one, each larger than those before, so that blocks' scales grow, in batches of one
    token a sequence at most and in batches that could hold two: the same cache bit for bit."""
    torch.manual_seed(d)
    rotary = turning(torch, qlm, 100, d // 2)
    table = torch.arange(6, dtype=torch.int32, device="cuda").view(3, 2)
    caches = [qlm.DeviceKvCache.empty(6, kv, d, getattr(torch, kind)) for _ in range(4)]
    for c in caches:
        clear(c)
    for step in range(1, 70):
        k, v, q = (torch.randn((3, h, d), device="cuda").bfloat16() * 1.3 ** (step % 50) for h in (kv, kv, 2))
        lengths = torch.full((3,), step, dtype=torch.int32, device="cuda")
        one = qlm.KvBatch(table, lengths)
        start = torch.arange(4, dtype=torch.int32, device="cuda")
        two = qlm.KvBatch(table, lengths, start, 3, 2)
        qlm.kv_append(caches[0], one, k, v)
        qlm.kv_append(caches[1], two, k, v)
        a = qlm.kv_append_rotated(caches[2], one, k, v, q, rotary)
        b = qlm.kv_append_rotated(caches[3], two, k, v, q, rotary)
        assert torch.equal(a, b)
        if step % 9 == 0 or step > 62:
            for x, y in (caches[:2], caches[2:]):
                assert all(torch.equal(m, n) for m, n in zip(slots(torch, x), slots(torch, y))), step
    held = torch.arange(6, device="cuda").view(3, 2)
    assert bool((caches[0].k_scale[held] != 0).all())
