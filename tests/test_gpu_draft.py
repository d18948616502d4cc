"""Verification of drafted tokens on the GPU against the definition in 64 bits, token for
token, and the distribution of what it draws."""
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


def drawn(w, u):
    """The least word whose running sum passes u of the whole; -1 of no sum."""
    total = w.sum()
    if not (total > 0 and np.isfinite(total)):
        return -1
    below = np.cumsum(w)
    return int(np.searchsorted(below, u * below[-1], side="right"))


def verified(counts, lengths, tokens, target, draft, uniform, most):
    """The definition; target and draft in 64 bits."""
    out = np.full((len(counts), most), -1)
    count, left = np.zeros(len(counts), int), np.array(lengths)
    vocab = target.shape[1] if len(target) else 0
    r = 0
    for s, n in enumerate(counts):
        if n == 0:
            continue
        kept = 0
        while kept < n - 1:
            t = tokens[r + kept + 1]
            if not 0 <= t < vocab:
                break
            q = 1.0 if draft is None else draft[r + kept, t]
            if not uniform[r + kept] * q < target[r + kept, t]:
                break
            out[s, kept] = t
            kept += 1
        p = target[r + kept]
        w = p
        if kept < n - 1:
            if draft is not None:
                q = draft[r + kept]
            else:
                q = np.zeros(vocab)
                if 0 <= tokens[r + kept + 1] < vocab:
                    q[tokens[r + kept + 1]] = 1.0
            w = np.where(p - q < 0, 0.0, p - q)
            if not (w.sum() > 0 and np.isfinite(w.sum())):
                w = p
        out[s, kept] = drawn(w, uniform[r + n - 1])
        count[s], left[s] = kept + 1, max(0, lengths[s] - (n - 1 - kept))
        r += n
    return out, count, left


class Step:
    """A step's batch and its probabilities, drafts near the target."""

    def __init__(self, torch, qlm, counts, vocab, kind="float32", drawn_=True, seed=0, near=0.7,
                 extra=0, lengths=None, pad=0, shift=0):
        torch.manual_seed(seed)
        self.torch, self.qlm, self.counts = torch, qlm, counts
        rows = sum(counts) + extra
        dt = getattr(torch, kind)
        logits = 2.0 * torch.randn((rows, vocab), device="cuda")
        near = logits + near * torch.randn((rows, vocab), device="cuda")

        def placed(x):
            big = torch.full((rows, vocab + pad), float("nan"), dtype=dt, device="cuda")
            view = big[:, shift:shift + vocab]
            view.copy_(x)
            return view

        self.target = placed(torch.softmax(logits, -1))
        near = torch.softmax(near, -1)
        self.draft = placed(near) if drawn_ else None
        noise = torch.rand((rows, vocab), device="cuda").clamp_(min=1e-9)
        self.tokens = torch.roll((near / -noise.log()).argmax(-1), 1).int() if rows else \
            torch.zeros(0, dtype=torch.int32, device="cuda")
        self.uniform = torch.rand(rows, device="cuda")
        self.lengths = [3 * i + n for i, n in enumerate(counts)] if lengths is None else lengths
        start = np.concatenate([[0], np.cumsum(counts)])
        i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")  # noqa: E731
        most = max([1] + counts)
        table = torch.zeros((len(counts), -(-max([1] + self.lengths) // 64)), dtype=torch.int32,
                            device="cuda")
        self.batch = qlm.KvBatch(table, i32(self.lengths), i32(start), rows, most)

    def run(self, **more):
        return self.qlm.draft_verify(self.batch, self.tokens, self.target, self.draft, self.uniform,
                                     **more)

    def check(self, **more):
        got = [x.cpu().numpy() for x in self.run(**more)]
        wide = lambda x: None if x is None else x.double().cpu().numpy()  # noqa: E731
        want = verified(self.counts, self.lengths, self.tokens.cpu().numpy(), wide(self.target),
                        wide(self.draft), wide(self.uniform), self.batch.max_new)
        for name, a, b in zip(("tokens", "count", "lengths"), got, want):
            assert (a == b).all(), (name, np.argwhere(a != b)[:4].tolist(), a[a != b][:4],
                                    b[a != b][:4])
        return got


COUNTS = [5, 1, 0, 2, 9, 3, 1, 6, 0, 4, 4, 4]


@pytest.mark.parametrize("kind", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("given", [True, False])
@pytest.mark.parametrize("vocab", [1, 2, 7, 63, 64, 257, 1000, 4096, 5001, 32000, 70001])
def test_vocabularies(torch, qlm, vocab, given, kind):
    Step(torch, qlm, COUNTS, vocab, kind, given, seed=vocab).check()


@pytest.mark.parametrize("counts", [[1], [2], [8], [1] * 70, [3] * 300, [0, 0, 0], [0, 0, 5, 0]])
def test_batches(torch, qlm, counts):
    Step(torch, qlm, counts, 3001, seed=len(counts)).check()


@pytest.mark.parametrize("kind", ["float32", "float16"])
@pytest.mark.parametrize("seqs,vocab", [(1, 300000), (2, 131072), (5, 200001), (70, 40000)])
def test_large(torch, qlm, seqs, vocab, kind):
    Step(torch, qlm, [4] * seqs, vocab, kind, seed=seqs).check()


@pytest.mark.parametrize("near,label", [(0.0, "all kept"), (0.05, "most kept"), (8.0, "few kept")])
def test_drafts_near_and_far(torch, qlm, near, label):
    got = Step(torch, qlm, [9] * 40, 500, near=near, seed=7).check()
    if label == "all kept":
        assert (got[1] == 9).all()


@pytest.mark.parametrize("drafts", [63, 64, 65, 130])
def test_many_drafts(torch, qlm, drafts):
    """More drafts than lanes, kept up to a place of our choice."""
    for stop in (0, 1, 63, 64, drafts - 1, drafts):
        s = Step(torch, qlm, [drafts + 1, 3], 50, seed=drafts)
        s.uniform[:drafts] = 0.0                     # accepted, whatever the probabilities
        if stop < drafts:
            s.target[stop, int(s.tokens[stop + 1])] = 0.0
        got = s.check()
        assert got[1][0] == min(stop, drafts) + 1


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
@pytest.mark.parametrize("pad,shift", [(1, 0), (3, 1), (5, 2), (8, 8), (9, 7)])
def test_strides(torch, qlm, pad, shift, kind):
    """Rows that stand anywhere on their 16 bytes, between not-a-numbers."""
    Step(torch, qlm, COUNTS, 1003, kind, pad=pad, shift=shift).check()


@pytest.mark.parametrize("kind", ["float32", "float16"])
def test_target_and_draft_placed_apart(torch, qlm, kind):
    s = Step(torch, qlm, COUNTS, 1003, kind, pad=5, shift=1)
    s.draft = torch.cat([s.draft, s.draft[:, :2]], 1)[:, :1003]
    s.check()


def test_borders(torch, qlm):
    """u on a border of the running sum: the next word; u = 0: the first word of any weight."""
    s = Step(torch, qlm, [1] * 6, 8)
    s.target.copy_(torch.tensor([0, 0.25, 0, 0.25, 0, 0, 0.5, 0]).expand(6, 8))
    s.uniform.copy_(torch.tensor([0.0, 0.25, 0.2499, 0.5, 0.75, 1 - 2.0 ** -24]))
    got = s.check()
    assert got[0][:, 0].tolist() == [1, 3, 1, 6, 6, 6]


@pytest.mark.parametrize("vocab", [3000, 131072])
@pytest.mark.parametrize("u", [1 - 2.0 ** -24, 1.0, 1.5, float("nan")])
def test_nothing_behind_the_last_weight(torch, qlm, vocab, u):
    """Words of no weight after the last one of any, and between: none of them is drawn, not by a
    uniform number that came out as 1 either."""
    s = Step(torch, qlm, [1] * 5, vocab, seed=8)
    s.target[:, vocab // 3:] = 0.0
    s.target[:, : vocab // 5] = 0.0
    s.target[1, vocab // 2] = 0.25
    s.target[2].fill_(0.0)
    s.target[2, 5] = 1e-30
    s.uniform.fill_(u)
    tokens = s.run()[0][:, 0].cpu().numpy()
    p = s.target.cpu().numpy()
    assert (p[np.arange(5), tokens] > 0).all()
    assert tokens[1] == vocab // 2 and tokens[2] == 5
    if not u < 1:
        assert (tokens == [np.flatnonzero(row)[-1] for row in p]).all()


def test_acceptance_border(torch, qlm):
    """u q < p exactly: equal is refused."""
    s = Step(torch, qlm, [2, 2, 2], 4)
    s.target.fill_(0.25)
    s.draft.fill_(0.5)
    s.tokens.fill_(2)
    for row, u in ((0, 0.5), (2, 0.5 - 2.0 ** -25), (4, 0.6)):
        s.uniform[row] = u
    got = s.check()
    assert got[1].tolist() == [1, 2, 1]


@pytest.mark.parametrize("given", [True, False])
def test_nothing_left(torch, qlm, given):
    """Weights that sum to nothing, to an infinity or not to a number."""
    s = Step(torch, qlm, [2] * 6, 300, drawn_=given, seed=4)
    s.uniform[0::2] = 0.999
    for r in range(0, 12, 2):
        s.target[r, int(s.tokens[r + 1])] = 0.0         # refused
    if given:
        s.draft.copy_(s.target * 2 + 1)                 # nothing is left: from the target
    s.target[2] = 0.0                                   # not even there
    s.target[4, 7] = float("nan")
    s.target[6, 9] = float("inf")
    if given:
        s.draft[8, 3] = float("nan")                    # (the target itself is fine)
        s.draft[10, 5] = float("inf")
    got = s.check()
    assert got[0][1, 0] == -1 and got[0][2, 0] == -1 and got[0][3, 0] == -1
    assert (got[0][4:, 0] >= 0).all()


@pytest.mark.parametrize("given", [True, False])
def test_tokens_outside_the_vocabulary(torch, qlm, given):
    s = Step(torch, qlm, [3, 3, 3], 100, drawn_=given)
    s.uniform[:] = 0.0
    s.tokens[1], s.tokens[5], s.tokens[7] = -1, 100, 2 ** 31 - 1
    assert s.check()[1].tolist() == [1, 2, 1]


def test_lengths_in_place(torch, qlm):
    """The batch's own lengths cut; a length shorter than its rows stays at 0."""
    s = Step(torch, qlm, [9, 1, 0, 9], 200, near=8.0, lengths=[100, 7, 5, 2])
    s.target[0, int(s.tokens[1])] = 0.0
    s.uniform[0] = 0.5
    got = s.check(lengths=s.batch.lengths)
    now = s.batch.lengths.cpu().tolist()
    assert now == got[2].tolist() and now[0] == 92 and now[1:3] == [7, 5]


def test_rows_of_no_sequence(torch, qlm):
    """Rows behind the last sequence's: nothing of them is read."""
    s = Step(torch, qlm, [3, 2], 100, extra=4)
    s.target[5:] = float("nan")
    s.draft[5:] = float("nan")
    s.check()


def test_without_row_start(torch, qlm):
    """One row a sequence: no drafts, a token drawn for each."""
    s = Step(torch, qlm, [1] * 9, 777)
    s.batch = qlm.KvBatch(s.batch.block_table, s.batch.lengths)
    assert (s.check()[1] == 1).all()


def test_distribution(torch, qlm):
    """A verified token is distributed as the target has it, whatever the draft: of N = 60000
    sequences each word's share is within 5 standard deviations (12 words: by Hoeffding's
    sharper form less than one run in 10^5 would not be, and the seed is fixed)."""
    n, vocab = 60000, 12
    torch.manual_seed(9)
    p = torch.softmax(torch.randn(vocab, device="cuda"), 0)
    q = torch.softmax(torch.randn(vocab, device="cuda"), 0)
    s = Step(torch, qlm, [2], vocab)
    table = torch.zeros((n, 1), dtype=torch.int32, device="cuda")
    start = torch.arange(n + 1, dtype=torch.int32, device="cuda") * 2
    lengths = torch.full((n,), 2, dtype=torch.int32, device="cuda")
    s.batch = qlm.KvBatch(table, lengths, start, 2 * n, 2)
    s.target, s.draft = p.expand(2 * n, vocab).contiguous(), q.expand(2 * n, vocab).contiguous()
    s.tokens = torch.multinomial(q, 2 * n, replacement=True).int()
    s.uniform = torch.rand(2 * n, device="cuda")
    tokens = s.run()[0][:, 0].long()
    share = torch.bincount(tokens, minlength=vocab).double() / n
    p = p.double() / p.double().sum()
    assert bool(((share - p).abs() <= 5 * (p * (1 - p) / n).sqrt()).all())


def test_captured_and_replayed(torch, qlm):
    s = Step(torch, qlm, COUNTS, 9000)
    ws = qlm.draft_verify_workspace(s.batch, 9000)
    s.run(ws=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = s.run(ws=ws)
    for i in range(5):
        s.uniform.copy_(torch.rand(s.uniform.shape, device="cuda"))
        s.target.copy_(s.target.roll(1, 0))
        for x in got:
            x.fill_(-9)
        graph.replay()
        torch.cuda.synchronize()
        want = s.check()
        for a, b in zip(got, want):
            assert (a.cpu().numpy() == b).all(), i


def test_on_a_side_stream(torch, qlm):
    s = Step(torch, qlm, COUNTS, 5000)
    want = s.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = s.run(stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
