"""Verification of drafted tokens over rows so long that their sums come from a launch before, and
over the largest vocabularies, on the GPU, against the definition in 64 bits."""
import pytest

from test_gpu_draft import Step

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


def whole(torch, s, start=0):
    """Probabilities that are whole numbers over 2^24, so that every order of adding them in double
    precision gives the same sums, whatever the words' number (in the step's type: small whole
    numbers then)."""
    for x in (s.target, s.draft):
        if x is not None:
            gen = torch.Generator(device="cuda").manual_seed(start)
            x.copy_(torch.randint(0, 4, x.shape, generator=gen, device="cuda") * 2.0 ** -24)
            start += 1


@pytest.mark.parametrize("given", [True, False])
@pytest.mark.parametrize("kind", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("seqs,vocab", [(1, 300001), (2, 262144)])
def test_sums_from_before(torch, qlm, seqs, vocab, kind, given):
    """(of 16 bits with drafts chosen, too, a row this long takes the launch before)"""
    s = Step(torch, qlm, [4] * seqs, vocab, kind, given, seed=seqs)
    assert qlm.draft_verify_workspace_bytes(s.batch, vocab) > 0
    whole(torch, s)
    s.check()


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
@pytest.mark.parametrize("given", [True, False])
def test_nothing_left(torch, qlm, given, kind):
    """Sums from before that come to nothing, to an infinity or not to a number are made anew."""
    vocab = 400001
    s = Step(torch, qlm, [2] * 6, vocab, kind, given, seed=4)
    assert qlm.draft_verify_workspace_bytes(s.batch, vocab) > 0
    whole(torch, s, 7)
    s.uniform[0::2] = 0.999
    for r in range(0, 12, 2):
        s.target[r, int(s.tokens[r + 1])] = 0.0         # refused
    if given:
        s.draft.copy_(s.target * 2 + 1)                 # nothing is left: from the target
    s.target[2] = 0.0                                   # not even there
    s.target[4, 7] = float("nan")
    s.target[6, vocab - 1] = float("inf")
    if given:
        s.draft[8, 3] = float("nan")                    # (the target itself is fine)
        s.draft[10, 5] = float("inf")
    got = s.check()
    assert got[0][1, 0] == -1 and got[0][2, 0] == -1 and got[0][3, 0] == -1
    assert (got[0][4:, 0] >= 0).all()


@pytest.mark.parametrize("seqs", [1, 70])
def test_the_largest_vocabularies(torch, qlm, seqs):
    """Segments of several turns of a wave: their sums from a launch before, or (70 sequences) in
    the same one; u on borders, at the ends and between."""
    vocab = (1 << 24) if seqs == 1 else (1 << 20) + 333
    s = Step(torch, qlm, [1] * seqs, 4, "bfloat16", False)
    assert (qlm.draft_verify_workspace_bytes(s.batch, vocab) > 0) == (seqs == 1)
    s.target = torch.empty((seqs, vocab), dtype=torch.bfloat16, device="cuda")
    whole(torch, s, 3)
    s.target[:, vocab // 2:vocab // 2 + 5000] = 0.0
    for u in (0.0, 0.25, 0.499, 0.5, 0.501, 1 - 2.0 ** -24):
        s.uniform.fill_(u)
        s.check()


@pytest.mark.parametrize("most", [1, 5])
def test_repeats_itself(torch, qlm, most):
    s = Step(torch, qlm, [most, 3], 500000, seed=9)
    assert qlm.draft_verify_workspace_bytes(s.batch, 500000) > 0
    one = s.run()
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(one, s.run()))
