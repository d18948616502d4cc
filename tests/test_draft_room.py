"""Workspaces of the drafting step's operators, without a GPU: at sizes that need room, none, too
little and misaligned room are refused."""
import pytest

from test_draft_checks import A, P, batch, lib, made, qlm  # noqa: F401


@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("seqs,vocab", [(1, 300000), (2, 131072), (60, 1 << 20)])
def test_verification(qlm, lib, seqs, vocab, drawn, dtype):  # noqa: F811
    b = batch(qlm, n_seqs=seqs, n_rows=seqs)
    need = lib.qlm_draft_verify_workspace_bytes(P(b), vocab)
    assert need > 0
    d = made(qlm.DraftStruct, dict(vocab=vocab, dtype=dtype, target=A, draft=A if drawn else None,
                                   target_stride=vocab, draft_stride=vocab, tokens=A, uniform=A), {})
    for ws, size in ((None, need), (A + 128, need), (A, need - 1), (A, 0)):
        assert lib.qlm_draft_verify(P(b), P(d), A, A, A, ws, size, None) == qlm.QLM_ERR_WORKSPACE


@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("rows,n_out,n_in", [(3414, 300, 13578), (466, 505, 13323), (256, 256, 1 << 24)])
def test_products_in_runs(qlm, lib, rows, n_out, n_in, dtype):  # noqa: F811
    w, r = qlm.F8Struct(n_out, n_in, A), qlm.F8CodesStruct(rows, n_in, A, A)
    need = lib.qlm_f8_workspace_bytes(P(w), rows)
    assert need >= 2 * 4 * rows * n_out
    for ws, size in ((None, need), (A + 128, need), (A, need - 1), (A, 0)):
        assert lib.qlm_f8_matmul(P(r), P(w), 2 * A, n_out, dtype, ws, size, None) == \
            qlm.QLM_ERR_WORKSPACE
