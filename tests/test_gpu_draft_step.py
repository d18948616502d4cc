"""A drafting instance's operators used together: turned appends, attention of several rows,
products of either weights, verification and the cut of the cache, step after step."""
import importlib.util
import os

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location(
        "instance_profile", os.path.join(ROOT, "examples", "instance_profile.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


@pytest.mark.parametrize("bits", ["4", "8"])
def test_example_runs(example, bits):
    got = example.main(["--layers", "2", "--hidden", "256", "--heads", "4", "--kv-heads", "2",
                        "--dim", "64", "--inner", "512", "--batch", "3", "--prompt", "150",
                        "--budget", "128", "--recent", "16", "--steps", "40", "--plans", "256",
                        "--bits", bits, "--drafts", "3", "--vocab", "500"])
    assert 0 <= got["best"] < 256 and got["score"] >= 0
    for g in got["measured"]:
        assert g["prefill"] > 0 and g["decode_time"] > 0 and g["kv_tokens"] > 0
        assert 1 <= g["tokens_a_step"] <= 4
        lengths = g["lengths"].cpu().numpy()
        assert (lengths >= 128).all() and (lengths <= 128 + 64).all()
    assert np.isfinite(got["profile"]["decode_time"]).all()


def test_example_runs_on_eight_bits(example):
    got = example.main(["--layers", "2", "--hidden", "256", "--heads", "4", "--kv-heads", "2",
                        "--dim", "64", "--inner", "512", "--batch", "3", "--prompt", "150",
                        "--budget", "128", "--recent", "16", "--steps", "20", "--plans", "256",
                        "--bits", "8"])
    assert all(g["decode_time"] > 0 for g in got["measured"])


def test_kept_tokens_are_as_their_prompt(example):
    """What a drafted step's rows give, of the tokens that stay, is what the same tokens give as
    one prompt: refused drafts leave no trace in later rows.  The outputs differ by the
    rounding of codes under other block scales (powers of two: of e4m3 codes only subnormals
    round anew) and of bfloat16, which the layer's few products pass on."""
    import torch
    model = example.Model(128, 4, 2, 32, 256, vocab=60)
    batch, n, steps = 3, 4, 12
    inst = example.Instance(model, 1, batch, 256, positions=100)
    gen = torch.Generator(device="cuda").manual_seed(3)
    seen = []
    forward = inst.forward

    def noted(x, new):
        y = forward(x, new)
        seen.append((x.view(batch, new, -1), y.view(batch, new, -1)))
        return y

    inst.forward = noted
    tokens = torch.tensor([1, 2, 3], dtype=torch.int32, device="cuda")
    counts = []
    for _ in range(steps):
        got, count = inst.drafted_step(tokens, n, gen)
        assert bool(((got >= 0).sum(1) == count).all())
        tokens = got.gather(1, (count - 1).long()[:, None])[:, 0].contiguous()
        counts.append(count.cpu().tolist())
    total = np.sum(counts, 0)
    assert inst.lengths.cpu().tolist() == total.tolist() == inst.next.cpu().tolist()
    assert steps * batch < total.sum() < steps * batch * (n + 1)     # (some kept, some refused)
    for s in range(batch):
        x = torch.cat([seen[i][0][s, :counts[i][s]] for i in range(steps)])
        rows = torch.cat([seen[i][1][s, :counts[i][s]] for i in range(steps)])
        whole = example.Instance(model, 1, 1, 256, positions=100).forward(x, x.shape[0])
        d = (whole.float() - rows.float()).abs()
        # a bfloat16 rounding of each of six results in a row (the turned queries among them),
        # and of the e4m3 codes' values far below it
        assert float(d.max()) <= 7 * 2.0 ** -8 * float(whole.float().abs().max())


def test_drafted_steps_do_not_wait(example, monkeypatch):
    """Drafted steps and cuts are queued without a read of device memory."""
    import torch
    monkeypatch.undo()                   # (the tests' filling of fresh memory waits for it)
    model = example.Model(128, 4, 2, 32, 256, layers=2, bits=8, vocab=100)
    inst = example.Instance(model, 2, 3, 192, positions=400)
    gen = torch.Generator(device="cuda").manual_seed(3)
    tokens = torch.zeros(3, dtype=torch.int32, device="cuda")
    inst.drafted(tokens, 3, 17, 64, 8, gen)
    torch.cuda.synchronize()
    torch.cuda.set_sync_debug_mode("error")
    try:
        total = inst.drafted(tokens, 3, 33, 64, 8, gen)
    finally:
        torch.cuda.set_sync_debug_mode("default")
    assert 33 * 3 <= int(total) <= 33 * 3 * 4
    assert (inst.lengths <= 128).all()
