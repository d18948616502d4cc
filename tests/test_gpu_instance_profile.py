"""The instance operators used together: the example that measures a hardware
profile, at a small size, and a layer's decode against its prompt."""
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


def test_example_runs(example):
    got = example.main(["--layers", "2", "--hidden", "256", "--heads", "4", "--kv-heads", "2",
                        "--dim", "64", "--inner", "512", "--batch", "3", "--prompt", "150",
                        "--budget", "128", "--recent", "16", "--steps", "70", "--plans", "256"])
    assert 0 <= got["best"] < 256 and got["score"] >= 0
    for g in got["measured"]:
        assert g["prefill"] > 0 and g["decode_time"] > 0 and g["kv_tokens"] > 0
        # every block that filled up was followed by a cut to the budget
        lengths = g["lengths"].cpu().numpy()
        assert (lengths >= 128).all() and (lengths < 128 + 64 + 2).all()
    assert np.isfinite(got["profile"]["decode_time"]).all()


def test_prompt_and_steps_agree(example):
    """The same tokens as one prompt and one after another: the outputs differ by the
    rounding of codes under other block scales (powers of two: of e4m3 codes only
    subnormals round anew) and of bfloat16, which the layer's few products pass on."""
    import torch
    model = example.Model(128, 4, 2, 32, 256)
    x = torch.randn((40, 128), device="cuda", dtype=torch.bfloat16)
    whole = example.Instance(model, 1, 1, 64).forward(x, 40)
    step = example.Instance(model, 1, 1, 64)
    rows = torch.cat([step.forward(x[i:i + 1], 1) for i in range(40)])
    d = (whole.float() - rows.float()).abs()
    # a bfloat16 rounding of each of five results in a row, and of the e4m3 codes'
    # values (2^-4 of a subnormal step) far below it
    assert float(d.max()) <= 6 * 2.0 ** -8 * float(whole.float().abs().max())


def test_layers_have_weights_of_their_own(example, monkeypatch):
    """A step reads as many weights as the layers count: no layer's come a second time."""
    seen = []
    real = example.qlm.w4_matmul

    def noted(x, w, **more):
        seen.append(w.packed.data_ptr())
        return real(x, w, **more)

    monkeypatch.setattr(example.qlm, "w4_matmul", noted)
    example.main(["--layers", "3", "--hidden", "128", "--heads", "4", "--kv-heads", "2",
                  "--dim", "32", "--inner", "256", "--batch", "2", "--prompt", "20",
                  "--budget", "64", "--recent", "8", "--steps", "2", "--plans", "64"])
    # the first pass: a prompt through three layers of four matrices
    assert len(set(seen[:12])) == 12 and set(seen) == set(seen[:12])


def test_decode_does_not_wait(example, monkeypatch):
    """Decode steps and cuts are queued without a read of device memory, whose wait would
    be timed with them; lengths and positions as counted by the host."""
    import torch
    monkeypatch.undo()                   # (the tests' filling of fresh memory waits for it)
    model = example.Model(128, 4, 2, 32, 256, layers=2)
    inst = example.Instance(model, 2, 3, 192)
    x = torch.randn((3, 128), device="cuda", dtype=torch.bfloat16)
    inst.forward(x.repeat_interleave(60, 0), 60)
    inst.evict(64, 8)
    inst.decode(x, 1, 64, 8)
    torch.cuda.synchronize()
    torch.cuda.set_sync_debug_mode("error")
    try:
        inst.decode(x, 80, 64, 8)
    finally:
        torch.cuda.set_sync_debug_mode("default")
    assert inst.position == 141 and inst.next.cpu().tolist() == [141] * 3
    # cut to 64 at 128 tokens, then 13 more
    assert inst.lengths.cpu().tolist() == [77] * 3
