"""Products with 4-bit weights on the GPU against their definition in 64 bits,
within the error bound of single-precision sums."""
import numpy as np
import pytest

import kv_oracle as ko

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


def matrix(torch, n, k, group, zero=True, seed=0):
    rng = np.random.default_rng(seed + n + k)
    codes = rng.integers(0, 16, size=(n, k), dtype=np.uint8)
    ng = -(-k // group)
    scale = (rng.uniform(0.001, 0.1, size=(n, ng)) * rng.choice([-1, 1], size=(n, ng))).astype(
        np.float16)
    z = rng.integers(0, 16, size=(n, ng), dtype=np.uint8) if zero else None
    dev = lambda x: None if x is None else torch.from_numpy(x).cuda()  # noqa: E731
    return (codes, scale.astype(np.float64), z), (dev(codes), dev(scale), dev(z))


def rows(torch, m, k, dtype, seed=1, pad=0, mean=0.0):
    x = np.random.default_rng(seed + m).normal(mean, 1.0, size=(m, k + pad))
    dt = torch.bfloat16 if dtype == "bf16" else torch.float16
    t = torch.from_numpy(x).cuda().to(dt)[:, pad:]
    return t, t.double().cpu().numpy()


def check(got, want, bound, dtype, label=""):
    e = np.abs(got.double().cpu().numpy() - want)
    lim = ko.out_bound(want, bound, dtype)
    assert (e <= lim).all(), (label, float((e / lim).max()))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("m", [1, 2, 15, 16, 17, 33, 64, 65, 130])
def test_rows(torch, qlm, dtype, group, m):
    n, k = 83, 640
    host, dev = matrix(torch, n, k, group)
    w = qlm.w4_pack(*dev, group=group)
    x, xh = rows(torch, m, k, dtype)
    want, bound = ko.w4(xh, *host, group)
    check(qlm.w4_matmul(x, w), want, bound, dtype)


@pytest.mark.parametrize("n,k,group", [(1, 1, 32), (16, 31, 32), (17, 33, 32), (5, 127, 64),
                                       (130, 129, 128), (1000, 4100, 64), (64, 20000, 128),
                                       (3, 9001, 32)])
@pytest.mark.parametrize("m", [1, 7, 40])
def test_odd_sizes(torch, qlm, n, k, group, m):
    """Groups and steps that end short, no zero points (8 everywhere)."""
    host, dev = matrix(torch, n, k, group, zero=False)
    w = qlm.w4_pack(*dev, group=group)
    x, xh = rows(torch, m, k, "f16", mean=0.5)
    want, bound = ko.w4(xh, *host, group)
    check(qlm.w4_matmul(x, w), want, bound, "f16")


@pytest.mark.parametrize("m,pad", [(1, 3), (9, 1), (30, 8), (70, 5)])
def test_strides(torch, qlm, m, pad):
    """Rows apart and unaligned, an output that is a part of a larger one."""
    host, dev = matrix(torch, 70, 300, 64)
    w = qlm.w4_pack(*dev)
    x, xh = rows(torch, m, 300, "bf16", pad=pad)
    big = torch.full((m, 90), 5.0, dtype=torch.bfloat16, device="cuda")
    got = qlm.w4_matmul(x, w, out=big[:, 10:80])
    want, bound = ko.w4(xh, *host, 64)
    check(got, want, bound, "bf16")
    assert bool((big[:, :10] == 5).all()) and bool((big[:, 80:] == 5).all())


def test_magnitudes(torch, qlm):
    """Rows of very different size beside each other, zeros, large scales."""
    host, dev = matrix(torch, 40, 256, 32)
    dev[1].mul_(300.0)
    host = (host[0], dev[1].double().cpu().numpy(), host[2])
    w = qlm.w4_pack(*dev)
    for m in (5, 20):
        x, _ = rows(torch, m, 256, "bf16")
        x *= torch.tensor([1e-30, 0.0, 1.0, 1e20, 1e-8] * (m // 5), device="cuda",
                          dtype=torch.bfloat16)[:, None]
        want, bound = ko.w4(x.double().cpu().numpy(), *host, 32)
        check(qlm.w4_matmul(x, w), want, bound, "bf16")


@pytest.mark.parametrize("m", [1, 4, 16, 20])
def test_largest_magnitudes(torch, qlm, m):
    """Rows of bfloat16 up to its largest value, beside one down at its least normal ones:
    outputs that fit are finite, whichever form the number of rows takes."""
    for group in (32, 128):
        host, dev = matrix(torch, 40, 300, group)
        dev[1].mul_(2.0 ** -9)
        host = (host[0], dev[1].double().cpu().numpy(), host[2])
        w = qlm.w4_pack(*dev, group=group)
        x, _ = rows(torch, m, 300, "bf16")
        size = torch.tensor([3e37, 1e-36, 1e38, 1e36], device="cuda", dtype=torch.float64)
        x.copy_((x.double() * size[torch.arange(m, device="cuda") % 4][:, None])
                .clamp(-3.3e38, 3.3e38))
        if m == 1:
            x.abs_()                         # (sums that no sign keeps small)
        want, bound = ko.w4(x.double().cpu().numpy(), *host, group)
        assert (np.abs(want) < 3e38).all()
        check(qlm.w4_matmul(x, w), want, bound, "bf16", group)


def test_not_finite_rows(torch, qlm):
    """A row that is not finite spoils itself alone."""
    host, dev = matrix(torch, 50, 256, 64)
    w = qlm.w4_pack(*dev)
    for m in (4, 20):
        x, xh = rows(torch, m, 256, "f16")
        x[1, 9], x[2, 100] = float("nan"), float("inf")
        got = qlm.w4_matmul(x, w)
        assert not got[1:3].isfinite().any()
        keep = [r for r in range(m) if r not in (1, 2)]
        want, bound = ko.w4(xh[keep], *host, 64)
        check(got[keep], want, bound, "f16")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("k,group,pad", [(5120, 128, 0), (5000, 32, 0), (5120, 64, 8),
                                         (5120, 128, 3)])
@pytest.mark.parametrize("m", [1, 9, 10, 15, 16])
def test_few_rows_many_outputs(torch, qlm, m, k, group, pad, dtype):
    """Up to 16 rows on either side of the sizes from which x is shared by 64 outputs."""
    n = 4100
    host, dev = matrix(torch, n, k, group)
    w = qlm.w4_pack(*dev, group=group)
    x, xh = rows(torch, m, k, dtype, pad=pad)
    want, bound = ko.w4(xh, *host, group)
    got = qlm.w4_matmul(x, w)
    check(got, want, bound, dtype)
    assert torch.equal(got, qlm.w4_matmul(x, w))
    x[0, 3] = float("nan")
    again = qlm.w4_matmul(x, w)
    assert not again[:1].isfinite().any() and torch.equal(again[1:], got[1:])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n,k,counts", [(83, 2816, (8, 33, 300)), (83, 2700, (40,)),
                                        (4096, 11008, (8, 32, 64)), (3584, 18944, (8, 32, 64)),
                                        (6144, 8192, (8, 32, 64))])
def test_split_ends(torch, qlm, n, k, counts, dtype):
    """Inputs split so that the last share would end inside a pair of steps: x is the front
    of a larger tensor whose every other element is a not-a-number, on the right and
    below, and none of them is read; a row that is a not-a-number leaves the others as they are."""
    group = 128
    host, dev = matrix(torch, n, k, group)
    w = qlm.w4_pack(*dev, group=group)
    x, xh = rows(torch, max(counts), k, dtype)
    want, bound = ko.w4(xh, *host, group)
    for m in counts:
        outs = []
        for right in (0, 256):
            big = torch.full((m + 2, k + right), float("nan"), dtype=x.dtype, device="cuda")
            view = big[:m, :k]
            view.copy_(x[:m])
            ws = torch.full((qlm.w4_workspace_bytes(w, m),), 255, dtype=torch.uint8,
                            device="cuda")
            outs.append(qlm.w4_matmul(view, w, ws=ws))
            check(outs[-1], want[:m], bound[:m], dtype, (m, right))
        assert torch.equal(outs[0], outs[1])
        view[m // 2] = float("nan")
        got = qlm.w4_matmul(view, w)
        assert not got[m // 2].isfinite().any()
        keep = torch.arange(m, device="cuda") != m // 2
        assert torch.equal(got[keep], outs[1][keep])


def test_repeats_stream_graph(torch, qlm):
    """The same bits again, on another stream, and in a replayed graph."""
    _, dev = matrix(torch, 500, 2048, 128)
    w = qlm.w4_pack(*dev)
    for m in (1, 40):
        x, _ = rows(torch, m, 2048, "bf16")
        ws = qlm.w4_workspace(w, m)
        want = qlm.w4_matmul(x, w).clone()
        out = torch.empty_like(want)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        qlm.w4_matmul(x, w, out=out, ws=ws, stream=side)
        side.synchronize()
        assert torch.equal(out, want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            qlm.w4_matmul(x, w, out=out, ws=ws)
        for _ in range(3):
            out.zero_()
            ws.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want)


def test_no_rows(torch, qlm):
    _, dev = matrix(torch, 20, 64, 32)
    w = qlm.w4_pack(*dev)
    x = torch.empty((0, 64), dtype=torch.float16, device="cuda")
    assert qlm.w4_matmul(x, w).shape == (0, 20)
