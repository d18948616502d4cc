"""Where the tensors of the instance operators' calls are: memory that a call allocates for
itself, and tensors left on the host."""
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


def test_memory_beside_another_stream(torch, qlm):
    """Calls on a stream of their own that allocate for themselves, while the current stream
    allocates and writes memory of the same sizes: results as on the current stream."""
    gen = torch.Generator(device="cuda").manual_seed(0)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda").half()  # noqa: E731
    lengths = torch.tensor([3000, 2000], dtype=torch.int32, device="cuda")
    table = torch.arange(100, dtype=torch.int32, device="cuda").view(2, 50)
    caches = [qlm.DeviceKvCache.empty(100, 2, 64) for _ in range(2)]
    start = torch.tensor([0, 3000, 5000], dtype=torch.int32, device="cuda")
    k, v, q = rnd(5000, 2, 64), rnd(5000, 2, 64), rnd(2, 8, 64)
    codes = torch.randint(0, 16, (700, 1024), generator=gen, device="cuda", dtype=torch.uint8)
    scale, x = rnd(700, 8), rnd(40, 1024)
    b = qlm.KvBatch(table, lengths)
    side = torch.cuda.Stream()

    def steps(cache, stream):
        got = [qlm.kv_attention(cache, b, q, weight_decay=0.0, stream=stream)]
        disturb()
        got.append(qlm.kv_evict(cache, b, 512, 32, stream=stream))
        disturb()
        w = qlm.w4_pack(codes, scale, stream=stream)
        got.append(qlm.w4_matmul(x, w, stream=stream))
        disturb()
        return got + [cache.weight, w.packed]

    def disturb():
        for n in (qlm.kv_attention_workspace_bytes(caches[0], b, 8, True),
                  qlm.kv_evict_workspace_bytes(caches[0], b, 512), 2 * 8 * 64 * 2, 1 << 18):
            torch.empty(n, dtype=torch.uint8, device="cuda").fill_(255)

    for cache in caches:
        cache.weight.zero_()
        qlm.kv_append(cache, qlm.KvBatch(table, lengths, start, 5000, 3000), k, v)
    want = steps(caches[0], None)
    side.wait_stream(torch.cuda.current_stream())
    got = steps(caches[1], side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_host_tensors_beside_device_tensors(torch, qlm):
    """One tensor of a call left in host memory."""
    i32 = dict(dtype=torch.int32)
    half = lambda *s, dev="cuda": torch.zeros(s, dtype=torch.float16, device=dev)  # noqa: E731
    c = qlm.DeviceKvCache.empty(4, 2, 32)
    there = torch.zeros((2, 3), device="cuda", **i32), torch.zeros(2, device="cuda", **i32)
    b, host = qlm.KvBatch(*there), qlm.KvBatch(*(x.cpu() for x in there))
    k, q, hk, hq = half(2, 2, 32), half(2, 4, 32), half(2, 2, 32, dev="cpu"), half(2, 4, 32, dev="cpu")
    w = qlm.w4_pack(torch.zeros((4, 64), dtype=torch.uint8, device="cuda"), half(4, 2))
    ws = torch.zeros(1 << 25, dtype=torch.uint8)
    calls = [lambda: qlm.kv_append(c, host, k, k), lambda: qlm.kv_append(c, b, hk, k),
             lambda: qlm.kv_append(c, b, k, hk),
             lambda: qlm.kv_append(c, b, k, k, torch.zeros(2, **i32)),
             lambda: qlm.kv_attention(c, host, q), lambda: qlm.kv_attention(c, b, hq),
             lambda: qlm.kv_attention(c, b, q, out=hq), lambda: qlm.kv_attention(c, b, q, ws=ws),
             lambda: qlm.kv_evict(c, host, 64),
             lambda: qlm.kv_evict(c, b, 64, out=torch.zeros(2, **i32)),
             lambda: qlm.kv_evict(c, b, 64, ws=ws),
             lambda: qlm.w4_pack(torch.zeros((4, 64), dtype=torch.uint8, device="cuda"),
                                 half(4, 2, dev="cpu")),
             lambda: qlm.w4_matmul(half(2, 64, dev="cpu"), w),
             lambda: qlm.w4_matmul(half(2, 64), w, out=half(2, 4, dev="cpu")),
             lambda: qlm.w4_matmul(half(2, 64), w, ws=ws)]
    for call in calls:
        with pytest.raises(ValueError, match="must be on the GPU"):
            call()
