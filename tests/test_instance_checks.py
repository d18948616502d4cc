"""The instance operators without a GPU: host-side argument checks of the C
interface and of the binding, before anything reaches the device."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def qlm():
    from paper_2407_00047_amd import qlm
    return qlm


@pytest.fixture(scope="module")
def lib(qlm):
    return qlm.library()


A = 0x100000          # a pointer that the checks never follow
P = ctypes.byref


def cache(qlm, **more):
    f = dict(n_blocks=8, n_kv_heads=2, head_dim=64, format=0, k_codes=A, v_codes=A, k_scale=A,
             v_scale=A, position=A, weight=A)
    f.update(more)
    return qlm.KvCacheStruct(*f.values())


def batch(qlm, **more):
    f = dict(n_seqs=2, n_rows=2, max_new=1, max_length=100, table_stride=2, block_table=A,
             lengths=A, row_start=None)
    f.update(more)
    return qlm.KvBatchStruct(*f.values())


def rows(qlm, **more):
    f = dict(data=A, row_stride=128, head_stride=64, dtype=0)
    f.update(more)
    return qlm.Rows(*f.values())


BAD_CACHE = [dict(n_blocks=0), dict(n_kv_heads=0), dict(n_kv_heads=1025), dict(head_dim=0),
             dict(head_dim=8), dict(head_dim=72), dict(head_dim=272), dict(format=2),
             dict(format=-1), dict(k_codes=None), dict(v_codes=None), dict(k_scale=None),
             dict(v_scale=None), dict(k_codes=A + 8), dict(v_codes=A + 4)]
BAD_BATCH = [dict(n_seqs=-1), dict(n_rows=-1), dict(max_new=0), dict(max_length=-1),
             dict(max_length=(1 << 28) + 1, table_stride=1 << 23), dict(table_stride=1),
             dict(block_table=None), dict(lengths=None), dict(n_rows=3), dict(max_new=2),
             dict(n_seqs=(1 << 20) + 1, n_rows=(1 << 20) + 1)]


def calls(qlm, lib, c, b):
    """The three calls with otherwise good arguments."""
    r = rows(qlm)
    out = rows(qlm, data=A + 4096)
    q = qlm.KvQuery(r, out, 4, 0.125, 0, 0.0)
    big = 1 << 40
    return [lib.qlm_kv_append(c, b, P(r), P(r), None, None),
            lib.qlm_kv_attention(c, b, P(q), A, big, None),
            lib.qlm_kv_evict(c, b, 64, 0, A, A, big, None)]


@pytest.mark.parametrize("bad", BAD_CACHE, ids=str)
def test_bad_caches(qlm, lib, bad):
    assert calls(qlm, lib, P(cache(qlm, **bad)), P(batch(qlm))) == [qlm.QLM_ERR_ARG] * 3


@pytest.mark.parametrize("bad", BAD_BATCH, ids=str)
def test_bad_batches(qlm, lib, bad):
    assert calls(qlm, lib, P(cache(qlm)), P(batch(qlm, **bad))) == [qlm.QLM_ERR_ARG] * 3


def test_null_structs(qlm, lib):
    assert calls(qlm, lib, None, P(batch(qlm))) == [qlm.QLM_ERR_ARG] * 3
    assert calls(qlm, lib, P(cache(qlm)), None) == [qlm.QLM_ERR_ARG] * 3
    assert b"batch" in lib.qlm_last_error()


def test_append_checks(qlm, lib):
    c, b = cache(qlm), batch(qlm)
    good = rows(qlm)
    for bad in (None, rows(qlm, data=None), rows(qlm, dtype=2), rows(qlm, data=A + 1)):
        p = None if bad is None else P(bad)
        assert lib.qlm_kv_append(P(c), P(b), p, P(good), None, None) == qlm.QLM_ERR_ARG
        assert lib.qlm_kv_append(P(c), P(b), P(good), p, None, None) == qlm.QLM_ERR_ARG
    # nothing to write: no device work
    none = batch(qlm, n_seqs=0, n_rows=0)
    assert lib.qlm_kv_append(P(c), P(none), None, None, None, None) == qlm.QLM_OK


def test_attention_checks(qlm, lib):
    c, b = cache(qlm), batch(qlm)
    good = dict(q=rows(qlm), out=rows(qlm, data=A + 4096), n_heads=4, scale=0.1, accumulate=0,
                weight_decay=0.0)
    need = lib.qlm_kv_attention_workspace_bytes(P(c), P(b), 4, 0)
    assert need > 0
    assert lib.qlm_kv_attention_workspace_bytes(P(c), P(b), 4, 1) > need
    assert lib.qlm_kv_attention_workspace_bytes(None, P(b), 4, 0) == 0
    assert lib.qlm_kv_attention_workspace_bytes(P(c), P(b), 0, 0) == 0

    def call(ws=A, size=need, cc=c, **more):
        f = dict(good)
        f.update(more)
        return lib.qlm_kv_attention(P(cc), P(b), P(qlm.KvQuery(*f.values())), ws, size, None)

    assert lib.qlm_kv_attention(P(c), P(b), None, A, need, None) == qlm.QLM_ERR_ARG
    nan, inf = float("nan"), float("inf")
    for bad in (dict(n_heads=0), dict(n_heads=3), dict(n_heads=1 << 17), dict(scale=nan),
                dict(scale=inf), dict(q=rows(qlm, data=None)), dict(out=rows(qlm, dtype=1)),
                dict(out=rows(qlm)), dict(accumulate=1, weight_decay=nan),
                dict(accumulate=1, weight_decay=-1.0), dict(accumulate=1, weight_decay=inf),
                dict(accumulate=1, cc=cache(qlm, weight=None))):
        assert call(**bad) == qlm.QLM_ERR_ARG, bad
    for bad in (dict(ws=None), dict(ws=A + 16), dict(size=need - 1)):
        assert call(**bad) == qlm.QLM_ERR_WORKSPACE, bad


def test_attention_capacity(qlm, lib):
    """Sizes whose index arithmetic would not fit are refused, whatever the workspace."""
    c = cache(qlm)
    q = qlm.KvQuery(rows(qlm), rows(qlm, data=A + 4096), 2 << 10, 0.1, 0, 0.0)
    huge = batch(qlm, n_seqs=1, n_rows=1, max_new=1 << 21, row_start=A)
    assert lib.qlm_kv_attention(P(c), P(huge), P(q), A, 1 << 62, None) == qlm.QLM_ERR_CAPACITY
    many = batch(qlm, n_seqs=1 << 20, n_rows=1 << 20, max_length=1 << 20, table_stride=1 << 14)
    assert lib.qlm_kv_attention(P(c), P(many), P(q), A, 1 << 62, None) == qlm.QLM_ERR_CAPACITY
    assert lib.qlm_kv_evict(P(c), P(many), 64 << 14, 0, A, A, 1 << 62, None) == \
        qlm.QLM_ERR_CAPACITY
    assert lib.qlm_kv_append(P(c), P(batch(qlm, n_seqs=1 << 20, n_rows=1 << 20, max_new=1 << 20,
                                           max_length=1 << 20, table_stride=1 << 14, row_start=A)),
                             P(rows(qlm)), P(rows(qlm)), None, None) == qlm.QLM_ERR_CAPACITY


def test_workspace_of_prompts_beside_steps(qlm, lib):
    """One prompt joins a decode step whose weights are kept: the scores' room does not
    grow with the sequences without end."""
    c = cache(qlm, n_blocks=48000, n_kv_heads=8, head_dim=128)
    need = lib.qlm_kv_attention_workspace_bytes

    def mixed(seqs, length):
        b = batch(qlm, n_seqs=seqs, n_rows=seqs - 1 + 2000, max_new=2000, max_length=length,
                  table_stride=length // 64, row_start=A)
        return need(P(c), P(b), 64, 1)

    assert mixed(48, 4096) < 1 << 30
    for seqs, length in ((192, 16000), (1000, 16000), (192, 100032)):
        # (beside the scores: rows laid out, parts and splits)
        assert mixed(seqs, length) < (4 << 30) + (1 << 28)
    # one sequence's scores are the least
    assert mixed(3, 1 << 22) < (8 << 30) + (1 << 28)


def test_launches_of_too_many_threads(qlm, lib):
    """A call whose last launch would have 2^32 threads is refused before its first one."""
    big = 1 << 62
    q = qlm.KvQuery(rows(qlm), rows(qlm, data=A + 4096), 8, 0.1, 1, 0.0)
    c = cache(qlm, n_kv_heads=8)
    # the weights of prompts: a workgroup of 256 to each of 8 heads and 2^21 blocks
    b = batch(qlm, n_seqs=1, n_rows=100, max_new=100, max_length=1 << 27, table_stride=1 << 21,
              row_start=A)
    assert lib.qlm_kv_attention(P(c), P(b), P(q), A, big, None) == qlm.QLM_ERR_CAPACITY
    assert b"threads" in lib.qlm_last_error()
    # prompts: to each of 8 heads, 16 sequences and 2^17 tiles of 128 columns
    b = batch(qlm, n_seqs=16, n_rows=17, max_new=1 << 24, max_length=100, row_start=A)
    assert lib.qlm_kv_attention(P(c), P(b), P(q), A, big, None) == qlm.QLM_ERR_CAPACITY
    # queries: to each 32 columns
    b = batch(qlm, n_seqs=1, n_rows=1 << 24, max_new=1 << 23, max_length=100, row_start=A)
    q4 = qlm.KvQuery(rows(qlm), rows(qlm, data=A + 4096), 64, 0.1, 0, 0.0)
    assert lib.qlm_kv_attention(P(c), P(b), P(q4), A, big, None) == qlm.QLM_ERR_CAPACITY
    # appends: to each of 8 heads and 2^21 blocks
    b = batch(qlm, n_seqs=128, n_rows=1 << 20, max_new=1 << 20, max_length=1 << 20,
              table_stride=1 << 14, row_start=A)
    assert lib.qlm_kv_append(P(c), P(b), P(rows(qlm)), P(rows(qlm)), None, None) == \
        qlm.QLM_ERR_CAPACITY
    # evictions: two waves to each of 8 heads and 2^22 blocks; sixteen to each of 2^22 heads
    b = batch(qlm, n_seqs=1 << 8, n_rows=1 << 8, max_length=1 << 20, table_stride=1 << 14)
    assert lib.qlm_kv_evict(P(c), P(b), 1 << 20, 0, A, A, big, None) == qlm.QLM_ERR_CAPACITY
    b = batch(qlm, n_seqs=1 << 19, n_rows=1 << 19, max_length=1 << 12, table_stride=1 << 6)
    assert lib.qlm_kv_evict(P(c), P(b), 64, 0, A, A, big, None) == qlm.QLM_ERR_CAPACITY
    # packing: a wave to each 16 outputs and 128 inputs
    w = qlm.W4Struct(1 << 24, 1 << 13, 128, A)
    assert lib.qlm_w4_pack(P(w), A, A, None, None) == qlm.QLM_ERR_CAPACITY


def test_evict_checks(qlm, lib):
    c, b = cache(qlm), batch(qlm)
    need = lib.qlm_kv_evict_workspace_bytes(P(c), P(b), 64)
    assert need > 0 and lib.qlm_kv_evict_workspace_bytes(P(c), P(b), 128) > need
    assert lib.qlm_kv_evict_workspace_bytes(P(c), P(b), 0) == 0

    def call(cc=c, budget=64, recent=0, out=A, ws=A, size=need):
        return lib.qlm_kv_evict(P(cc), P(b), budget, recent, out, ws, size, None)

    for bad in (dict(budget=0), dict(budget=-64), dict(budget=63), dict(budget=100),
                dict(recent=-1), dict(recent=65), dict(out=None), dict(cc=cache(qlm, weight=None)),
                dict(cc=cache(qlm, position=None))):
        assert call(**bad) == qlm.QLM_ERR_ARG, bad
    for bad in (dict(ws=None), dict(ws=A + 64), dict(size=need - 1)):
        assert call(**bad) == qlm.QLM_ERR_WORKSPACE, bad


def test_w4_checks(qlm, lib):
    good = dict(n_out=100, n_in=4096, group=64, packed=A)
    for bad in (dict(n_out=0), dict(n_in=0), dict(group=16), dict(group=0), dict(group=256),
                dict(packed=None), dict(packed=A + 128), dict(n_in=(1 << 24) + 1)):
        w = qlm.W4Struct(*{**good, **bad}.values())
        assert lib.qlm_w4_pack(P(w), A, A, None, None) == qlm.QLM_ERR_ARG, bad
        assert lib.qlm_w4_matmul(P(w), A, 4096, 2 * A, 100, 1, 0, A, 1 << 40, None) == \
            qlm.QLM_ERR_ARG, bad
    w = qlm.W4Struct(*good.values())
    assert lib.qlm_w4_pack(P(w), None, A, None, None) == qlm.QLM_ERR_ARG
    assert lib.qlm_w4_pack(P(w), A, None, None, None) == qlm.QLM_ERR_ARG
    assert lib.qlm_w4_pack(None, A, A, None, None) == qlm.QLM_ERR_ARG
    mm = lib.qlm_w4_matmul
    big = 1 << 40
    assert mm(P(w), None, 4096, 2 * A, 100, 1, 0, A, big, None) == qlm.QLM_ERR_ARG
    assert mm(P(w), A, 4096, None, 100, 1, 0, A, big, None) == qlm.QLM_ERR_ARG
    assert mm(P(w), A, 4096, A, 100, 1, 0, A, big, None) == qlm.QLM_ERR_ARG
    assert mm(P(w), A, 4095, 2 * A, 100, 1, 0, A, big, None) == qlm.QLM_ERR_ARG
    assert mm(P(w), A, 4096, 2 * A, 99, 1, 0, A, big, None) == qlm.QLM_ERR_ARG
    assert mm(P(w), A, 4096, 2 * A, 100, -1, 0, A, big, None) == qlm.QLM_ERR_ARG
    assert mm(P(w), A, 4096, 2 * A, 100, 1, 2, A, big, None) == qlm.QLM_ERR_ARG
    assert mm(P(w), A, 4096, 2 * A, 100, 0, 0, None, 0, None) == qlm.QLM_OK
    need = lib.qlm_w4_workspace_bytes(P(w), 64)
    if need:
        assert mm(P(w), A, 4096, 2 * A, 100, 64, 0, None, need, None) == qlm.QLM_ERR_WORKSPACE
        assert mm(P(w), A, 4096, 2 * A, 100, 64, 0, A, need - 1, None) == qlm.QLM_ERR_WORKSPACE
    assert lib.qlm_w4_packed_bytes(16, 128, 128) == 1024 + 64
    assert lib.qlm_w4_packed_bytes(17, 129, 32) == 4 * (1024 + 256)
    assert lib.qlm_w4_packed_bytes(17, 129, 48) == 0


def test_binding_refusals(qlm):
    """Shapes and types that the binding turns down (host tensors: nothing is launched)."""
    import torch
    i32 = torch.int32
    c = qlm.DeviceKvCache.empty(4, 2, 32, device="cpu")
    with pytest.raises(ValueError):
        qlm.DeviceKvCache(c.k_codes, c.v_codes.view(torch.int8), c.k_scale, c.v_scale)
    with pytest.raises(ValueError):
        qlm.DeviceKvCache(c.k_codes, c.k_codes, c.k_scale, c.v_scale)
    with pytest.raises(ValueError):
        qlm.DeviceKvCache(c.k_codes, c.v_codes, c.k_scale.double(), c.v_scale)
    with pytest.raises(ValueError):
        qlm.DeviceKvCache(c.k_codes, c.v_codes, c.k_scale, c.v_scale, position=c.weight)
    t, n = torch.zeros((2, 3), dtype=i32), torch.zeros(2, dtype=i32)
    for bad in (dict(block_table=t.long(), lengths=n), dict(block_table=t[0], lengths=n),
                dict(block_table=t, lengths=n.long()), dict(block_table=t.t(), lengths=n),
                dict(block_table=t, lengths=n, max_length=193),
                dict(block_table=t, lengths=n, row_start=n, n_rows=2),
                dict(block_table=t, lengths=n, row_start=torch.zeros(3, dtype=i32))):
        with pytest.raises(ValueError):
            qlm.KvBatch(**bad)
    b = qlm.KvBatch(t, n)
    half = lambda *s: torch.zeros(s, dtype=torch.float16)  # noqa: E731
    for k in (half(3, 2, 32), half(2, 1, 32), half(2, 2, 16), half(2, 2, 32).float(),
              half(2, 32, 2).transpose(1, 2)):
        with pytest.raises(ValueError):
            qlm.kv_append(c, b, k, half(2, 2, 32))
    with pytest.raises(ValueError):
        qlm.kv_append(c, b, half(2, 2, 32), half(2, 2, 32), first_position=n.long())
    with pytest.raises(ValueError):
        qlm.kv_attention(c, b, half(2, 4, 32), out=half(2, 4, 16), ws=n)
    with pytest.raises(ValueError):
        qlm.kv_evict(c, b, 64, out=n.long())
    u8 = torch.zeros((4, 64), dtype=torch.uint8)
    for codes, scale, zero in ((u8.int(), half(4, 2), None), (u8, half(4, 3), None),
                               (u8, half(3, 2), None), (u8, half(4, 2).float(), None),
                               (u8, half(4, 2), half(4, 2)), (u8.t(), half(4, 2), None)):
        with pytest.raises(ValueError):
            qlm.w4_pack(codes, scale, zero)
    w = qlm.W4(torch.zeros(1024 + 128, dtype=torch.uint8), 16, 64, 32)
    for x in (half(2, 63), half(64), half(2, 64).float(), half(64, 2).t()[:, :1]):
        with pytest.raises(ValueError):
            qlm.w4_matmul(x, w)
    with pytest.raises(ValueError):
        qlm.w4_matmul(half(2, 64), w, out=half(2, 15))


def test_host_tensors_are_refused(qlm, monkeypatch):
    """Tensors of the right shape and type in host memory: their addresses reach no kernel."""
    import torch
    reached = []

    class Library:
        """The sizes as they are; no call of a kernel."""

        def __getattr__(self, name):
            if name.endswith("_bytes"):
                return getattr(real, name)
            return lambda *args: reached.append(name) or 0

    real = qlm.library()
    monkeypatch.setattr(qlm, "_lib", Library())
    monkeypatch.setattr(qlm, "_raw_stream", lambda stream: None)
    monkeypatch.setattr(qlm, "_stream", lambda stream: None)
    i32 = dict(dtype=torch.int32)
    half = lambda *s: torch.zeros(s, dtype=torch.float16)  # noqa: E731
    c = qlm.DeviceKvCache.empty(4, 2, 32, device="cpu")
    b = qlm.KvBatch(torch.zeros((2, 3), **i32), torch.zeros(2, **i32))
    u8 = torch.zeros((4, 64), dtype=torch.uint8)
    w = qlm.W4(torch.zeros(1024 + 128, dtype=torch.uint8), 16, 64, 64)
    calls = [lambda: qlm.kv_append(c, b, half(2, 2, 32), half(2, 2, 32)),
             lambda: qlm.kv_attention(c, b, half(2, 4, 32)),
             lambda: qlm.kv_evict(c, b, 64),
             lambda: qlm.w4_pack(u8, half(4, 2)),
             lambda: qlm.w4_matmul(half(2, 64), w)]
    for call in calls:
        with pytest.raises(ValueError, match="must be on the GPU"):
            call()
    assert not reached
    # a cache or a batch in two places
    with pytest.raises(ValueError, match="must be where"):
        qlm.DeviceKvCache(c.k_codes, c.v_codes, c.k_scale, c.v_scale.to("meta"))
    with pytest.raises(ValueError, match="must be where"):
        qlm.KvBatch(torch.zeros((2, 3), device="meta", **i32), torch.zeros(2, **i32))


def test_memory_of_the_calls_stream(qlm, monkeypatch):
    """Outputs and workspaces that a call allocates itself are memory of the stream that it
    runs on, whose order decides when the allocator hands them out again; what the caller gets
    is also recorded on the stream that was current."""
    import contextlib

    import torch
    current, made, recorded, launched = ["main"], [], [], []

    class Library:
        def __getattr__(self, name):
            if name.endswith("_bytes"):
                return lambda *args: 64
            return lambda *args: launched.append(name) or 0

    @contextlib.contextmanager
    def on(stream):
        current.append(stream)
        yield
        current.pop()

    def noted(make):
        return lambda *a, **k: (made.append(current[-1]), make(*a, **k))[1]

    i32 = dict(dtype=torch.int32)
    half = lambda *s: torch.zeros(s, dtype=torch.float16)  # noqa: E731
    c = qlm.DeviceKvCache.empty(4, 2, 32, device="cpu")
    b = qlm.KvBatch(torch.zeros((2, 3), **i32), torch.zeros(2, **i32))
    u8 = torch.zeros((4, 64), dtype=torch.uint8)
    w = qlm.W4(torch.zeros(1024 + 128, dtype=torch.uint8), 16, 64, 64)
    monkeypatch.setattr(qlm, "_lib", Library())
    for name in ("_raw_stream", "_stream"):
        monkeypatch.setattr(qlm, name, lambda stream: None)
    monkeypatch.setattr(qlm, "_refuse_place", lambda *a, **k: None)   # (no GPU here)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: current[-1])
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: recorded.append(s))
    for name in ("empty", "empty_like"):
        monkeypatch.setattr(torch, name, noted(getattr(torch, name)))
    calls = [(lambda s: qlm.kv_attention(c, b, half(2, 4, 32), stream=s), 2),
             (lambda s: qlm.kv_evict(c, b, 64, stream=s), 2),
             (lambda s: qlm.w4_pack(u8, half(4, 2), stream=s), 1),
             (lambda s: qlm.w4_matmul(half(2, 64), w, stream=s), 2)]
    for call, n in calls:
        for stream, where in ((None, "main"), ("side", "side")):
            made.clear(), recorded.clear(), launched.clear()
            call(stream)
            assert made == [where] * n and len(launched) == 1
            assert recorded == (["main"] if stream else [])
