"""The operators of an instance that checks drafted tokens, without a GPU: argument
checks of the C interface and of the binding, before anything reaches the device."""
import contextlib
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
BIG = 1 << 40


def made(kind, fields, more):
    return kind(*{**fields, **more}.values())


def cache(qlm, **more):
    return made(qlm.KvCacheStruct, dict(n_blocks=8, n_kv_heads=2, head_dim=64, format=0, k_codes=A,
                                        v_codes=A, k_scale=A, v_scale=A, position=A, weight=A), more)


def batch(qlm, **more):
    return made(qlm.KvBatchStruct, dict(n_seqs=2, n_rows=2, max_new=1, max_length=100,
                                        table_stride=2, block_table=A, lengths=A, row_start=None),
                more)


def rows(qlm, **more):
    return made(qlm.Rows, dict(data=A, row_stride=128, head_stride=64, dtype=0), more)


def rotary(qlm, **more):
    return made(qlm.RotaryStruct, dict(rotary_dim=64, interleaved=0, n_positions=100, n_axes=1,
                                       cos=A, sin=A, axis=None, position=None), more)


def test_rotated_append_checks(qlm, lib):
    good = dict(c=cache(qlm), b=batch(qlm), k=rows(qlm), v=rows(qlm), q=rows(qlm),
                out=rows(qlm, data=2 * A), heads=4, r=rotary(qlm))

    def call(**more):
        f = {**good, **more}
        ref = lambda x: None if x is None else P(x)  # noqa: E731
        return lib.qlm_kv_append_rotated(*(ref(f[n]) for n in ("c", "b", "k", "v", "q", "out")),
                                         f["heads"], ref(f["r"]), None, None)

    for name in good:
        if name != "heads":
            assert call(**{name: None}) == qlm.QLM_ERR_ARG, name
    for bad in (dict(rotary_dim=0), dict(rotary_dim=1), dict(rotary_dim=33), dict(rotary_dim=66),
                dict(rotary_dim=-2), dict(n_positions=0), dict(n_axes=0), dict(n_axes=5, position=A),
                dict(n_axes=3), dict(cos=None), dict(sin=None), dict(cos=A + 2), dict(sin=A + 1)):
        assert call(r=rotary(qlm, **bad)) == qlm.QLM_ERR_ARG, bad
    for bad in (dict(heads=-1), dict(heads=0), dict(heads=(1 << 16) + 1),
                dict(q=rows(qlm, dtype=2), out=rows(qlm, data=2 * A, dtype=2)),
                dict(out=rows(qlm, data=2 * A, dtype=1)), dict(q=rows(qlm, data=A + 1)),
                dict(out=rows(qlm, row_stride=256)), dict(out=rows(qlm, head_stride=32)),
                # (k and v stand at A as q does: their places are not the queries')
                dict(q=rows(qlm, data=4 * A), out=rows(qlm)),
                dict(c=cache(qlm, head_dim=72)), dict(b=batch(qlm, table_stride=1))):
        assert call(**bad) == qlm.QLM_ERR_ARG, bad
    # nothing to write: no device work
    assert call(b=batch(qlm, n_seqs=0, n_rows=0), k=None, v=None, q=None, out=None) == qlm.QLM_OK
    # a workgroup of 256 to each four rows of queries
    huge = batch(qlm, n_seqs=1, n_rows=1 << 26, max_new=1, row_start=A)
    assert call(b=huge) == qlm.QLM_ERR_CAPACITY


def test_f8_checks(qlm, lib):
    weight, coded = dict(n_out=100, n_in=300, packed=A), dict(n_rows=5, n_in=300, codes=A, scale=A)
    w, r = qlm.F8Struct(*weight.values()), qlm.F8CodesStruct(*coded.values())
    mm = lib.qlm_f8_matmul
    for bad in (dict(n_out=0), dict(n_in=0), dict(n_out=(1 << 24) + 1), dict(n_in=(1 << 24) + 1),
                dict(packed=None), dict(packed=A + 128)):
        b = made(qlm.F8Struct, weight, bad)
        assert lib.qlm_f8_pack(P(b), A, A, None) == qlm.QLM_ERR_ARG, bad
        assert mm(P(r), P(b), 2 * A, 100, 1, A, BIG, None) == qlm.QLM_ERR_ARG, bad
    for bad in (dict(n_rows=-1), dict(n_rows=(1 << 31) - 1), dict(n_in=0), dict(n_in=(1 << 24) + 1),
                dict(codes=None), dict(scale=None), dict(codes=A + 8), dict(scale=A + 2)):
        b = made(qlm.F8CodesStruct, coded, bad)
        assert lib.qlm_f8_rows(P(b), A, 1 << 25, 0, None) == qlm.QLM_ERR_ARG, bad
        assert mm(P(b), P(w), 2 * A, 100, 1, A, BIG, None) == qlm.QLM_ERR_ARG, bad
    assert lib.qlm_f8_pack(None, A, A, None) == qlm.QLM_ERR_ARG
    assert lib.qlm_f8_pack(P(w), None, A, None) == qlm.QLM_ERR_ARG
    assert lib.qlm_f8_pack(P(w), A, None, None) == qlm.QLM_ERR_ARG
    assert lib.qlm_f8_pack(P(w), A, A + 2, None) == qlm.QLM_ERR_ARG
    for args in ((None, A, 300, 0), (P(r), None, 300, 0), (P(r), A + 1, 300, 0), (P(r), A, 299, 0),
                 (P(r), A, 300, 2), (P(r), A, 300, -1)):
        assert lib.qlm_f8_rows(*args, None) == qlm.QLM_ERR_ARG
    other = made(qlm.F8CodesStruct, coded, dict(n_in=299))
    for args in ((None, P(w), 2 * A, 100, 1), (P(r), None, 2 * A, 100, 1), (P(other), P(w), 2 * A, 100, 1),
                 (P(r), P(w), None, 100, 1), (P(r), P(w), A, 100, 1), (P(r), P(w), 2 * A, 99, 1),
                 (P(r), P(w), 2 * A, 100, 3), (P(r), P(w), 2 * A + 1, 100, 1),
                 (P(r), P(w), 2 * A + 2, 100, 2)):
        assert mm(*args, A, BIG, None) == qlm.QLM_ERR_ARG
    none = made(qlm.F8CodesStruct, coded, dict(n_rows=0, codes=None, scale=None))
    assert lib.qlm_f8_rows(P(none), None, 300, 0, None) == qlm.QLM_OK
    assert mm(P(none), P(w), None, 100, 1, None, 0, None) == qlm.QLM_OK
    # tiles of 16 x 128 bytes, a scale for 128 x 128
    assert lib.qlm_f8_packed_bytes(16, 128) == 2048 + 4
    assert lib.qlm_f8_packed_bytes(129, 129) == 9 * 2 * 2048 + 4 * 4
    assert lib.qlm_f8_packed_bytes(0, 128) == 0 and lib.qlm_f8_packed_bytes(16, 0) == 0
    # launches of 2^32 threads
    big = qlm.F8Struct(1 << 24, 1 << 24, A)
    assert lib.qlm_f8_pack(P(big), A, A, None) == qlm.QLM_ERR_CAPACITY
    many = qlm.F8CodesStruct(1 << 30, 1 << 20, A, A)
    assert lib.qlm_f8_rows(P(many), A, 1 << 20, 0, None) == qlm.QLM_ERR_CAPACITY
    most = qlm.F8Struct(1 << 24, 1 << 20, A)
    assert mm(P(many), P(most), 2 * A, 1 << 24, 1, A, 1 << 62, None) == qlm.QLM_ERR_CAPACITY


def test_f8_workspace(qlm, lib):
    for n_out, n_in in ((100, 300), (4096, 4096), (300, 16384)):
        w = qlm.F8Struct(n_out, n_in, A)
        for m in (1, 16, 33, 100, 1000):
            need = lib.qlm_f8_workspace_bytes(P(w), m)
            r = qlm.F8CodesStruct(m, n_in, A, A)
            if need:
                for ws, size in ((None, need), (A + 128, need), (A, need - 1)):
                    assert lib.qlm_f8_matmul(P(r), P(w), 2 * A, n_out, 1, ws, size, None) == \
                        qlm.QLM_ERR_WORKSPACE
    assert lib.qlm_f8_workspace_bytes(None, 5) == 0


def test_verify_checks(qlm, lib):
    good = dict(vocab=100, dtype=2, target=A, draft=A, target_stride=100, draft_stride=100, tokens=A,
                uniform=A)

    def call(b=None, out=A, count=A, lengths=A, **more):
        d = made(qlm.DraftStruct, good, more)
        return lib.qlm_draft_verify(P(batch(qlm) if b is None else b), P(d), out, count, lengths, A,
                                    BIG, None)

    for bad in (dict(vocab=0), dict(vocab=(1 << 24) + 1), dict(dtype=3), dict(dtype=-1),
                dict(target=None), dict(tokens=None), dict(uniform=None), dict(target=A + 2),
                dict(draft=A + 2), dict(target=A + 1, dtype=0), dict(target_stride=99),
                dict(draft_stride=99), dict(out=None), dict(count=None),
                dict(b=batch(qlm, n_seqs=-1)), dict(b=batch(qlm, lengths=None)),
                dict(b=batch(qlm, n_rows=3))):
        assert call(**bad) == qlm.QLM_ERR_ARG, bad
    assert lib.qlm_draft_verify(None, P(made(qlm.DraftStruct, good, {})), A, A, A, A, BIG, None) == \
        qlm.QLM_ERR_ARG
    assert lib.qlm_draft_verify(P(batch(qlm)), None, A, A, A, A, BIG, None) == qlm.QLM_ERR_ARG
    none = batch(qlm, n_seqs=0, n_rows=0)
    assert call(b=none, target=None, tokens=None, uniform=None, out=None, count=None) == qlm.QLM_OK
    assert lib.qlm_draft_verify_workspace_bytes(None, 100) == 0
    need = lib.qlm_draft_verify_workspace_bytes(P(batch(qlm)), 100)
    if need:
        d = made(qlm.DraftStruct, good, {})
        for ws, size in ((None, need), (A + 128, need), (A, need - 1)):
            assert lib.qlm_draft_verify(P(batch(qlm)), P(d), A, A, A, ws, size, None) == \
                qlm.QLM_ERR_WORKSPACE


class Host:
    """Arguments of the right shapes and types in host memory."""

    def __init__(self, qlm):
        import torch
        self.qlm, self.torch = qlm, torch
        i32 = dict(dtype=torch.int32)
        self.half = lambda *s: torch.zeros(s, dtype=torch.float16)
        self.cache = qlm.DeviceKvCache.empty(4, 2, 32, device="cpu")
        self.batch = qlm.KvBatch(torch.zeros((2, 3), **i32), torch.zeros(2, **i32))
        self.table = torch.zeros((10, 8))
        self.rotary = qlm.Rotary(self.table, self.table)
        self.f8 = lambda *s: torch.zeros(s, dtype=torch.uint8).view(torch.float8_e4m3fn)
        self.rows = qlm.F8Rows(self.f8(1, 1, 8, 16, 16), torch.zeros((1, 16)), 2, 64)
        self.weight = qlm.F8(torch.zeros(2048 + 4, dtype=torch.uint8), 16, 64)
        self.tokens, self.uniform = torch.zeros(2, **i32), torch.zeros(2)
        self.probs = torch.zeros((2, 50))

    def append(self, **more):
        f = dict(k=self.half(2, 2, 32), v=self.half(2, 2, 32), q=self.half(2, 4, 32),
                 rotary=self.rotary)
        f.update(more)
        return self.qlm.kv_append_rotated(self.cache, self.batch, **f)

    def verify(self, **more):
        f = dict(tokens=self.tokens, target=self.probs, draft=self.probs, uniform=self.uniform)
        f.update(more)
        return self.qlm.draft_verify(self.batch, **f)


def test_binding_refusals(qlm):
    import torch
    h = Host(qlm)
    half, i32 = h.half, dict(dtype=torch.int32)
    t = h.table
    for bad in (dict(cos=t[0], sin=t[0]), dict(cos=t.double(), sin=t), dict(cos=t, sin=t[:5]),
                dict(cos=t.t(), sin=t.t()), dict(cos=t, sin=t, axis=torch.zeros(8)),
                dict(cos=t, sin=t, axis=torch.zeros(7, **i32)),
                dict(cos=t, sin=torch.zeros((10, 8), device="meta"))):
        with pytest.raises(ValueError):
            qlm.Rotary(**bad)
    for bad in (dict(q=half(2, 4, 16)), dict(q=half(3, 4, 32)), dict(q=half(2, 128)),
                dict(k=half(2, 1, 32)), dict(v=half(2, 2, 32).float()), dict(out=half(2, 3, 32)),
                dict(out=half(2, 4, 32).bfloat16()), dict(q=None, out=half(2, 4, 32)),
                dict(position=torch.zeros(3, **i32)), dict(position=torch.zeros(2)),
                dict(position=torch.zeros((2, 3), **i32).t()),
                dict(first_position=torch.zeros(2)), dict(first_position=torch.zeros(3, **i32))):
        with pytest.raises(ValueError):
            h.append(**bad)
    f8 = h.f8
    for codes, scale in ((f8(4, 64).view(torch.uint8), torch.zeros((1, 1))),
                         (f8(4, 64), torch.zeros((1, 2))), (f8(4, 64), torch.zeros((1, 1)).double()),
                         (f8(4, 64).t(), torch.zeros((1, 1))), (f8(64), torch.zeros((1, 1)))):
        with pytest.raises(ValueError):
            qlm.f8_pack(codes, scale)
    for bad in ((f8(1, 1, 8, 16, 16), torch.zeros((1, 16)), 17, 64),
                (f8(1, 1, 8, 16, 16), torch.zeros((1, 16)), 2, 129),
                (f8(1, 1, 8, 16, 16), torch.zeros((1, 15)), 2, 64),
                (f8(1, 1, 8, 16, 16).view(torch.int8), torch.zeros((1, 16)), 2, 64),
                (f8(1, 1, 8, 16, 16), torch.zeros((1, 16), device="meta"), 2, 64)):
        with pytest.raises(ValueError):
            qlm.F8Rows(*bad)
    for x in (half(64), half(2, 64).float(), half(64, 2).t()):
        with pytest.raises(ValueError):
            qlm.f8_rows(x)
    with pytest.raises(ValueError):
        qlm.f8_rows(half(3, 64), out=h.rows)
    for bad in (dict(weight=qlm.F8(h.weight.packed, 16, 65)), dict(out=half(2, 15)),
                dict(dtype=torch.float64), dict(out=torch.zeros((2, 16)).double()),
                dict(out=half(2, 16), dtype=torch.bfloat16), dict(out=half(16, 2).t())):
        with pytest.raises(ValueError):
            qlm.f8_matmul(h.rows, **{"weight": h.weight, **bad})
    p = h.probs
    for bad in (dict(target=p[:1]), dict(target=p.double(), draft=None), dict(draft=p.half()),
                dict(draft=p[:, :49]), dict(target=torch.zeros((50, 2)).t()),
                dict(tokens=h.tokens.long()), dict(tokens=torch.zeros(3, **i32)),
                dict(uniform=h.uniform.double()), dict(uniform=torch.zeros(1)),
                dict(lengths=torch.zeros(2)), dict(lengths=torch.zeros(3, **i32))):
        with pytest.raises(ValueError):
            h.verify(**bad)


def test_host_tensors_are_refused(qlm, monkeypatch):
    """Tensors of the right shape and type in host memory: their addresses reach no kernel."""
    import torch
    reached = []
    real = qlm.library()

    class Library:
        """The sizes as they are; no call of a kernel."""

        def __getattr__(self, name):
            if name.endswith("_bytes"):
                return getattr(real, name)
            return lambda *args: reached.append(name) or 0

    h = Host(qlm)
    monkeypatch.setattr(qlm, "_lib", Library())
    monkeypatch.setattr(qlm, "_stream_on", lambda index, stream: None)
    for call in (h.append, h.verify, lambda: qlm.f8_pack(h.f8(4, 64), torch.zeros((1, 1))),
                 lambda: qlm.f8_rows(h.half(2, 64)), lambda: qlm.f8_matmul(h.rows, h.weight)):
        with pytest.raises(ValueError, match="must be on the GPU"):
            call()
    assert not reached


def test_memory_of_the_calls_stream(qlm, monkeypatch):
    """Outputs and workspaces that a call allocates itself are memory of the stream that it
    runs on; what the caller gets is also recorded on the stream that was current."""
    import torch
    current, allocated, recorded, launched = ["main"], [], [], []

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
        return lambda *a, **k: (allocated.append(current[-1]), make(*a, **k))[1]

    h = Host(qlm)
    weights = torch.zeros((1, 1))
    append = dict(k=h.half(2, 2, 32), v=h.half(2, 2, 32), q=h.half(2, 4, 32))
    codes, x = h.f8(4, 64), h.half(2, 64)
    monkeypatch.setattr(qlm, "_lib", Library())
    monkeypatch.setattr(qlm, "_stream_on", lambda index, stream: None)
    monkeypatch.setattr(qlm, "_refuse_place", lambda *a, **k: None)   # (no GPU here)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: current[-1])
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: recorded.append(s))
    for name in ("empty", "empty_like"):
        monkeypatch.setattr(torch, name, noted(getattr(torch, name)))
    # (call, what it allocates, what of that the caller gets)
    for call, n, kept in ((lambda s: h.append(stream=s, **append), 1, 1),
                          (lambda s: qlm.f8_pack(codes, weights, stream=s), 1, 1),
                          (lambda s: qlm.f8_rows(x, stream=s), 2, 2),
                          (lambda s: qlm.f8_matmul(h.rows, h.weight, stream=s), 2, 1),
                          (lambda s: h.verify(stream=s), 4, 3)):
        for stream, where in ((None, "main"), ("side", "side")):
            allocated.clear(), recorded.clear(), launched.clear()
            call(stream)
            assert allocated == [where] * n and len(launched) == 1
            assert recorded == (["main"] * kept if stream else [])


def test_stream_of_another_gpu(qlm, monkeypatch):
    """Tensors of one GPU and the current stream, or a given one, of another."""
    import torch

    class Side:
        device_index, cuda_stream = 1, 77

    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: 50 + i, raising=False)
    assert qlm._stream_on(0, None) == 50 and qlm._stream_on(1, Side) == 77
    for index, stream in ((1, None), (0, Side)):
        with pytest.raises(ValueError, match="stream on GPU"):
            qlm._stream_on(index, stream)
