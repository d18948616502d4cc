"""Python binding of libqlm (include/qlm.h): argument marshalling only.

Every step of the scoring path runs in the HIP kernels of ``csrc/qlm.hip``;
PyTorch supplies device memory and the current stream.  The binding refuses to
run when the library is not built (there is no fallback of any kind).

Function names follow the C interface: ``rwt_score``, ``rwt_score_exact``,
``best_plan`` (with ``best_plan_workspace_bytes``), ``validate_plans``,
``validate_problem``, ``search_n_moves``, ``search_workspace_bytes``,
``search_moves``, ``search_screen``, ``local_search``, ``seed_plans``,
``place_group``; and of a serving instance's decode step ``kv_append``,
``kv_append_rotated``, ``kv_attention``, ``kv_evict``, ``w4_pack``, ``w4_matmul``,
``f8_pack``, ``f8_rows``, ``f8_matmul``, ``draft_verify``.
"""
from __future__ import annotations

import ctypes
import os
import struct
import threading

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libqlm.so")
_lock = threading.Lock()
_lib = None

QLM_OK, QLM_ERR_ARG, QLM_ERR_CAPACITY, QLM_ERR_WORKSPACE, QLM_ERR_HIP = range(5)


class QlmError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__("qlm status %d: %s" % (status, message))
        self.status = status


class Problem(ctypes.Structure):
    _fields_ = [("n_groups", ctypes.c_int32), ("n_instances", ctypes.c_int32),
                ("n_models", ctypes.c_int32), ("n_classes", ctypes.c_int32),
                ("grp_count", ctypes.c_void_p), ("grp_mu", ctypes.c_void_p),
                ("grp_var", ctypes.c_void_p), ("grp_model", ctypes.c_void_p),
                ("grp_slo", ctypes.c_void_p), ("inst_tput", ctypes.c_void_p),
                ("inst_class", ctypes.c_void_p), ("inst_model0", ctypes.c_void_p),
                ("swap_cost", ctypes.c_void_p), ("evict_cost", ctypes.c_float)]


class Plans(ctypes.Structure):
    _fields_ = [("n_plans", ctypes.c_int64), ("plan_stride", ctypes.c_int64),
                ("perm", ctypes.c_void_p), ("qoff", ctypes.c_void_p),
                ("evict_bits", ctypes.c_void_p)]


class PlansOut(ctypes.Structure):
    _fields_ = [("plan_stride", ctypes.c_int64), ("perm", ctypes.c_void_p),
                ("qoff", ctypes.c_void_p), ("evict_bits", ctypes.c_void_p)]


class Detail(ctypes.Structure):
    _fields_ = [("plan_begin", ctypes.c_int64), ("plan_count", ctypes.c_int64),
                ("wait_mean", ctypes.c_void_p), ("wait_sd", ctypes.c_void_p),
                ("prob", ctypes.c_void_p)]


class Profile(ctypes.Structure):
    _fields_ = [("prefill", ctypes.c_void_p), ("decode_time", ctypes.c_void_p),
                ("ineff", ctypes.c_void_p), ("max_tokens", ctypes.c_void_p),
                ("kv_tokens", ctypes.c_void_p), ("mean_tokens", ctypes.c_void_p)]


class KvCacheStruct(ctypes.Structure):
    _fields_ = [("n_blocks", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("format", ctypes.c_int32),
                ("k_codes", ctypes.c_void_p), ("v_codes", ctypes.c_void_p),
                ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("position", ctypes.c_void_p), ("weight", ctypes.c_void_p)]


class KvBatchStruct(ctypes.Structure):
    _fields_ = [("n_seqs", ctypes.c_int32), ("n_rows", ctypes.c_int32),
                ("max_new", ctypes.c_int32), ("max_length", ctypes.c_int32),
                ("table_stride", ctypes.c_int64), ("block_table", ctypes.c_void_p),
                ("lengths", ctypes.c_void_p), ("row_start", ctypes.c_void_p)]


class Rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("row_stride", ctypes.c_int64),
                ("head_stride", ctypes.c_int64), ("dtype", ctypes.c_int32)]


class KvQuery(ctypes.Structure):
    _fields_ = [("q", Rows), ("out", Rows), ("n_heads", ctypes.c_int32),
                ("scale", ctypes.c_float), ("accumulate", ctypes.c_int32),
                ("weight_decay", ctypes.c_float)]


class W4Struct(ctypes.Structure):
    _fields_ = [("n_out", ctypes.c_int32), ("n_in", ctypes.c_int32), ("group", ctypes.c_int32),
                ("packed", ctypes.c_void_p)]


class F8Struct(ctypes.Structure):
    _fields_ = [("n_out", ctypes.c_int32), ("n_in", ctypes.c_int32), ("packed", ctypes.c_void_p)]


class F8CodesStruct(ctypes.Structure):
    _fields_ = [("n_rows", ctypes.c_int32), ("n_in", ctypes.c_int32), ("codes", ctypes.c_void_p),
                ("scale", ctypes.c_void_p)]


class RotaryStruct(ctypes.Structure):
    _fields_ = [("rotary_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32),
                ("n_positions", ctypes.c_int32), ("n_axes", ctypes.c_int32),
                ("cos", ctypes.c_void_p), ("sin", ctypes.c_void_p), ("axis", ctypes.c_void_p),
                ("position", ctypes.c_void_p)]


class DraftStruct(ctypes.Structure):
    _fields_ = [("vocab", ctypes.c_int32), ("dtype", ctypes.c_int32), ("target", ctypes.c_void_p),
                ("draft", ctypes.c_void_p), ("target_stride", ctypes.c_int64),
                ("draft_stride", ctypes.c_int64), ("tokens", ctypes.c_void_p),
                ("uniform", ctypes.c_void_p)]


PROFILE_FIELDS = ("prefill", "decode_time", "ineff", "max_tokens", "kv_tokens", "mean_tokens")


def library():
    """The loaded libqlm; raises when it has not been built."""
    global _lib
    with _lock:
        if _lib is None:
            if not os.path.exists(LIB_PATH):
                raise RuntimeError("libqlm.so is not built (run __graft_entry__.build() or "
                                   "python -m paper_2407_00047_amd.build)")
            lib = ctypes.CDLL(LIB_PATH)
            P, PL, D = ctypes.POINTER(Problem), ctypes.POINTER(Plans), ctypes.POINTER(Detail)
            vp, i64 = ctypes.c_void_p, ctypes.c_int64
            lib.qlm_rwt_score.argtypes = [P, PL, vp, vp, D, vp]
            lib.qlm_rwt_score_exact.argtypes = [P, PL, vp, i64, vp, vp]
            lib.qlm_best_plan_workspace_bytes.argtypes = [P, i64]
            lib.qlm_best_plan_workspace_bytes.restype = ctypes.c_size_t
            lib.qlm_best_plan.argtypes = [P, PL, vp, ctypes.c_size_t, vp, vp, vp]
            lib.qlm_best_plan_static.argtypes = [P, PL, vp, vp, vp]
            lib.qlm_score_form.argtypes = [P, ctypes.c_int32, vp, vp]
            lib.qlm_validate_plans.argtypes = [P, PL, vp, vp, vp]
            lib.qlm_validate_problem.argtypes = [P, vp, vp]
            lib.qlm_max_groups.argtypes = [ctypes.c_int32] * 4
            lib.qlm_max_groups.restype = ctypes.c_int32
            lib.qlm_status_string.argtypes = [ctypes.c_int]
            lib.qlm_status_string.restype = ctypes.c_char_p
            lib.qlm_last_error.restype = ctypes.c_char_p
            lib.qlm_timing_enable.argtypes = [ctypes.c_int]
            lib.qlm_timing_read.argtypes = [ctypes.POINTER(ctypes.c_int64),
                                            ctypes.POINTER(ctypes.c_double)]
            i32 = ctypes.c_int32
            lib.qlm_search_n_moves.argtypes = [i32, i32, i32]
            lib.qlm_search_n_moves.restype = i64
            lib.qlm_search_workspace_bytes.argtypes = [P, i64, i32]
            lib.qlm_search_workspace_bytes.restype = ctypes.c_size_t
            lib.qlm_search_moves.argtypes = [P, PL, i32, vp, ctypes.c_size_t, vp, vp]
            lib.qlm_search_screen.argtypes = [P, PL, i32, vp, ctypes.c_size_t, vp, vp, vp]
            lib.qlm_place_group.argtypes = [P, PL, ctypes.POINTER(PlansOut), i32, vp,
                                            ctypes.c_size_t, vp, vp, vp]
            lib.qlm_seed_workspace_bytes.argtypes = [P, i32]
            lib.qlm_seed_workspace_bytes.restype = ctypes.c_size_t
            lib.qlm_seed_plans.argtypes = [P, i32, ctypes.POINTER(ctypes.c_int32),
                                           ctypes.POINTER(PlansOut), vp, ctypes.c_size_t, vp]
            lib.qlm_local_search.argtypes = [P, PL, ctypes.POINTER(PlansOut), i32, i32, vp,
                                             ctypes.c_size_t, vp, vp, vp, vp]
            sz = ctypes.c_size_t
            lib.qlm_fcfs_workspace_bytes.argtypes = [P, i64, i64, i64]
            lib.qlm_fcfs_workspace_bytes.restype = sz
            lib.qlm_fcfs_score.argtypes = [P, PL, vp, i64, vp, sz, vp, vp]
            lib.qlm_fcfs_score_exact.argtypes = [P, PL, vp, i64, vp, i64, vp, sz, vp, vp]
            lib.qlm_fcfs_best_plan.argtypes = [P, PL, vp, i64, vp, sz, vp, vp, vp]
            lib.qlm_apply_profile.argtypes = [P, ctypes.POINTER(Profile), vp, vp, vp, vp, vp, i64,
                                              vp, vp]
            lib.qlm_place_begin.argtypes = [P, PL, vp, sz, vp]
            lib.qlm_place_step.argtypes = [P, i64, i32, vp, sz, vp, vp, vp]
            lib.qlm_place_end.argtypes = [P, i64, ctypes.POINTER(PlansOut), vp, sz, vp, vp]
            C, B = ctypes.POINTER(KvCacheStruct), ctypes.POINTER(KvBatchStruct)
            W = ctypes.POINTER(W4Struct)
            lib.qlm_kv_append.argtypes = [C, B, vp, vp, vp, vp]  # (rows packed as bytes)
            lib.qlm_kv_attention_workspace_bytes.argtypes = [C, B, i32, i32]
            lib.qlm_kv_attention_workspace_bytes.restype = ctypes.c_size_t
            lib.qlm_kv_attention.argtypes = [C, B, vp, vp, sz, vp]
            lib.qlm_kv_evict_workspace_bytes.argtypes = [C, B, i32]
            lib.qlm_kv_evict_workspace_bytes.restype = ctypes.c_size_t
            lib.qlm_kv_evict.argtypes = [C, B, i32, i32, vp, vp, sz, vp]
            lib.qlm_w4_packed_bytes.argtypes = [i32, i32, i32]
            lib.qlm_w4_packed_bytes.restype = ctypes.c_size_t
            lib.qlm_w4_pack.argtypes = [W, vp, vp, vp, vp]
            lib.qlm_w4_workspace_bytes.argtypes = [W, i32]
            lib.qlm_w4_workspace_bytes.restype = ctypes.c_size_t
            lib.qlm_w4_matmul.argtypes = [W, vp, i64, vp, i64, i32, i32, vp, sz, vp]
            lib.qlm_kv_append_rotated.argtypes = [C, B, vp, vp, vp, vp, i32, vp, vp, vp]
            F, R = ctypes.POINTER(F8Struct), vp                  # (coded rows packed as bytes)
            lib.qlm_f8_packed_bytes.argtypes = [i32, i32]
            lib.qlm_f8_packed_bytes.restype = ctypes.c_size_t
            lib.qlm_f8_pack.argtypes = [F, vp, vp, vp]
            lib.qlm_f8_rows.argtypes = [R, vp, i64, i32, vp]
            lib.qlm_f8_workspace_bytes.argtypes = [F, i32]
            lib.qlm_f8_workspace_bytes.restype = ctypes.c_size_t
            lib.qlm_f8_matmul.argtypes = [R, F, vp, i64, i32, vp, sz, vp]
            lib.qlm_draft_verify_workspace_bytes.argtypes = [B, i32]
            lib.qlm_draft_verify_workspace_bytes.restype = ctypes.c_size_t
            lib.qlm_draft_verify.argtypes = [B, vp, vp, vp, vp, vp, sz, vp]
            for name in ("qlm_kv_append", "qlm_kv_attention", "qlm_kv_evict", "qlm_w4_pack",
                         "qlm_w4_matmul", "qlm_kv_append_rotated", "qlm_f8_pack", "qlm_f8_rows",
                         "qlm_f8_matmul", "qlm_draft_verify"):
                getattr(lib, name).restype = ctypes.c_int
            for name in ("qlm_rwt_score", "qlm_rwt_score_exact", "qlm_best_plan", "qlm_best_plan_static",
                         "qlm_score_form",
                         "qlm_validate_plans", "qlm_validate_problem", "qlm_timing_enable",
                         "qlm_timing_read", "qlm_search_moves", "qlm_search_screen",
                         "qlm_local_search", "qlm_seed_plans", "qlm_place_group",
                         "qlm_fcfs_score", "qlm_fcfs_score_exact", "qlm_fcfs_best_plan",
                         "qlm_apply_profile", "qlm_place_begin", "qlm_place_step",
                         "qlm_place_end"):
                getattr(lib, name).restype = ctypes.c_int
            _lib = lib
    return _lib


def _check(rc: int):
    if rc != QLM_OK:
        lib = library()
        raise QlmError(rc, lib.qlm_last_error().decode())


def _stream(stream):
    import torch
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def _ptr(t):
    return None if t is None else t.data_ptr()


class DeviceProblem:
    """Problem tables in device memory (torch tensors) plus the C struct."""

    def __init__(self, problem, device="cuda"):
        import torch

        def dev(x, dt):
            if x is None:
                return None
            return torch.as_tensor(np.ascontiguousarray(x)).to(device=device, dtype=dt)

        self.n_groups = int(problem["n_groups"])
        self.n_instances = int(problem["n_instances"])
        self.n_models = int(problem["n_models"])
        self.n_classes = int(problem["n_classes"])
        self.grp_count = dev(problem["grp_count"], torch.int32)
        self.grp_mu = dev(problem["grp_mu"], torch.float32)
        self.grp_var = dev(problem["grp_var"], torch.float32)
        self.grp_model = dev(problem["grp_model"], torch.int32)
        self.grp_slo = dev(problem["grp_slo"], torch.float32)
        self.inst_tput = dev(problem["inst_tput"], torch.float32)
        self.inst_class = dev(problem["inst_class"], torch.int32)
        self.inst_model0 = dev(problem.get("inst_model0"), torch.int32)
        self.swap_cost = dev(problem.get("swap_cost"), torch.float32)
        self.evict_cost = float(problem.get("evict_cost", 0.0))
        self.total_requests = int(np.asarray(problem["grp_count"], np.int64).sum())
        self.struct = Problem(self.n_groups, self.n_instances, self.n_models, self.n_classes,
                              _ptr(self.grp_count), _ptr(self.grp_mu), _ptr(self.grp_var),
                              _ptr(self.grp_model), _ptr(self.grp_slo), _ptr(self.inst_tput),
                              _ptr(self.inst_class), _ptr(self.inst_model0),
                              _ptr(self.swap_cost), self.evict_cost)


class DevicePlans:
    """A slot-major plan batch in device memory plus the C struct.  ``perm`` is
    [G, stride] int32, ``qoff`` [I+1, stride] int32, ``evict_bits``
    [ceil(G/32), stride] int32 (bit patterns) or None."""

    def __init__(self, perm, qoff, evict_bits=None, n_plans=None):
        self.perm = perm
        self.qoff = qoff
        self.evict_bits = evict_bits
        stride = int(perm.shape[1])
        self.n_plans = stride if n_plans is None else int(n_plans)
        self.struct = Plans(self.n_plans, stride, _ptr(perm), _ptr(qoff), _ptr(evict_bits))

    @classmethod
    def from_host(cls, plans, device="cuda"):
        import torch
        perm = torch.from_numpy(np.ascontiguousarray(plans["perm"])).to(device)
        qoff = torch.from_numpy(np.ascontiguousarray(plans["qoff"])).to(device)
        ev = plans.get("evict_bits")
        if ev is not None:
            ev = torch.from_numpy(np.ascontiguousarray(ev).view(np.int32)).to(device)
        return cls(perm, qoff, ev, plans.get("n_plans"))


def rwt_score(problem: DeviceProblem, plans: DevicePlans, penalty: bool = False,
              detail: tuple[int, int] | None = None, stream=None, out=None):
    """Screening scores (and optionally penalties and per-slot detail for plans
    [begin, begin+count)).  Returns dict of device tensors."""
    import torch
    dev = plans.perm.device
    P = plans.n_plans
    # (the library writes every entry: a fill before would be a launch each)
    score = out if out is not None else torch.empty((P,), dtype=torch.float64, device=dev)
    pen = torch.empty((P,), dtype=torch.float64, device=dev) if penalty else None
    det = None
    res = {"score": score, "penalty": pen}
    if detail is not None:
        b, c = detail
        G = problem.n_groups
        wm = torch.empty((G, c), dtype=torch.float32, device=dev)
        ws = torch.empty((G, c), dtype=torch.float32, device=dev)
        pr = torch.empty((G, c), dtype=torch.float32, device=dev)
        det = Detail(b, c, _ptr(wm), _ptr(ws), _ptr(pr))
        res.update(wait_mean=wm, wait_sd=ws, prob=pr)
    _check(library().qlm_rwt_score(ctypes.byref(problem.struct), ctypes.byref(plans.struct),
                                   _ptr(score), _ptr(pen),
                                   ctypes.byref(det) if det is not None else None,
                                   _stream(stream)))
    return res


def rwt_score_exact(problem: DeviceProblem, plans: DevicePlans, plan_index, stream=None):
    import torch
    idx = torch.as_tensor(plan_index, dtype=torch.int64).to(plans.perm.device)
    out = torch.empty((idx.numel(),), dtype=torch.float64, device=plans.perm.device)
    _check(library().qlm_rwt_score_exact(ctypes.byref(problem.struct), ctypes.byref(plans.struct),
                                         _ptr(idx), idx.numel(), _ptr(out), _stream(stream)))
    return out


def best_plan_workspace_bytes(problem: DeviceProblem, n_plans: int) -> int:
    return int(library().qlm_best_plan_workspace_bytes(ctypes.byref(problem.struct), n_plans))


def workspace(problem: DeviceProblem, n_plans: int, device="cuda"):
    import torch
    nbytes = best_plan_workspace_bytes(problem, n_plans)
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


def best_plan(problem: DeviceProblem, plans: DevicePlans, ws=None, stream=None, out=None):
    """(best_index, best_score) as device tensors of shape [1]."""
    import torch
    dev = plans.perm.device
    if ws is None:
        ws = workspace(problem, plans.n_plans, dev)
    if out is None:
        bi = torch.empty((1,), dtype=torch.int64, device=dev)
        bs = torch.empty((1,), dtype=torch.float64, device=dev)
    else:
        bi, bs = out
    _check(library().qlm_best_plan(ctypes.byref(problem.struct), ctypes.byref(plans.struct),
                                   _ptr(ws), ws.numel(), _ptr(bi), _ptr(bs), _stream(stream)))
    return bi, bs


def best_plan_static(problem: DeviceProblem, plans: DevicePlans, stream=None, out=None):
    """qlm_best_plan_static: (best_index, best_score) as device tensors of
    shape [1], with the library's static scratch as the workspace."""
    import torch
    dev = plans.perm.device
    if out is None:
        bi = torch.empty((1,), dtype=torch.int64, device=dev)
        bs = torch.empty((1,), dtype=torch.float64, device=dev)
    else:
        bi, bs = out
    _check(library().qlm_best_plan_static(ctypes.byref(problem.struct), ctypes.byref(plans.struct),
                                          _ptr(bi), _ptr(bs), _stream(stream)))
    return bi, bs


def score_form(problem: DeviceProblem, with_eviction: bool, stream=None) -> int:
    """1 when qlm_rwt_score / qlm_best_plan take their fast path for this
    problem, 0 when they take the general exact walk (synchronizes)."""
    import torch
    f = torch.empty((1,), dtype=torch.int32, device=problem.grp_count.device)
    _check(library().qlm_score_form(ctypes.byref(problem.struct), int(bool(with_eviction)),
                                    _ptr(f), _stream(stream)))
    return int(f.item())


def validate_plans(problem: DeviceProblem, plans: DevicePlans, stream=None):
    """(n_invalid tensor [1], per-plan status tensor [P])."""
    import torch
    dev = plans.perm.device
    n = torch.empty(1, dtype=torch.int64, device=dev)
    st = torch.empty(max(plans.n_plans, 1), dtype=torch.int32, device=dev)
    _check(library().qlm_validate_plans(ctypes.byref(problem.struct), ctypes.byref(plans.struct),
                                        _ptr(n), _ptr(st), _stream(stream)))
    return n, st[:plans.n_plans]


def validate_problem(problem: DeviceProblem, stream=None):
    import torch
    n = torch.empty(1, dtype=torch.int64, device=problem.grp_count.device)
    _check(library().qlm_validate_problem(ctypes.byref(problem.struct), _ptr(n), _stream(stream)))
    return n


def max_groups(n_models: int, n_classes: int, n_instances: int, with_eviction: bool) -> int:
    return int(library().qlm_max_groups(n_models, n_classes, n_instances, int(with_eviction)))


def timing_enable(on: bool = True):
    _check(library().qlm_timing_enable(int(on)))


def timing_read():
    """(number of scoring launches, total milliseconds) since the last read."""
    n = ctypes.c_int64(0)
    ms = ctypes.c_double(0.0)
    _check(library().qlm_timing_read(ctypes.byref(n), ctypes.byref(ms)))
    return int(n.value), float(ms.value)


# -- plan search --------------------------------------------------------------

def plans_like(plans: DevicePlans, n_groups: int) -> DevicePlans:
    """Output plans shaped like `plans`, always with eviction words (a
    relocation sets flags even in plans that had none)."""
    import torch
    ev = plans.evict_bits
    ev = torch.empty_like(ev) if ev is not None else torch.empty(
        ((n_groups + 31) // 32, plans.perm.shape[1]), dtype=torch.int32, device=plans.perm.device)
    return DevicePlans(torch.empty_like(plans.perm), torch.empty_like(plans.qoff), ev,
                       plans.n_plans)


def search_n_moves(n_groups: int, n_instances: int, window: int) -> int:
    return int(library().qlm_search_n_moves(n_groups, n_instances, window))


def search_workspace_bytes(problem: DeviceProblem, n_plans: int, window: int) -> int:
    return int(library().qlm_search_workspace_bytes(ctypes.byref(problem.struct), n_plans,
                                                    window))


def search_workspace(problem: DeviceProblem, n_plans: int, window: int, device="cuda"):
    import torch
    nbytes = search_workspace_bytes(problem, n_plans, window)
    return torch.empty(max(nbytes, 1), dtype=torch.uint8, device=device)


def search_moves(problem: DeviceProblem, plans: DevicePlans, window: int, ws=None, stream=None,
                 out=None):
    """Exact score of every move of every plan: device tensor [P, n_moves]
    (+inf where a move number names no move)."""
    import torch
    dev = plans.perm.device
    nm = search_n_moves(problem.n_groups, problem.n_instances, window)
    if ws is None:
        ws = search_workspace(problem, plans.n_plans, window, dev)
    if out is None:
        out = torch.empty((plans.n_plans, nm), dtype=torch.float64, device=dev)
    _check(library().qlm_search_moves(ctypes.byref(problem.struct), ctypes.byref(plans.struct),
                                      window, _ptr(ws), ws.numel(), _ptr(out), _stream(stream)))
    return out


def search_screen(problem: DeviceProblem, plans: DevicePlans, window: int, ws=None, stream=None):
    """Screened score and its error bound for every move of every plan: two
    device tensors [P, n_moves] (score +inf, bound 0 where a move number names
    no move; bound +inf where the screen cannot bound the move)."""
    import torch
    dev = plans.perm.device
    nm = search_n_moves(problem.n_groups, problem.n_instances, window)
    if ws is None:
        ws = search_workspace(problem, plans.n_plans, window, dev)
    score = torch.empty((plans.n_plans, nm), dtype=torch.float64, device=dev)
    bound = torch.empty((plans.n_plans, nm), dtype=torch.float64, device=dev)
    _check(library().qlm_search_screen(ctypes.byref(problem.struct), ctypes.byref(plans.struct),
                                       window, _ptr(ws), ws.numel(), _ptr(score), _ptr(bound),
                                       _stream(stream)))
    return score, bound


def local_search(problem: DeviceProblem, plans: DevicePlans, window: int, max_steps: int,
                 trace: bool = False, ws=None, stream=None, out: DevicePlans | None = None):
    """Steepest-descent search from every plan.  Returns a dict with the final
    plans (a DevicePlans), their exact scores [P] f64, the steps applied [P]
    int32 and, when asked, the trace [P, max_steps] int64."""
    import torch
    dev = plans.perm.device
    P = plans.n_plans
    if ws is None:
        ws = search_workspace(problem, P, window, dev)
    if out is None:
        out = plans_like(plans, problem.n_groups)
    o = PlansOut(int(out.perm.shape[1]), _ptr(out.perm), _ptr(out.qoff), _ptr(out.evict_bits))
    score = torch.empty((P,), dtype=torch.float64, device=dev)
    steps = torch.empty((P,), dtype=torch.int32, device=dev)
    tr = torch.empty((P, max(max_steps, 1)), dtype=torch.int64, device=dev) if trace else None
    _check(library().qlm_local_search(ctypes.byref(problem.struct), ctypes.byref(plans.struct),
                                      ctypes.byref(o), window, max_steps, _ptr(ws), ws.numel(),
                                      _ptr(score), _ptr(steps), _ptr(tr), _stream(stream)))
    res = {"plans": out, "score": score, "steps": steps}
    if trace:
        res["trace"] = tr[:, :max_steps]
    return res


EDF, GROUPED = 0, 1


def seed_workspace_bytes(problem: DeviceProblem, n_seeds: int) -> int:
    return int(library().qlm_seed_workspace_bytes(ctypes.byref(problem.struct), n_seeds))


def seed_plans(problem: DeviceProblem, policies=(EDF, GROUPED), evict: bool = False, ws=None,
               stream=None, device="cuda"):
    """Seed plans (one per policy: EDF = 0, GROUPED = 1) as a DevicePlans; with
    evict=True the plans carry (cleared) eviction bits."""
    import torch
    n = len(policies)
    G, I = problem.n_groups, problem.n_instances
    perm = torch.empty((G, max(n, 1)), dtype=torch.int32, device=device)
    qoff = torch.empty((I + 1, max(n, 1)), dtype=torch.int32, device=device)
    ev = torch.empty(((G + 31) // 32, max(n, 1)), dtype=torch.int32, device=device) if evict else None
    if ws is None:
        ws = torch.empty(max(seed_workspace_bytes(problem, n), 1), dtype=torch.uint8, device=device)
    pol = (ctypes.c_int32 * max(n, 1))(*policies)
    o = PlansOut(int(perm.shape[1]), _ptr(perm), _ptr(qoff), _ptr(ev))
    _check(library().qlm_seed_plans(ctypes.byref(problem.struct), n, pol, ctypes.byref(o),
                                    _ptr(ws), ws.numel(), _stream(stream)))
    return DevicePlans(perm, qoff, ev, n)


def place_group(problem: DeviceProblem, plans: DevicePlans, group: int, ws=None, stream=None,
                out: DevicePlans | None = None):
    """Every plan with `group` moved to its best place: the EDF position after
    the head of queue c, or (c >= I) the head of queue c - I with its eviction
    flag set; a group at its queue's head stays.  Returns a dict with the
    placed plans (DevicePlans, with eviction words), their exact scores [P] f64
    and the chosen places c [P] int32."""
    import torch
    dev = plans.perm.device
    P = plans.n_plans
    if ws is None:
        ws = search_workspace(problem, P, 0, dev)
    if out is None:
        out = plans_like(plans, problem.n_groups)
    o = PlansOut(int(out.perm.shape[1]), _ptr(out.perm), _ptr(out.qoff), _ptr(out.evict_bits))
    score = torch.empty((P,), dtype=torch.float64, device=dev)
    queue = torch.empty((P,), dtype=torch.int32, device=dev)
    _check(library().qlm_place_group(ctypes.byref(problem.struct), ctypes.byref(plans.struct),
                                     ctypes.byref(o), int(group), _ptr(ws), ws.numel(),
                                     _ptr(score), _ptr(queue), _stream(stream)))
    return {"plans": out, "score": score, "queue": queue}


# -- per-request (first come, first served) variant ---------------------------

def device_requests(req_slo, device="cuda"):
    """Per-request SLOs (group by group, each group's in arrival order) as a
    float32 device tensor."""
    import torch
    return torch.as_tensor(np.ascontiguousarray(req_slo, dtype=np.float32)).to(device)


def fcfs_workspace_bytes(problem: DeviceProblem, n_plans: int, n_requests: int,
                         chunk_plans: int = 0) -> int:
    return int(library().qlm_fcfs_workspace_bytes(ctypes.byref(problem.struct), int(n_plans),
                                                  int(n_requests), int(chunk_plans)))


def fcfs_workspace(problem: DeviceProblem, n_plans: int, n_requests: int, device="cuda",
                   chunk_plans: int = 0):
    """A workspace for chunks of chunk_plans plans (0 = the default size)."""
    import torch
    nbytes = fcfs_workspace_bytes(problem, n_plans, n_requests, chunk_plans)
    return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)


def fcfs_score(problem: DeviceProblem, plans: DevicePlans, req_slo, ws=None, stream=None,
               out=None):
    """Screened per-request scores of every plan: device tensor [P] f64."""
    import torch
    dev = plans.perm.device
    if ws is None:
        ws = fcfs_workspace(problem, plans.n_plans, req_slo.numel(), dev)
    if out is None:
        out = torch.empty((max(plans.n_plans, 1),), dtype=torch.float64, device=dev)
    _check(library().qlm_fcfs_score(ctypes.byref(problem.struct), ctypes.byref(plans.struct),
                                    _ptr(req_slo), req_slo.numel(), _ptr(ws), ws.numel(),
                                    _ptr(out), _stream(stream)))
    return out[:plans.n_plans]


def fcfs_score_exact(problem: DeviceProblem, plans: DevicePlans, req_slo, plan_index, ws=None,
                     stream=None):
    """Exact per-request scores of the listed plans: device tensor [n] f64."""
    import torch
    dev = plans.perm.device
    idx = torch.as_tensor(plan_index, dtype=torch.int64).to(dev)
    if ws is None:
        ws = fcfs_workspace(problem, plans.n_plans, req_slo.numel(), dev)
    out = torch.full((max(idx.numel(), 1),), float("nan"), dtype=torch.float64, device=dev)
    _check(library().qlm_fcfs_score_exact(ctypes.byref(problem.struct),
                                          ctypes.byref(plans.struct), _ptr(req_slo),
                                          req_slo.numel(), _ptr(idx), idx.numel(), _ptr(ws),
                                          ws.numel(), _ptr(out), _stream(stream)))
    return out[:idx.numel()]


def fcfs_best_plan(problem: DeviceProblem, plans: DevicePlans, req_slo, ws=None, stream=None,
                   out=None):
    """(best_index, best_score) of the per-request score, device tensors [1]."""
    import torch
    dev = plans.perm.device
    if ws is None:
        ws = fcfs_workspace(problem, plans.n_plans, req_slo.numel(), dev)
    if out is None:
        bi = torch.empty((1,), dtype=torch.int64, device=dev)
        bs = torch.empty((1,), dtype=torch.float64, device=dev)
    else:
        bi, bs = out
    _check(library().qlm_fcfs_best_plan(ctypes.byref(problem.struct), ctypes.byref(plans.struct),
                                        _ptr(req_slo), req_slo.numel(), _ptr(ws), ws.numel(),
                                        _ptr(bi), _ptr(bs), _stream(stream)))
    return bi, bs


# -- problem tables from a hardware profile -----------------------------------

def apply_profile(problem: DeviceProblem, profile, inst_model=None, req_slo=None, stream=None):
    """The problem with the profile's prefill, drain and throughput folded into
    its SLO, swap and throughput tables (a new DeviceProblem sharing the other
    arrays), and the per-request SLOs less the prefill when req_slo is given.
    ``profile`` maps the qlm_profile field names to arrays (or None)."""
    import copy
    import torch
    dev = problem.grp_count.device
    M, C = problem.n_models, problem.n_classes
    keep = {}
    for f in PROFILE_FIELDS:
        x = profile.get(f)
        keep[f] = None if x is None else torch.as_tensor(
            np.ascontiguousarray(x, dtype=np.float32).reshape(-1)).to(dev)
    sizes = {"prefill": M, "decode_time": C * M, "ineff": C * M, "max_tokens": M,
             "kv_tokens": C * M, "mean_tokens": M}
    for f, x in keep.items():
        if x is not None and x.numel() != sizes[f]:
            raise ValueError(f + " has the wrong size")
    im = None if inst_model is None else torch.as_tensor(
        np.ascontiguousarray(inst_model, dtype=np.int32)).to(dev)
    if im is not None and im.numel() != problem.n_instances:
        raise ValueError("inst_model must have n_instances entries")
    pf = Profile(*[_ptr(keep[f]) for f in PROFILE_FIELDS])
    out = copy.copy(problem)
    out.swap_cost = torch.empty(C * M * M, dtype=torch.float32, device=dev)
    out.grp_slo = torch.empty(problem.n_groups, dtype=torch.float32, device=dev)
    out.inst_tput = torch.empty(problem.n_instances, dtype=torch.float32, device=dev)
    rs = None
    if req_slo is not None:
        rs = torch.empty_like(req_slo)
    _check(library().qlm_apply_profile(ctypes.byref(problem.struct), ctypes.byref(pf), _ptr(im),
                                       _ptr(out.swap_cost), _ptr(out.grp_slo),
                                       _ptr(out.inst_tput), _ptr(req_slo),
                                       0 if req_slo is None else req_slo.numel(), _ptr(rs),
                                       _stream(stream)))
    out._profile_keep = (keep, im)
    out.struct = Problem(out.n_groups, out.n_instances, out.n_models, out.n_classes,
                         _ptr(out.grp_count), _ptr(out.grp_mu), _ptr(out.grp_var),
                         _ptr(out.grp_model), _ptr(out.grp_slo), _ptr(out.inst_tput),
                         _ptr(out.inst_class), _ptr(out.inst_model0), _ptr(out.swap_cost),
                         out.evict_cost)
    return out, rs


class PlaceSession:
    """A placement session (qlm_place_begin / step / end): the plans stay in
    the workspace while groups are placed one after another, on one stream
    (`stream`, or the current stream when the session begins)."""

    def __init__(self, problem: DeviceProblem, plans: DevicePlans, ws=None, stream=None):
        import torch
        if stream is None:
            stream = torch.cuda.current_stream()
        self.problem = problem
        self.n_plans = plans.n_plans
        self.has_evict = plans.evict_bits is not None
        self.like = plans
        self.dev = plans.perm.device
        self.ws = ws if ws is not None else search_workspace(problem, plans.n_plans, 0, self.dev)
        self.stream = stream
        _check(library().qlm_place_begin(ctypes.byref(problem.struct), ctypes.byref(plans.struct),
                                         _ptr(self.ws), self.ws.numel(), _stream(stream)))
        self.score = torch.full((max(self.n_plans, 1),), float("nan"), dtype=torch.float64,
                                device=self.dev)
        self.queue = torch.full((max(self.n_plans, 1),), -2, dtype=torch.int32, device=self.dev)
        # a step's arguments but the group, formed once (a step is a few tens of
        # microseconds of GPU work; marshalling them per call would add as much)
        self._fn = library().qlm_place_step
        self._args = (ctypes.byref(problem.struct), self.n_plans)
        self._rest = (_ptr(self.ws), self.ws.numel(), _ptr(self.score), _ptr(self.queue),
                      _stream(stream))
        self._out = (self.score[:self.n_plans], self.queue[:self.n_plans])

    def step(self, group: int):
        """Places `group` in every plan; returns (scores [P], places [P]) (device)."""
        _check(self._fn(*self._args, int(group), *self._rest))
        return self._out

    def end(self, out: DevicePlans | None = None):
        """The plans as they stand (DevicePlans) and their exact scores."""
        import torch
        if out is None:
            out = plans_like(self.like, self.problem.n_groups)
        o = PlansOut(int(out.perm.shape[1]), _ptr(out.perm), _ptr(out.qoff), _ptr(out.evict_bits))
        score = torch.empty(max(self.n_plans, 1), dtype=torch.float64, device=self.dev)
        _check(library().qlm_place_end(ctypes.byref(self.problem.struct), self.n_plans,
                                       ctypes.byref(o), _ptr(self.ws), self.ws.numel(),
                                       _ptr(score), _stream(self.stream)))
        return out, score[:self.n_plans]


# -- a serving instance's decode step ------------------------------------------

KV_BLOCK = 64
_KV_FORMATS = ("float8_e4m3fn", "int8")


# A decode step makes these calls once a layer, each of a few microseconds on
# the GPU: their structs are packed as bytes and the stream is taken as a number
# (a few microseconds less a call than ctypes objects and torch.cuda.Stream).
_ROWS = struct.Struct("@Pqqi0P")
_KV_QUERY = struct.Struct("@Pqqi0PPqqi0Pifif0P")
_ROTARY = struct.Struct("@iiiiPPPP")
_DRAFT = struct.Struct("@iiPPqqPP")
_F8_CODES = struct.Struct("@iiPP")
_row_types = {}
_word_types = {}


def _row_type(t, what):
    if not _row_types:
        import torch
        _row_types.update({torch.float16: 0, torch.bfloat16: 1})
    kind = _row_types.get(t.dtype)
    if kind is None:
        raise ValueError("%s must be float16 or bfloat16" % what)
    return kind


def _rows(t, n_rows, heads, dim, what):
    """(pointer, row stride, head stride, type) of rows [n_rows, heads, dim]."""
    if t.shape != (n_rows, heads, dim):
        raise ValueError("%s must be [%d rows, %d, %d]" % (what, n_rows, heads, dim))
    row, head, one = t.stride()
    if one != 1:
        raise ValueError("%s: a head's dims must be contiguous" % what)
    return t.data_ptr(), row, head, _row_type(t, what)


def _allocated(stream, make, returned=True):
    """What `make` allocates for a call on `stream` (None: the current one).  The
    allocator hands memory out again in the order of the stream it was allocated on, and
    that must be the stream whose kernels use it: not memory that the current one still
    works in, nor given away by it while the call is queued.  What the caller gets is kept
    from reuse until the current stream has passed the point where it was dropped, too."""
    if stream is None:
        return make()
    import torch
    with torch.cuda.stream(stream):
        t = make()
    if returned:
        t.record_stream(torch.cuda.current_stream())
    return t


def _refuse_place(index, **tensors):
    """Names the tensor that is not on GPU `index`, that of the call's cache or matrix
    (-1 of host memory): a kernel would follow its address."""
    for name, t in tensors.items():
        if index < 0 or (t is not None and t.get_device() != index):
            raise ValueError("%s must be on the GPU, together with the call's other tensors" % name)


def _raw_stream(stream):
    if stream is not None:
        return stream.cuda_stream
    import torch
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _stream_on(index, stream):
    """The raw stream of a call whose tensors are on GPU `index`: a launch goes to the stream's
    GPU, so that has to be theirs."""
    import torch
    at = torch._C._cuda_getDevice() if stream is None else stream.device_index
    if at != index:
        raise ValueError("the call's tensors are on GPU %d, its stream on GPU %d" % (index, at))
    return torch._C._cuda_getCurrentRawStream(at) if stream is None else stream.cuda_stream


class DeviceKvCache:
    """An 8-bit token cache in device memory plus the C struct (qlm_kv_cache).

    k_codes   [n_blocks, n_kv_heads, 64, head_dim], float8_e4m3fn or int8
    v_codes   [n_blocks, n_kv_heads, 4, head_dim, 16], the same type: slot t of a
              block stands in group (t // 4) % 4, there at place (t // 16) * 4 + t % 4
    k_scale, v_scale   [n_blocks, n_kv_heads] float32
    position  [n_blocks, n_kv_heads, 64] int32 or None
    weight    [n_blocks, n_kv_heads, 64] float32 or None

    Every tensor is contiguous.  ``DeviceKvCache.empty`` allocates one."""

    def __init__(self, k_codes, v_codes, k_scale, v_scale, position=None, weight=None):
        import torch
        if k_codes.dim() != 4 or k_codes.shape[2] != KV_BLOCK:
            raise ValueError("k_codes must be [n_blocks, n_kv_heads, 64, head_dim]")
        nb, h, _, d = k_codes.shape
        kinds = [getattr(torch, n) for n in _KV_FORMATS]
        if k_codes.dtype not in kinds or v_codes.dtype != k_codes.dtype:
            raise ValueError("codes must be float8_e4m3fn or int8, keys and values alike")
        want = {"v_codes": (v_codes, (nb, h, 4, d, 16), v_codes.dtype),
                "k_scale": (k_scale, (nb, h), torch.float32),
                "v_scale": (v_scale, (nb, h), torch.float32),
                "position": (position, (nb, h, KV_BLOCK), torch.int32),
                "weight": (weight, (nb, h, KV_BLOCK), torch.float32),
                "k_codes": (k_codes, (nb, h, KV_BLOCK, d), k_codes.dtype)}
        for name, (x, shape, dtype) in want.items():
            if x is None and name in ("position", "weight"):
                continue
            if tuple(x.shape) != shape or x.dtype != dtype or not x.is_contiguous():
                raise ValueError("%s must be contiguous %s of %s" % (name, shape, dtype))
            if x.device != k_codes.device:
                raise ValueError("%s must be where k_codes is" % name)
        self.index = k_codes.get_device()
        self.n_blocks, self.n_kv_heads, self.head_dim = int(nb), int(h), int(d)
        self.k_codes, self.v_codes = k_codes, v_codes
        self.k_scale, self.v_scale = k_scale, v_scale
        self.position, self.weight = position, weight
        self.struct = KvCacheStruct(self.n_blocks, self.n_kv_heads, self.head_dim,
                                    kinds.index(k_codes.dtype), _ptr(k_codes), _ptr(v_codes),
                                    _ptr(k_scale), _ptr(v_scale), _ptr(position), _ptr(weight))
        self._ref = ctypes.byref(self.struct)

    @classmethod
    def empty(cls, n_blocks, n_kv_heads, head_dim, dtype=None, keep_weights=True, device="cuda"):
        """An unwritten cache; positions and weights are kept unless
        keep_weights is False."""
        import torch
        dtype = torch.float8_e4m3fn if dtype is None else dtype
        codes = lambda *s: torch.empty(s, dtype=torch.uint8, device=device).view(dtype)  # noqa: E731
        slots = (n_blocks, n_kv_heads, KV_BLOCK)
        return cls(codes(*slots, head_dim), codes(n_blocks, n_kv_heads, 4, head_dim, 16),
                   torch.empty((n_blocks, n_kv_heads), dtype=torch.float32, device=device),
                   torch.empty((n_blocks, n_kv_heads), dtype=torch.float32, device=device),
                   torch.empty(slots, dtype=torch.int32, device=device) if keep_weights else None,
                   torch.empty(slots, dtype=torch.float32, device=device) if keep_weights else None)


class KvBatch:
    """The sequences of a call (qlm_kv_batch): ``block_table`` [n_seqs, blocks]
    int32, ``lengths`` [n_seqs] int32 (new tokens included), ``row_start``
    [n_seqs + 1] int32 or None (one row each), ``n_rows`` rows in all, at most
    ``max_new`` of a sequence, which holds at most ``max_length`` slots (default:
    what the table's rows can hold)."""

    def __init__(self, block_table, lengths, row_start=None, n_rows=None, max_new=1,
                 max_length=None):
        import torch
        for name, x in (("block_table", block_table), ("lengths", lengths),
                        ("row_start", row_start)):
            if x is not None and x.dtype != torch.int32:
                raise ValueError(name + " must be int32")
        n = int(lengths.numel())
        if block_table.dim() != 2 or block_table.shape[0] != n or not lengths.is_contiguous():
            raise ValueError("block_table must be [n_seqs, blocks] and lengths [n_seqs]")
        if block_table.shape[1] > 1 and block_table.stride(1) != 1:
            raise ValueError("a row of block_table must be contiguous")
        if row_start is not None and (row_start.numel() != n + 1 or not row_start.is_contiguous()):
            raise ValueError("row_start must be [n_seqs + 1]")
        if row_start is not None and n_rows is None:
            raise ValueError("n_rows is required with row_start")
        if any(x is not None and x.device != lengths.device for x in (block_table, row_start)):
            raise ValueError("block_table and row_start must be where lengths is")
        self.index = lengths.get_device()
        width = int(block_table.shape[1])
        if max_length is None:
            max_length = width * KV_BLOCK
        if max_length > width * KV_BLOCK:
            raise ValueError("max_length exceeds the blocks of block_table's rows")
        self.block_table, self.lengths, self.row_start = block_table, lengths, row_start
        self.n_seqs, self.max_new, self.max_length = n, int(max_new), int(max_length)
        self.n_rows = n if row_start is None else int(n_rows)
        # (the stride of a table of one row says nothing)
        stride = int(block_table.stride(0)) if n > 1 else width
        self.struct = KvBatchStruct(n, self.n_rows, self.max_new, self.max_length, stride,
                                    _ptr(block_table), _ptr(lengths), _ptr(row_start))
        self._ref = ctypes.byref(self.struct)


def kv_append(cache: DeviceKvCache, batch: KvBatch, k, v, first_position=None, stream=None):
    """Writes the new tokens' keys and values [n_rows, n_kv_heads, head_dim]
    (float16 or bfloat16) into the last slots of their sequences.
    first_position [n_seqs] int32: the position of each sequence's first new
    token (the slot's number when None)."""
    if first_position is not None and (first_position.dtype != batch.lengths.dtype or
                                       first_position.numel() != batch.n_seqs or
                                       not first_position.is_contiguous()):
        raise ValueError("first_position must be [n_seqs] int32")
    rk = _rows(k, batch.n_rows, cache.n_kv_heads, cache.head_dim, "k")
    rv = _rows(v, batch.n_rows, cache.n_kv_heads, cache.head_dim, "v")
    if not 0 <= cache.index == batch.index == k.get_device() == v.get_device() or \
            (first_position is not None and first_position.get_device() != cache.index):
        _refuse_place(cache.index, cache=cache.k_codes, batch=batch.lengths, k=k, v=v,
                      first_position=first_position)
    rc = (_lib or library()).qlm_kv_append(
        cache._ref, batch._ref, _ROWS.pack(*rk), _ROWS.pack(*rv),
        None if first_position is None else first_position.data_ptr(), _raw_stream(stream))
    if rc:
        _check(rc)


class Rotary:
    """Tables of a rotation by position: ``cos`` and ``sin`` [n_positions, pairs]
    float32, contiguous; twice the pairs' number of a head's dims turn, dim i with
    dim i + pairs, or 2i with 2i + 1 where ``interleaved``.  ``axis`` [pairs] int32:
    which of a token's positions turns the pair (the first one where None)."""

    def __init__(self, cos, sin, interleaved=False, axis=None):
        import torch
        for name, x in (("cos", cos), ("sin", sin)):
            if x.dim() != 2 or x.dtype != torch.float32 or not x.is_contiguous() or \
                    x.shape != cos.shape:
                raise ValueError(name + " must be contiguous [n_positions, pairs] float32")
        if axis is not None and (axis.dtype != torch.int32 or axis.shape != cos.shape[1:] or
                                 not axis.is_contiguous()):
            raise ValueError("axis must be [pairs] int32")
        if any(x is not None and x.device != cos.device for x in (sin, axis)):
            raise ValueError("sin and axis must be where cos is")
        self.cos, self.sin, self.axis, self.interleaved = cos, sin, axis, bool(interleaved)
        self.n_positions, self.pairs = (int(x) for x in cos.shape)
        self.index = cos.get_device()
        self._tables = (_ptr(cos), _ptr(sin), _ptr(axis) or 0)


def kv_append_rotated(cache: DeviceKvCache, batch: KvBatch, k, v, q, rotary: Rotary,
                      position=None, first_position=None, out=None, stream=None):
    """``kv_append`` of keys turned by their positions, together with the rows'
    queries q [n_rows, n_heads, head_dim] (None: no queries); returns the turned
    queries (``out``, which may be q itself).  position [axes, n_rows] (or [n_rows])
    int32: each row's positions on the rotation's axes; None: the position that the
    cache keeps for its slot, counted from first_position."""
    if first_position is not None and (first_position.dtype != batch.lengths.dtype or
                                       first_position.numel() != batch.n_seqs or
                                       not first_position.is_contiguous()):
        raise ValueError("first_position must be [n_seqs] int32")
    n, kv, dim = batch.n_rows, cache.n_kv_heads, cache.head_dim
    axes, at = 1, 0
    if position is not None:
        shape = position.shape
        if position.dtype != batch.lengths.dtype or not position.is_contiguous() or \
                len(shape) not in (1, 2) or shape[-1] != n:
            raise ValueError("position must be contiguous [axes, %d rows] int32" % n)
        axes, at = shape[0] if len(shape) == 2 else 1, position.data_ptr()
    rk, rv = _rows(k, n, kv, dim, "k"), _rows(v, n, kv, dim, "v")
    index, heads, rq, ro = cache.index, 0, None, None
    here = 0 <= index == batch.index == rotary.index == k.get_device() == v.get_device() and \
        (position is None or position.get_device() == index) and \
        (first_position is None or first_position.get_device() == index)
    if q is not None:
        if q.dim() != 3:
            raise ValueError("q must be [rows, n_heads, head_dim]")
        heads = q.shape[1]
        rq = _rows(q, n, heads, dim, "q")
        if out is None:
            import torch
            make = lambda: torch.empty_like(q, memory_format=torch.contiguous_format)  # noqa: E731
            out = make() if stream is None else _allocated(stream, make)
            ro = (out.data_ptr(), heads * dim, dim, rq[3])
        elif out.shape != q.shape or out.dtype != q.dtype:
            raise ValueError("out must have q's shape and type")
        else:
            ro = _rows(out, n, heads, dim, "out")
        here = here and q.get_device() == index == out.get_device()
    elif out is not None:
        raise ValueError("out is of queries, and there are none")
    if not here:
        _refuse_place(index, cache=cache.k_codes, batch=batch.lengths, k=k, v=v, q=q, out=out,
                      rotary=rotary.cos, position=position, first_position=first_position)
    rc = (_lib or library()).qlm_kv_append_rotated(
        cache._ref, batch._ref, _ROWS.pack(*rk), _ROWS.pack(*rv),
        _ROWS.pack(*rq) if heads else None, _ROWS.pack(*ro) if heads else None, heads,
        _ROTARY.pack(2 * rotary.pairs, rotary.interleaved, rotary.n_positions, axes,
                     *rotary._tables, at),
        None if first_position is None else first_position.data_ptr(), _stream_on(index, stream))
    if rc:
        _check(rc)
    return out


def kv_attention_workspace_bytes(cache: DeviceKvCache, batch: KvBatch, n_heads: int,
                                 accumulate: bool = False) -> int:
    return int(library().qlm_kv_attention_workspace_bytes(cache._ref, batch._ref, int(n_heads),
                                                          int(bool(accumulate))))


def kv_attention_workspace(cache: DeviceKvCache, batch: KvBatch, n_heads: int,
                           accumulate: bool = False):
    import torch
    nbytes = kv_attention_workspace_bytes(cache, batch, n_heads, accumulate)
    return torch.empty(max(nbytes, 1), dtype=torch.uint8, device=cache.k_codes.device)


def kv_attention(cache: DeviceKvCache, batch: KvBatch, q, scale=None, weight_decay=None,
                 out=None, ws=None, stream=None):
    """Attention of the batch's rows q [n_rows, n_heads, head_dim] over their
    sequences' slots; the outputs, of q's shape and type.  scale: of the
    scores, head_dim ** -0.5 when None.  weight_decay: when given, the cache's
    weights become weight_decay * weight plus the step's attention weights."""
    import torch
    if q.dim() != 3:
        raise ValueError("q must be [rows, n_heads, head_dim]")
    heads, dim = q.shape[1], cache.head_dim
    rq = _rows(q, batch.n_rows, heads, dim, "q")
    if out is None:
        out = _allocated(stream, lambda: torch.empty(q.shape, dtype=q.dtype, device=q.device))
    elif out.shape != q.shape or out.dtype != q.dtype:
        raise ValueError("out must have q's shape and type")
    if ws is None:
        ws = _allocated(stream, lambda: kv_attention_workspace(cache, batch, heads,
                                                               weight_decay is not None), False)
    query = _KV_QUERY.pack(*rq, *_rows(out, batch.n_rows, heads, dim, "out"), heads,
                           dim ** -0.5 if scale is None else scale, weight_decay is not None,
                           weight_decay or 0.0)
    if not 0 <= cache.index == batch.index == q.get_device() == out.get_device() == ws.get_device():
        _refuse_place(cache.index, cache=cache.k_codes, batch=batch.lengths, q=q, out=out, ws=ws)
    rc = (_lib or library()).qlm_kv_attention(cache._ref, batch._ref, query, ws.data_ptr(),
                                              ws.numel(), _raw_stream(stream))
    if rc:
        _check(rc)
    return out


def kv_evict_workspace_bytes(cache: DeviceKvCache, batch: KvBatch, budget: int) -> int:
    return int(library().qlm_kv_evict_workspace_bytes(cache._ref, batch._ref, int(budget)))


def kv_evict_workspace(cache: DeviceKvCache, batch: KvBatch, budget: int):
    import torch
    return torch.empty(max(kv_evict_workspace_bytes(cache, batch, budget), 1), dtype=torch.uint8,
                       device=cache.k_codes.device)


def kv_evict(cache: DeviceKvCache, batch: KvBatch, budget: int, recent: int = 0, out=None,
             ws=None, stream=None):
    """Cuts the sequences to `budget` slots (a multiple of 64) for each kv head:
    the slots of the `recent` newest positions and those of the greatest weight
    stay.  Returns the new lengths [n_seqs] int32 (`out`, which may be the
    batch's own lengths)."""
    if out is None:
        import torch
        out = _allocated(stream, lambda: torch.empty_like(batch.lengths))
    elif out.dtype != batch.lengths.dtype or out.numel() != batch.n_seqs or not out.is_contiguous():
        raise ValueError("out must be [n_seqs] int32")
    if ws is None:
        ws = _allocated(stream, lambda: kv_evict_workspace(cache, batch, budget), False)
    if not 0 <= cache.index == batch.index == out.get_device() == ws.get_device():
        _refuse_place(cache.index, cache=cache.k_codes, batch=batch.lengths, out=out, ws=ws)
    rc = (_lib or library()).qlm_kv_evict(cache._ref, batch._ref, budget, recent, out.data_ptr(),
                                          ws.data_ptr(), ws.numel(), _raw_stream(stream))
    if rc:
        _check(rc)
    return out


class W4:
    """A matrix of 4-bit weights as the kernels read it (qlm_w4): made by
    ``w4_pack``."""

    def __init__(self, packed, n_out, n_in, group):
        self.packed, self.n_out, self.n_in, self.group = packed, n_out, n_in, group
        self.index = packed.get_device()
        self.struct = W4Struct(n_out, n_in, group, _ptr(packed))
        self._ref = ctypes.byref(self.struct)


def w4_pack(codes, scale, zero=None, group=None, stream=None):
    """Lays out 4-bit weights (code - zero) * scale once: ``codes`` [n_out, n_in]
    uint8 (0..15), ``scale`` [n_out, groups] float16, ``zero`` [n_out, groups]
    uint8 (8 everywhere when None), a group for each 32, 64 or 128 inputs
    (found from the shapes when None)."""
    import torch
    if codes.dim() != 2 or codes.dtype != torch.uint8 or not codes.is_contiguous():
        raise ValueError("codes must be contiguous [n_out, n_in] uint8")
    n, k = (int(x) for x in codes.shape)
    fits = [g for g in (128, 64, 32) if scale.dim() == 2 and -(-k // g) == scale.shape[1]]
    if group is None:
        if not fits:
            raise ValueError("scale's groups fit no group of 32, 64 or 128 inputs")
        group = fits[0]
    if group not in fits or scale.shape[0] != n or scale.dtype != torch.float16 or \
            not scale.is_contiguous():
        raise ValueError("scale must be contiguous [n_out, ceil(n_in / group)] float16")
    if zero is not None and (zero.shape != scale.shape or zero.dtype != torch.uint8 or
                             not zero.is_contiguous()):
        raise ValueError("zero must be contiguous uint8 of scale's shape")
    _refuse_place(codes.get_device(), codes=codes, scale=scale, zero=zero)
    nbytes = int(library().qlm_w4_packed_bytes(n, k, group))
    packed = _allocated(stream, lambda: torch.empty(nbytes, dtype=torch.uint8, device=codes.device))
    w = W4(packed, n, k, group)
    _check(library().qlm_w4_pack(w._ref, _ptr(codes), _ptr(scale), _ptr(zero), _stream(stream)))
    return w


def w4_workspace_bytes(weight: W4, n_rows: int) -> int:
    return int(library().qlm_w4_workspace_bytes(weight._ref, int(n_rows)))


def w4_workspace(weight: W4, n_rows: int):
    import torch
    return torch.empty(max(w4_workspace_bytes(weight, n_rows), 1), dtype=torch.uint8,
                       device=weight.packed.device)


def w4_matmul(x, weight: W4, out=None, ws=None, stream=None):
    """x [n_rows, n_in] (float16 or bfloat16) times the matrix: [n_rows, n_out]
    of x's type."""
    import torch
    if x.dim() != 2 or x.shape[1] != weight.n_in or (x.stride(1) != 1 and weight.n_in > 1):
        raise ValueError("x must be [rows, %d] with contiguous rows" % weight.n_in)
    kind = _row_type(x, "x")
    n = x.shape[0]
    if out is None:
        out = _allocated(stream, lambda: torch.empty((n, weight.n_out), dtype=x.dtype,
                                                     device=x.device))
    elif tuple(out.shape) != (n, weight.n_out) or out.dtype != x.dtype or \
            (out.stride(1) != 1 and weight.n_out > 1):
        raise ValueError("out must be [rows, %d] of x's type with contiguous rows" % weight.n_out)
    if ws is None:
        ws = _allocated(stream, lambda: w4_workspace(weight, n), False)
    # (the stride of a matrix of one row says nothing)
    xs, os_ = (x.stride(0), out.stride(0)) if n > 1 else (weight.n_in, weight.n_out)
    if not 0 <= weight.index == x.get_device() == out.get_device() == ws.get_device():
        _refuse_place(weight.index, weight=weight.packed, x=x, out=out, ws=ws)
    rc = (_lib or library()).qlm_w4_matmul(weight._ref, x.data_ptr(), xs, out.data_ptr(), os_, n,
                                           kind, ws.data_ptr(), ws.numel(), _raw_stream(stream))
    if rc:
        _check(rc)
    return out


F8_BLOCK, F8_TILE = 128, 16


class F8:
    """A matrix of e4m3 weights as the kernels read it (qlm_f8): made by
    ``f8_pack``."""

    def __init__(self, packed, n_out, n_in):
        self.packed, self.n_out, self.n_in = packed, n_out, n_in
        self.index = packed.get_device()
        self.struct = F8Struct(n_out, n_in, _ptr(packed))
        self._ref = ctypes.byref(self.struct)


class F8Rows:
    """Rows in e4m3 with a scale for each row and 128 inputs (qlm_f8_codes): made by
    ``f8_rows``, or from

    codes  [ceil(n_rows / 16), ceil(n_in / 128), 8, 16, 16] float8_e4m3fn: input k of
           row r of a tile at [k % 128 // 16, r, k % 16], zeros past the last row and
           input
    scale  [ceil(n_in / 128), 16 * ceil(n_rows / 16)] float32

    both contiguous."""

    def __init__(self, codes, scale, n_rows, n_in):
        import torch
        tiles, blocks = -(-n_rows // F8_TILE), -(-n_in // F8_BLOCK)
        if tuple(codes.shape) != (tiles, blocks, 8, F8_TILE, 16) or \
                codes.dtype != torch.float8_e4m3fn or not codes.is_contiguous():
            raise ValueError("codes must be contiguous [%d, %d, 8, 16, 16] float8_e4m3fn"
                             % (tiles, blocks))
        if tuple(scale.shape) != (blocks, tiles * F8_TILE) or scale.dtype != torch.float32 or \
                not scale.is_contiguous():
            raise ValueError("scale must be contiguous [%d, %d] float32"
                             % (blocks, tiles * F8_TILE))
        if scale.device != codes.device:
            raise ValueError("scale must be where codes is")
        self._hold(codes, scale, int(n_rows), int(n_in))

    def _hold(self, codes, scale, n_rows, n_in):
        self.codes, self.scale, self.n_rows, self.n_in = codes, scale, n_rows, n_in
        self.index = codes.get_device()
        self._struct = _F8_CODES.pack(n_rows, n_in, codes.data_ptr(), scale.data_ptr())

    @classmethod
    def _empty(cls, n_rows, n_in, device, stream):
        """Room for so many rows, as a call on `stream` allocates it."""
        import torch
        tiles, blocks = -(-n_rows // F8_TILE), -(-n_in // F8_BLOCK)
        kind, at, by = torch.float8_e4m3fn, (tiles, blocks, 8, F8_TILE, 16), (blocks, tiles * F8_TILE)
        if stream is None:
            codes = torch.empty(at, dtype=kind, device=device)
            scale = torch.empty(by, dtype=torch.float32, device=device)
        else:
            codes = _allocated(stream, lambda: torch.empty(at, dtype=kind, device=device))
            scale = _allocated(stream, lambda: torch.empty(by, dtype=torch.float32, device=device))
        rows = cls.__new__(cls)
        rows._hold(codes, scale, n_rows, n_in)
        return rows


def f8_pack(codes, scale, stream=None):
    """Lays out 8-bit weights code * scale once: ``codes`` [n_out, n_in]
    float8_e4m3fn, ``scale`` [ceil(n_out / 128), ceil(n_in / 128)] float32."""
    import torch
    if codes.dim() != 2 or codes.dtype != torch.float8_e4m3fn or not codes.is_contiguous():
        raise ValueError("codes must be contiguous [n_out, n_in] float8_e4m3fn")
    n, k = (int(x) for x in codes.shape)
    if tuple(scale.shape) != (-(-n // F8_BLOCK), -(-k // F8_BLOCK)) or \
            scale.dtype != torch.float32 or not scale.is_contiguous():
        raise ValueError("scale must be contiguous [ceil(n_out / 128), ceil(n_in / 128)] float32")
    _refuse_place(codes.get_device(), codes=codes, scale=scale)
    nbytes = int(library().qlm_f8_packed_bytes(n, k))
    packed = _allocated(stream, lambda: torch.empty(nbytes, dtype=torch.uint8, device=codes.device))
    w = F8(packed, n, k)
    _check(library().qlm_f8_pack(w._ref, _ptr(codes), _ptr(scale), _stream_on(w.index, stream)))
    return w


def f8_rows(x, out=None, stream=None):
    """x [n_rows, n_in] (float16 or bfloat16) as e4m3 codes with a scale for each row
    and 128 inputs: an F8Rows (``out``, of x's sizes, when given)."""
    import torch
    if x.dim() != 2 or (x.stride(1) != 1 and x.shape[1] > 1) or x.shape[1] < 1:
        raise ValueError("x must be [rows, inputs] with contiguous rows")
    kind = _row_type(x, "x")
    n, k = x.shape
    if out is None:
        out = F8Rows._empty(n, k, x.device, stream)
    elif out.n_rows != n or out.n_in != k:
        raise ValueError("out must be of %d rows of %d inputs" % (n, k))
    if not 0 <= out.index == x.get_device():
        _refuse_place(x.get_device(), x=x, out=out.codes)
    # (the stride of a matrix of one row says nothing)
    rc = (_lib or library()).qlm_f8_rows(out._struct, x.data_ptr(), x.stride(0) if n > 1 else k,
                                         kind, _stream_on(out.index, stream))
    if rc:
        _check(rc)
    return out


def f8_workspace_bytes(weight: F8, n_rows: int) -> int:
    return int(library().qlm_f8_workspace_bytes(weight._ref, int(n_rows)))


def f8_workspace(weight: F8, n_rows: int):
    import torch
    return torch.empty(max(f8_workspace_bytes(weight, n_rows), 1), dtype=torch.uint8,
                       device=weight.packed.device)


def _word_type(dtype, what):
    """The number of a row type, of which float32 is one too."""
    if not _word_types:
        import torch
        _word_types.update({torch.float16: 0, torch.bfloat16: 1, torch.float32: 2})
    kind = _word_types.get(dtype)
    if kind is None:
        raise ValueError("%s must be float16, bfloat16 or float32" % what)
    return kind


def f8_matmul(x: F8Rows, weight: F8, out=None, dtype=None, ws=None, stream=None):
    """Coded rows times the matrix: [n_rows, n_out] of ``dtype`` (bfloat16 when None;
    out's where out is given).  float32 outputs too hold sums of the 8-bit matrix
    instructions, which keep 13 bits below the largest of eight neighbouring products:
    1.5e-5 to 3e-5 of the outputs' norm."""
    import torch
    if x.n_in != weight.n_in:
        raise ValueError("x must be rows of %d inputs" % weight.n_in)
    n = x.n_rows
    if out is None:
        dtype = torch.bfloat16 if dtype is None else dtype
        kind = _word_type(dtype, "dtype")
        shape, dev = (n, weight.n_out), x.codes.device
        if stream is None:
            out = torch.empty(shape, dtype=dtype, device=dev)
        else:
            out = _allocated(stream, lambda: torch.empty(shape, dtype=dtype, device=dev))
    elif tuple(out.shape) != (n, weight.n_out) or (dtype is not None and out.dtype != dtype) or \
            (out.stride(1) != 1 and weight.n_out > 1):
        raise ValueError("out must be [%d, %d] with contiguous rows" % (n, weight.n_out))
    else:
        kind = _word_type(out.dtype, "out")
    if ws is None:
        ws = _allocated(stream, lambda: f8_workspace(weight, n), False)
    if not 0 <= weight.index == x.index == out.get_device() == ws.get_device():
        _refuse_place(weight.index, weight=weight.packed, x=x.codes, out=out, ws=ws)
    rc = (_lib or library()).qlm_f8_matmul(x._struct, weight._ref, out.data_ptr(),
                                           out.stride(0) if n > 1 else weight.n_out, kind,
                                           ws.data_ptr(), ws.numel(), _stream_on(weight.index, stream))
    if rc:
        _check(rc)
    return out


def draft_verify_workspace_bytes(batch: KvBatch, vocab: int) -> int:
    return int(library().qlm_draft_verify_workspace_bytes(batch._ref, int(vocab)))


def draft_verify_workspace(batch: KvBatch, vocab: int):
    import torch
    return torch.empty(max(draft_verify_workspace_bytes(batch, vocab), 1), dtype=torch.uint8,
                       device=batch.lengths.device)


def draft_verify(batch: KvBatch, tokens, target, draft, uniform, lengths=None, ws=None,
                 stream=None):
    """Verifies the drafted tokens of a step.  The batch's rows are a token of each
    sequence and the drafts behind it; tokens [n_rows] int32; target [n_rows, vocab]
    the probabilities behind each row, draft the same of the drafting model (None:
    the drafts were chosen, not drawn), float16, bfloat16 or float32 alike; uniform
    [n_rows] float32 in [0, 1).  Returns (tokens [n_seqs, max_new] int32: accepted
    drafts, the token drawn, -1; their number [n_seqs] int32; the lengths that stay
    in the cache [n_seqs] int32: ``lengths``, which may be the batch's own)."""
    import torch
    n, seqs, index = batch.n_rows, batch.n_seqs, batch.index
    shape, stride = target.shape, target.stride()
    if len(shape) != 2 or shape[0] != n or shape[1] < 1 or (stride[1] != 1 and shape[1] > 1):
        raise ValueError("target must be [%d rows, vocab] with contiguous rows" % n)
    vocab = shape[1]
    kind = _word_type(target.dtype, "target")
    near, apart = 0, vocab
    if draft is not None:
        if draft.shape != shape or draft.dtype != target.dtype or \
                (draft.stride(1) != 1 and vocab > 1):
            raise ValueError("draft must have target's shape and type, with contiguous rows")
        near, apart = draft.data_ptr(), draft.stride(0)
    if tokens.dtype != torch.int32 or tokens.numel() != n or not tokens.is_contiguous():
        raise ValueError("tokens must be [%d rows] int32" % n)
    if uniform.dtype != torch.float32 or uniform.numel() != n or not uniform.is_contiguous():
        raise ValueError("uniform must be [%d rows] float32" % n)
    have = batch.lengths
    if lengths is not None and (lengths.dtype != torch.int32 or lengths.numel() != seqs or
                                not lengths.is_contiguous()):
        raise ValueError("lengths must be [n_seqs] int32")
    one = lambda: torch.empty_like(have)  # noqa: E731
    rows = lambda: torch.empty((seqs, batch.max_new), dtype=torch.int32,  # noqa: E731
                               device=have.device)
    if stream is None:
        out, count, lengths = rows(), one(), one() if lengths is None else lengths
    else:
        out, count = _allocated(stream, rows), _allocated(stream, one)
        lengths = _allocated(stream, one) if lengths is None else lengths
    if ws is None:
        ws = _allocated(stream, lambda: draft_verify_workspace(batch, vocab), False)
    if not 0 <= index == tokens.get_device() == target.get_device() == uniform.get_device() == \
            lengths.get_device() == ws.get_device() or \
            (draft is not None and draft.get_device() != index):
        _refuse_place(index, batch=batch.lengths, tokens=tokens, target=target, draft=draft,
                      uniform=uniform, lengths=lengths, ws=ws)
    # (the stride of a matrix of one row says nothing)
    rc = (_lib or library()).qlm_draft_verify(
        batch._ref,
        _DRAFT.pack(vocab, kind, target.data_ptr(), near, stride[0] if n > 1 else vocab,
                    apart if n > 1 else vocab, tokens.data_ptr(), uniform.data_ptr()),
        out.data_ptr(), count.data_ptr(), lengths.data_ptr(), ws.data_ptr(), ws.numel(),
        _stream_on(index, stream))
    if rc:
        _check(rc)
    return out, count, lengths
