"""Binding of libpcpp.so: argument marshalling only (torch tensors -> device pointers), by ctypes, and by compiled code for the
operators whose calls are short."""
from __future__ import annotations

import ctypes
import importlib.util
import os
import threading
from dataclasses import dataclass

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libpcpp.so")

PCPP_F32, PCPP_BF16 = 0, 1
PLAN_FWD, PLAN_BWD_INPUT, PLAN_SPATIAL = 1, 2, 4
BUILD_TEST_SHORT_LISTS, BUILD_TEST_WIDE_KEYS, BUILD_VOXEL = 0x100, 0x200, 0x400
PLAN_MASK = PLAN_FWD | PLAN_BWD_INPUT | PLAN_SPATIAL
NORM_NONE, NORM_RMS, NORM_LAYER = 0, 1, 2
ACT_NONE, ACT_RELU, ACT_SILU, ACT_GELU = 0, 1, 2, 3
DROP_ELEMENTS, DROP_ROWS, DROP_CLOUDS = 0, 1, 2
ERR_CAPACITY = -2

EXPORTS = ("pcpp_last_error", "pcpp_version", "pcpp_build_triplets_workspace_bytes",
           "pcpp_build_triplets_workspace_bytes_for", "pcpp_plan_bytes",
           "pcpp_build_triplets", "pcpp_mvmr_workspace_bytes", "pcpp_mvmr_fwd", "pcpp_mvmr_bwd_input",
           "pcpp_mvmr_bwd_weight", "pcpp_static_scratch_bytes", "pcpp_mvmr_fwd_static",
           "pcpp_build_triplets_batched", "pcpp_voxel_subsample_workspace_bytes", "pcpp_voxel_subsample",
           "pcpp_act_code_bytes", "pcpp_act_pack", "pcpp_act_unpack", "pcpp_mvmr_packed_workspace_bytes",
           "pcpp_mvmr_bwd_weight_packed", "pcpp_block_norm_fwd", "pcpp_block_norm_workspace_bytes", "pcpp_block_norm_bwd",
           "pcpp_log_probs_workspace_bytes", "pcpp_log_probs_fwd", "pcpp_log_probs_bwd",
           "pcpp_dropout_fwd", "pcpp_dropout_bwd", "pcpp_group_norm_workspace_bytes", "pcpp_group_norm_fwd", "pcpp_group_norm_bwd",
           "pcpp_mx_row_bytes", "pcpp_mx_scale_bytes", "pcpp_mx_pack", "pcpp_mx_unpack", "pcpp_mx_product_workspace_bytes",
           "pcpp_mx_product", "pcpp_mx_linear_workspace_bytes", "pcpp_mx_linear")


class PcppError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__(f"pcpp error {code}: {message}")
        self.code = code


_lib = None


def library() -> ctypes.CDLL:
    """Load libpcpp.so (building it first only if no built library exists).  Raises if unavailable."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        from .build import build
        build()
    L = ctypes.CDLL(LIB_PATH)
    i64, i32, f32, vp, sz = ctypes.c_int64, ctypes.c_int, ctypes.c_float, ctypes.c_void_p, ctypes.c_size_t
    L.pcpp_last_error.restype = ctypes.c_char_p
    L.pcpp_last_error.argtypes = []
    L.pcpp_version.restype = i32
    L.pcpp_build_triplets_workspace_bytes.restype = sz
    L.pcpp_build_triplets_workspace_bytes.argtypes = [i64, i64, i32]
    L.pcpp_build_triplets_workspace_bytes_for.restype = sz
    L.pcpp_build_triplets_workspace_bytes_for.argtypes = [i64, i64, i32, i64]
    L.pcpp_plan_bytes.restype = sz
    L.pcpp_plan_bytes.argtypes = [i64, i64, i32, i64, i32]
    L.pcpp_build_triplets.restype = i32
    L.pcpp_build_triplets.argtypes = [vp, i64, vp, i64, f32, i32, vp, vp, vp, i64, vp,
                                      ctypes.POINTER(i64), vp, sz, i32, vp, sz, vp]
    L.pcpp_build_triplets_batched.restype = i32
    L.pcpp_build_triplets_batched.argtypes = [vp, i64, vp, i64, vp, vp, i32, f32, i32, vp, vp, vp, i64, vp,
                                              ctypes.POINTER(i64), vp, sz, i32, vp, sz, vp]
    L.pcpp_voxel_subsample_workspace_bytes.restype = sz
    L.pcpp_voxel_subsample_workspace_bytes.argtypes = [i64]
    L.pcpp_voxel_subsample.restype = i32
    L.pcpp_voxel_subsample.argtypes = [vp, i64, f32, vp, ctypes.POINTER(i64), vp, sz, vp]
    L.pcpp_mvmr_workspace_bytes.restype = sz
    L.pcpp_mvmr_workspace_bytes.argtypes = [i32, i64, i64, i64, i32, i32, i32, i32]
    head = [i64, i64, i32, i32, i32, vp, vp, vp, vp, i64, vp, sz, i32]     # sizes, triplets, plan
    tail = head + [vp, sz, vp]                                             # workspace, stream
    L.pcpp_mvmr_fwd.restype = i32
    L.pcpp_mvmr_fwd.argtypes = [vp, vp, vp, i32, i32] + tail
    L.pcpp_mvmr_bwd_input.restype = i32
    L.pcpp_mvmr_bwd_input.argtypes = [vp, vp, vp, i32, i32] + tail
    L.pcpp_mvmr_bwd_weight.restype = i32
    L.pcpp_mvmr_bwd_weight.argtypes = [vp, vp, vp, i32] + tail
    L.pcpp_tune_workspace_bytes.restype = sz
    L.pcpp_tune_workspace_bytes.argtypes = [i64, i64, i32, i64, i32, i32, i32, i32]
    L.pcpp_tune_plan_order.restype = i32
    L.pcpp_tune_plan_order.argtypes = [vp, i64, vp, i64, f32, i32, i32, i64, i32, i32, i32, i32, vp, sz,
                                       ctypes.POINTER(i32), ctypes.POINTER(f32), ctypes.POINTER(f32), vp]
    L.pcpp_static_scratch_bytes.restype = sz
    L.pcpp_static_scratch_bytes.argtypes = []
    L.pcpp_mvmr_fwd_static.restype = i32
    L.pcpp_mvmr_fwd_static.argtypes = [vp, vp, vp, i32, i32] + head + [vp]
    L.pcpp_act_code_bytes.restype = sz
    L.pcpp_act_code_bytes.argtypes = [i32]
    L.pcpp_act_pack.restype = i32
    L.pcpp_act_pack.argtypes = [vp, i32, i64, i32, vp, vp, vp]
    L.pcpp_act_unpack.restype = i32
    L.pcpp_act_unpack.argtypes = [vp, vp, i64, i32, vp, i32, vp]
    L.pcpp_mvmr_packed_workspace_bytes.restype = sz
    L.pcpp_mvmr_packed_workspace_bytes.argtypes = [i64, i64, i64, i32, i32, i32, i32]
    L.pcpp_mvmr_bwd_weight_packed.restype = i32
    L.pcpp_mvmr_bwd_weight_packed.argtypes = [vp, vp, vp, vp, i32] + tail
    block = [vp, i64, i32, vp, vp, i32, i32, f32, f32, i64, i32, i32, i32]     # gate, weights, norms, sizes, types
    L.pcpp_block_norm_fwd.restype = i32
    L.pcpp_block_norm_fwd.argtypes = [vp, vp, i64] + block + [vp, vp, vp, vp, vp, vp, vp]
    L.pcpp_block_norm_workspace_bytes.restype = sz
    L.pcpp_block_norm_workspace_bytes.argtypes = [i64, i32]
    L.pcpp_block_norm_bwd.restype = i32
    L.pcpp_block_norm_bwd.argtypes = [vp, vp, vp, vp, i64, vp, vp] + block + [vp, vp, vp, vp, vp, vp, sz, vp]
    L.pcpp_log_probs_workspace_bytes.restype = sz
    L.pcpp_log_probs_workspace_bytes.argtypes = [i64, i64, i32]
    L.pcpp_log_probs_fwd.restype = i32
    L.pcpp_log_probs_fwd.argtypes = [vp, i32, i64, i64, i64, vp, i32, vp, vp, vp, vp, vp, vp, sz, vp]
    L.pcpp_log_probs_bwd.restype = i32
    L.pcpp_log_probs_bwd.argtypes = [vp, i32, i64, i64, i64, vp, vp, vp, vp, vp, vp, i64, vp]
    u32 = ctypes.c_uint32
    drop = [vp, u32, f32]                                                  # random state, site, p
    L.pcpp_dropout_fwd.restype = i32
    L.pcpp_dropout_fwd.argtypes = [vp, i64, vp] + drop + [i32, vp, i32, i64, i32, i32, i32, vp, vp]
    L.pcpp_dropout_bwd.restype = i32
    L.pcpp_dropout_bwd.argtypes = [vp] + drop + [i32, vp, i32, i64, i32, i32, i32, vp, vp]
    L.pcpp_group_norm_workspace_bytes.restype = sz
    L.pcpp_group_norm_workspace_bytes.argtypes = [i64, i32, i32, i32, i32]
    L.pcpp_group_norm_fwd.restype = i32
    L.pcpp_group_norm_fwd.argtypes = [vp, i64, vp, vp, vp, i32, i32, i32, f32] + drop + [i64, i32, i32, vp, vp, vp, sz, vp]
    L.pcpp_group_norm_bwd.restype = i32
    L.pcpp_group_norm_bwd.argtypes = [vp, vp, i64, vp, vp, vp, vp, i32, i32, i32] + drop + [i64, i32, i32, vp, vp, vp, vp, sz, vp]
    L.pcpp_mx_row_bytes.restype = sz
    L.pcpp_mx_row_bytes.argtypes = [i64]
    L.pcpp_mx_scale_bytes.restype = sz
    L.pcpp_mx_scale_bytes.argtypes = [i64]
    L.pcpp_mx_pack.restype = i32
    L.pcpp_mx_pack.argtypes = [vp, i64, i32, i64, i64, vp, u32, vp, vp, vp, vp, vp]
    L.pcpp_mx_unpack.restype = i32
    L.pcpp_mx_unpack.argtypes = [vp, vp, i64, i64, vp, i32, vp]
    L.pcpp_mx_product_workspace_bytes.restype = sz
    L.pcpp_mx_product_workspace_bytes.argtypes = [i64, i64, i64]
    L.pcpp_mx_product.restype = i32
    L.pcpp_mx_product.argtypes = [vp, vp, vp, vp, vp, i32, i64, i64, i64, vp, i32, vp, sz, vp]
    L.pcpp_mx_linear_workspace_bytes.restype = sz
    L.pcpp_mx_linear_workspace_bytes.argtypes = [i64, i64, i64]
    L.pcpp_mx_linear.restype = i32
    L.pcpp_mx_linear.argtypes = [vp, i64, i32, vp, vp, vp, i32, i64, i64, i64, vp, i32, vp, sz, vp]
    _lib = L
    return L


_landing = threading.local()


def _landing_word():
    """Pinned host word that the device writes a count into (one per host thread), as the pointer that the calls take; word[0] is
    the count."""
    word = getattr(_landing, "word", None)
    if word is None:
        _landing.memory = torch.zeros(8, dtype=torch.int64, pin_memory=True)
        word = _landing.word = ctypes.cast(_landing.memory.data_ptr(), ctypes.POINTER(ctypes.c_int64))
    return word


def _check(rc: int):
    if rc != 0:
        raise PcppError(rc, library().pcpp_last_error().decode())


def _capacity_error(capacity: int, needed: int) -> PcppError:
    # (made here: an exception held by the frame that raises it would keep that frame's tensors until a collection)
    err = PcppError(ERR_CAPACITY, f"capacity {capacity} too small, need {needed}")
    err.needed = needed
    return err


def _ptr(t):
    return ctypes.c_void_p(t.data_ptr()) if t is not None else None


def _stream() -> int:
    """The current device's current stream as the calls take it (0.2 us; by way of torch.cuda.current_stream() 3)."""
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return PCPP_F32
    if t.dtype == torch.bfloat16:
        return PCPP_BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def _bytes(n: int, device) -> torch.Tensor:
    return torch.empty(max(int(n), 256), dtype=torch.uint8, device=device)


def _room(given: torch.Tensor | None, n: int) -> bool:
    """Whether a caller's buffer has n bytes in one piece (an expanded tensor's numel() are not there)."""
    return given is not None and given.is_contiguous() and given.numel() >= n


def _written(*given: torch.Tensor | None):
    """Tensors of the caller's that a call has written: autograd is to refuse to go on with what it saved of them."""
    for t in given:
        if t is not None and not t.is_inference():
            torch.autograd.graph.increment_version(t)


@dataclass
class Triplets:
    """Result of pcpp_build_triplets: T in (k, o, i) order plus the plan the compute calls read."""
    tri_o: torch.Tensor
    tri_i: torch.Tensor
    tri_k: torch.Tensor
    seg_offsets: torch.Tensor
    n_triplets: int
    n_in: int
    n_out: int
    t: int
    plan: torch.Tensor
    plan_flags: int

    @property
    def K(self) -> int:
        return self.t ** 3


def pcpp_count_triplets(in_xyz: torch.Tensor, out_xyz: torch.Tensor, radius: float, t: int,
                        workspace: torch.Tensor | None = None) -> int:
    L = library()
    n_in, n_out = in_xyz.shape[0], out_xyz.shape[0]
    ws_bytes = L.pcpp_build_triplets_workspace_bytes(n_in, n_out, t)
    ws = workspace if _room(workspace, 0) else _bytes(ws_bytes, in_xyz.device)
    n = _landing_word()
    _check(L.pcpp_build_triplets(_ptr(in_xyz), n_in, _ptr(out_xyz), n_out, float(radius), int(t), None, None, None,
                                 0, None, n, None, 0, 0, _ptr(ws), ws.numel(), _stream()))
    return int(n[0])


def pcpp_build_triplets(in_xyz: torch.Tensor, out_xyz: torch.Tensor, radius: float, t: int,
                        plan_flags: int = PLAN_FWD | PLAN_BWD_INPUT, capacity: int | None = None,
                        buffers: dict | None = None, in_offsets: torch.Tensor | None = None,
                        out_offsets: torch.Tensor | None = None) -> Triplets:
    """Triplet construction (Sec. 3.2 with the fixed-radius search of Sec. 4.1) and reordering by (k, o, i).

    in_xyz [n_in,3], out_xyz [n_out,3]: contiguous float32 CUDA tensors.  Without `capacity` room for 48
    triplets per output point is provided; if that is too little the call reports the exact count and is
    repeated once with it (so the search runs once in the common case).  `buffers` may carry preallocated
    'tri_o','tri_i','tri_k','seg_offsets','plan','workspace' tensors to reuse.  plan_flags may include
    PLAN_SPATIAL (tiles follow a space-filling order; for wide layers), BUILD_VOXEL (the degraded, sparse-voxel
    operator of Sec. 3.2: `radius` is the voxel pitch) and the BUILD_TEST_* aids.  in_offsets / out_offsets: int32
    CUDA tensors [n_batches + 1] for a batch of clouds held as concatenated arrays (Sec. 4.1).
    """
    if capacity is None:
        guess = max(48 * int(out_xyz.shape[0]), 1024)
        try:
            return pcpp_build_triplets(in_xyz, out_xyz, radius, t, plan_flags, guess, buffers, in_offsets, out_offsets)
        except PcppError as e:
            if e.code != ERR_CAPACITY:
                raise
            needed = e.needed
        # outside the handler: the first attempt's buffers are free again
        return pcpp_build_triplets(in_xyz, out_xyz, radius, t, plan_flags, needed, buffers, in_offsets, out_offsets)
    L = library()
    assert in_xyz.is_cuda and out_xyz.is_cuda and in_xyz.dtype == torch.float32 and out_xyz.dtype == torch.float32
    assert in_xyz.is_contiguous() and out_xyz.is_contiguous()
    dev = in_xyz.device
    n_in, n_out = int(in_xyz.shape[0]), int(out_xyz.shape[0])
    K = t ** 3
    buffers = buffers or {}
    ws = buffers.get("workspace")
    cap = max(int(capacity), 1)
    # with room for the neighbour lists that all passes read
    ws_bytes = L.pcpp_build_triplets_workspace_bytes_for(n_in, n_out, t, cap)
    if ws_bytes == 0:
        raise PcppError(-1, "invalid sizes or t")
    if not _room(ws, ws_bytes):
        ws = _bytes(ws_bytes, dev)

    given = []

    def buf(name, numel, dtype):
        b = buffers.get(name)
        if not _room(b, numel) or b.dtype != dtype:
            b = torch.empty(numel, dtype=dtype, device=dev)
        else:
            given.append(b)
        return b

    tri_o, tri_i, tri_k = (buf(nm, cap, torch.int32) for nm in ("tri_o", "tri_i", "tri_k"))
    seg = buf("seg_offsets", K + 1, torch.int64)
    want_plan = bool(plan_flags & PLAN_MASK)
    plan_bytes = L.pcpp_plan_bytes(n_in, n_out, t, cap, plan_flags & PLAN_MASK) if want_plan else 0
    plan = buffers.get("plan")
    if want_plan and not _room(plan, plan_bytes):
        plan = _bytes(plan_bytes, dev)
    n = _landing_word()
    n_batches = 1
    if in_offsets is not None or out_offsets is not None:
        assert in_offsets is not None and out_offsets is not None and in_offsets.is_cuda and out_offsets.is_cuda
        assert in_offsets.dtype == torch.int32 and out_offsets.dtype == torch.int32
        assert in_offsets.numel() == out_offsets.numel() >= 2
        n_batches = in_offsets.numel() - 1
    rc = L.pcpp_build_triplets_batched(_ptr(in_xyz), n_in, _ptr(out_xyz), n_out, _ptr(in_offsets), _ptr(out_offsets),
                                       n_batches, float(radius), int(t),
                                       _ptr(tri_o), _ptr(tri_i), _ptr(tri_k), cap, _ptr(seg), n,
                                       _ptr(plan) if want_plan else None, plan.numel() if want_plan else 0, plan_flags,
                                       _ptr(ws), ws.numel(), _stream())
    nt = int(n[0])
    _written(*given)
    if rc == ERR_CAPACITY:
        raise _capacity_error(cap, nt)
    _check(rc)
    return Triplets(tri_o[:nt], tri_i[:nt], tri_k[:nt], seg[:K + 1], nt, n_in, n_out, t, plan, plan_flags & PLAN_MASK)


def pcpp_voxel_subsample(xyz: torch.Tensor, pitch: float) -> torch.Tensor:
    """Voxel-grid down-sampling that keeps original coordinates (Sec. 4.1): indices (ascending, int32) of the
    lowest-index point of every occupied voxel of the given pitch."""
    L = library()
    assert xyz.is_cuda and xyz.is_contiguous() and xyz.dtype == torch.float32
    n = int(xyz.shape[0])
    kept = torch.empty(max(n, 1), dtype=torch.int32, device=xyz.device)
    ws = _bytes(L.pcpp_voxel_subsample_workspace_bytes(n), xyz.device)
    cnt = _landing_word()
    _check(L.pcpp_voxel_subsample(_ptr(xyz), n, float(pitch), _ptr(kept), cnt, _ptr(ws), ws.numel(), _stream()))
    return kept[:int(cnt[0])]


def pcpp_tune_plan_order(in_xyz: torch.Tensor, out_xyz: torch.Tensor, radius: float, t: int, n_triplets: int,
                         c_in: int, c_out: int, dtype: torch.dtype, ops: int = PLAN_FWD | PLAN_BWD_INPUT,
                         build_flags: int = 0) -> tuple[int, float, float]:
    """The plan order (Sec. 3.3.2, closing remark on auto-tuning) that runs this layer faster on this cloud:
    returns (plan flags to build with, ms per pass in index order, ms per pass in spatial order)."""
    L = library()
    assert in_xyz.is_cuda and in_xyz.is_contiguous() and out_xyz.is_contiguous() and in_xyz.dtype == torch.float32
    n_in, n_out = int(in_xyz.shape[0]), int(out_xyz.shape[0])
    code = 1 if dtype == torch.bfloat16 else 0
    ws = _bytes(L.pcpp_tune_workspace_bytes(n_in, n_out, t, n_triplets, c_in, c_out, code, ops), in_xyz.device)
    best, ms_a, ms_b = ctypes.c_int32(0), ctypes.c_float(0), ctypes.c_float(0)
    _check(L.pcpp_tune_plan_order(_ptr(in_xyz), n_in, _ptr(out_xyz), n_out, float(radius), t, build_flags, n_triplets,
                                  c_in, c_out, code, ops, _ptr(ws), ws.numel(), ctypes.byref(best), ctypes.byref(ms_a),
                                  ctypes.byref(ms_b), _stream()))
    return int(best.value), float(ms_a.value), float(ms_b.value)


def _plan_args(T: Triplets):
    if T.plan is None:
        return None, 0, T.plan_flags
    return _ptr(T.plan), T.plan.numel(), T.plan_flags


def _mvmr_ws(op, T: Triplets, c_in, c_out, code, dev, workspace):
    need = library().pcpp_mvmr_workspace_bytes(op, T.n_in, T.n_out, T.n_triplets, c_in, c_out, T.K, code)
    if not _room(workspace, need):
        workspace = _bytes(need, dev)
    return workspace


def pcpp_mvmr_fwd(x: torch.Tensor, w: torch.Tensor, T: Triplets, out: torch.Tensor | None = None,
                  out_dtype: torch.dtype = torch.float32, workspace: torch.Tensor | None = None) -> torch.Tensor:
    """Eq. (1): out[o] = sum_{(o,i,k) in T} W[k] x[i];  x [n_in,c_in], w [K,c_out,c_in] -> out [n_out,c_out]."""
    L = library()
    assert x.is_cuda and x.is_contiguous() and w.is_contiguous() and x.dtype == w.dtype
    K, c_out, c_in = w.shape
    assert K == T.K and x.shape == (T.n_in, c_in)
    given = out
    if out is None:
        out = torch.empty((T.n_out, c_out), dtype=out_dtype, device=x.device)
    ws = _mvmr_ws(0, T, c_in, c_out, _dtype_code(x), x.device, workspace)
    _check(L.pcpp_mvmr_fwd(_ptr(x), _ptr(w), _ptr(out), _dtype_code(x), _dtype_code(out), T.n_in, T.n_out, c_in, c_out,
                           K, _ptr(T.tri_o), _ptr(T.tri_i), _ptr(T.tri_k), _ptr(T.seg_offsets), T.n_triplets,
                           *_plan_args(T), _ptr(ws), ws.numel(), _stream()))
    _written(given)
    return out


def pcpp_mvmr_fwd_static(x: torch.Tensor, w: torch.Tensor, T: Triplets, out: torch.Tensor,
                         out_dtype: torch.dtype = torch.float32) -> torch.Tensor:
    """pcpp_mvmr_fwd without a workspace: the packed weights go to the library's own device array, and the call
    allocates nothing (`out` must be given)."""
    L = library()
    assert x.is_cuda and x.is_contiguous() and w.is_contiguous() and x.dtype == w.dtype
    K, c_out, c_in = w.shape
    assert K == T.K and x.shape == (T.n_in, c_in) and out.shape == (T.n_out, c_out)
    _check(L.pcpp_mvmr_fwd_static(_ptr(x), _ptr(w), _ptr(out), _dtype_code(x), _dtype_code(out), T.n_in, T.n_out, c_in,
                                  c_out, K, _ptr(T.tri_o), _ptr(T.tri_i), _ptr(T.tri_k), _ptr(T.seg_offsets),
                                  T.n_triplets, *_plan_args(T), _stream()))
    _written(out)
    return out


def pcpp_mvmr_bwd_input(dy: torch.Tensor, w: torch.Tensor, T: Triplets, dx: torch.Tensor | None = None,
                        out_dtype: torch.dtype = torch.float32, workspace: torch.Tensor | None = None) -> torch.Tensor:
    """Sec. 3.3.3: dx[i] = sum_{(o,i,k) in T} W[k]^T dy[o];  dy [n_out,c_out] -> dx [n_in,c_in]."""
    L = library()
    assert dy.is_cuda and dy.is_contiguous() and w.is_contiguous() and dy.dtype == w.dtype
    K, c_out, c_in = w.shape
    assert K == T.K and dy.shape == (T.n_out, c_out)
    if not (T.plan_flags & PLAN_BWD_INPUT):
        raise PcppError(-1, "triplets were built without PLAN_BWD_INPUT")
    given = dx
    if dx is None:
        dx = torch.empty((T.n_in, c_in), dtype=out_dtype, device=dy.device)
    ws = _mvmr_ws(1, T, c_in, c_out, _dtype_code(dy), dy.device, workspace)
    _check(L.pcpp_mvmr_bwd_input(_ptr(dy), _ptr(w), _ptr(dx), _dtype_code(dy), _dtype_code(dx), T.n_in, T.n_out, c_in,
                                 c_out, K, _ptr(T.tri_o), _ptr(T.tri_i), _ptr(T.tri_k), _ptr(T.seg_offsets),
                                 T.n_triplets, *_plan_args(T), _ptr(ws), ws.numel(), _stream()))
    _written(given)
    return dx


def pcpp_mvmr_bwd_weight(x: torch.Tensor, dy: torch.Tensor, T: Triplets, dw: torch.Tensor | None = None,
                         workspace: torch.Tensor | None = None) -> torch.Tensor:
    """Eq. (5): dW[k] = sum_{(o,i,k) in T} dy[o] (outer) x[i] -> float32 [K,c_out,c_in]."""
    L = library()
    assert x.is_cuda and x.is_contiguous() and dy.is_contiguous() and x.dtype == dy.dtype
    c_in, c_out = x.shape[1], dy.shape[1]
    assert x.shape[0] == T.n_in and dy.shape[0] == T.n_out
    given = dw
    if dw is None:
        dw = torch.empty((T.K, c_out, c_in), dtype=torch.float32, device=x.device)
    ws = _mvmr_ws(2, T, c_in, c_out, _dtype_code(x), x.device, workspace)
    _check(L.pcpp_mvmr_bwd_weight(_ptr(x), _ptr(dy), _ptr(dw), _dtype_code(x), T.n_in, T.n_out, c_in, c_out, T.K,
                                  _ptr(T.tri_o), _ptr(T.tri_i), _ptr(T.tri_k), _ptr(T.seg_offsets), T.n_triplets,
                                  *_plan_args(T), _ptr(ws), ws.numel(), _stream()))
    _written(given)
    return dw


# ---- the operators around the convolution ------------------------------------------------------------------------
# Their smallest calls take the GPU 3 us, so tensors are checked, outputs made and the library called by compiled code
# (csrc/torch_calls.cpp); what does not fit raises AssertionError or TypeError there, and a call's status PcppError here.

_calls = None


def _compiled():
    """The compiled side of the calls, bound to the library (built first only if there is none for this Python and torch).  Raises if
    unavailable."""
    global _calls
    if _calls is None:
        from .build import build_calls, calls_lib
        handle = library()._handle
        path = calls_lib()
        if not os.path.exists(path):
            build_calls()
        spec = importlib.util.spec_from_file_location("_torch_calls", path)
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
        module.bind(handle)
        _calls = module
    return _calls


def _where():
    """The current device and its stream."""
    device = torch._C._cuda_getDevice()
    return device, torch._C._cuda_getCurrentRawStream(device)


def _outputs(result):
    """A call's outputs, or its error."""
    if type(result) is int:
        _check(result)
    return result


_CODES = {torch.float32: PCPP_F32, torch.bfloat16: PCPP_BF16}


def _code_or(dtype: torch.dtype | None) -> int:
    if dtype is None:
        return -1
    code = _CODES.get(dtype)
    if code is None:
        raise TypeError(f"unsupported dtype {dtype}")
    return code


@dataclass
class Packed:
    """Rows in 8 bits: values q * 2^(code - 127), one code for 32 channels (255: not finite)."""
    q: torch.Tensor          # int8 [n, c]
    codes: torch.Tensor      # uint8 [n, pcpp_act_code_bytes(c)]


def pcpp_act_pack(x: torch.Tensor, out: Packed | None = None) -> Packed:
    """Activations in 8 bits for a later backward pass: blocks of 32 channels of a row share a power of two."""
    q, codes = (None, None) if out is None else (out.q, out.codes)
    return Packed(*_outputs(_compiled().act_pack(x, q, codes, *_where())))


def pcpp_act_unpack(p: Packed, dtype: torch.dtype = torch.bfloat16, out: torch.Tensor | None = None) -> torch.Tensor:
    """The values of rows in 8 bits; bfloat16 holds them exactly."""
    return _outputs(_compiled().act_unpack(p.q, p.codes, _code_or(dtype), out, *_where()))[0]


def pcpp_mvmr_bwd_weight_packed(x: Packed, dy: torch.Tensor, T: Triplets, dw: torch.Tensor | None = None,
                                workspace: torch.Tensor | None = None) -> torch.Tensor:
    """pcpp_mvmr_bwd_weight from an input that was kept in 8 bits: dW[k] = sum dy[o] (outer) x[i].  T.plan may be None unless x in dy's
    type, dy or the triplets' indices take 4 GiB."""
    return _outputs(_compiled().weight_packed(x.q, x.codes, dy, T.tri_o, T.tri_i, T.tri_k, T.seg_offsets, T.plan, T.plan_flags,
                                              T.n_triplets, T.n_in, T.n_out, T.K, dw, workspace, *_where()))[0]


@dataclass
class BlockNorm:
    """Result of pcpp_block_norm_fwd: the residual stream behind the block, the next block's input, 8-bit copies."""
    r: torch.Tensor | None
    h: torch.Tensor | None
    f_packed: Packed | None = None
    h_packed: Packed | None = None


@dataclass
class BlockNormGrads:
    """Result of pcpp_block_norm_bwd; what does not apply is None."""
    dx: torch.Tensor
    df: torch.Tensor | None
    dgate: torch.Tensor | None
    dw_post: torch.Tensor | None
    dw_pre: torch.Tensor | None


def pcpp_block_norm_fwd(x: torch.Tensor, f: torch.Tensor | None = None, gate: torch.Tensor | None = None,
                        w_post: torch.Tensor | None = None, w_pre: torch.Tensor | None = None, *,
                        post_norm: int = NORM_RMS, pre_norm: int = NORM_RMS, residual_scale: float = 1.0,
                        eps: float = 1e-6, dtype: torch.dtype | None = None, pack_f: bool = False,
                        pack_h: bool = False) -> BlockNorm:
    """Between two blocks: r = residual_scale x + sigmoid(gate) w_post norm(f),  h = w_pre norm(r).

    x [n, c]: the residual stream, f [n, c]: the block's output (None: r is x, only h is formed), gate [n, c] or [n, 1]:
    logits; f and gate may be column slices.  post_norm / pre_norm: NORM_NONE, NORM_RMS or NORM_LAYER (pre_norm
    NORM_NONE: no h).  dtype: type of h where there is no f.  pack_f, pack_h: copies in 8 bits for the backward pass.
    """
    r, h, fq, fe, hq, he = _outputs(_compiled().block_norm_fwd(x, f, gate, w_post, w_pre, post_norm, pre_norm, residual_scale, eps,
                                                               _code_or(dtype), pack_f, pack_h, *_where()))
    return BlockNorm(x if f is None else r, h, Packed(fq, fe) if pack_f else None, Packed(hq, he) if pack_h else None)


def pcpp_block_norm_bwd(dr: torch.Tensor | None, dh: torch.Tensor | None, r: torch.Tensor | None,
                        f: torch.Tensor | Packed | None = None, gate: torch.Tensor | None = None,
                        w_post: torch.Tensor | None = None, w_pre: torch.Tensor | None = None, *,
                        post_norm: int = NORM_RMS, pre_norm: int = NORM_RMS, residual_scale: float = 1.0,
                        eps: float = 1e-6, dtype: torch.dtype | None = None, block: bool | None = None,
                        workspace: torch.Tensor | None = None) -> BlockNormGrads:
    """Gradients of pcpp_block_norm_fwd.  dr (None: zero) and dh flow to its r and h; r is what it wrote, f what it was
    given or its copy in 8 bits.  `block`: there was a block, though nothing of f is needed (neither post norm nor gate;
    default: f is not None).  dtype: type of the block's tensors where neither dh nor f says it."""
    fq = fe = None
    if block is None:
        block = f is not None
    if isinstance(f, Packed):
        f, fq, fe = None, f.q, f.codes
    return BlockNormGrads(*_outputs(_compiled().block_norm_bwd(dr, dh, r, f, fq, fe, gate, w_post, w_pre, post_norm, pre_norm,
                                                               residual_scale, eps, _code_or(dtype), block, workspace,
                                                               *_where())))


class LogProbs:
    """Result of pcpp_log_probs_fwd, fp32 [n]; max_log_sum [n, 2]: the row's maximum and the logarithm of its sum of exp(x - maximum);
    top_* [n, n_top], the most probable classes in descending order."""
    __slots__ = ("log_prob", "entropy", "max_log_sum", "_top_log_prob", "_top_index")

    def __init__(self, log_prob, entropy, max_log_sum, top_log_prob=None, top_index=None):
        self.log_prob, self.entropy, self.max_log_sum = log_prob, entropy, max_log_sum
        self._top_log_prob, self._top_index = top_log_prob, top_index

    @property
    def lse(self) -> torch.Tensor:
        return self.max_log_sum.sum(1)

    # (without alternatives the empty tensors are made when they are asked for: a training step never does)
    @property
    def top_log_prob(self) -> torch.Tensor:
        return self.entropy.new_empty((self.entropy.shape[0], 0)) if self._top_log_prob is None else self._top_log_prob

    @property
    def top_index(self) -> torch.Tensor:
        return self.entropy.new_empty((self.entropy.shape[0], 0), dtype=torch.int32) if self._top_index is None else self._top_index


def pcpp_log_probs_fwd(logits: torch.Tensor, labels: torch.Tensor | None = None, n_top: int = 0,
                       workspace: torch.Tensor | None = None) -> LogProbs:
    """Log probability of every row's label (a label outside 0 .. v - 1: none, 0), the entropy, and the n_top most probable
    classes.  logits [n, v], rows may be a slice of wider ones; labels int32 [n]."""
    return LogProbs(*_outputs(_compiled().log_probs_fwd(logits, labels, n_top, workspace, *_where())))


def pcpp_log_probs_bwd(logits: torch.Tensor, labels: torch.Tensor | None, forward: LogProbs,
                       d_log_prob: torch.Tensor | None = None, d_entropy: torch.Tensor | None = None,
                       out: torch.Tensor | None = None) -> torch.Tensor:
    """Gradient of the logits from what flows to log_prob and to entropy (fp32 [n]).  out: where it goes, by default a new
    tensor; it may be the logits."""
    return _outputs(_compiled().log_probs_bwd(logits, labels, forward.max_log_sum, forward.entropy, d_log_prob, d_entropy, out,
                                              *_where()))[0]


# ---- the pointwise layers ----------------------------------------------------------------------------------------

@dataclass
class Random:
    """Where an operator's random numbers come from: a program's state, int64 [2] on the GPU (seed, step), read when the kernel runs, and
    the operator's own number among those that draw from it.  The same state, site and shape draw the same numbers."""
    state: torch.Tensor
    site: int = 0


def _draws(random: Random | None):
    return (None, 0) if random is None else (random.state, random.site)


def pcpp_dropout_fwd(x: torch.Tensor, p: float, random: Random, residual: torch.Tensor | None = None, *, scope: int = DROP_ELEMENTS,
                     offsets: torch.Tensor | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
    """residual + dropout(x): elements (DROP_ELEMENTS), whole rows (DROP_ROWS) or whole clouds (DROP_CLOUDS, with the batch's
    offsets, int32 [clouds + 1]) go with probability p, in steps of 2^-16, and what stays is scaled up.  x [n, c] may be a
    slice of wider rows; the residual (x's type or float32) and out are contiguous.  No mask is kept: the backward pass draws it again."""
    return _outputs(_compiled().dropout_fwd(x, residual, *_draws(random), p, scope, offsets, out, *_where()))[0]


def pcpp_dropout_bwd(dy: torch.Tensor, p: float, random: Random, *, scope: int = DROP_ELEMENTS, offsets: torch.Tensor | None = None,
                     dtype: torch.dtype | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
    """Gradient of x (of type `dtype`, default dy's); the residual's is dy itself."""
    return _outputs(_compiled().dropout_bwd(dy, *_draws(random), p, scope, offsets, _code_or(dtype), out, *_where()))[0]


@dataclass
class GroupNorm:
    """Result of pcpp_group_norm_fwd; mean_rstd float32 [clouds, groups, 2] is what the backward pass needs of it."""
    y: torch.Tensor
    mean_rstd: torch.Tensor | None


@dataclass
class GroupNormGrads:
    """Result of pcpp_group_norm_bwd; what is not wanted is None."""
    dx: torch.Tensor | None
    dw: torch.Tensor | None
    db: torch.Tensor | None


def pcpp_group_norm_fwd(x: torch.Tensor, groups: int, w: torch.Tensor | None = None, b: torch.Tensor | None = None,
                        offsets: torch.Tensor | None = None, *, act: int = ACT_NONE, eps: float = 1e-5, p: float = 0.0,
                        random: Random | None = None, statistics: bool = True, out: torch.Tensor | None = None,
                        workspace: torch.Tensor | None = None) -> GroupNorm:
    """y = dropout(act(w v + b)), v: x [n, c] normalised over the rows of each cloud (offsets int32 [clouds + 1]; None: one cloud) and
    the neighbouring channels of each group.  x may be a slice of wider rows.  statistics = False: an answer only.  Rows that belong to
    no cloud are not written."""
    return GroupNorm(*_outputs(_compiled().group_norm_fwd(x, groups, w, b, offsets, act, eps, *_draws(random), p, statistics, out,
                                                          workspace, *_where())))


def pcpp_group_norm_bwd(dy: torch.Tensor, x: torch.Tensor, mean_rstd: torch.Tensor, w: torch.Tensor | None = None,
                        b: torch.Tensor | None = None, offsets: torch.Tensor | None = None, *, act: int = ACT_NONE, p: float = 0.0,
                        random: Random | None = None, of_x: bool = True, of_weights: bool = True,
                        workspace: torch.Tensor | None = None) -> GroupNormGrads:
    """Gradients of pcpp_group_norm_fwd from what flows to y; the arguments are the forward pass's, mean_rstd what it returned."""
    return GroupNormGrads(*_outputs(_compiled().group_norm_bwd(dy, x, mean_rstd, w, b, offsets, act, *_draws(random), p, of_x, of_weights,
                                                               workspace, *_where())))


@dataclass
class MxRows:
    """Rows in microscaled 4-bit floating point: two elements a byte, a power of two for 32 channels."""
    q: torch.Tensor          # uint8 [n, pcpp_mx_row_bytes(c)]
    scales: torch.Tensor     # uint8 [n, pcpp_mx_scale_bytes(c)]
    c: int


@dataclass
class Mx:
    """Result of pcpp_mx_pack: the rows of x [n, c], and its columns as c rows of n elements; what is not wanted is None."""
    rows: MxRows | None
    columns: MxRows | None


def pcpp_mx_pack(x: torch.Tensor, *, rows: bool = True, columns: bool = False, random: Random | None = None) -> Mx:
    """x [n, c] in 4 bits, to nearest, or at random (unbiased) with `random`.  A product sums over what shares a power of two: rows
    for y = x W^T and dx = dy W, columns for dW = dy^T x.  Both at once read x once."""
    q, s, qt, st = _outputs(_compiled().mx_pack(x, rows, columns, *_draws(random), *_where()))
    return Mx(MxRows(q, s, x.shape[1]) if rows else None, MxRows(qt, st, x.shape[0]) if columns else None)


def pcpp_mx_unpack(m: MxRows, dtype: torch.dtype = torch.bfloat16, out: torch.Tensor | None = None) -> torch.Tensor:
    """The values of rows in 4 bits; bfloat16 holds them exactly."""
    return _outputs(_compiled().mx_unpack(m.q, m.scales, m.c, _code_or(dtype), out, *_where()))[0]


def pcpp_mx_product(a: MxRows, b: MxRows, bias: torch.Tensor | None = None, *, act: int = ACT_NONE, dtype: torch.dtype = torch.bfloat16,
                    out: torch.Tensor | None = None, workspace: torch.Tensor | None = None) -> torch.Tensor:
    """act(a b^T + bias): every row of a with every row of b, summed in fp32, bias float32 [rows of b].  Columns of a batch without rows
    are rows of no elements: act(bias), so zeros for its weights' gradient."""
    return _outputs(_compiled().mx_product(a.q, a.scales, a.c, b.q, b.scales, b.c, bias, act, _code_or(dtype), out, workspace, *_where()))[0]


def pcpp_mx_linear(x: torch.Tensor, w: MxRows, bias: torch.Tensor | None = None, *, act: int = ACT_NONE, dtype: torch.dtype | None = None,
                   out: torch.Tensor | None = None, workspace: torch.Tensor | None = None) -> torch.Tensor:
    """act(x w^T + bias) with x [n, k] rounded to 4 bits on the way, as pcpp_mx_pack does to nearest.  dtype: the result's, default x's."""
    return _outputs(_compiled().mx_linear(x, w.q, w.scales, w.c, bias, act, _code_or(dtype), out, workspace, *_where()))[0]
