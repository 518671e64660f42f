"""ctypes binding of libprunedctc: argument marshalling only.

Every step of the computation runs in the library's CUDA kernels; torch is
used for device memory and the current stream.  There is no CPU path: calls
raise if the library is missing or returns an error status.
"""

from __future__ import annotations

import ctypes
import os
from typing import Optional

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libprunedctc.so")

PCTC_BF16, PCTC_FP32 = 0, 1
GEMM_AUTO, GEMM_SIMT = 0, 1
UTT_INFEASIBLE, UTT_NONFINITE, UTT_BAD_TARGET, UTT_SUBSET_OVERFLOW, UTT_STATE_FULL = 1, 2, 4, 8, 16

EXPORTS = ("pctc_workspace_bytes", "pctc_chunk_width", "pruned_ctc_fwd_bwd", "pruned_ctc_fwd_bwd_traced", "pctc_gemm_bf16",
           "pctc_workspace_status", "pctc_status_string", "pctc_host_call_scratch_bytes",
           "pruned_ctc_fwd_bwd_host", "pctc_subset_relabel_noalloc", "pctc_greedy_workspace_bytes",
           "pctc_greedy_decode", "pctc_topk_workspace_bytes", "pctc_topk_decode",
           "pctc_clip_workspace_bytes", "pctc_clip_grad_norm", "pctc_grad_sqsum", "pctc_grad_scale",
           "pctc_prefix_state_bytes", "pctc_prefix_advance", "pctc_prefix_read",
           "pctc_prefix_decode", "pctc_beam_workspace_bytes", "pctc_beam_select",
           "pctc_beam_reorder")
NOALLOC_MAX_V = 262144

PHASES = ("prep", "lse", "subset_logp", "dp", "dlogits", "dh", "dw", "dbias", "finish")


class Problem(ctypes.Structure):
    _fields_ = [
        ("N", ctypes.c_int32), ("T", ctypes.c_int32), ("D", ctypes.c_int32),
        ("V", ctypes.c_int64),
        ("dtype", ctypes.c_int32), ("blank_id", ctypes.c_int32),
        ("beam", ctypes.c_float),
        ("chunk", ctypes.c_int32), ("target_stride", ctypes.c_int32), ("gemm_path", ctypes.c_int32),
        ("skip_dW", ctypes.c_int32), ("accumulate_dW", ctypes.c_int32), ("forward_only", ctypes.c_int32),
        ("max_K", ctypes.c_int32),
        ("utt_weights", ctypes.c_void_p),
    ]


class PrefixProblem(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int32) for name in ("N", "T", "k", "beams", "blank_id", "max_frames")]


class BeamProblem(ctypes.Structure):
    _fields_ = [("N", ctypes.c_int32), ("B", ctypes.c_int32), ("K", ctypes.c_int32), ("V", ctypes.c_int64),
                ("stride_n", ctypes.c_int64), ("stride_b", ctypes.c_int64), ("dtype", ctypes.c_int32),
                ("eos_id", ctypes.c_int32)]


class BeamState(ctypes.Structure):
    _fields_ = [("src", ctypes.c_void_p), ("dst", ctypes.c_void_p),
                ("src_stride_n", ctypes.c_int64), ("src_stride_b", ctypes.c_int64),
                ("dst_stride_n", ctypes.c_int64), ("dst_stride_b", ctypes.c_int64),
                ("segments", ctypes.c_int64), ("segment_stride", ctypes.c_int64),
                ("units", ctypes.c_int64), ("unit_bytes", ctypes.c_int64),
                ("timed", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class TraceStruct(ctypes.Structure):
    _fields_ = [("events", ctypes.POINTER(ctypes.c_void_p)), ("capacity", ctypes.c_int32),
                ("used", ctypes.c_int32), ("kinds", ctypes.POINTER(ctypes.c_int32))]


class Trace:
    """Caller-owned CUDA events for pruned_ctc_fwd_bwd_traced (one timeline per call)."""

    def __init__(self, capacity: int):
        import torch

        self.capacity = int(capacity)
        self.events = [torch.cuda.Event(enable_timing=True) for _ in range(self.capacity)]
        for e in self.events:          # torch creates the CUDA event at its first record
            e.record()
        torch.cuda.synchronize()
        self._handles = (ctypes.c_void_p * self.capacity)(*[int(e.cuda_event) for e in self.events])
        self._kinds = (ctypes.c_int32 * self.capacity)()
        self.struct = TraceStruct(ctypes.cast(self._handles, ctypes.POINTER(ctypes.c_void_p)), self.capacity, 0,
                                  ctypes.cast(self._kinds, ctypes.POINTER(ctypes.c_int32)))

    def spans(self):
        """[(phase index, milliseconds)] of the last call; synchronise the stream first."""
        n = self.struct.used
        return [(int(self._kinds[i]), self.events[i].elapsed_time(self.events[i + 1])) for i in range(n - 1)]

    @staticmethod
    def capacity_for(V: int, chunk: int) -> int:
        return 12 + 4 * ((V + chunk - 1) // chunk)


class PctcError(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__(f"{what}: status {status} ({status_string(status)})")
        self.status = status


_lib = None


def load() -> ctypes.CDLL:
    """Load the shared library (no build here; see build.build())."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: run paper_2609_33645_b200.build.build() first; "
                           "there is no fallback implementation")
    _lib = _configure(ctypes.CDLL(LIB_PATH))
    return _lib


def load_variant(path: str) -> ctypes.CDLL:
    """A test variant of the library (build.build_variant), loaded beside the regular one: call its
    entry points directly, e.g. ``gemm_bf16(..., lib=load_variant(path))``."""
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: run paper_2609_33645_b200.build.build_variant() first")
    return _configure(ctypes.CDLL(path))


def _configure(lib: ctypes.CDLL) -> ctypes.CDLL:
    vp, i32p = ctypes.c_void_p, ctypes.POINTER(ctypes.c_int32)
    lib.pctc_workspace_bytes.restype = ctypes.c_int
    lib.pctc_workspace_bytes.argtypes = [ctypes.POINTER(Problem), i32p, i32p, ctypes.POINTER(ctypes.c_size_t)]
    lib.pctc_chunk_width.restype = ctypes.c_int
    lib.pctc_chunk_width.argtypes = [ctypes.POINTER(Problem), i32p, i32p, i32p, i32p]
    lib.pruned_ctc_fwd_bwd.restype = ctypes.c_int
    lib.pruned_ctc_fwd_bwd.argtypes = [ctypes.POINTER(Problem), vp, vp, vp, vp, i32p, i32p,
                                       vp, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.pruned_ctc_fwd_bwd_traced.restype = ctypes.c_int
    lib.pruned_ctc_fwd_bwd_traced.argtypes = lib.pruned_ctc_fwd_bwd.argtypes + [ctypes.POINTER(TraceStruct)]
    lib.pruned_ctc_fwd_bwd_host.restype = ctypes.c_int
    lib.pruned_ctc_fwd_bwd_host.argtypes = lib.pruned_ctc_fwd_bwd.argtypes
    lib.pctc_host_call_scratch_bytes.restype = ctypes.c_int
    lib.pctc_host_call_scratch_bytes.argtypes = [ctypes.POINTER(Problem), i32p, i32p, ctypes.c_int32,
                                                 ctypes.POINTER(ctypes.c_size_t)]
    lib.pctc_subset_relabel_noalloc.restype = ctypes.c_int
    lib.pctc_subset_relabel_noalloc.argtypes = [vp, vp, ctypes.c_int32, ctypes.c_int32, ctypes.c_int64,
                                                ctypes.c_int32, vp, vp, vp, vp, vp]
    lib.pctc_greedy_workspace_bytes.restype = ctypes.c_int
    lib.pctc_greedy_workspace_bytes.argtypes = [ctypes.POINTER(Problem), i32p, ctypes.POINTER(ctypes.c_size_t)]
    lib.pctc_greedy_decode.restype = ctypes.c_int
    lib.pctc_greedy_decode.argtypes = [ctypes.POINTER(Problem), vp, vp, vp, i32p, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.pctc_topk_workspace_bytes.restype = ctypes.c_int
    lib.pctc_topk_workspace_bytes.argtypes = [ctypes.POINTER(Problem), i32p, ctypes.c_int32,
                                              ctypes.POINTER(ctypes.c_size_t)]
    lib.pctc_topk_decode.restype = ctypes.c_int
    lib.pctc_topk_decode.argtypes = [ctypes.POINTER(Problem), vp, vp, vp, i32p, ctypes.c_int32, vp, vp, vp,
                                     ctypes.c_size_t, vp]
    i64p, vpp, size_p = ctypes.POINTER(ctypes.c_int64), ctypes.POINTER(vp), ctypes.POINTER(ctypes.c_size_t)
    lib.pctc_clip_workspace_bytes.restype = ctypes.c_int
    lib.pctc_clip_workspace_bytes.argtypes = [ctypes.c_int32, size_p]
    lib.pctc_clip_grad_norm.restype = ctypes.c_int
    lib.pctc_clip_grad_norm.argtypes = [ctypes.c_int32, vpp, vpp, i64p, i32p, i32p, ctypes.c_float, ctypes.c_float,
                                        vp, vp, ctypes.c_size_t, vp]
    lib.pctc_grad_sqsum.restype = ctypes.c_int
    lib.pctc_grad_sqsum.argtypes = [ctypes.c_int32, vpp, i64p, i32p, vp, vp, ctypes.c_size_t, vp]
    lib.pctc_grad_scale.restype = ctypes.c_int
    lib.pctc_grad_scale.argtypes = [ctypes.c_int32, vpp, vpp, i64p, i32p, i32p, vp, ctypes.c_float, ctypes.c_float,
                                    vp, vp]
    prefix_p = ctypes.POINTER(PrefixProblem)
    lib.pctc_prefix_state_bytes.restype = ctypes.c_int
    lib.pctc_prefix_state_bytes.argtypes = [prefix_p, size_p]
    lib.pctc_prefix_advance.restype = ctypes.c_int
    lib.pctc_prefix_advance.argtypes = [prefix_p, vp, vp, i32p, ctypes.c_int32, vp, ctypes.c_size_t, vp]
    lib.pctc_prefix_read.restype = ctypes.c_int
    lib.pctc_prefix_read.argtypes = [prefix_p, vp, ctypes.c_size_t, vp, ctypes.c_int32, vp, vp, vp, vp]
    lib.pctc_prefix_decode.restype = ctypes.c_int
    lib.pctc_prefix_decode.argtypes = [prefix_p, vp, vp, i32p, vp, ctypes.c_size_t, vp, ctypes.c_int32, vp, vp, vp, vp]
    lib.pctc_beam_select.restype = ctypes.c_int
    lib.pctc_beam_select.argtypes = [ctypes.POINTER(BeamProblem)] + [vp] * 9 + [ctypes.c_size_t, vp]
    lib.pctc_beam_workspace_bytes.restype = ctypes.c_int
    lib.pctc_beam_workspace_bytes.argtypes = [ctypes.POINTER(BeamProblem), size_p]
    lib.pctc_beam_reorder.restype = ctypes.c_int
    lib.pctc_beam_reorder.argtypes = [ctypes.c_int32, ctypes.POINTER(BeamState), ctypes.c_int32, ctypes.c_int32,
                                      ctypes.c_int32, vp, vp, vp]
    lib.pctc_gemm_bf16.restype = ctypes.c_int
    lib.pctc_gemm_bf16.argtypes = [vp, vp, vp, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                                   ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, vp, vp]
    lib.pctc_workspace_status.restype = ctypes.c_int
    lib.pctc_workspace_status.argtypes = [vp, vp, i32p]
    lib.pctc_status_string.restype = ctypes.c_char_p
    lib.pctc_status_string.argtypes = [ctypes.c_int]
    return lib


def status_string(status: int) -> str:
    return load().pctc_status_string(int(status)).decode()


def _i32(a) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(a), dtype=np.int32)


def _ptr_i32(a: np.ndarray):
    return a.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))


def make_problem(N, T, D, V, dtype, blank_id, beam=0.0, chunk=0, target_stride=0, gemm_path=GEMM_AUTO,
                 skip_dW=False, accumulate_dW=False, utt_weights_ptr=None, max_K=0, forward_only=False) -> Problem:
    return Problem(int(N), int(T), int(D), int(V), int(dtype), int(blank_id), float(beam), int(chunk),
                   int(target_stride), int(gemm_path), int(bool(skip_dW)), int(bool(accumulate_dW)),
                   int(bool(forward_only)), int(max_K), utt_weights_ptr)


def workspace_bytes(problem: Problem, input_lengths, target_lengths) -> int:
    il, tl = _i32(input_lengths), _i32(target_lengths)
    out = ctypes.c_size_t(0)
    st = load().pctc_workspace_bytes(ctypes.byref(problem), _ptr_i32(il), _ptr_i32(tl), ctypes.byref(out))
    if st != 0:
        raise PctcError(st, "pctc_workspace_bytes")
    return int(out.value)


def chunk_width(problem: Problem, input_lengths, target_lengths):
    """(C, number of chunks) the library will use for this problem (its default when problem.chunk is 0)."""
    il, tl = _i32(input_lengths), _i32(target_lengths)
    c, n = ctypes.c_int32(0), ctypes.c_int32(0)
    st = load().pctc_chunk_width(ctypes.byref(problem), _ptr_i32(il), _ptr_i32(tl), ctypes.byref(c), ctypes.byref(n))
    if st != 0:
        raise PctcError(st, "pctc_chunk_width")
    return int(c.value), int(n.value)


def _dptr(t) -> Optional[int]:
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def pruned_ctc_fwd_bwd(hidden, W, bias, targets, input_lengths, target_lengths, blank_id, *, beam=0.0,
                       chunk=0, gemm_path=GEMM_AUTO, workspace=None, out=None, check_status=False,
                       trace: Optional[Trace] = None, skip_dW=False, accumulate_dW=False, utt_weights=None,
                       max_K=0, forward_only=False, lib_handle=None):
    """Algorithm 1 on CUDA tensors.

    hidden [N,T,D], W [V,D], bias [V] or None (bf16 or fp32, same dtype), targets
    [N,stride] int32 on the device; input_lengths / target_lengths are host
    integer sequences.  Returns a dict of device tensors: loss [N] fp32, dH, dW,
    dbias (or None), subset [1+sum U], K [1], relabeled [N,stride], flags [N],
    plus "workspace" (reusable) and "workspace_bytes".  `out` may carry
    preallocated tensors from an earlier call with the same shapes.
    skip_dW: frozen head, dW is None.  accumulate_dW: add into out["dW"] / out["dbias"].
    utt_weights: fp32 CUDA tensor [N] of upstream gradients of the utterance losses.
    lib_handle: a test variant of the library from load_variant() instead of the regular one.
    """
    import torch

    lib = lib_handle or load()
    if not (hidden.is_cuda and W.is_cuda and hidden.is_contiguous() and W.is_contiguous()):
        raise ValueError("hidden and W must be contiguous CUDA tensors")
    if hidden.dtype != W.dtype or hidden.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("hidden and W must both be bf16 or both fp32")
    dt = PCTC_BF16 if hidden.dtype == torch.bfloat16 else PCTC_FP32
    N, T, D = hidden.shape
    V = W.shape[0]
    il, tl = _i32(input_lengths), _i32(target_lengths)
    if targets is None:
        targets = torch.zeros((N, 1), dtype=torch.int32, device=hidden.device)
    if targets.dtype != torch.int32 or not targets.is_contiguous():
        raise ValueError("targets must be a contiguous int32 CUDA tensor")
    stride = targets.shape[1]
    if utt_weights is not None and (utt_weights.dtype != torch.float32 or tuple(utt_weights.shape) != (N,)):
        raise ValueError("utt_weights must be an fp32 CUDA tensor of shape [N]")
    prob = make_problem(N, T, D, V, dt, blank_id, beam, chunk, stride, gemm_path, skip_dW, accumulate_dW,
                        None if utt_weights is None else utt_weights.data_ptr(), max_K, forward_only)
    need = workspace_bytes(prob, il, tl)          # host-only arithmetic, the same in every variant
    dev = hidden.device
    if workspace is None or workspace.numel() < need:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    o = out or {}

    def buf(name, shape, dtype):
        t = o.get(name)
        if t is None or tuple(t.shape) != tuple(shape) or t.dtype != dtype:
            t = torch.empty(shape, dtype=dtype, device=dev)
        return t

    ksum = int(tl.sum()) + 1
    if max_K:
        ksum = min(ksum, int(max_K))
    res = dict(
        loss=buf("loss", (N,), torch.float32),
        dH=None if forward_only else buf("dH", (N, T, D), hidden.dtype),
        dW=None if (skip_dW or forward_only) else buf("dW", (V, D), hidden.dtype),
        dbias=buf("dbias", (V,), hidden.dtype) if (bias is not None and not forward_only) else None,
        subset=buf("subset", (ksum,), torch.int32),
        K=buf("K", (1,), torch.int32),
        relabeled=buf("relabeled", (N, stride), torch.int32),
        flags=buf("flags", (N,), torch.int32),
        workspace=workspace, workspace_bytes=need,
    )
    stream = ctypes.c_void_p(torch.cuda.current_stream(dev).cuda_stream)
    args = [ctypes.byref(prob), _dptr(hidden), _dptr(W), _dptr(bias), _dptr(targets), _ptr_i32(il), _ptr_i32(tl),
            _dptr(res["loss"]), _dptr(res["dH"]), _dptr(res["dW"]), _dptr(res["dbias"]),
            _dptr(res["subset"]), _dptr(res["K"]), _dptr(res["relabeled"]), _dptr(res["flags"]),
            _dptr(workspace), ctypes.c_size_t(workspace.numel()), stream]
    if trace is None:
        st = lib.pruned_ctc_fwd_bwd(*args)
    else:
        st = lib.pruned_ctc_fwd_bwd_traced(*args, ctypes.byref(trace.struct))
    if st != 0:
        raise PctcError(st, "pruned_ctc_fwd_bwd")
    if check_status:
        code = workspace_status(workspace, lib_handle=lib)
        if code != 0:
            raise PctcError(6 if code < 0x100 else 1, f"device status word {code:#x}")
    return res


def workspace_status(workspace, lib_handle=None) -> int:
    """Synchronise the current stream and return the device status word: 0 nothing to report, 1-4 a
    bounded wait gave up, 0x100 more selected classes than max_K, 0x201.. (debug build) a bad index."""
    import torch

    host = ctypes.c_int32(0)
    stream = ctypes.c_void_p(torch.cuda.current_stream(workspace.device).cuda_stream)
    st = (lib_handle or load()).pctc_workspace_status(_dptr(workspace), stream, ctypes.byref(host))
    if st not in (0, 1, 6):
        raise PctcError(st, "pctc_workspace_status")
    return int(host.value)


def gemm_bf16(A, B, m, n, k, a_mn_major=False, b_mn_major=False, gemm_path=GEMM_AUTO):
    """C[m,n] (fp32) = sum_k A(i,k) B(j,k) for bf16 CUDA tensors; see prunedctc.h."""
    import torch

    C = torch.empty((m, n), dtype=torch.float32, device=A.device)
    status = torch.zeros(64, dtype=torch.int32, device=A.device)
    stream = ctypes.c_void_p(torch.cuda.current_stream(A.device).cuda_stream)
    st = load().pctc_gemm_bf16(_dptr(A), _dptr(B), _dptr(C), m, n, k, int(a_mn_major), int(b_mn_major),
                               int(gemm_path), _dptr(status), stream)
    if st != 0:
        raise PctcError(st, "pctc_gemm_bf16")
    code = int(status[0].item())
    if code != 0:
        raise PctcError(6, f"device status word {code}")
    return C


def pruned_ctc_fwd_bwd_host(hidden, W, bias, targets, input_lengths, target_lengths, blank_id, *, beam=0.0,
                            chunk=0, gemm_path=GEMM_AUTO, scratch=None, out=None, device=None):
    """Algorithm 1 on HOST tensors (pinned torch CPU tensors): copies in, computes, copies out.

    Returns host tensors loss, dH, dW, dbias, subset, K, relabeled, flags (pinned; valid after the
    current stream has been synchronised) plus "scratch", the reusable device buffer.
    """
    import torch

    lib = load()
    dev = torch.device(device or "cuda:0")
    if hidden.is_cuda or W.is_cuda:
        raise ValueError("the host entry point takes CPU tensors")
    dt = PCTC_BF16 if hidden.dtype == torch.bfloat16 else PCTC_FP32
    N, T, D = hidden.shape
    V = W.shape[0]
    il, tl = _i32(input_lengths), _i32(target_lengths)
    stride = targets.shape[1]
    prob = make_problem(N, T, D, V, dt, blank_id, beam, chunk, stride, gemm_path)
    need = ctypes.c_size_t(0)
    st = lib.pctc_host_call_scratch_bytes(ctypes.byref(prob), _ptr_i32(il), _ptr_i32(tl),
                                          int(bias is not None), ctypes.byref(need))
    if st != 0:
        raise PctcError(st, "pctc_host_call_scratch_bytes")
    if scratch is None or scratch.numel() < need.value:
        scratch = torch.empty(need.value, dtype=torch.uint8, device=dev)
    o = out or {}

    def buf(name, shape, dtype):
        t = o.get(name)
        if t is None or tuple(t.shape) != tuple(shape) or t.dtype != dtype:
            t = torch.empty(shape, dtype=dtype, pin_memory=True)
        return t

    res = dict(
        loss=buf("loss", (N,), torch.float32), dH=buf("dH", (N, T, D), hidden.dtype),
        dW=buf("dW", (V, D), hidden.dtype),
        dbias=buf("dbias", (V,), hidden.dtype) if bias is not None else None,
        subset=buf("subset", (int(tl.sum()) + 1,), torch.int32), K=buf("K", (1,), torch.int32),
        relabeled=buf("relabeled", (N, stride), torch.int32), flags=buf("flags", (N,), torch.int32),
        scratch=scratch, scratch_bytes=int(need.value),
    )
    stream = ctypes.c_void_p(torch.cuda.current_stream(dev).cuda_stream)
    st = lib.pruned_ctc_fwd_bwd_host(
        ctypes.byref(prob), _dptr(hidden), _dptr(W), _dptr(bias), _dptr(targets), _ptr_i32(il), _ptr_i32(tl),
        _dptr(res["loss"]), _dptr(res["dH"]), _dptr(res["dW"]), _dptr(res["dbias"]),
        _dptr(res["subset"]), _dptr(res["K"]), _dptr(res["relabeled"]), _dptr(res["flags"]),
        _dptr(scratch), ctypes.c_size_t(scratch.numel()), stream)
    if st != 0:
        raise PctcError(st, "pruned_ctc_fwd_bwd_host")
    return res


def subset_relabel_noalloc(targets, target_lengths, V, blank_id, out):
    """Algorithm 1 lines 2-3 through the entry point that allocates nothing.

    For callers that may not allocate device memory: every buffer, including the
    outputs in `out` (subset, K, relabeled, flags: int32 CUDA tensors), is the
    caller's; the library's own scratch is a fixed array inside it, so V may be
    at most NOALLOC_MAX_V.  targets [N,stride] and target_lengths [N] are int32
    CUDA tensors.  Runs on the current stream; returns `out`.
    """
    import torch

    N, stride = targets.shape
    stream = ctypes.c_void_p(torch.cuda.current_stream(targets.device).cuda_stream)
    st = load().pctc_subset_relabel_noalloc(_dptr(targets), _dptr(target_lengths), int(N), int(stride), int(V),
                                            int(blank_id), _dptr(out["subset"]), _dptr(out["K"]),
                                            _dptr(out["relabeled"]), _dptr(out["flags"]), stream)
    if st != 0:
        raise PctcError(st, "pctc_subset_relabel_noalloc")
    return out


def greedy_decode(hidden, W, bias, input_lengths, blank_id, *, gemm_path=GEMM_AUTO, workspace=None):
    """Greedy CTC recognition: frame arg-max of the head, repeats merged, blanks dropped.

    Returns device tensors frame_labels [N,T] (-1 on padded frames), tokens [N,T] (padded with
    -1), token_lengths [N], and the reusable workspace.
    """
    import torch

    lib = load()
    dt = PCTC_BF16 if hidden.dtype == torch.bfloat16 else PCTC_FP32
    N, T, D = hidden.shape
    V = W.shape[0]
    il = _i32(input_lengths)
    prob = make_problem(N, T, D, V, dt, blank_id, gemm_path=gemm_path)
    need = ctypes.c_size_t(0)
    st = lib.pctc_greedy_workspace_bytes(ctypes.byref(prob), _ptr_i32(il), ctypes.byref(need))
    if st != 0:
        raise PctcError(st, "pctc_greedy_workspace_bytes")
    dev = hidden.device
    if workspace is None or workspace.numel() < need.value:
        workspace = torch.empty(need.value, dtype=torch.uint8, device=dev)
    frame_labels = torch.empty((N, T), dtype=torch.int32, device=dev)
    tokens = torch.empty((N, T), dtype=torch.int32, device=dev)
    token_lengths = torch.empty((N,), dtype=torch.int32, device=dev)
    stream = ctypes.c_void_p(torch.cuda.current_stream(dev).cuda_stream)
    st = lib.pctc_greedy_decode(ctypes.byref(prob), _dptr(hidden), _dptr(W), _dptr(bias), _ptr_i32(il),
                                _dptr(frame_labels), _dptr(tokens), _dptr(token_lengths), _dptr(workspace),
                                ctypes.c_size_t(workspace.numel()), stream)
    if st != 0:
        raise PctcError(st, "pctc_greedy_decode")
    return dict(frame_labels=frame_labels, tokens=tokens, token_lengths=token_lengths, workspace=workspace)


def topk_decode(hidden, W, bias, input_lengths, k, *, chunk=0, gemm_path=GEMM_AUTO, workspace=None):
    """The k best classes of every frame (k in 1, 2, 4, 8) and their log-probabilities under the
    full-vocabulary softmax: device tensors classes [N,T,k] int32 (-1 on padded frames) and logprobs
    [N,T,k] fp32 (-inf there), plus the reusable workspace."""
    import torch

    lib = load()
    dt = PCTC_BF16 if hidden.dtype == torch.bfloat16 else PCTC_FP32
    N, T, D = hidden.shape
    V = W.shape[0]
    il = _i32(input_lengths)
    prob = make_problem(N, T, D, V, dt, 0, chunk=chunk, gemm_path=gemm_path)
    need = ctypes.c_size_t(0)
    st = lib.pctc_topk_workspace_bytes(ctypes.byref(prob), _ptr_i32(il), int(k), ctypes.byref(need))
    if st != 0:
        raise PctcError(st, "pctc_topk_workspace_bytes")
    dev = hidden.device
    if workspace is None or workspace.numel() < need.value:
        workspace = torch.empty(need.value, dtype=torch.uint8, device=dev)
    classes = torch.empty((N, T, k), dtype=torch.int32, device=dev)
    logprobs = torch.empty((N, T, k), dtype=torch.float32, device=dev)
    stream = ctypes.c_void_p(torch.cuda.current_stream(dev).cuda_stream)
    st = lib.pctc_topk_decode(ctypes.byref(prob), _dptr(hidden), _dptr(W), _dptr(bias), _ptr_i32(il), int(k),
                              _dptr(classes), _dptr(logprobs), _dptr(workspace), ctypes.c_size_t(workspace.numel()),
                              stream)
    if st != 0:
        raise PctcError(st, "pctc_topk_decode")
    return dict(classes=classes, logprobs=logprobs, workspace=workspace)


_marshal = None


def _native():
    """The compiled argument marshalling (csrc/marshal.cpp), bound to the loaded library."""
    global _marshal
    if _marshal is None:
        import torch  # noqa: F401  (its libraries come first)

        lib = load()
        try:
            from . import _marshal as module
        except ImportError as e:
            raise RuntimeError("_marshal.so is missing: run paper_2609_33645_b200.build.build() first; "
                               "there is no fallback implementation") from e
        names = ("pctc_clip_workspace_bytes", "pctc_clip_grad_norm", "pctc_grad_sqsum", "pctc_grad_scale",
                 "pctc_beam_workspace_bytes", "pctc_beam_select", "pctc_beam_reorder", "pctc_prefix_state_bytes",
                 "pctc_prefix_advance", "pctc_prefix_read", "pctc_prefix_decode")
        module.bind([ctypes.cast(getattr(lib, name), ctypes.c_void_p).value for name in names], PctcError)
        _marshal = module
    return _marshal


def clip_workspace_bytes(n: int) -> int:
    """Workspace of clip_grad_norm / grad_sqsum for n tensors."""
    need = ctypes.c_size_t(0)
    st = load().pctc_clip_workspace_bytes(int(n), ctypes.byref(need))
    if st != 0:
        raise PctcError(st, "pctc_clip_workspace_bytes")
    return int(need.value)


def clip_grad_norm(grads, max_norm, *, out=None, eps=1e-6, workspace=None):
    """Clip gradients by their global norm: every tensor times min(1, max_norm / (norm + eps)).

    grads: contiguous CUDA tensors of one device, bf16 and fp32 in any mixture, scaled in place, or
    into the tensors of `out` (same shapes; each of its gradient's type or fp32).  Returns a dict:
    norm [1] fp32 on the device (nothing waits for it), grads (the scaled tensors) and the workspace, which
    later calls on the same stream may take.  If the norm is not finite nothing is scaled.  The same tensor may
    not be given twice.  Autograd does not record the scaling; the written tensors' versions count up.
    """
    grads = list(grads)
    out = None if out is None else list(out)
    norm, workspace = _native().clip_grad_norm(grads, out, max_norm, eps, workspace)
    return dict(norm=norm, grads=grads if out is None else out, workspace=workspace)


def grad_sqsum(grads, *, workspace=None):
    """Sum of the squares of all values of `grads` (as in clip_grad_norm): sqsum [1] fp64 on the device, and
    the workspace.  Ranks that hold different shards add these up before grad_scale."""
    sqsum, workspace = _native().grad_sqsum(list(grads), workspace)
    return dict(sqsum=sqsum, workspace=workspace)


def grad_scale(grads, sqsum, max_norm, *, out=None, eps=1e-6):
    """The second half of clip_grad_norm, from a sum of squares [1] fp64 on the device."""
    grads = list(grads)
    out = None if out is None else list(out)
    norm = _native().grad_scale(grads, out, sqsum, max_norm, eps)
    return dict(norm=norm, grads=grads if out is None else out)


class PrefixBeam:
    """A CTC prefix beam search in progress, for frames that arrive in portions.

    `advance(classes, logprobs, lengths)` takes the next frames (classes [N,t,k] int32 and logprobs
    [N,t,k] fp32 as topk_decode gives them, any t, 0 too; lengths: host integers, how many of the t count
    per utterance, None for all); `read()` returns the hypotheses so far.  The state lives in one device
    buffer with room for max_frames frames an utterance.  Calls on one object belong on one stream.  An advance
    that is captured into a CUDA graph replays with the lengths of its capture, and starts the search anew if it was
    the first one; frames of replays are not counted here, but a state that is full still takes no more.
    """

    def __init__(self, N, beams, max_frames, blank_id, device):
        import torch

        self.N, self.beams, self.max_frames, self.blank_id = int(N), int(beams), int(max_frames), int(blank_id)
        self.device = torch.device(device)
        if self.device.type != "cuda":
            raise ValueError("the state of a prefix search lives on a CUDA device")
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.frames = [0] * self.N
        self.started = False
        self.state = _native().prefix_start(self.N, self.beams, self.blank_id, self.max_frames, self.device.index)

    def advance(self, classes, logprobs, lengths=None):
        native = _native()
        native.prefix_check(classes, logprobs, self.N, -1 if self.device.index is None else self.device.index)
        lengths = [classes.shape[1]] * self.N if lengths is None else [int(n) for n in lengths]
        if len(lengths) != self.N:
            raise ValueError("one length per utterance is required")
        frames = [f + n for f, n in zip(self.frames, lengths)]
        if max(frames) > self.max_frames:
            raise ValueError("more frames than the state has room for")
        native.prefix_advance(self.state, classes, logprobs, lengths, self.N, self.beams, self.blank_id, self.max_frames,
                              0 if self.started else 1)
        self.started = True
        self.frames = frames

    def read(self, max_tokens=None):
        """Device tensors, best hypothesis first: tokens [N,beams,max_tokens] int32 (-1 behind the last; max_tokens
        defaults to the frames taken so far), token_lengths [N,beams], scores [N,beams] fp32 (log-probabilities,
        -inf where there are fewer hypotheses than beams), flags [N]."""
        if not self.started:
            raise ValueError("no frames yet")
        width = max(1, max(self.frames)) if max_tokens is None else int(max_tokens)
        return _native().prefix_read(self.state, self.N, self.beams, self.blank_id, self.max_frames, width)


def prefix_beam_decode(classes, logprobs, input_lengths, blank_id, beams):
    """CTC prefix beam search over whole utterances: classes [N,T,k] int32 and logprobs [N,T,k] fp32 as
    topk_decode gives them, input_lengths host integers.  Returns the dict of PrefixBeam.read() with tokens
    [N,beams,T] (one label wide where T is 0), plus the PrefixBeam itself as "search"."""
    lengths = [int(n) for n in input_lengths]
    res, state = _native().prefix_decode(classes, logprobs, lengths, beams, blank_id)
    search = PrefixBeam.__new__(PrefixBeam)
    search.N, search.beams, search.blank_id = len(lengths), int(beams), int(blank_id)
    search.max_frames = max(1, classes.shape[1])
    search.device, search.state, search.frames, search.started = classes.device, state, lengths, True
    res["search"] = search
    return res


def beam_decode(hidden, W, bias, input_lengths, blank_id, beams, *, k=8, chunk=0, gemm_path=GEMM_AUTO, workspace=None):
    """CTC prefix beam search with the head: topk_decode's k best classes of every frame, then
    prefix_beam_decode over them.  Returns the latter's dict plus the head's workspace."""
    best = topk_decode(hidden, W, bias, input_lengths, k, chunk=chunk, gemm_path=gemm_path, workspace=workspace)
    res = prefix_beam_decode(best["classes"], best["logprobs"], input_lengths, blank_id, beams)
    res["workspace"] = best["workspace"]
    return res


def beam_select(logits, scores, beams, *, finished=None, eos_id=None):
    """One step of beam search: the `beams` best continuations of every utterance over beams and vocabulary.

    logits [N,B,V] bf16 or fp32 with contiguous rows (any strides between rows, e.g. a view of a padded
    vocabulary), scores [N,B] fp32 (-inf: a dead beam), finished [N,B] bool or None (ended hypotheses, which
    keep their score in one candidate with token eos_id), eos_id the token that ends a hypothesis or None.
    Returns device tensors: scores [N,beams] fp32, parents and tokens [N,beams] int32 (-1 where there are
    fewer candidates than beams), finished [N,beams] bool and flags [N] int32 (UTT_NONFINITE).  Best
    first; among equals the lowest beam, then the lowest token.  Not differentiable: the scores carry no gradient.
    """
    return _native().beam_select(logits, scores, beams, finished, eos_id)


def beam_reorder(states, parents, *, lengths=None, time_axes=None, out=None):
    """Move decoder states to the beams that were selected: state[n, k] = state[n, parents[n, k]] for every tensor
    of `states` ([N, B, ...] of any type, contiguous behind the beam dimension), in one launch.  Bytes are moved, so
    a lazily conjugated or negated view has to be resolved first.

    parents [N, K] int32 (beam_select's; entries outside [0, B) leave their slot as it is).  out: tensors
    [N, K, ...] to write to; None: in place (K == B).  time_axes: for each state the dimension of which only
    the first lengths[n] entries (lengths [N] int32 on the device) are moved, or None for whole rows; what lies
    behind is left as it is.  Returns the list of written tensors; autograd does not record the move, and their
    versions count up.
    """
    states = list(states)
    out = None if out is None else list(out)
    _native().beam_reorder(states, parents, lengths, None if time_axes is None else list(time_axes), out)
    return states if out is None else out
