"""ctypes binding of the C ABI in include/solo.h (argument marshalling only).

Every step of the optimizer runs in the CUDA library; this module passes raw device
pointers of torch tensors and the current CUDA stream.  If the shared library is not
there, loading raises: there is no other implementation to fall back to.
"""
from __future__ import annotations

import bisect
import ctypes as C
import functools
import math
import operator
import threading
import weakref
from pathlib import Path

import torch

_PKG = Path(__file__).resolve().parent
LIB_PATH = _PKG / "libsolo_b200.so"

SOLO_OK, SOLO_EINVAL, SOLO_EALIGN, SOLO_ENOMEM, SOLO_ECUDA, SOLO_ESTATE = 0, -1, -2, -3, -4, -5
SOLO_ELIMIT = -6
STATIC_MAX_TENSORS = 1024


class SoloError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {strerror(status)} ({status})")


class Hyper(C.Structure):
    """solo_hyper_t"""

    _fields_ = [
        ("lr", C.c_float), ("beta1", C.c_float), ("beta2", C.c_float), ("eps", C.c_float),
        ("weight_decay", C.c_float), ("p_quantile", C.c_float), ("fixed_alpha", C.c_float),
        ("adamw", C.c_int32), ("bias_correction", C.c_int32), ("round_m", C.c_int32),
        ("round_v", C.c_int32), ("param_dtype", C.c_int32), ("belief", C.c_int32),
        ("param_round", C.c_int32), ("v_codebook", C.c_int32),
        ("seed", C.c_uint64),
    ]


class TensorList(C.Structure):
    """solo_tensor_list_t"""

    _fields_ = [
        ("num_tensors", C.c_int32), ("param", C.c_void_p), ("grad", C.c_void_p),
        ("numel", C.c_void_p), ("state", C.c_void_p),
    ]


class HostList(C.Structure):
    """solo_host_list_t: every pointer is a host array"""

    _fields_ = [
        ("num_tensors", C.c_int32), ("param_dev", C.c_void_p), ("grad_host", C.c_void_p),
        ("param_out_host", C.c_void_p), ("numel", C.c_void_p), ("chunk_elems", C.c_int64),
        ("state", C.c_void_p),
    ]


class RawState(C.Structure):
    """solo_raw_state_t: caller-owned state buffers for solo_multi_step_static"""

    _fields_ = [
        ("codes_m", C.c_void_p), ("codes_v", C.c_void_p), ("scale_m", C.c_void_p),
        ("scale_v", C.c_void_p), ("alpha", C.c_void_p),
        ("bits_m", C.c_int32), ("bits_v", C.c_int32), ("block", C.c_int32),
    ]


class GradList(C.Structure):
    """solo_grad_list_t"""

    _fields_ = [("grads", C.c_void_p), ("data", C.c_void_p), ("dtype", C.c_int32)]


class GradRows(C.Structure):
    """solo_grad_rows_t"""

    _fields_ = [
        ("acc", C.c_void_p), ("num_rows", C.c_int64), ("width", C.c_int64), ("tokens", C.c_void_p),
        ("token_bytes", C.c_int32), ("grad_dtype", C.c_int32), ("grad", C.c_void_p), ("grad_stride", C.c_int64),
        ("num_tokens", C.c_int64),
    ]


def hyper(lr=1e-3, beta1=0.8, beta2=0.999, eps=1e-8, weight_decay=0.01, p_quantile=0.1,
          adamw=1, bias_correction=1, round_m=0, round_v=1, param_dtype=0, seed=0, belief=0, fixed_alpha=0.0,
          param_round=0, v_codebook=0) -> Hyper:
    return Hyper(lr, beta1, beta2, eps, weight_decay, p_quantile, fixed_alpha, adamw, bias_correction,
                 round_m, round_v, param_dtype, belief, param_round, v_codebook, seed)


_lib = None


def lib() -> C.CDLL:
    """Loads libsolo_b200.so from the package directory; raises if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not LIB_PATH.exists():
        raise ImportError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2505_00347_b200._build` "
            "(nvcc, sm_100a).  There is no CPU or PyTorch fallback.")
    L = C.CDLL(str(LIB_PATH))
    vp, i64, i32 = C.c_void_p, C.c_int64, C.c_int
    L.solo_state_create.argtypes = [i64, i32, i32, i32, C.POINTER(vp)]
    L.solo_state_create_multi.argtypes = [C.POINTER(C.c_int64), i32, i32, i32, i32, C.POINTER(vp)]
    L.solo_state_destroy.argtypes = [vp]
    L.solo_state_bytes.argtypes = [i64, i32, i32, i32, C.POINTER(C.c_size_t)]
    L.solo_step.argtypes = [vp, vp, vp, C.POINTER(Hyper), i64, vp]
    L.solo_multi_step.argtypes = [C.POINTER(TensorList), C.POINTER(Hyper), i64, vp]
    L.solo_dequant.argtypes = [vp, i32, vp, vp]
    L.solo_state_raw.argtypes = [vp, i32, C.POINTER(vp), C.POINTER(C.c_size_t)]
    L.solo_state_info.argtypes = [vp, C.POINTER(C.c_int64), C.POINTER(C.c_int64),
                                  C.POINTER(C.c_int32), C.POINTER(C.c_int32),
                                  C.POINTER(C.c_int32), C.POINTER(C.c_int32)]
    L.solo_state_status.argtypes = [vp, C.POINTER(C.c_int)]
    L.solo_codebook_m.argtypes = [i32, C.POINTER(C.c_float)]
    L.solo_codebook_v.argtypes = [i32, i32, C.POINTER(C.c_float)]
    L.solo_codebook_v.restype = C.c_int
    L.solo_default_beta1.argtypes = [i32, i32]
    L.solo_default_beta1.restype = C.c_float
    L.solo_set_kernel_policy.argtypes = [i32]
    L.solo_debug_check_fast_log.argtypes = [C.c_uint32, C.c_uint32, C.POINTER(C.c_float),
                                            C.POINTER(C.c_float)]
    L.solo_debug_check_update_math.argtypes = [C.c_uint32, C.c_uint32, C.POINTER(C.c_uint64)]
    L.solo_debug_check_update_math.restype = C.c_int
    L.solo_multi_step_static.argtypes = [C.c_int32, vp, vp, C.POINTER(C.c_int64), C.POINTER(RawState),
                                         C.POINTER(Hyper), i64, vp]
    L.solo_multi_step_static.restype = C.c_int
    L.solo_multi_step_host.argtypes = [C.POINTER(HostList), C.POINTER(Hyper), i64, vp]
    L.solo_multi_step_host.restype = C.c_int
    L.solo_state_export_bytes.argtypes = [vp, C.POINTER(C.c_size_t)]
    L.solo_state_export.argtypes = [vp, vp, C.c_size_t, vp]
    L.solo_state_import.argtypes = [vp, vp, C.c_size_t, vp]
    L.solo_state_set_origin.argtypes = [vp, C.POINTER(C.c_int32), C.POINTER(C.c_int64)]
    L.solo_state_set_origin.restype = C.c_int
    L.solo_static_status.argtypes = [C.POINTER(C.c_int), vp]
    L.solo_static_status.restype = C.c_int
    L.solo_debug_stall_copy.argtypes = [i64]
    L.solo_debug_stall_copy.restype = C.c_int
    L.solo_launch_count.argtypes = []
    L.solo_launch_count.restype = C.c_int64
    L.solo_strerror.argtypes = [i32]
    gl, f32 = C.POINTER(GradList), C.c_float
    L.solo_grads_create.argtypes = [C.POINTER(C.c_int64), i32, vp, vp, C.POINTER(vp)]
    L.solo_grads_destroy.argtypes = [vp]
    L.solo_grads_workspace.argtypes = [vp, C.POINTER(C.c_size_t)]
    L.solo_grad_norm.argtypes = [gl, i32, f32, vp, vp, vp, vp]
    L.solo_grad_clip.argtypes = [gl, gl, vp, i32, i32, f32, f32, vp]
    L.solo_grad_clip_norm.argtypes = [gl, gl, i32, f32, f32, vp, vp, vp, vp]
    L.solo_grad_accumulate.argtypes = [gl, gl, f32, i32, i32, vp, vp, vp, vp]
    L.solo_grad_rows_workspace.argtypes = [i64, i64, C.POINTER(C.c_size_t)]
    L.solo_grad_accumulate_rows.argtypes = [C.POINTER(GradRows), f32, vp, vp]
    L.solo_strerror.restype = C.c_char_p
    for name in ("solo_state_create", "solo_state_create_multi", "solo_state_destroy",
                 "solo_state_bytes", "solo_step", "solo_multi_step", "solo_dequant",
                 "solo_state_raw", "solo_state_info", "solo_state_status", "solo_codebook_m",
                 "solo_set_kernel_policy", "solo_debug_check_fast_log", "solo_state_export_bytes",
                 "solo_state_export", "solo_state_import", "solo_grads_create", "solo_grads_destroy",
                 "solo_grads_workspace", "solo_grad_norm", "solo_grad_clip", "solo_grad_clip_norm",
                 "solo_grad_accumulate", "solo_grad_rows_workspace", "solo_grad_accumulate_rows"):
        getattr(L, name).restype = C.c_int
    _lib = L
    return L


def strerror(status: int) -> str:
    return lib().solo_strerror(status).decode()


def _check(rc: int, what: str) -> None:
    if rc != SOLO_OK:
        raise SoloError(rc, what)


_raw_stream = None            # (device) -> handle of its current stream, once CUDA is initialised


def _stream() -> int:
    # torch.cuda.current_stream() builds a Stream object on every call: 1 us of a 4 us launch.  The functions beneath it are
    # not public: the first call goes through the public one, which also initialises CUDA, and so do all where they are missing.
    global _raw_stream
    if _raw_stream is not None:
        return _raw_stream(torch._C._cuda_getDevice())
    handle = torch.cuda.current_stream().cuda_stream
    if hasattr(torch._C, "_cuda_getDevice"):
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return handle


def _current_device() -> int:
    return torch._C._cuda_getDevice() if _raw_stream is not None else torch.cuda.current_device()


RAW = {"codes_m": 0, "codes_v": 1, "scale_m": 2, "scale_v": 3, "alpha": 4}
_RAW_DTYPE = {0: torch.uint8, 1: torch.uint8, 2: torch.float32, 3: torch.float32, 4: torch.float32}


class State:
    """Owner of a solo_state_t handle (single tensor or tensor list)."""

    def __init__(self, numel, bits_m: int, bits_v: int, block: int = 128):
        self.handle = C.c_void_p()
        self.sizes = [int(numel)] if isinstance(numel, int) else [int(n) for n in numel]
        if isinstance(numel, int):
            rc = lib().solo_state_create(numel, bits_m, bits_v, block, C.byref(self.handle))
        else:
            arr = (C.c_int64 * len(self.sizes))(*self.sizes)
            rc = lib().solo_state_create_multi(arr, len(self.sizes), bits_m, bits_v, block,
                                               C.byref(self.handle))
        _check(rc, "solo_state_create")
        self.bits_m, self.bits_v, self.block = bits_m, bits_v, block
        self.device = torch.device("cuda", torch.cuda.current_device())

    def destroy(self) -> None:
        if getattr(self, "handle", None) is not None and self.handle:
            lib().solo_state_destroy(self.handle)
            self.handle = C.c_void_p()

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    def set_origin(self, stream_ids=None, elem_offsets=None) -> None:
        """solo_state_set_origin: where each tensor of this state sits in the random stream (the
        tensor's stream number and the index of its first element within the whole tensor)."""
        T = len(self.sizes)
        ids = (C.c_int32 * T)(*[int(x) for x in stream_ids]) if stream_ids is not None else None
        offs = (C.c_int64 * T)(*[int(x) for x in elem_offsets]) if elem_offsets is not None else None
        _check(lib().solo_state_set_origin(self.handle, ids, offs), "solo_state_set_origin")

    def info(self) -> dict:
        n, nb = C.c_int64(), C.c_int64()
        t, bm, bv, blk = C.c_int32(), C.c_int32(), C.c_int32(), C.c_int32()
        _check(lib().solo_state_info(self.handle, C.byref(n), C.byref(nb), C.byref(t), C.byref(bm),
                                     C.byref(bv), C.byref(blk)), "solo_state_info")
        return dict(numel=n.value, num_blocks=nb.value, num_tensors=t.value, bits_m=bm.value,
                    bits_v=bv.value, block=blk.value)

    def raw_ptr(self, which) -> tuple[int, int]:
        w = RAW[which] if isinstance(which, str) else which
        p, b = C.c_void_p(), C.c_size_t()
        _check(lib().solo_state_raw(self.handle, w, C.byref(p), C.byref(b)), "solo_state_raw")
        return p.value or 0, b.value

    def raw_get(self, which) -> torch.Tensor:
        """Copy of one state buffer as a CPU tensor (uint8 codes / float32 scales)."""
        w = RAW[which] if isinstance(which, str) else which
        ptr, nbytes = self.raw_ptr(w)
        out = torch.empty(nbytes, dtype=torch.uint8)
        torch.cuda.synchronize()
        _cuda_memcpy(out.data_ptr(), ptr, nbytes, 2)
        return out if _RAW_DTYPE[w] == torch.uint8 else out.view(torch.float32)

    def raw_set(self, which, value: torch.Tensor) -> None:
        """Overwrite one state buffer from a CPU tensor of the same byte size."""
        w = RAW[which] if isinstance(which, str) else which
        ptr, nbytes = self.raw_ptr(w)
        v = value.contiguous().view(torch.uint8).cpu()
        if v.numel() != nbytes:
            raise ValueError(f"expected {nbytes} bytes, got {v.numel()}")
        torch.cuda.synchronize()
        _cuda_memcpy(ptr, v.data_ptr(), nbytes, 1)

    def export(self) -> torch.Tensor:
        """The whole state as one CPU uint8 tensor (solo_state_export)."""
        n = C.c_size_t()
        _check(lib().solo_state_export_bytes(self.handle, C.byref(n)), "solo_state_export_bytes")
        out = torch.empty(n.value, dtype=torch.uint8)
        _check(lib().solo_state_export(self.handle, out.data_ptr(), n.value,
                                       torch.cuda.current_stream().cuda_stream), "solo_state_export")
        return out

    def load(self, blob: torch.Tensor) -> None:
        """Restores a state written by export() into this one (solo_state_import)."""
        b = blob.contiguous().view(torch.uint8).cpu()
        _check(lib().solo_state_import(self.handle, b.data_ptr(), b.numel(),
                                       torch.cuda.current_stream().cuda_stream), "solo_state_import")

    def status(self) -> int:
        s = C.c_int()
        _check(lib().solo_state_status(self.handle, C.byref(s)), "solo_state_status")
        return s.value


_cudart = None


def _cuda_memcpy(dst: int, src: int, nbytes: int, kind: int) -> None:
    """cudaMemcpy through the runtime that torch already loaded (kind 1 = H2D, 2 = D2H)."""
    global _cudart
    if nbytes == 0:
        return
    if _cudart is None:
        _cudart = C.CDLL(_find_cudart())
        _cudart.cudaMemcpy.argtypes = [C.c_void_p, C.c_void_p, C.c_size_t, C.c_int]
        _cudart.cudaMemcpy.restype = C.c_int
    rc = _cudart.cudaMemcpy(dst, src, nbytes, kind)
    if rc:
        raise RuntimeError(f"cudaMemcpy failed with {rc}")


def _find_cudart() -> str:
    import glob
    import os
    cands = []
    for root in (os.path.join(os.path.dirname(torch.__file__), "lib"),
                 os.path.join(os.path.dirname(os.path.dirname(torch.__file__)), "nvidia",
                              "cuda_runtime", "lib"),
                 "/usr/local/cuda/lib64"):
        cands += sorted(glob.glob(os.path.join(root, "libcudart.so*")))
    if not cands:
        raise ImportError("libcudart.so not found")
    return cands[0]


def state_bytes(numel: int, bits_m: int, bits_v: int, block: int = 128) -> int:
    out = C.c_size_t()
    _check(lib().solo_state_bytes(numel, bits_m, bits_v, block, C.byref(out)), "solo_state_bytes")
    return out.value


def solo_step(param: torch.Tensor, grad: torch.Tensor, state: State, h: Hyper, step: int) -> None:
    """One fused step on a single tensor, on the current stream."""
    _check_tensor(param, grad, h)
    rc = (_lib or lib()).solo_step(param.data_ptr(), grad.data_ptr(), state.handle, C.byref(h), step, _stream())
    if rc:
        _check(rc, "solo_step")


def _check_tensor(param: torch.Tensor, grad: torch.Tensor, h: Hyper) -> None:
    want = torch.bfloat16 if h.param_dtype == 1 else torch.float32
    if not (param.is_cuda and grad.is_cuda and param.is_contiguous() and grad.is_contiguous()):
        raise ValueError("param and grad must be contiguous CUDA tensors")
    if param.dtype != want or grad.dtype != torch.bfloat16 or param.numel() != grad.numel():
        raise ValueError("param must be fp32/bf16 per hyper.param_dtype, grad bf16, same numel")


class TensorSet:
    """Device-side descriptor arrays of a tensor list (built once, reused every step)."""

    def __init__(self, params: list[torch.Tensor], grads: list[torch.Tensor], state: State):
        if len(params) != len(grads) or len(params) != len(state.sizes):
            raise ValueError("params, grads and state must have the same number of tensors")
        for p, g, n in zip(params, grads, state.sizes):
            if p.numel() != n or g.numel() != n or g.dtype != torch.bfloat16:
                raise ValueError("tensor sizes / dtypes do not match the state")
            if not (p.is_cuda and g.is_cuda and p.is_contiguous() and g.is_contiguous()):
                raise ValueError("tensors must be contiguous CUDA tensors")
        dev = params[0].device
        self.params, self.grads, self.state = params, grads, state
        self.param_ptrs = torch.tensor([p.data_ptr() for p in params], dtype=torch.int64, device=dev)
        self.grad_ptrs = torch.tensor([g.data_ptr() for g in grads], dtype=torch.int64, device=dev)
        self.numel = torch.tensor(state.sizes, dtype=torch.int64, device=dev)
        self.desc = TensorList(len(params), self.param_ptrs.data_ptr(), self.grad_ptrs.data_ptr(),
                               self.numel.data_ptr(), state.handle)


def solo_multi_step(ts: TensorSet, h: Hyper, step: int) -> None:
    """One fused step over the whole tensor list, in one launch or two (solo_multi_step in solo.h), on the current stream."""
    rc = (_lib or lib()).solo_multi_step(C.byref(ts.desc), C.byref(h), step, _stream())
    if rc:
        _check(rc, "solo_multi_step")


def solo_dequant(state: State, which: int) -> torch.Tensor:
    """Dequantized first (0) or second (1) moment of every element, as a float32 CUDA tensor."""
    out = torch.empty(sum(state.sizes), dtype=torch.float32, device=state.device)
    _check(lib().solo_dequant(state.handle, which, out.data_ptr(), _stream()), "solo_dequant")
    return out


def solo_multi_step_static(params: list[torch.Tensor], grads: list[torch.Tensor], sizes: list[int],
                           buffers: dict, bits_m: int, bits_v: int, block: int, h: Hyper, step: int,
                           param_ptrs: torch.Tensor = None, grad_ptrs: torch.Tensor = None) -> None:
    """The allocation-free step: `buffers` maps codes_m / codes_v (uint8) and scale_m / scale_v /
    alpha (float32) to CUDA tensors that the caller allocated in the library's state layout.
    `param_ptrs` / `grad_ptrs` are int64 CUDA tensors of the tensors' data pointers (built here,
    with torch, when not given; the library call itself allocates nothing)."""
    if param_ptrs is None:
        param_ptrs = torch.tensor([p.data_ptr() for p in params], dtype=torch.int64, device=params[0].device)
    if grad_ptrs is None:
        grad_ptrs = torch.tensor([g.data_ptr() for g in grads], dtype=torch.int64, device=params[0].device)
    raw = RawState(buffers["codes_m"].data_ptr(), buffers["codes_v"].data_ptr(),
                   buffers["scale_m"].data_ptr(), buffers["scale_v"].data_ptr(),
                   buffers["alpha"].data_ptr(), bits_m, bits_v, block)
    numel = (C.c_int64 * len(sizes))(*[int(n) for n in sizes])
    _check(lib().solo_multi_step_static(len(sizes), param_ptrs.data_ptr(), grad_ptrs.data_ptr(), numel,
                                        C.byref(raw), C.byref(h), step, _stream()),
           "solo_multi_step_static")


def solo_multi_step_host(params: list[torch.Tensor], grads_host: list[torch.Tensor],
                         params_out_host, state: State, h: Hyper, step: int, chunk_elems: int = 0) -> None:
    """The step with gradients in host memory (CPU bf16 tensors, pinned for overlap) and, when
    `params_out_host` is a list of CPU tensors of the parameters' type, a host copy of the updated
    parameters.  `params` are the resident CUDA tensors."""
    T = len(params)
    want = torch.bfloat16 if h.param_dtype == 1 else torch.float32
    for i in range(T):
        if not (params[i].is_cuda and params[i].is_contiguous() and params[i].dtype == want):
            raise ValueError("params must be contiguous CUDA tensors of the type hyper.param_dtype names")
        if grads_host[i].is_cuda or grads_host[i].dtype != torch.bfloat16 or not grads_host[i].is_contiguous() \
                or grads_host[i].numel() != params[i].numel():
            raise ValueError("grads_host must be contiguous CPU bf16 tensors of the parameters' sizes")
        if params_out_host is not None:
            o = params_out_host[i]
            if o.is_cuda or o.dtype != want or not o.is_contiguous() or o.numel() != params[i].numel():
                raise ValueError("params_out_host must be contiguous CPU tensors like the parameters")
    vp = C.c_void_p * T
    pd = vp(*[p.data_ptr() for p in params])
    gh = vp(*[g.data_ptr() for g in grads_host])
    po = vp(*[o.data_ptr() for o in params_out_host]) if params_out_host is not None else None
    numel = (C.c_int64 * T)(*[int(p.numel()) for p in params])
    lst = HostList(T, C.cast(pd, C.c_void_p), C.cast(gh, C.c_void_p),
                   C.cast(po, C.c_void_p) if po is not None else None, C.cast(numel, C.c_void_p),
                   int(chunk_elems), state.handle)
    _check(lib().solo_multi_step_host(C.byref(lst), C.byref(h), step, _stream()), "solo_multi_step_host")


_GRAD_DTYPE = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_NORM_TYPE = {math.inf: 0, 1: 1, 2: 2}


class GradSet:
    """Descriptor of a list of contiguous gradient tensors of one type: fp32, bf16 or fp16.  Built once and reused every step where
    the tensors keep their memory, as accumulators do (making one takes the host 20 us and 0.7 us for each tensor); gradients of
    several types make a list each, whose norms solo_grad_clip joins.  Made on the current stream, not while it is capturing;
    work on other streams is ordered after that by the caller.  It outlives the work and the captured graphs that use it, as the
    tensors do."""

    def __init__(self, grads: list[torch.Tensor]):
        if not grads:
            raise ValueError("a gradient list has at least one tensor")
        dtype, dev = grads[0].dtype, grads[0].device
        if dtype not in _GRAD_DTYPE:
            raise ValueError("gradients must be fp32, bf16 or fp16")
        index = dev.index
        for g in grads:
            if not (g.is_cuda and g.is_contiguous()) or g.dtype != dtype or g.get_device() != index:
                raise ValueError("gradients must be contiguous CUDA tensors of one type on one device")
        if index != torch.cuda.current_device():
            raise ValueError("gradients must be on the current device")
        self.grads, self.dtype, self.device = list(grads), dtype, dev
        self.sizes = [g.numel() for g in grads]
        ptrs = [g.data_ptr() for g in grads]
        _aligned(ptrs, grads[0].element_size())
        self.ptrs = torch.tensor(ptrs, dtype=torch.int64).to(dev, non_blocking=True)      # staged before it returns
        self.geom = torch.empty(2 * len(grads) + 1, dtype=torch.int64, device=dev)
        self.handle = C.c_void_p()
        arr = (C.c_int64 * len(grads))(*self.sizes)
        _check(lib().solo_grads_create(arr, len(grads), self.geom.data_ptr(), _stream(), C.byref(self.handle)), "solo_grads_create")
        # a list that is written must not have two tensors over the same memory
        self._spans = [(p, p + n * grads[0].element_size()) for p, n in zip(ptrs, self.sizes) if n]
        self._in_order = sorted(self._spans)
        self._apart = _disjoint(self._in_order)
        self._low = self._in_order[0][0] if self._spans else 0
        self._high = 0 if not self._spans else self._in_order[-1][1] if self._apart else max(b for _, b in self._spans)
        self._clear_of = None         # set of the lists that this one was found to lie clear of
        n = C.c_size_t()
        _check(lib().solo_grads_workspace(self.handle, C.byref(n)), "solo_grads_workspace")
        self.desc = GradList(self.handle.value, self.ptrs.data_ptr(), _GRAD_DTYPE[dtype])
        self._ref = C.byref(self.desc)
        self._workspace_bytes, self._lengths = n.value, [1, len(grads)]
        self._workspaces = {}         # by stream: calls on one stream follow one another
        self._turn = threading.Lock()

    def __del__(self):
        try:
            if self.handle:
                lib().solo_grads_destroy(self.handle)
        except Exception:
            pass

    def _workspace(self, stream: int) -> torch.Tensor:
        """The list's workspace on a stream.  What is captured into a graph gets one of its own."""
        if torch.cuda.is_current_stream_capturing():
            return torch.empty(self._workspace_bytes, dtype=torch.uint8, device=self.device)
        ws = self._workspaces.get(stream)
        if ws is None:
            ws = torch.zeros(self._workspace_bytes, dtype=torch.uint8, device=self.device)
            # kept for a stream of the list's device alone: another device's may have the same handle, and its call is refused; the
            # zeros would then be of no stream that a later call follows
            if self.device.index == _current_device():
                self._workspaces[stream] = ws
        return ws

    def _norms(self, per_tensor: bool) -> torch.Tensor:
        return torch.empty(1 + len(self.sizes) if per_tensor else 1, dtype=torch.float32, device=self.device)


def _aligned(ptrs: list, size: int) -> None:
    if functools.reduce(operator.or_, ptrs) & (size - 1):         # (memory of other libraries may begin anywhere)
        raise ValueError("gradients must be aligned to their elements")


def _disjoint(spans) -> bool:
    return all(a[1] <= b[0] for a, b in zip(spans, spans[1:]))


def _union(spans) -> list:
    out = []
    for a, b in sorted(spans):
        if out and a <= out[-1][1]:
            out[-1] = (out[-1][0], max(b, out[-1][1]))
        else:
            out.append((a, b))
    return out


def _written(gs: GradSet, read: GradSet):
    """gs as the list that a call writes while it reads `read`: the same tensors in the same type, or none of their memory."""
    if not gs._apart:
        raise ValueError("tensors of a list that is written must not overlap")
    if read is not gs and read._low < gs._high and gs._low < read._high:
        if gs._clear_of is None or read not in gs._clear_of:
            same = read._spans == gs._spans and read.dtype == gs.dtype
            if not same and not _disjoint(sorted(gs._spans + _union(read._spans))):
                raise ValueError("the lists of a call must not overlap, unless they are the same")
            if gs._clear_of is None:
                gs._clear_of = weakref.WeakSet()
            gs._clear_of.add(read)
    return gs._ref


def _reaches_into(low: int, high: int, apart: list) -> bool:
    """Whether [low, high) shares memory with one of the spans, which are in order and apart."""
    i = bisect.bisect_left(apart, (high,))
    return i > 0 and apart[i - 1][1] > low


def _norm_type(p) -> int:
    if p not in _NORM_TYPE:
        raise ValueError("norm_type must be 1, 2 or infinity")
    return _NORM_TYPE[p]


def solo_grad_norm(gs: GradSet, norm_type=2, scale: float = 1.0, per_tensor: bool = False):
    """|scale| times the norm (1, 2 or infinity) of the whole list, as a float32 CUDA tensor of one element; with
    `per_tensor` also one of every tensor's norm.  On the current stream, without waiting, as all of these calls."""
    p, stream = _norm_type(norm_type), _stream()
    out = gs._norms(per_tensor)
    at = out.data_ptr()
    with gs._turn:
        rc = (_lib or lib()).solo_grad_norm(gs._ref, p, scale, at, at + 4 if per_tensor else None, gs._workspace(stream).data_ptr(), stream)
    if rc:
        _check(rc, "solo_grad_norm")
    return out.split_with_sizes(gs._lengths) if per_tensor else out


def solo_grad_clip(src: GradSet, norms, max_norm: float, dst: GradSet = None, norm_type=2, scale: float = 1.0) -> None:
    """dst (default: src, in place) = src * scale * min(1, max_norm / (N + 1e-6)), N the norm of the whole from the
    `norms` of its parts (a float32 CUDA tensor, outside of dst); norms=None: scaling and conversion alone."""
    n, to = 0, dst or src
    if norms is not None:
        if not isinstance(norms, torch.Tensor) or not norms.is_cuda or norms.dtype != torch.float32 or not norms.is_contiguous() or norms.device != src.device:
            raise ValueError("norms must be a contiguous float32 tensor on the gradients' device")
        n = norms.numel()
        if n == 0:
            raise ValueError("norms has no element")
        at = norms.data_ptr()
        if at < to._high and to._low < at + 4 * n and to._apart and _reaches_into(at, at + 4 * n, to._in_order):
            raise ValueError("norms must not lie in what is written")
    rc = (_lib or lib()).solo_grad_clip(src._ref, _written(to, src), at if n else None, n,
                                        _norm_type(norm_type), max_norm if n else 0.0, scale, _stream())
    if rc:
        _check(rc, "solo_grad_clip")


def solo_grad_clip_norm(src: GradSet, max_norm: float, dst: GradSet = None, norm_type=2, scale: float = 1.0,
                        per_tensor: bool = False):
    """solo_grad_norm, and solo_grad_clip by its result, in one call; returns what solo_grad_norm does."""
    p, stream, to = _norm_type(norm_type), _stream(), _written(dst or src, src)
    out = src._norms(per_tensor)
    at = out.data_ptr()
    with src._turn:
        rc = (_lib or lib()).solo_grad_clip_norm(src._ref, to, p, max_norm, scale, at, at + 4 if per_tensor else None,
                                                 src._workspace(stream).data_ptr(), stream)
    if rc:
        _check(rc, "solo_grad_clip_norm")
    return out.split_with_sizes(src._lengths) if per_tensor else out


def solo_grad_accumulate(acc: GradSet, grads: GradSet, scale: float = 1.0, first: bool = False, norm_type=None,
                         per_tensor: bool = False):
    """acc (fp32) += scale * grads, or = scale * grads with `first`; with a `norm_type` returns the norm of the new acc
    as solo_grad_norm does, from the same pass."""
    if norm_type is None:
        rc = (_lib or lib()).solo_grad_accumulate(_written(acc, grads), grads._ref, scale, 1 if first else 0, -1, None, None, None, _stream())
        if rc:
            _check(rc, "solo_grad_accumulate")
        return None
    p, stream, to = _norm_type(norm_type), _stream(), _written(acc, grads)
    out = acc._norms(per_tensor)
    at = out.data_ptr()
    with acc._turn:
        rc = (_lib or lib()).solo_grad_accumulate(to, grads._ref, scale, 1 if first else 0, p, at, at + 4 if per_tensor else None,
                                                  acc._workspace(stream).data_ptr(), stream)
    if rc:
        _check(rc, "solo_grad_accumulate")
    return out.split_with_sizes(acc._lengths) if per_tensor else out


_TOKEN_BYTES = {torch.int32: 4, torch.int64: 8}


@functools.lru_cache(maxsize=1024)
def _rows_workspace(num_tokens: int, width: int) -> int:
    size = C.c_size_t()
    _check(lib().solo_grad_rows_workspace(num_tokens, width, C.byref(size)), "solo_grad_rows_workspace")
    return size.value


def solo_grad_accumulate_rows(acc: torch.Tensor, tokens: torch.Tensor, grad: torch.Tensor, scale: float = 1.0) -> None:
    """acc[tokens[i], :] += scale * grad[i, :], the gradient of an embedding.  acc: fp32 [rows, width], contiguous; tokens:
    int32 or int64 of any shape, contiguous; grad: fp32, bf16 or fp16 of that shape and a last dimension of width, contiguous
    or, with one dimension of tokens, with rows any distance apart.  Tokens outside the table contribute nothing.  acc shares no
    memory with tokens or the rows of grad: refused."""
    if acc.dim() != 2 or acc.dtype != torch.float32 or not acc.is_cuda or not acc.is_contiguous():
        raise ValueError("acc must be a contiguous float32 CUDA matrix")
    num_rows, width = acc.shape
    dev = acc.get_device()
    if tokens.dtype not in _TOKEN_BYTES or not tokens.is_cuda or tokens.get_device() != dev or not tokens.is_contiguous():
        raise ValueError("tokens must be contiguous int32 or int64 on the accumulator's device")
    if grad.dtype not in _GRAD_DTYPE or not grad.is_cuda or grad.get_device() != dev or grad.shape != (*tokens.shape, width):
        raise ValueError("grad must be fp32, bf16 or fp16 of the tokens' shape and the accumulator's width, on its device")
    stream = _stream()
    if dev != _current_device():
        raise ValueError("tensors must be on the current device")
    n = tokens.numel()
    if grad.is_contiguous():
        stride = width
    elif grad.dim() == 2 and (width == 1 or grad.stride(1) == 1):
        stride = grad.stride(0)
    else:
        raise ValueError("grad must be contiguous, or a matrix with contiguous rows")
    if n == 0 or num_rows == 0 or width == 0:
        return
    size = _rows_workspace(n, width)
    ws = torch.empty(size, dtype=torch.uint8, device=acc.device) if size else None
    desc = GradRows(acc.data_ptr(), num_rows, width, tokens.data_ptr(), _TOKEN_BYTES[tokens.dtype], _GRAD_DTYPE[grad.dtype],
                    grad.data_ptr(), stride, n)
    rc = (_lib or lib()).solo_grad_accumulate_rows(C.byref(desc), scale, ws.data_ptr() if size else None, stream)
    if rc:
        _check(rc, "solo_grad_accumulate_rows")


def codebook_m(bits: int) -> torch.Tensor:
    buf = (C.c_float * (1 << bits))()
    _check(lib().solo_codebook_m(bits, buf), "solo_codebook_m")
    return torch.tensor(list(buf), dtype=torch.float32)


def codebook_v(v_codebook: int, bits: int) -> torch.Tensor:
    buf = (C.c_float * (1 << bits))()
    _check(lib().solo_codebook_v(v_codebook, bits, buf), "solo_codebook_v")
    return torch.tensor(list(buf), dtype=torch.float32)


def default_beta1(bits_m: int, from_scratch: bool = False) -> float:
    return float(lib().solo_default_beta1(bits_m, 1 if from_scratch else 0))


def set_kernel_policy(policy: int) -> None:
    """0: fastest kernel that applies (default); 1: always the general kernel; 2: like 0 without the
    sixteen-elements-per-thread kernel; 3: that kernel wherever it exists, whatever the tensor sizes."""
    _check(lib().solo_set_kernel_policy(policy), "solo_set_kernel_policy")


def debug_check_fast_log(lo_bits: int, hi_bits: int) -> tuple[float, float]:
    """(largest excess of the lg2 approximation over the relative bound, assumed absolute bound)."""
    ex, ab = C.c_float(), C.c_float()
    _check(lib().solo_debug_check_fast_log(lo_bits, hi_bits, C.byref(ex), C.byref(ab)),
           "solo_debug_check_fast_log")
    return ex.value, ab.value


def debug_check_update_math(lo_bits: int, hi_bits: int) -> int:
    """Results of the pairwise square root and division that differ from the IEEE operations'."""
    n = C.c_uint64()
    _check(lib().solo_debug_check_update_math(lo_bits, hi_bits, C.byref(n)), "solo_debug_check_update_math")
    return n.value


def static_status() -> int:
    """Status word of the last solo_multi_step_static call on the current device (waits for the
    current stream)."""
    out = C.c_int(-1)
    _check(lib().solo_static_status(C.byref(out), _stream()), "solo_static_status")
    return out.value


def debug_stall_copy(tile: int) -> None:
    """Test hook: the next step over-announces the input copy of tile `tile`, so the bounded wait
    for it runs out."""
    _check(lib().solo_debug_stall_copy(int(tile)), "solo_debug_stall_copy")


def launch_count() -> int:
    return int(lib().solo_launch_count())
