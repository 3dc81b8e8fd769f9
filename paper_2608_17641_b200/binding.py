"""ctypes binding of ``librlcs.so``: same names as the C ABI, argument marshalling only.

Every function takes CUDA ``torch.Tensor`` arguments (fp32 / uint8 / bool, contiguous), passes their
device pointers and the current CUDA stream to the C entry point and returns the output tensors.
Nothing is computed here; there is no CPU path.  A missing library raises at first use.
"""
from __future__ import annotations

import ctypes
import functools
import os
import threading

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "librlcs.so")

RLCS_OK = 0
RLCS_ERR_NULL, RLCS_ERR_SIZE, RLCS_ERR_ARG, RLCS_ERR_ALIGN = 1, 2, 3, 4
RLCS_ERR_WORKSPACE, RLCS_ERR_CUDA, RLCS_ERR_TIMEOUT, RLCS_ERR_LIMIT, RLCS_ERR_CAPTURE = 5, 6, 7, 8, 9

_vp, _i64, _f, _sz, _int = ctypes.c_void_p, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t, ctypes.c_int
_i32 = ctypes.c_int32
_TAIL = [_vp, _sz, _vp]          # workspace, workspace_bytes, cuda_stream

# name -> argtypes, exactly the declarations of include/rlcs.h
SIGNATURES = {
    "rlcs_status_string": ([_int], ctypes.c_char_p),
    "rlcs_workspace_bytes": ([_i64, _i64], _sz),
    "rlcs_workspace_init": ([_vp, _sz, _vp], _int),
    "rlcs_last_device_status": ([_vp, _vp], _int),
    "rlcs_gae": ([_vp] * 8 + [_i64, _i64, _f, _f] + _TAIL, _int),
    "rlcs_gae_normalized": ([_vp] * 8 + [_i64, _i64, _f, _f, _f, _int] + _TAIL, _int),
    "rlcs_gae_normalized_workspace_bytes": ([_i64, _i64], _sz),
    "rlcs_vtrace": ([_vp] * 9 + [_i64, _i64, _f, _f, _f] + _TAIL, _int),
    "rlcs_retrace": ([_vp] * 9 + [_i64, _i64, _f, _f, _f] + _TAIL, _int),
    "rlcs_retrace_probs": ([_vp] * 10 + [_i64, _i64, _i64, _f, _f, _f] + _TAIL, _int),
    "rlcs_td_lambda": ([_vp] * 7 + [_i64, _i64, _f, _f] + _TAIL, _int),
    "rlcs_discounted_return": ([_vp] * 6 + [_i64, _i64, _f] + _TAIL, _int),
    "rlcs_elig_trace": ([_vp] * 3 + [_i64, _i64, _f, _f] + _TAIL, _int),
    "rlcs_elig_trace_vec": ([_vp] * 3 + [_i64, _i64, _i64, _f, _f] + _TAIL, _int),
    "rlcs_elig_trace_vec_workspace_bytes": ([_i64, _i64, _i64], _sz),
    "rlcs_elig_trace_vec_beta": ([_vp] * 4 + [_i64, _i64, _i64] + _TAIL, _int),
    "rlcs_elig_trace_vec_beta_workspace_bytes": ([_i64, _i64, _i64], _sz),
    "rlcs_episodic_prefix_sum": ([_vp] * 3 + [_i64, _i64, _int] + _TAIL, _int),
    "rlcs_gae_skip": ([_vp] * 10 + [_i64, _i64, _f, _f] + _TAIL, _int),
    "rlcs_gae_no_alloc": ([_vp] * 8 + [_i64, _i64, _f, _f, _vp], _int),
    "rlcs_no_alloc_scratch_bytes": ([], _sz),
    "rlcs_no_alloc_last_device_status": ([_vp], _int),
    "rlcs_gae_carry_bytes": ([_i64, _i64, _int, _int], _sz),
    "rlcs_time_major_workspace_bytes": ([_i64, _i64], _sz),
    "rlcs_gae_time_major": ([_vp] * 8 + [_i64, _i64, _f, _f] + _TAIL, _int),
    "rlcs_vtrace_time_major": ([_vp] * 9 + [_i64, _i64, _f, _f, _f] + _TAIL, _int),
    "rlcs_retrace_time_major": ([_vp] * 9 + [_i64, _i64, _f, _f, _f] + _TAIL, _int),
    "rlcs_td_lambda_time_major": ([_vp] * 7 + [_i64, _i64, _f, _f] + _TAIL, _int),
    "rlcs_discounted_return_time_major": ([_vp] * 6 + [_i64, _i64, _f] + _TAIL, _int),
    "rlcs_elig_trace_time_major": ([_vp] * 3 + [_i64, _i64, _f, _f] + _TAIL, _int),
    "rlcs_episodic_prefix_sum_time_major": ([_vp] * 3 + [_i64, _i64, _int] + _TAIL, _int),
    "rlcs_gae_bf16": ([_vp] * 8 + [_i64, _i64, _f, _f] + _TAIL, _int),
    "rlcs_vtrace_bf16": ([_vp] * 9 + [_i64, _i64, _f, _f, _f] + _TAIL, _int),
    "rlcs_retrace_bf16": ([_vp] * 9 + [_i64, _i64, _f, _f, _f] + _TAIL, _int),
    "rlcs_td_lambda_bf16": ([_vp] * 7 + [_i64, _i64, _f, _f] + _TAIL, _int),
    "rlcs_discounted_return_bf16": ([_vp] * 6 + [_i64, _i64, _f] + _TAIL, _int),
    "rlcs_elig_trace_bf16": ([_vp] * 3 + [_i64, _i64, _f, _f] + _TAIL, _int),
    "rlcs_episodic_prefix_sum_bf16": ([_vp] * 3 + [_i64, _i64, _int] + _TAIL, _int),
    "rlcs_sample_actions": ([_vp, _i64] + [_vp] * 5 + [_f, _i32, _f, _f] + [_vp] * 3 + [_i64, _i64, _vp], _int),
    "rlcs_sample_actions_bf16": ([_vp, _i64] + [_vp] * 5 + [_f, _i32, _f, _f] + [_vp] * 3 + [_i64, _i64, _vp], _int),
    "rlcs_policy_grad": ([_vp, _i64] + [_vp] * 8 + [_i64] * 3 + [_f] * 4 + [_vp], _int),
    "rlcs_policy_grad_bf16": ([_vp, _i64] + [_vp] * 8 + [_i64] * 3 + [_f] * 4 + [_vp], _int),
    "rlcs_prefix_attention_workspace_bytes": ([_i64] * 8, _sz),
    "rlcs_prefix_attention_bf16": ([_vp, _i64, _vp, _vp] + [_i64] * 4 + [_vp, _i64, _vp, _vp, _vp, _i64] + [_vp] * 3 + [_i64] * 8
                                   + [_f] + _TAIL, _int),
    "rlcs_block_tables": ([_vp] * 8 + [_i64] * 5 + [_vp], _int),
    "rlcs_chunk_attention_workspace_bytes": ([_i64] * 8, _sz),
    "rlcs_chunk_attention_bf16": ([_vp, _i64, _vp, _vp] + [_i64] * 4 + [_vp, _i64] + [_vp] * 4 + [_i64] * 8 + [_f] + _TAIL, _int),
    "rlcs_verify_drafts_workspace_bytes": ([_i64] * 2, _sz),
    "rlcs_verify_drafts": ([_vp, _i64, _vp, _i64] + [_vp] * 5 + [_f] + [_vp] * 3 + [_i64] * 3 + _TAIL, _int),
    "rlcs_verify_drafts_bf16": ([_vp, _i64, _vp, _i64] + [_vp] * 5 + [_f] + [_vp] * 3 + [_i64] * 3 + _TAIL, _int),
    "rlcs_distill_grad": ([_vp, _i64] + [_vp] * 5 + [_i64] * 4 + [_f] * 2 + [_vp], _int),
    "rlcs_distill_grad_bf16": ([_vp, _i64] + [_vp] * 5 + [_i64] * 4 + [_f] * 2 + [_vp], _int),
    "rlcs_fork_block_tables_workspace_bytes": ([_i64] * 2, _sz),
    "rlcs_fork_block_tables": ([_vp] * 8 + [_i64] * 5 + _TAIL, _int),
    "rlcs_copy_pages_bf16": ([_vp] * 2 + [_i64] * 4 + [_vp] * 2 + [_i64] * 4 + [_vp], _int),
    "rlcs_free_pages_workspace_bytes": ([_i64], _sz),
    "rlcs_free_pages": ([_vp] * 6 + [_i64] * 6 + _TAIL, _int),
    "rlcs_affine_scan": ([_vp] * 3 + [_i64, _i64, _int] + _TAIL, _int),
    "rlcs_debug_set_tile_variant": ([_int], _int),
    "rlcs_debug_tile_elems": ([_int], _int),
    "rlcs_debug_set_carry_fault": ([_i64, _i64], _int),
    "rlcs_debug_set_wait_polls": ([_int], _int),
    "rlcs_debug_time_major_path": ([_int], None),
    "rlcs_debug_vec_trace_plan": ([_int, _int], None),
    "rlcs_debug_stream_copy": ([_vp, _vp, _sz, _sz, _vp], _int),
    "rlcs_debug_force_wide_index": ([_int], _int),
    "rlcs_debug_allow_cluster_carry": ([_int], _int),
    "rlcs_debug_set_dependent_launch": ([_int], _int),
    "rlcs_debug_allow_row_tiles": ([_int], _int),
    "rlcs_debug_set_row_blocks": ([_int], _int),
    "rlcs_debug_variant_for": ([_int, _int, _i64, _i64], _int),
    "rlcs_debug_variant_built": ([_int], _int),
    "rlcs_debug_variant_info": ([_int] + [ctypes.POINTER(ctypes.c_int)] * 4, _int),
}

_lib = None
_lock = threading.Lock()


class RlcsError(RuntimeError):
    def __init__(self, status: int):
        self.status = status
        super().__init__(lib().rlcs_status_string(status).decode())


_recording = threading.local()        # .calls, .held: lists while prepare() runs a wrapper, absent otherwise
_preparing = False                    # whether it does, in any thread


class _Recorder:
    """Stands in for the library while prepare() runs a wrapper: records (C function, arguments) of
    every compute call instead of making it; anything else (size queries, ...) goes to the library."""

    def __init__(self, real):
        self._real = real

    def __getattr__(self, name):
        fn = getattr(self._real, name)
        compute = (fn.restype is _int and fn.argtypes and fn.argtypes[-1] is _vp and not name.startswith("rlcs_debug")
                   and name not in ("rlcs_workspace_init", "rlcs_last_device_status", "rlcs_no_alloc_last_device_status"))
        if not compute:
            return fn

        def record(*args):
            _recording.calls.append((fn, args))
            return RLCS_OK
        return record


class Prepared:
    """A call whose arguments were checked and marshalled once (prepare()).  Calling it only makes the
    C call(s) -- a few microseconds of host time instead of the 12-28 that dtype, shape, device and
    pointer marshalling cost per call -- on the current stream, or on `stream_handle` (a raw
    cudaStream_t as int) when given.  The tensors are kept alive by this object, those too that the
    wrapper made for itself (a workspace); `outputs` is what the wrapper would have returned.  The caller must not free or resize them while it is in use, and must
    call it with the device current on which it was prepared."""

    def __init__(self, calls, outputs, keep):
        self._calls, self.outputs, self._keep = calls, outputs, keep

    def __call__(self, stream_handle=None):
        h = _stream() if stream_handle is None else stream_handle
        for fn, args in self._calls:
            st = fn(*args[:-1], h)
            if st != RLCS_OK:
                raise RlcsError(st)
        return self.outputs


def prepare(wrapper, *args, **kwargs) -> Prepared:
    """Run one of this module's rlcs_* wrappers in recording mode: all of its checks happen now,
    outputs and workspace are allocated (and the workspace initialised) now -- pass them in to control
    that -- and no kernel is launched.  Not thread-safe: no other thread may use this module meanwhile.
    The returned object repeats the call at C-call cost, e.g. inside a training loop on fixed buffers:

        step = prepare(rlcs_gae, rewards, values, dones, gamma=0.99, lam=0.95, workspace=ws)
        ...
        adv, ret = step()
    """
    real = lib()
    global _lib, _preparing
    _recording.calls, _recording.held = [], []
    _preparing = True
    with _lock:
        _lib = _Recorder(real)
    try:
        outputs = wrapper(*args, **kwargs)
        calls, held = _recording.calls, _recording.held
    finally:
        with _lock:
            _lib = real
        _preparing = False
        del _recording.calls, _recording.held
    if not calls:
        raise ValueError("prepare() takes one of the rlcs_* compute wrappers of this module")
    return Prepared(calls, outputs, (args, kwargs, held))


def lib() -> ctypes.CDLL:
    """The loaded C library (loaded once).  Raises if it has not been built."""
    global _lib
    with _lock:
        if _lib is None:
            if not os.path.exists(LIB_PATH):
                raise RuntimeError(
                    f"{LIB_PATH} is missing: build it with `python -m paper_2608_17641_b200.build` "
                    "(there is no fallback path)")
            L = ctypes.CDLL(LIB_PATH)
            for name, (argtypes, restype) in SIGNATURES.items():
                fn = getattr(L, name)
                fn.argtypes = argtypes
                fn.restype = restype
            _lib = L
    return _lib


def _check(status: int):
    if status != RLCS_OK:
        raise RlcsError(status)


_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


_cuda_current_device = None


def _current_device() -> int:
    global _cuda_current_device
    if _cuda_current_device is None:
        _cuda_current_device = _torch().cuda.current_device
    return _cuda_current_device()


def _require_current_device(t, what: str = "tensor"):
    """The library launches on the current device and the current stream of that device: a tensor
    (or workspace) that lives on another GPU would hand the kernel a pointer it must not touch."""
    index, cur = t.get_device(), _current_device()
    if index is not None and index >= 0 and index != cur:
        raise ValueError(f"{what} is on cuda:{index} but the current device is cuda:{cur}; "
                         f"call under torch.cuda.device({index})")


def _ptr(t, dtype_kind: str, shape=None):
    """Device pointer of a tensor (None -> NULL) after dtype / device / layout checks."""
    if t is None:
        return None
    torch = _torch()
    if not t.is_cuda:
        raise TypeError("rlcs takes CUDA tensors (device pointers); there is no CPU path")
    _require_current_device(t)
    if dtype_kind == "f32":
        if t.dtype != torch.float32:
            raise TypeError(f"expected float32, got {t.dtype}")     # the method is fp32-only
    elif dtype_kind == "bf16":
        if t.dtype != torch.bfloat16:
            raise TypeError(f"expected bfloat16, got {t.dtype}")
    elif t.dtype not in (torch.uint8, torch.bool):
        raise TypeError(f"expected a uint8/bool mask, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError("rlcs takes contiguous row-major tensors")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"expected shape {tuple(shape)}, got {tuple(t.shape)}")
    return t.data_ptr()


def _alloc(shape, dtype, device):
    """Device memory for outputs and workspaces the binding creates itself (torch's allocator).  A
    module-level function so that a test harness can substitute an allocator that adds guard bands."""
    n = len(shape)                                            # with strides given, torch takes 1.5 us instead of 2.4
    if n == 1:
        return _torch().empty_strided(shape, (1,), dtype=dtype, device=device)
    if n == 2:
        return _torch().empty_strided(shape, (shape[1], 1), dtype=dtype, device=device)
    if n == 3:
        return _torch().empty_strided(shape, (shape[1] * shape[2], shape[2], 1), dtype=dtype, device=device)
    return _torch().empty(shape, dtype=dtype, device=device)


def _held(t):
    """A tensor whose pointer goes into a C call: under prepare(), which repeats the call later, it is kept for as long."""
    if _preparing:
        held = getattr(_recording, "held", None)
        if held is not None:
            held.append(t)
    return t


def _new(shape, dtype, device):
    return _held(_alloc(shape, dtype, device))


_raw_stream = None


def _stream(stream=None):
    """Raw handle of the given stream, or of the current one (asked for without building a Stream object where torch allows)."""
    global _raw_stream
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None:
        torch = _torch()
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda device: torch.cuda.current_stream().cuda_stream)
    return _raw_stream(_current_device())


class Workspace:
    """Caller-owned carry workspace (device memory held by a torch tensor), initialised once."""

    def __init__(self, N: int, T: int, device="cuda", stream=None, nbytes: int | None = None):
        torch = _torch()
        self.nbytes = int(lib().rlcs_workspace_bytes(N, T)) if nbytes is None else int(nbytes)
        self.buf = _new((max(self.nbytes, 16),), torch.uint8, device) if self.nbytes else None
        if self.buf is not None:
            if stream is not None:
                self.buf.record_stream(stream)     # the caching allocator must not hand it out again before that stream is done
            _check(lib().rlcs_workspace_init(self.buf.data_ptr(), self.nbytes, _stream(stream)))

    @property
    def ptr(self):
        return None if self.buf is None else self.buf.data_ptr()

    def device_status(self, stream=None) -> int:
        return lib().rlcs_last_device_status(self.ptr, _stream(stream))


def workspace_bytes(N: int, T: int) -> int:
    return int(lib().rlcs_workspace_bytes(N, T))


def _ws(ws: Workspace | None):
    if ws is None:
        return (None, 0)
    if ws.buf is not None:
        _require_current_device(ws.buf, "workspace")
    return (ws.ptr, ws.nbytes)


def _out(like, out):
    torch = _torch()
    return _new(tuple(like.shape), torch.float32, like.device) if out is None else out


def rlcs_gae(rewards, values, dones, truncs=None, trunc_bootstrap=None, bootstrap=None, *, gamma, lam,
             advantages=None, returns=None, want_returns=True, workspace=None, stream=None):
    N, T = rewards.shape
    adv = _out(rewards, advantages)
    ret = (_out(rewards, returns) if want_returns else None)
    wp, wb = _ws(workspace)
    _check(lib().rlcs_gae(_ptr(rewards, "f32"), _ptr(values, "f32", (N, T)), _ptr(dones, "u8", (N, T)),
                          _ptr(truncs, "u8", (N, T)), _ptr(trunc_bootstrap, "f32", (N, T)),
                          _ptr(bootstrap, "f32", (N,)), _ptr(adv, "f32", (N, T)), _ptr(ret, "f32", (N, T)),
                          N, T, gamma, lam, wp, wb, _stream(stream)))
    return (adv, ret) if want_returns else adv


def rlcs_gae_normalized(rewards, values, dones, truncs=None, trunc_bootstrap=None, bootstrap=None, *, gamma, lam,
                        eps=1e-8, ddof=1, advantages=None, returns=None, want_returns=True, workspace=None, stream=None):
    """GAE + advantage normalisation over all N*T steps.  `workspace` must be a Workspace created with
    nbytes=rlcs_gae_normalized_workspace_bytes(N, T) (one is made on the fly when omitted)."""
    N, T = rewards.shape
    adv = _out(rewards, advantages)
    ret = (_out(rewards, returns) if want_returns else None)
    if workspace is None:
        workspace = Workspace(N, T, device=rewards.device, stream=stream,
                              nbytes=int(lib().rlcs_gae_normalized_workspace_bytes(N, T)))
    wp, wb = _ws(workspace)
    _check(lib().rlcs_gae_normalized(_ptr(rewards, "f32"), _ptr(values, "f32", (N, T)), _ptr(dones, "u8", (N, T)),
                                     _ptr(truncs, "u8", (N, T)), _ptr(trunc_bootstrap, "f32", (N, T)),
                                     _ptr(bootstrap, "f32", (N,)), _ptr(adv, "f32", (N, T)), _ptr(ret, "f32", (N, T)),
                                     N, T, gamma, lam, eps, ddof, wp, wb, _stream(stream)))
    return (adv, ret) if want_returns else adv


def rlcs_gae_skip(rewards, values, dones, truncs=None, trunc_bootstrap=None, bootstrap=None, *, skip, gamma, lam,
                  values_filled=None, advantages=None, returns=None, want_returns=True, workspace=None, stream=None):
    """GAE with observation-skip masking (skip != 0: masked, transparent step).  Returns
    (advantages, returns = A + W, values_filled = W), or (advantages, values_filled) without returns."""
    N, T = rewards.shape
    fil = _out(rewards, values_filled)
    adv = _out(rewards, advantages)
    ret = (_out(rewards, returns) if want_returns else None)
    wp, wb = _ws(workspace)
    _check(lib().rlcs_gae_skip(_ptr(rewards, "f32"), _ptr(values, "f32", (N, T)), _ptr(dones, "u8", (N, T)),
                               _ptr(truncs, "u8", (N, T)), _ptr(trunc_bootstrap, "f32", (N, T)),
                               _ptr(bootstrap, "f32", (N,)), _ptr(skip, "u8", (N, T)), _ptr(fil, "f32", (N, T)),
                               _ptr(adv, "f32", (N, T)), _ptr(ret, "f32", (N, T)), N, T, gamma, lam, wp, wb,
                               _stream(stream)))
    return (adv, ret, fil) if want_returns else (adv, fil)


def rlcs_gae_no_alloc(rewards, values, dones, truncs=None, trunc_bootstrap=None, bootstrap=None, *, gamma, lam,
                      advantages=None, returns=None, want_returns=True, stream=None):
    """GAE through the entry point that takes no workspace: the carry scratch is a fixed device
    array inside the library, so this call path performs no device allocation (pass `advantages`
    and `returns` to keep torch from allocating the outputs either).  Calls must not overlap on
    the GPU; the first call on a device should happen outside stream capture."""
    N, T = rewards.shape
    adv = _out(rewards, advantages)
    ret = (_out(rewards, returns) if want_returns else None)
    _check(lib().rlcs_gae_no_alloc(_ptr(rewards, "f32"), _ptr(values, "f32", (N, T)), _ptr(dones, "u8", (N, T)),
                                   _ptr(truncs, "u8", (N, T)), _ptr(trunc_bootstrap, "f32", (N, T)),
                                   _ptr(bootstrap, "f32", (N,)), _ptr(adv, "f32", (N, T)), _ptr(ret, "f32", (N, T)),
                                   N, T, gamma, lam, _stream(stream)))
    return (adv, ret) if want_returns else adv


def rlcs_no_alloc_last_device_status(stream=None) -> int:
    """Device status of the rlcs_gae_no_alloc calls on the current device (synchronises the stream,
    clears the word): RLCS_OK or RLCS_ERR_TIMEOUT."""
    return int(lib().rlcs_no_alloc_last_device_status(_stream(stream)))


def rlcs_vtrace(rewards, values, log_rhos, dones, truncs=None, trunc_bootstrap=None, bootstrap=None, *,
                gamma, rho_bar=1.0, c_bar=1.0, vs=None, pg_advantages=None, want_advantages=True,
                workspace=None, stream=None):
    N, T = rewards.shape
    vs = _out(rewards, vs)
    adv = (_out(rewards, pg_advantages) if want_advantages else None)
    wp, wb = _ws(workspace)
    _check(lib().rlcs_vtrace(_ptr(rewards, "f32"), _ptr(values, "f32", (N, T)), _ptr(log_rhos, "f32", (N, T)),
                             _ptr(dones, "u8", (N, T)), _ptr(truncs, "u8", (N, T)),
                             _ptr(trunc_bootstrap, "f32", (N, T)), _ptr(bootstrap, "f32", (N,)),
                             _ptr(vs, "f32", (N, T)), _ptr(adv, "f32", (N, T)), N, T, gamma, rho_bar, c_bar,
                             wp, wb, _stream(stream)))
    return (vs, adv) if want_advantages else vs


def rlcs_retrace(rewards, q_sa, expected_q, log_rhos, dones, truncs=None, trunc_bootstrap=None,
                 bootstrap=None, *, gamma, lam, c_bar=1.0, q_targets=None, workspace=None, stream=None):
    N, T = rewards.shape
    out = _out(rewards, q_targets)
    wp, wb = _ws(workspace)
    _check(lib().rlcs_retrace(_ptr(rewards, "f32"), _ptr(q_sa, "f32", (N, T)), _ptr(expected_q, "f32", (N, T)),
                              _ptr(log_rhos, "f32", (N, T)), _ptr(dones, "u8", (N, T)), _ptr(truncs, "u8", (N, T)),
                              _ptr(trunc_bootstrap, "f32", (N, T)), _ptr(bootstrap, "f32", (N,)),
                              _ptr(out, "f32", (N, T)), N, T, gamma, lam, c_bar, wp, wb, _stream(stream)))
    return out


def rlcs_retrace_probs(rewards, q_values, target_probs, behaviour_probs, actions, dones, truncs=None,
                       trunc_bootstrap=None, bootstrap=None, *, gamma, lam, c_bar=1.0, q_targets=None, workspace=None,
                       stream=None):
    """Retrace(lambda) from [N,T,A] Q-values / target / behaviour probabilities and int32 actions [N,T]."""
    torch = _torch()
    N, T = rewards.shape
    A = q_values.shape[2]
    if actions.dtype != torch.int32 or not actions.is_cuda or not actions.is_contiguous() or tuple(actions.shape) != (N, T):
        raise TypeError("actions must be a contiguous CUDA int32 tensor of shape [N, T]")
    out = _out(rewards, q_targets)
    wp, wb = _ws(workspace)
    _check(lib().rlcs_retrace_probs(_ptr(rewards, "f32"), _ptr(q_values, "f32", (N, T, A)),
                                    _ptr(target_probs, "f32", (N, T, A)), _ptr(behaviour_probs, "f32", (N, T, A)),
                                    actions.data_ptr(), _ptr(dones, "u8", (N, T)), _ptr(truncs, "u8", (N, T)),
                                    _ptr(trunc_bootstrap, "f32", (N, T)), _ptr(bootstrap, "f32", (N,)),
                                    _ptr(out, "f32", (N, T)), N, T, A, gamma, lam, c_bar, wp, wb, _stream(stream)))
    return out


def rlcs_td_lambda(rewards, values, dones, truncs=None, trunc_bootstrap=None, bootstrap=None, *, gamma, lam,
                   returns=None, workspace=None, stream=None):
    N, T = rewards.shape
    out = _out(rewards, returns)
    wp, wb = _ws(workspace)
    _check(lib().rlcs_td_lambda(_ptr(rewards, "f32"), _ptr(values, "f32", (N, T)), _ptr(dones, "u8", (N, T)),
                                _ptr(truncs, "u8", (N, T)), _ptr(trunc_bootstrap, "f32", (N, T)),
                                _ptr(bootstrap, "f32", (N,)), _ptr(out, "f32", (N, T)), N, T, gamma, lam,
                                wp, wb, _stream(stream)))
    return out


def rlcs_discounted_return(rewards, dones, truncs=None, trunc_bootstrap=None, bootstrap=None, *, gamma,
                           returns=None, workspace=None, stream=None):
    N, T = rewards.shape
    out = _out(rewards, returns)
    wp, wb = _ws(workspace)
    _check(lib().rlcs_discounted_return(_ptr(rewards, "f32"), _ptr(dones, "u8", (N, T)), _ptr(truncs, "u8", (N, T)),
                                        _ptr(trunc_bootstrap, "f32", (N, T)), _ptr(bootstrap, "f32", (N,)),
                                        _ptr(out, "f32", (N, T)), N, T, gamma, wp, wb, _stream(stream)))
    return out


def rlcs_elig_trace(x, dones, *, gamma, lam, traces=None, workspace=None, stream=None):
    N, T = x.shape
    out = _out(x, traces)
    wp, wb = _ws(workspace)
    _check(lib().rlcs_elig_trace(_ptr(x, "f32"), _ptr(dones, "u8", (N, T)), _ptr(out, "f32", (N, T)), N, T,
                                 gamma, lam, wp, wb, _stream(stream)))
    return out


def rlcs_elig_trace_vec(x, dones, *, gamma, lam, traces=None, workspace=None, stream=None):
    """Vector-valued eligibility trace: x [N,T,D], dones [N,T].  A workspace is made on the fly when the
    time axis has to be cut and none is given."""
    N, T, D = x.shape
    out = _out(x, traces)
    if workspace is None:
        nbytes = int(lib().rlcs_elig_trace_vec_workspace_bytes(N, T, D))
        workspace = Workspace(N, T, device=x.device, stream=stream, nbytes=nbytes) if nbytes else None
    wp, wb = _ws(workspace)
    _check(lib().rlcs_elig_trace_vec(_ptr(x, "f32"), _ptr(dones, "u8", (N, T)), _ptr(out, "f32", (N, T, D)), N, T, D,
                                     gamma, lam, wp, wb, _stream(stream)))
    return out


def rlcs_elig_trace_vec_beta(x, beta, dones, *, traces=None, workspace=None, stream=None):
    """Eligibility trace with a decay per component and step: x, beta [N,T,D], dones [N,T]."""
    N, T, D = x.shape
    out = _out(x, traces)
    if workspace is None:
        nbytes = int(lib().rlcs_elig_trace_vec_beta_workspace_bytes(N, T, D))
        workspace = Workspace(N, T, device=x.device, stream=stream, nbytes=nbytes) if nbytes else None
    wp, wb = _ws(workspace)
    _check(lib().rlcs_elig_trace_vec_beta(_ptr(x, "f32"), _ptr(beta, "f32", (N, T, D)), _ptr(dones, "u8", (N, T)),
                                          _ptr(out, "f32", (N, T, D)), N, T, D, wp, wb, _stream(stream)))
    return out


def rlcs_episodic_prefix_sum(x, dones, *, starts_at=False, sums=None, workspace=None, stream=None):
    N, T = x.shape
    out = _out(x, sums)
    wp, wb = _ws(workspace)
    _check(lib().rlcs_episodic_prefix_sum(_ptr(x, "f32"), _ptr(dones, "u8", (N, T)), _ptr(out, "f32", (N, T)),
                                          N, T, int(bool(starts_at)), wp, wb, _stream(stream)))
    return out


def rlcs_affine_scan(alpha, beta, *, forward=False, out=None, workspace=None, stream=None):
    N, T = alpha.shape
    out = _out(alpha, out)
    wp, wb = _ws(workspace)
    _check(lib().rlcs_affine_scan(_ptr(alpha, "f32"), _ptr(beta, "f32", (N, T)), _ptr(out, "f32", (N, T)), N, T,
                                  int(bool(forward)), wp, wb, _stream(stream)))
    return out


def rlcs_debug_set_tile_variant(variant: int):
    _check(lib().rlcs_debug_set_tile_variant(variant))


def rlcs_debug_tile_elems(variant: int) -> int:
    return int(lib().rlcs_debug_tile_elems(variant))


ALGORITHM_IDS = {"gae": 0, "td_lambda": 1, "discounted_return": 2, "vtrace": 3, "retrace": 4, "elig_trace": 5,
                 "episodic_prefix_sum": 6}


def rlcs_debug_variant_for(algorithm: str, has_truncs: bool, N: int, T: int) -> dict:
    """The kernel variant a call would use, as {variant, threads, steps_per_thread, blocks_per_sm, ring_stages}."""
    v = int(lib().rlcs_debug_variant_for(ALGORITHM_IDS[algorithm], int(bool(has_truncs)), N, T))
    out = [ctypes.c_int() for _ in range(4)]
    _check(lib().rlcs_debug_variant_info(v, *[ctypes.byref(o) for o in out]))
    return dict(variant=v, threads=out[0].value, steps_per_thread=out[1].value, blocks_per_sm=out[2].value,
                ring_stages=out[3].value)


def rlcs_debug_set_row_blocks(mode: int = -1):
    """Test hook: one thread block per row: -1 = when there are enough rows (default), 0 = never, 1 = whenever legal."""
    _check(lib().rlcs_debug_set_row_blocks(int(mode)))


def rlcs_debug_allow_row_tiles(on: bool):
    """Test hook: allow (default) or forbid row-aligned tiling; without it short rows that do not divide the tile use the look-back."""
    _check(lib().rlcs_debug_allow_row_tiles(int(bool(on))))


def rlcs_debug_variant_built(variant: int) -> bool:
    """Whether that tile variant is compiled into the loaded library."""
    return bool(lib().rlcs_debug_variant_built(int(variant)))


def rlcs_debug_set_dependent_launch(on: bool):
    """Measurement hook: launch the row-major scan kernels with (default) or without programmatic stream serialisation."""
    _check(lib().rlcs_debug_set_dependent_launch(int(bool(on))))


def rlcs_debug_allow_cluster_carry(on: bool):
    _check(lib().rlcs_debug_allow_cluster_carry(int(bool(on))))


def rlcs_debug_force_wide_index(on: bool):
    _check(lib().rlcs_debug_force_wide_index(int(bool(on))))


def rlcs_debug_set_carry_fault(mute_tile: int = -1, spin_cap: int = 0):
    _check(lib().rlcs_debug_set_carry_fault(mute_tile, spin_cap))


def rlcs_debug_set_wait_polls(polls: int = -1):
    """Test hook: polls after which a wait of the policy-loss and attention kernels gives up (0: at once; negative: default)."""
    _check(lib().rlcs_debug_set_wait_polls(int(polls)))


def rlcs_debug_stream_copy(src, dst, read_bytes: int, write_bytes: int, stream=None):
    """Streaming read of read_bytes from src and write of write_bytes to dst (measurement hook)."""
    _check(lib().rlcs_debug_stream_copy(src.data_ptr(), dst.data_ptr(), int(read_bytes), int(write_bytes), _stream(stream)))


def rlcs_debug_vec_trace_plan(batch: int = 0, chunks: int = 0):
    """Test hook: force the load-ahead depth (8/16/32) and the number of time chunks of the vector traces."""
    lib().rlcs_debug_vec_trace_plan(int(batch), int(chunks))


def rlcs_debug_time_major_path(path: int = 0):
    """1 = register walk only; anything else = shared-memory ring wherever alignment allows (default)."""
    lib().rlcs_debug_time_major_path(int(path))


# ------------------------------------------------------------------------------------------ bfloat16 tensors
def _out16(like, out):
    torch = _torch()
    return _new(tuple(like.shape), torch.bfloat16, like.device) if out is None else out


def rlcs_gae_bf16(rewards, values, dones, truncs=None, trunc_bootstrap=None, bootstrap=None, *, gamma, lam,
                  advantages=None, returns=None, want_returns=True, workspace=None, stream=None):
    """GAE on bfloat16 tensors (fp32 arithmetic on chip, outputs rounded to bfloat16 on store)."""
    N, T = rewards.shape
    adv = _out16(rewards, advantages)
    ret = (_out16(rewards, returns) if want_returns else None)
    wp, wb = _ws(workspace)
    _check(lib().rlcs_gae_bf16(_ptr(rewards, "bf16"), _ptr(values, "bf16", (N, T)), _ptr(dones, "u8", (N, T)),
                               _ptr(truncs, "u8", (N, T)), _ptr(trunc_bootstrap, "bf16", (N, T)),
                               _ptr(bootstrap, "bf16", (N,)), _ptr(adv, "bf16", (N, T)), _ptr(ret, "bf16", (N, T)),
                               N, T, gamma, lam, wp, wb, _stream(stream)))
    return (adv, ret) if want_returns else adv


def rlcs_vtrace_bf16(rewards, values, log_rhos, dones, truncs=None, trunc_bootstrap=None, bootstrap=None, *,
                     gamma, rho_bar=1.0, c_bar=1.0, vs=None, pg_advantages=None, want_advantages=True,
                     workspace=None, stream=None):
    N, T = rewards.shape
    vs = _out16(rewards, vs)
    adv = (_out16(rewards, pg_advantages) if want_advantages else None)
    wp, wb = _ws(workspace)
    _check(lib().rlcs_vtrace_bf16(_ptr(rewards, "bf16"), _ptr(values, "bf16", (N, T)), _ptr(log_rhos, "bf16", (N, T)),
                                  _ptr(dones, "u8", (N, T)), _ptr(truncs, "u8", (N, T)),
                                  _ptr(trunc_bootstrap, "bf16", (N, T)), _ptr(bootstrap, "bf16", (N,)),
                                  _ptr(vs, "bf16", (N, T)), _ptr(adv, "bf16", (N, T)), N, T, gamma, rho_bar, c_bar,
                                  wp, wb, _stream(stream)))
    return (vs, adv) if want_advantages else vs


def rlcs_retrace_bf16(rewards, q_sa, expected_q, log_rhos, dones, truncs=None, trunc_bootstrap=None, bootstrap=None, *,
                      gamma, lam, c_bar=1.0, q_targets=None, workspace=None, stream=None):
    N, T = rewards.shape
    out = _out16(rewards, q_targets)
    wp, wb = _ws(workspace)
    _check(lib().rlcs_retrace_bf16(_ptr(rewards, "bf16"), _ptr(q_sa, "bf16", (N, T)), _ptr(expected_q, "bf16", (N, T)),
                                   _ptr(log_rhos, "bf16", (N, T)), _ptr(dones, "u8", (N, T)), _ptr(truncs, "u8", (N, T)),
                                   _ptr(trunc_bootstrap, "bf16", (N, T)), _ptr(bootstrap, "bf16", (N,)),
                                   _ptr(out, "bf16", (N, T)), N, T, gamma, lam, c_bar, wp, wb, _stream(stream)))
    return out


def rlcs_td_lambda_bf16(rewards, values, dones, truncs=None, trunc_bootstrap=None, bootstrap=None, *, gamma, lam,
                        returns=None, workspace=None, stream=None):
    N, T = rewards.shape
    out = _out16(rewards, returns)
    wp, wb = _ws(workspace)
    _check(lib().rlcs_td_lambda_bf16(_ptr(rewards, "bf16"), _ptr(values, "bf16", (N, T)), _ptr(dones, "u8", (N, T)),
                                     _ptr(truncs, "u8", (N, T)), _ptr(trunc_bootstrap, "bf16", (N, T)),
                                     _ptr(bootstrap, "bf16", (N,)), _ptr(out, "bf16", (N, T)), N, T, gamma, lam,
                                     wp, wb, _stream(stream)))
    return out


def rlcs_discounted_return_bf16(rewards, dones, truncs=None, trunc_bootstrap=None, bootstrap=None, *, gamma,
                                returns=None, workspace=None, stream=None):
    N, T = rewards.shape
    out = _out16(rewards, returns)
    wp, wb = _ws(workspace)
    _check(lib().rlcs_discounted_return_bf16(_ptr(rewards, "bf16"), _ptr(dones, "u8", (N, T)), _ptr(truncs, "u8", (N, T)),
                                             _ptr(trunc_bootstrap, "bf16", (N, T)), _ptr(bootstrap, "bf16", (N,)),
                                             _ptr(out, "bf16", (N, T)), N, T, gamma, wp, wb, _stream(stream)))
    return out


def rlcs_elig_trace_bf16(x, dones, *, gamma, lam, traces=None, workspace=None, stream=None):
    N, T = x.shape
    out = _out16(x, traces)
    wp, wb = _ws(workspace)
    _check(lib().rlcs_elig_trace_bf16(_ptr(x, "bf16"), _ptr(dones, "u8", (N, T)), _ptr(out, "bf16", (N, T)), N, T,
                                      gamma, lam, wp, wb, _stream(stream)))
    return out


def rlcs_episodic_prefix_sum_bf16(x, dones, *, starts_at=False, sums=None, workspace=None, stream=None):
    N, T = x.shape
    out = _out16(x, sums)
    wp, wb = _ws(workspace)
    _check(lib().rlcs_episodic_prefix_sum_bf16(_ptr(x, "bf16"), _ptr(dones, "u8", (N, T)), _ptr(out, "bf16", (N, T)),
                                               N, T, int(bool(starts_at)), wp, wb, _stream(stream)))
    return out


# ------------------------------------------------------------------------------------------ time-major [T, N] entry points
def _tm_ws(T, N, like, workspace, stream):
    if workspace is not None:
        return _ws(workspace)
    nbytes = int(lib().rlcs_time_major_workspace_bytes(N, T))
    if not nbytes:
        return None, 0
    # Scratch for this one call; it needs no initialisation.  Freed memory goes back to torch's caching
    # allocator, which reuses it in stream order on the allocating stream; a caller-chosen stream is
    # recorded on the buffer so that the same holds there.
    buf = _torch().empty(nbytes, dtype=_torch().uint8, device=like.device)
    if stream is not None:
        buf.record_stream(stream)
    return buf.data_ptr(), nbytes




def rlcs_gae_time_major(rewards, values, dones, truncs=None, trunc_bootstrap=None, bootstrap=None, *, gamma, lam,
                        advantages=None, returns=None, want_returns=True, workspace=None, stream=None):
    """GAE on [T, N] tensors (element (t, n) at t*N + n); bootstrap [N]."""
    T, N = rewards.shape
    adv = _out(rewards, advantages)
    ret = (_out(rewards, returns) if want_returns else None)
    wp, wb = _tm_ws(T, N, rewards, workspace, stream)
    _check(lib().rlcs_gae_time_major(_ptr(rewards, "f32"), _ptr(values, "f32", (T, N)), _ptr(dones, "u8", (T, N)),
                                     _ptr(truncs, "u8", (T, N)), _ptr(trunc_bootstrap, "f32", (T, N)),
                                     _ptr(bootstrap, "f32", (N,)), _ptr(adv, "f32", (T, N)), _ptr(ret, "f32", (T, N)),
                                     N, T, gamma, lam, wp, wb, _stream(stream)))
    return (adv, ret) if want_returns else adv


def rlcs_vtrace_time_major(rewards, values, log_rhos, dones, truncs=None, trunc_bootstrap=None, bootstrap=None, *,
                           gamma, rho_bar=1.0, c_bar=1.0, vs=None, pg_advantages=None, workspace=None, stream=None):
    T, N = rewards.shape
    vs, adv = _out(rewards, vs), _out(rewards, pg_advantages)
    wp, wb = _tm_ws(T, N, rewards, workspace, stream)
    _check(lib().rlcs_vtrace_time_major(_ptr(rewards, "f32"), _ptr(values, "f32", (T, N)), _ptr(log_rhos, "f32", (T, N)),
                                        _ptr(dones, "u8", (T, N)), _ptr(truncs, "u8", (T, N)),
                                        _ptr(trunc_bootstrap, "f32", (T, N)), _ptr(bootstrap, "f32", (N,)),
                                        _ptr(vs, "f32", (T, N)), _ptr(adv, "f32", (T, N)), N, T, gamma, rho_bar, c_bar,
                                        wp, wb, _stream(stream)))
    return vs, adv


def rlcs_retrace_time_major(rewards, q_sa, expected_q, log_rhos, dones, truncs=None, trunc_bootstrap=None,
                            bootstrap=None, *, gamma, lam, c_bar=1.0, q_targets=None, workspace=None, stream=None):
    T, N = rewards.shape
    out = _out(rewards, q_targets)
    wp, wb = _tm_ws(T, N, rewards, workspace, stream)
    _check(lib().rlcs_retrace_time_major(_ptr(rewards, "f32"), _ptr(q_sa, "f32", (T, N)), _ptr(expected_q, "f32", (T, N)),
                                         _ptr(log_rhos, "f32", (T, N)), _ptr(dones, "u8", (T, N)),
                                         _ptr(truncs, "u8", (T, N)), _ptr(trunc_bootstrap, "f32", (T, N)),
                                         _ptr(bootstrap, "f32", (N,)), _ptr(out, "f32", (T, N)), N, T, gamma, lam, c_bar,
                                         wp, wb, _stream(stream)))
    return out


def rlcs_td_lambda_time_major(rewards, values, dones, truncs=None, trunc_bootstrap=None, bootstrap=None, *, gamma, lam,
                              returns=None, workspace=None, stream=None):
    T, N = rewards.shape
    out = _out(rewards, returns)
    wp, wb = _tm_ws(T, N, rewards, workspace, stream)
    _check(lib().rlcs_td_lambda_time_major(_ptr(rewards, "f32"), _ptr(values, "f32", (T, N)), _ptr(dones, "u8", (T, N)),
                                           _ptr(truncs, "u8", (T, N)), _ptr(trunc_bootstrap, "f32", (T, N)),
                                           _ptr(bootstrap, "f32", (N,)), _ptr(out, "f32", (T, N)), N, T, gamma, lam,
                                           wp, wb, _stream(stream)))
    return out


def rlcs_discounted_return_time_major(rewards, dones, truncs=None, trunc_bootstrap=None, bootstrap=None, *, gamma,
                                      returns=None, workspace=None, stream=None):
    T, N = rewards.shape
    out = _out(rewards, returns)
    wp, wb = _tm_ws(T, N, rewards, workspace, stream)
    _check(lib().rlcs_discounted_return_time_major(_ptr(rewards, "f32"), _ptr(dones, "u8", (T, N)),
                                                   _ptr(truncs, "u8", (T, N)), _ptr(trunc_bootstrap, "f32", (T, N)),
                                                   _ptr(bootstrap, "f32", (N,)), _ptr(out, "f32", (T, N)), N, T, gamma,
                                                   wp, wb, _stream(stream)))
    return out


def rlcs_elig_trace_time_major(x, dones, *, gamma, lam, traces=None, workspace=None, stream=None):
    T, N = x.shape
    out = _out(x, traces)
    wp, wb = _tm_ws(T, N, x, workspace, stream)
    _check(lib().rlcs_elig_trace_time_major(_ptr(x, "f32"), _ptr(dones, "u8", (T, N)), _ptr(out, "f32", (T, N)), N, T,
                                            gamma, lam, wp, wb, _stream(stream)))
    return out


def rlcs_episodic_prefix_sum_time_major(x, dones, *, starts_at=False, sums=None, workspace=None, stream=None):
    T, N = x.shape
    out = _out(x, sums)
    wp, wb = _tm_ws(T, N, x, workspace, stream)
    _check(lib().rlcs_episodic_prefix_sum_time_major(_ptr(x, "f32"), _ptr(dones, "u8", (T, N)), _ptr(out, "f32", (T, N)),
                                                     N, T, int(bool(starts_at)), wp, wb, _stream(stream)))
    return out


# ------------------------------------------------------------------ rollout and policy operators
def _on_stream(wrapper):
    """stream= makes that stream current for the whole call: what the call allocates then belongs to the stream that writes it, and
    is not handed out again, or taken from a pending use, in another stream's order.  (Inputs of another stream stay the caller's
    to order and to record.)"""
    @functools.wraps(wrapper)
    def call(*args, stream=None, **kwargs):
        if stream is None:
            return wrapper(*args, **kwargs)
        with _torch().cuda.stream(stream):
            return wrapper(*args, stream=stream, **kwargs)
    return call


_KINDS = {"f32": "float32", "bf16": "bfloat16", "i32": "int32", "i64": "int64"}
_dtypes: dict = {}


def _dtype(kind: str):
    dt = _dtypes.get(kind)
    if dt is None:
        dt = _dtypes[kind] = getattr(_torch(), _KINDS[kind])
    return dt


def _device_for(t) -> int:
    """The current device, once the call's first tensor is known to be a CUDA tensor."""
    if not t.is_cuda:
        raise TypeError("rlcs takes CUDA tensors (device pointers); there is no CPU path")
    return _current_device()


def _refuse(t, kind, shape, what):
    """Says why _typed() or _rows() does not take a tensor."""
    if not t.is_cuda:
        raise TypeError("rlcs takes CUDA tensors (device pointers); there is no CPU path")
    _require_current_device(t, what)
    if t.dtype != _dtype(kind):
        raise TypeError(f"expected {_KINDS[kind]} for {what}, got {t.dtype}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"expected shape {tuple(shape)} for {what}, got {tuple(t.shape)}")
    raise ValueError(f"{what} must be contiguous")


def _typed(t, kind: str, shape, what: str, device: int):
    """Pointer of a contiguous tensor of one of _KINDS on the current device (None -> NULL)."""
    if t is None:
        return None
    if not (t.dtype == _dtype(kind) and t.is_cuda and t.get_device() == device and t.is_contiguous()
            and (shape is None or t.shape == shape)):
        _refuse(t, kind, shape, what)
    return t.data_ptr()


def _output(t, kind: str, shape, what: str, device: int):
    """(tensor, pointer) of an output: the caller's, checked, or a new one on the current device."""
    if t is None:
        t = _alloc(shape, _dtype(kind), device)
        if _preparing:
            _held(t)
        return t, t.data_ptr()
    return t, _typed(t, kind, shape, what, device)


def _rows(t, kind: str, what: str, device: int, shape=None):
    """(pointer, row stride) of a 2-D tensor whose rows are contiguous and do not overlap."""
    if not (t.dtype == _dtype(kind) and t.is_cuda and t.get_device() == device and (shape is None or t.shape == shape)):
        _refuse(t, kind, shape, what)
    if t.dim() != 2:
        raise ValueError(f"{what} must be 2-D [rows, actions]")
    R, A = t.shape
    ld = t.stride(0) if R > 1 else max(A, 1)
    if (A > 1 and t.stride(1) != 1) or ld < A:
        raise ValueError(f"rows of {what} must be contiguous and must not overlap")
    return t.data_ptr(), ld


def _per_row(value, kind: str, shape, default, what: str, device: int):
    """A per-row parameter: (pointer, unused) for an [R] tensor, (NULL, value) for a number or None."""
    if value is None:
        return None, default
    if isinstance(value, (int, float)):
        return None, value
    return _typed(value, kind, shape, what, device), default


def _sample_actions(name, kind, logits, uniforms, temperature, top_k, top_p, min_p, actions, log_probs, kept_log_probs, stream):
    dev = _device_for(logits)
    ptr, ld = _rows(logits, kind, "logits", dev)
    R, A = logits.shape
    n = (R,)
    t, t_all = _per_row(temperature, "f32", n, 1.0, "temperature", dev)
    k, k_all = _per_row(top_k, "i32", n, 0, "top_k", dev)
    p, p_all = _per_row(top_p, "f32", n, 1.0, "top_p", dev)
    m, m_all = _per_row(min_p, "f32", n, 0.0, "min_p", dev)
    a, ap = _output(actions, "i32", n, "actions", dev)
    lp, lpp = _output(log_probs, "f32", n, "log_probs", dev)
    kp, kpp = _output(kept_log_probs, "f32", n, "kept_log_probs", dev)
    _check(getattr(lib(), name)(ptr, ld, _typed(uniforms, "f32", n, "uniforms", dev), t, k, p, m, t_all, max(0, min(int(k_all), 2 ** 31 - 1)),
                                p_all, m_all, ap, lpp, kpp, R, A, _stream(stream)))
    return a, lp, kp


@_on_stream
def rlcs_sample_actions(logits, uniforms, *, temperature=None, top_k=None, top_p=None, min_p=None, actions=None, log_probs=None,
                        kept_log_probs=None, stream=None):
    """Actions drawn from float32 logits [R, A] (rows may be strided) with one uniform a row; temperature, top_k (int32), top_p
    and min_p are numbers or [R] tensors.  Returns (actions int32, log_probs, kept_log_probs), all [R]."""
    return _sample_actions("rlcs_sample_actions", "f32", logits, uniforms, temperature, top_k, top_p, min_p, actions, log_probs,
                           kept_log_probs, stream)


@_on_stream
def rlcs_sample_actions_bf16(logits, uniforms, *, temperature=None, top_k=None, top_p=None, min_p=None, actions=None, log_probs=None,
                             kept_log_probs=None, stream=None):
    """rlcs_sample_actions on bfloat16 logits."""
    return _sample_actions("rlcs_sample_actions_bf16", "bf16", logits, uniforms, temperature, top_k, top_p, min_p, actions, log_probs,
                           kept_log_probs, stream)


def _policy_grad(name, kind, logits, actions, advantages, old_log_probs, mask, temperature, clip, entropy_coef, scale, want_grad,
                 loss, log_probs, entropy, dlogits, stream):
    dev = _device_for(logits)
    ptr, ld = _rows(logits, kind, "logits", dev)
    R, A = logits.shape
    n = (R,)
    lp, lpp = _output(log_probs, "f32", n, "log_probs", dev)
    ent, entp = _output(entropy, "f32", n, "entropy", dev)
    dptr, ldd, lossp = None, 0, None
    if advantages is None:
        if old_log_probs is not None or loss is not None or dlogits is not None:
            raise ValueError("old_log_probs, loss and dlogits go with advantages")
    else:
        loss, lossp = _output(loss, "f32", n, "loss", dev)
        if dlogits is not None:
            dptr, ldd = _rows(dlogits, kind, "dlogits", dev, (R, A))
        elif want_grad:
            dlogits, ldd = _gradient_like(logits, ptr, ld, dev)
            dptr = dlogits.data_ptr()
    _check(getattr(lib(), name)(ptr, ld, _typed(actions, "i32", n, "actions", dev), _ptr(mask, "u8", n),
                                _typed(advantages, "f32", n, "advantages", dev), _typed(old_log_probs, "f32", n, "old_log_probs", dev),
                                lossp, lpp, entp, dptr, ldd, R, A, temperature, clip, entropy_coef, scale,
                                _stream(stream)))
    if advantages is None:
        return lp, ent
    return (loss, lp, ent, dlogits) if dlogits is not None else (loss, lp, ent)


@_on_stream
def rlcs_policy_grad(logits, actions, advantages=None, *, old_log_probs=None, mask=None, temperature=1.0, clip=0.2, entropy_coef=0.0,
                     scale=1.0, want_grad=True, loss=None, log_probs=None, entropy=None, dlogits=None, stream=None):
    """Policy loss of float32 logits [R, A] (rows may be strided) and its gradient: (loss, log_probs, entropy, dlogits), without
    dlogits if want_grad is False, and (log_probs, entropy) alone without advantages.  dlogits may be logits itself."""
    return _policy_grad("rlcs_policy_grad", "f32", logits, actions, advantages, old_log_probs, mask, temperature, clip, entropy_coef,
                        scale, want_grad, loss, log_probs, entropy, dlogits, stream)


@_on_stream
def rlcs_policy_grad_bf16(logits, actions, advantages=None, *, old_log_probs=None, mask=None, temperature=1.0, clip=0.2,
                          entropy_coef=0.0, scale=1.0, want_grad=True, loss=None, log_probs=None, entropy=None, dlogits=None,
                          stream=None):
    """rlcs_policy_grad on bfloat16 logits (dlogits bfloat16, the per-row outputs float32)."""
    return _policy_grad("rlcs_policy_grad_bf16", "bf16", logits, actions, advantages, old_log_probs, mask, temperature, clip,
                        entropy_coef, scale, want_grad, loss, log_probs, entropy, dlogits, stream)


_attention_bytes: dict = {}            # workspace bytes by sizes


@_on_stream
def rlcs_prefix_attention_bf16(q, k_cache, v_cache, prefix_table, prefix_lens, group_offsets, block_table, lens, *, scale,
                               max_prefix_len=None, max_len=None, want_lse=True, out=None, lse=None, workspace=None, stream=None):
    """One query a row over its group's paged prefix and its own pages.  q [B, H, d] (rows may be strided), caches
    [pages, page, Hk, d] (any strides with contiguous d), tables and lengths int32; prefix_table, prefix_lens and group_offsets
    None: no prefixes.  Returns (out, lse), or out without lse."""
    if q.dim() != 3 or k_cache.dim() != 4 or v_cache.shape != k_cache.shape:
        raise ValueError("expected q [B, H, d] and caches [pages, page, Hk, d] of one shape")
    dev = _device_for(q)
    for t, what in ((q, "q"), (k_cache, "k_cache"), (v_cache, "v_cache")):
        if not (t.dtype == _dtype("bf16") and t.is_cuda and t.get_device() == dev):
            _refuse(t, "bf16", None, what)
    B, H, d = q.shape
    pages, page, Hk, dk = k_cache.shape
    sq, sk = q.stride(), k_cache.stride()
    if dk != d or (d > 1 and sq[2] != 1) or (H > 1 and sq[1] != d) or sk[3] != 1:
        raise ValueError("q and the caches must agree in d, with heads of q and d of both contiguous")
    if sk != v_cache.stride():
        raise ValueError("k_cache and v_cache must have the same strides")
    if (prefix_table is None) != (prefix_lens is None) or (prefix_table is None) != (group_offsets is None):
        raise ValueError("prefix_table, prefix_lens and group_offsets go together")
    groups, prefix_width = (0, 0) if prefix_table is None else prefix_table.shape
    own_width = block_table.shape[1]
    mp = prefix_width * page if max_prefix_len is None else min(int(max_prefix_len), prefix_width * page)
    ml = own_width * page if max_len is None else min(int(max_len), own_width * page)
    out, outp = _output(out, "bf16", (B, H, d), "out", dev)
    lsep = None
    if lse is not None or want_lse:
        lse, lsep = _output(lse, "f32", (B, H), "lse", dev)
    if workspace is None or callable(workspace):
        sizes = (B, H, Hk, d, page, groups, mp, ml)
        need = _attention_bytes.get(sizes)
        if need is None:
            if len(_attention_bytes) >= 4096:
                _attention_bytes.clear()
            need = _attention_bytes[sizes] = int(lib().rlcs_prefix_attention_workspace_bytes(*sizes))
    if workspace is None:
        workspace, room = _new((max(need, 16),), _torch().uint8, dev), max(need, 16)
    else:
        if callable(workspace):
            workspace = _held(workspace(need))
        if not getattr(workspace, "is_cuda", False):
            raise TypeError("workspace must be a CUDA tensor")
        if workspace.get_device() != dev:
            _require_current_device(workspace, "workspace")
        if not workspace.is_contiguous():
            raise ValueError("workspace must be contiguous")
        room = workspace.numel() * workspace.element_size()
    _check(lib().rlcs_prefix_attention_bf16(
        q.data_ptr(), sq[0] if B > 1 else H * d, k_cache.data_ptr(), v_cache.data_ptr(), pages, sk[0], sk[1], sk[2],
        _typed(prefix_table, "i32", (groups, prefix_width), "prefix_table", dev), prefix_width,
        _typed(prefix_lens, "i32", (groups,), "prefix_lens", dev), _typed(group_offsets, "i32", (groups + 1,), "group_offsets", dev),
        _typed(block_table, "i32", (B, own_width), "block_table", dev), own_width, _typed(lens, "i32", (B,), "lens", dev),
        outp, lsep, B, H, Hk, d, page, groups, mp, ml, scale,
        workspace.data_ptr(), room, _stream(stream)))
    return out if lse is None else (out, lse)


@_on_stream
def rlcs_block_tables(cached, added, free_pages, block_table, *, page_size, num_slots, slots=None, positions=None, offsets=None,
                      page_offsets=None, stream=None):
    """One step's page tables (block_table [B, width], in place), slot map and positions from int32 lengths on the GPU.  Returns
    (slots int64 [num_slots], positions int32 [num_slots], offsets int32 [B + 1], page_offsets int32 [B + 1])."""
    if cached.dim() != 1 or free_pages.dim() != 1 or block_table.dim() != 2:
        raise ValueError("expected cached [B], free_pages [F], block_table [B, width]")
    B, width = block_table.shape
    dev = _device_for(cached)
    slots, sp = _output(slots, "i64", (num_slots,), "slots", dev)
    positions, pp = _output(positions, "i32", (num_slots,), "positions", dev)
    offsets, op = _output(offsets, "i32", (B + 1,), "offsets", dev)
    page_offsets, gp = _output(page_offsets, "i32", (B + 1,), "page_offsets", dev)
    _check(lib().rlcs_block_tables(
        _typed(cached, "i32", (B,), "cached", dev), _typed(added, "i32", (B,), "added", dev),
        _typed(free_pages, "i32", None, "free_pages", dev), _typed(block_table, "i32", None, "block_table", dev),
        sp, pp, op, gp, B, width, free_pages.shape[0], num_slots, page_size, _stream(stream)))
    return slots, positions, offsets, page_offsets


# ------------------------------------------------------------------ speculative rollouts and distillation
_scratch_bytes: dict = {}              # workspace bytes by entry point, device and sizes


def _scratch(query: str, sizes, workspace, device: int):
    """(pointer, bytes, tensor) of a call's workspace: the caller's, checked, or one of the call's own from torch's allocator."""
    if workspace is None:
        key = (query, device, *sizes)
        need = _scratch_bytes.get(key)
        if need is None:
            if len(_scratch_bytes) >= 4096:
                _scratch_bytes.clear()
            need = _scratch_bytes[key] = int(getattr(lib(), query)(*sizes))
        if need == 0:
            return None, 0, None
        workspace = _new((need,), _torch().uint8, device)
        return workspace.data_ptr(), need, workspace
    if not getattr(workspace, "is_cuda", False):
        raise TypeError("workspace must be a CUDA tensor")
    if workspace.get_device() != device:
        _require_current_device(workspace, "workspace")
    if not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size(), workspace


def _caches(k_cache, v_cache, device: int):
    """Strides of a pair of caches [pages, page, Hk, d] whose rows of d are contiguous."""
    if k_cache.dim() != 4 or (v_cache is not None and v_cache.shape != k_cache.shape):
        raise ValueError("expected caches [pages, page, Hk, d] of one shape")
    bf16 = _dtype("bf16")
    if k_cache.dtype != bf16 or k_cache.get_device() != device:
        _refuse(k_cache, "bf16", None, "k_cache")
    if v_cache is not None and (v_cache.dtype != bf16 or v_cache.get_device() != device):
        _refuse(v_cache, "bf16", None, "v_cache")
    s = k_cache.stride()
    if s[3] != 1:
        raise ValueError("d of the caches must be contiguous")
    if v_cache is not None and v_cache.stride() != s:
        raise ValueError("k_cache and v_cache must have the same strides")
    return s


@_on_stream
def rlcs_chunk_attention_bf16(q, k_cache, v_cache, block_table, offsets, lens, *, scale, max_new=None, max_len=None, want_lse=True,
                              out=None, lse=None, workspace=None, stream=None):
    """Queries of chunks of new tokens, q [T, H, d] (tokens may be strided), over their trajectories' paged keys up to their own: tokens
    offsets[b] to offsets[b+1]-1 are the last of the lens[b] tokens in the pages block_table[b].  Caches as for
    rlcs_prefix_attention_bf16.  Returns (out, lse), or out without lse; tokens outside every trajectory are not written."""
    if q.dim() != 3 or block_table.dim() != 2:
        raise ValueError("expected q [T, H, d] and block_table [B, width]")
    dev = _device_for(q)
    if not (q.dtype == _dtype("bf16") and q.get_device() == dev):
        _refuse(q, "bf16", None, "q")
    sk = _caches(k_cache, v_cache, dev)
    T, H, d = q.shape
    pages, page, Hk, dk = k_cache.shape
    sq = q.stride()
    if dk != d or (d > 1 and sq[2] != 1) or (H > 1 and sq[1] != d):
        raise ValueError("q and the caches must agree in d, with heads of q contiguous")
    B, width = block_table.shape
    mn = T if max_new is None else min(int(max_new), T)
    ml = width * page if max_len is None else min(int(max_len), width * page)
    out, outp = _output(out, "bf16", (T, H, d), "out", dev)
    lsep = None
    if lse is not None or want_lse:
        lse, lsep = _output(lse, "f32", (T, H), "lse", dev)
    wp, room, workspace = _scratch("rlcs_chunk_attention_workspace_bytes", (T, B, H, Hk, d, page, mn, ml), workspace, dev)
    _check(lib().rlcs_chunk_attention_bf16(
        q.data_ptr(), sq[0] if T > 1 else H * d, k_cache.data_ptr(), v_cache.data_ptr(), pages, sk[0], sk[1], sk[2],
        _typed(block_table, "i32", (B, width), "block_table", dev), width, _typed(offsets, "i32", (B + 1,), "offsets", dev),
        _typed(lens, "i32", (B,), "lens", dev), outp, lsep, T, B, H, Hk, d, page, mn, ml, scale, wp, room, _stream(stream)))
    return out if lse is None else (out, lse)


def _verify_drafts(name, kind, logits, tokens, offsets, uniforms, draw_uniforms, draft_logits, temperature, out_tokens, log_probs, accepted,
                   workspace, stream):
    dev = _device_for(logits)
    ptr, ld = _rows(logits, kind, "logits", dev)
    T, A = logits.shape
    dptr, ldd = (None, 0) if draft_logits is None else _rows(draft_logits, kind, "draft_logits", dev, (T, A))
    if offsets.dim() != 1 or offsets.shape[0] < 1:
        raise ValueError("expected offsets [B + 1]")
    B = offsets.shape[0] - 1
    t, t_all = _per_row(temperature, "f32", (B,), 1.0, "temperature", dev)
    out, outp = _output(out_tokens, "i32", (T,), "out_tokens", dev)
    lp, lpp = _output(log_probs, "f32", (T,), "log_probs", dev)
    acc, accp = _output(accepted, "i32", (B,), "accepted", dev)
    wp, room, workspace = _scratch("rlcs_verify_drafts_workspace_bytes", (T, B), workspace, dev)
    _check(getattr(lib(), name)(ptr, ld, dptr, ldd, _typed(tokens, "i32", (T,), "tokens", dev), _typed(offsets, "i32", (B + 1,), "offsets", dev),
                                _typed(uniforms, "f32", (T,), "uniforms", dev), _typed(draw_uniforms, "f32", (B,), "draw_uniforms", dev),
                                t, t_all, outp, lpp, accp, T, B, A, wp, room, _stream(stream)))
    return out, lp, acc


@_on_stream
def rlcs_verify_drafts(logits, tokens, offsets, uniforms, draw_uniforms, *, draft_logits=None, temperature=None, out_tokens=None,
                       log_probs=None, accepted=None, workspace=None, stream=None):
    """Drafts tokens[t+1] against the target's float32 logits [T, A] (rows may be strided), trajectory b in rows offsets[b] to
    offsets[b+1]-1; temperature is a number or one a trajectory.  Returns (out_tokens int32 [T], log_probs [T], accepted int32 [B])."""
    return _verify_drafts("rlcs_verify_drafts", "f32", logits, tokens, offsets, uniforms, draw_uniforms, draft_logits, temperature, out_tokens,
                          log_probs, accepted, workspace, stream)


@_on_stream
def rlcs_verify_drafts_bf16(logits, tokens, offsets, uniforms, draw_uniforms, *, draft_logits=None, temperature=None, out_tokens=None,
                            log_probs=None, accepted=None, workspace=None, stream=None):
    """rlcs_verify_drafts on bfloat16 logits."""
    return _verify_drafts("rlcs_verify_drafts_bf16", "bf16", logits, tokens, offsets, uniforms, draw_uniforms, draft_logits, temperature,
                          out_tokens, log_probs, accepted, workspace, stream)


def _gradient_like(logits, ptr: int, ld: int, device: int):
    """A gradient for logits [R, A]: rows as far apart, and as far from a 16-byte boundary, as theirs where that costs little memory, so
    that both are walked in whole vectors (rows of up to 64 actions leave as one block of memory, which wants them close together)."""
    R, A = logits.shape
    ldd, lead = (ld, ptr % 16 // logits.element_size()) if A > 64 and ld - A <= A // 8 + 16 else (A, 0)
    if ldd == A and lead == 0:
        return _new((R, A), logits.dtype, device), ldd
    flat = _new((R * ldd + lead,), logits.dtype, device)
    return flat.as_strided((R, A), (ldd, 1), flat.storage_offset() + lead), ldd


def _distill_grad(name, kind, logits, teacher_ids, teacher_logits, mask, temperature, scale, want_grad, loss, dlogits, stream):
    dev = _device_for(logits)
    ptr, ld = _rows(logits, kind, "logits", dev)
    R, A = logits.shape
    if teacher_ids.dim() != 2:
        raise ValueError("expected teacher_ids and teacher_logits [rows, K]")
    K = teacher_ids.shape[1]
    loss, lossp = _output(loss, "f32", (R,), "loss", dev)
    dptr, ldd = None, 0
    if dlogits is not None:
        dptr, ldd = _rows(dlogits, kind, "dlogits", dev, (R, A))
    elif want_grad:
        dlogits, ldd = _gradient_like(logits, ptr, ld, dev)
        dptr = dlogits.data_ptr()
    _check(getattr(lib(), name)(ptr, ld, _typed(teacher_ids, "i32", (R, K), "teacher_ids", dev),
                                _typed(teacher_logits, "f32", (R, K), "teacher_logits", dev), _ptr(mask, "u8", (R,)), lossp, dptr, ldd, R, A, K,
                                temperature, scale, _stream(stream)))
    return loss if dlogits is None else (loss, dlogits)


@_on_stream
def rlcs_distill_grad(logits, teacher_ids, teacher_logits, *, mask=None, temperature=1.0, scale=1.0, want_grad=True, loss=None, dlogits=None,
                      stream=None):
    """Loss of float32 student logits [R, A] (rows may be strided) towards a teacher's logits [R, K] of teacher_ids [R, K] (int32; outside
    [0, A): absent) and its gradient: (loss, dlogits), or loss alone if want_grad is False.  dlogits may be logits itself."""
    return _distill_grad("rlcs_distill_grad", "f32", logits, teacher_ids, teacher_logits, mask, temperature, scale, want_grad, loss, dlogits, stream)


@_on_stream
def rlcs_distill_grad_bf16(logits, teacher_ids, teacher_logits, *, mask=None, temperature=1.0, scale=1.0, want_grad=True, loss=None,
                           dlogits=None, stream=None):
    """rlcs_distill_grad on bfloat16 logits (dlogits bfloat16; loss and teacher float32)."""
    return _distill_grad("rlcs_distill_grad_bf16", "bf16", logits, teacher_ids, teacher_logits, mask, temperature, scale, want_grad, loss, dlogits,
                         stream)


@_on_stream
def rlcs_fork_block_tables(block_table, lens, sources, free_pages, *, page_size, new_table=None, copy_from=None, copy_to=None, pages_used=None,
                           workspace=None, stream=None):
    """Page tables of rows that continue rows `sources` [N] of block_table [B, width]: whole pages shared, part-filled last ones copied
    for all but the first row that ends in them (for all that do, where another new row has the page whole).  Returns (new_table [N, width], copy_from [N], copy_to [N], pages_used [1])."""
    if block_table.dim() != 2 or sources.dim() != 1 or free_pages.dim() != 1:
        raise ValueError("expected block_table [B, width], sources [N], free_pages [F]")
    dev = _device_for(block_table)
    B, width = block_table.shape
    N = sources.shape[0]
    new_table, tp = _output(new_table, "i32", (N, width), "new_table", dev)
    copy_from, fp = _output(copy_from, "i32", (N,), "copy_from", dev)
    copy_to, cp = _output(copy_to, "i32", (N,), "copy_to", dev)
    pages_used, up = _output(pages_used, "i32", (1,), "pages_used", dev)
    old = _typed(block_table, "i32", None, "block_table", dev)
    if N * width and tp == old:
        raise ValueError("new_table must not be block_table")
    wp, room, workspace = _scratch("rlcs_fork_block_tables_workspace_bytes", (B, N), workspace, dev)
    _check(lib().rlcs_fork_block_tables(old, _typed(lens, "i32", (B,), "lens", dev), _typed(sources, "i32", None, "sources", dev),
                                        _typed(free_pages, "i32", None, "free_pages", dev), tp, fp, cp, up, B, N, width, free_pages.shape[0],
                                        page_size, wp, room, _stream(stream)))
    return new_table, copy_from, copy_to, pages_used


@_on_stream
def rlcs_copy_pages_bf16(k_cache, v_cache, copy_from, copy_to, *, stream=None):
    """Pages copy_from[i] -> copy_to[i] (int32; negative: none) copied within k_cache and v_cache (None: keys alone)."""
    if copy_from.dim() != 1:
        raise ValueError("expected copy_from [N] and copy_to [N]")
    dev = _device_for(k_cache)
    s = _caches(k_cache, v_cache, dev)
    pages, page, Hk, d = k_cache.shape
    n = copy_from.shape[0]
    _check(lib().rlcs_copy_pages_bf16(k_cache.data_ptr(), None if v_cache is None else v_cache.data_ptr(), pages, s[0], s[1], s[2],
                                      _typed(copy_from, "i32", (n,), "copy_from", dev), _typed(copy_to, "i32", (n,), "copy_to", dev), n, page, Hk,
                                      d, _stream(stream)))
    return k_cache if v_cache is None else (k_cache, v_cache)


@_on_stream
def rlcs_free_pages(block_table, lens, prefix_table=None, prefix_lens=None, *, num_pages, page_size, free_pages=None, free_count=None,
                    workspace=None, stream=None):
    """The pages below num_pages that no row of block_table [B, width] (lens [B]) or prefix_table (prefix_lens) names, ascending:
    (free_pages int32 [num_pages], -1 behind the last, free_count int32 [1])."""
    if block_table.dim() != 2 or (prefix_table is None) != (prefix_lens is None) or (prefix_table is not None and prefix_table.dim() != 2):
        raise ValueError("expected block_table [B, width], and prefix_table [groups, width] with prefix_lens or neither")
    dev = _device_for(block_table)
    B, width = block_table.shape
    groups, prefix_width = (0, 0) if prefix_table is None else prefix_table.shape
    free_pages, fp = _output(free_pages, "i32", (num_pages,), "free_pages", dev)
    free_count, cp = _output(free_count, "i32", (1,), "free_count", dev)
    wp, room, workspace = _scratch("rlcs_free_pages_workspace_bytes", (num_pages,), workspace, dev)
    _check(lib().rlcs_free_pages(_typed(block_table, "i32", None, "block_table", dev), _typed(lens, "i32", (B,), "lens", dev),
                                 _typed(prefix_table, "i32", None, "prefix_table", dev), _typed(prefix_lens, "i32", (groups,), "prefix_lens", dev),
                                 fp, cp, B, width, groups, prefix_width, num_pages, page_size, wp, room, _stream(stream)))
    return free_pages, free_count
