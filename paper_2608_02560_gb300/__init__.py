"""PRECOG hot path on GB300: Python binding of the C-ABI library ``libprecog.so``.

Thin ctypes marshalling only: every step of the path (scan with state capture,
top-1 retrieval, state injection and query prefill) runs in the library's CUDA
kernels. PyTorch tensors are accepted for device memory and the current CUDA
stream; nothing here computes. If the library is missing the import fails
loudly: there is no CPU fallback.

Functions carry the C names:

* :func:`precog_encode_chunks`    -- offline indexing (Sec. 4.2)
* :func:`precog_encode_chunks_ordered` -- the same, chunks taken up in a given order
* :func:`precog_encode_trajectory` -- K-dial trajectory capture (Sec. 5.2)
* :func:`precog_retrieve`         -- exact top-1 retrieval (Sec. 4.2)
* :func:`precog_prefill_from_state` -- injection (Eq. 2) + query prefill
* :func:`precog_retrieve_topk`    -- top-k retrieval (Sec. 4.2 / 5.4)
* :func:`precog_retrieve_keys`, :func:`precog_decode_keys` -- row-sharded retrieval
* :func:`precog_prefill_composed` -- softmax-weighted top-k injection (Sec. 4.4) + prefill
* :func:`precog_smc_route`, :func:`precog_smc_consolidate` -- SMC (Sec. 5)
* :func:`precog_delta_scan`, :func:`precog_delta_step` -- the gated delta rule: chunks or queries
  from injected matrix states, and one token of each sequence on a table of states
* :func:`precog_qk_norm_rope`     -- norms of query and key heads with the position rotation
* :func:`precog_token_logprobs`   -- log probabilities of given tokens, entropy, best entries
* :func:`precog_causal_conv`, :func:`precog_conv_step` -- the short causal convolution in front of a
  scan: chunks or queries from injected windows, and one token of each sequence
* :func:`precog_scan_step`        -- one token of the diagonal scan of each sequence on a table of states
* :func:`precog_block_norm`       -- skip, gate, norm and residual at the end of a block, the next one's norm
* :func:`precog_adjust_logits`    -- penalties for repeated tokens, biases and grammar masks on logits
* :func:`precog_retrieve_noalloc`  -- top-1 retrieval without a caller workspace
* :func:`precog_device_status`    -- device-side status word; :func:`precog_status_string`,
  :func:`precog_last_error`, :func:`precog_abi_version`, :func:`precog_launch_count`
"""
from __future__ import annotations

import ctypes
import os
import struct

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libprecog.so")

PRECOG_F32, PRECOG_BF16, PRECOG_F16 = 0, 1, 2
PRECOG_OK = 0
PRECOG_NORM_NONE, PRECOG_NORM_L2, PRECOG_NORM_RMS = 0, 1, 2
PRECOG_A_GENERAL, PRECOG_A_POWER, PRECOG_A_COMPLEX = 0, 1, 2
PRECOG_DEV_BAD_OFFSETS, PRECOG_DEV_BAD_INDEX, PRECOG_DEV_TIMEOUT, PRECOG_DEV_BAD_A = 0x1, 0x2, 0x4, 0x8
STATUS_NAMES = {0: "PRECOG_OK", 1: "PRECOG_ERR_INVALID_ARG", 2: "PRECOG_ERR_UNSUPPORTED",
                3: "PRECOG_ERR_CUDA", 4: "PRECOG_ERR_TIMEOUT", 5: "PRECOG_ERR_DEVICE"}


class PrecogError(RuntimeError):
    def __init__(self, status: int, detail: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {detail}")
        self.status = status
        self.detail = detail


class ScanInputs(ctypes.Structure):
    """Mirror of ``precog_scan_inputs`` (include/precog.h)."""
    _fields_ = [("n_layers", ctypes.c_int32), ("D", ctypes.c_int32), ("N", ctypes.c_int32),
                ("in_dtype", ctypes.c_int32), ("a_kind", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("x", ctypes.c_void_p), ("dt", ctypes.c_void_p),
                ("B", ctypes.c_void_p), ("C", ctypes.c_void_p), ("A", ctypes.c_void_p),
                ("layer_stride_xd", ctypes.c_int64), ("layer_stride_bc", ctypes.c_int64)]
    rows = device = None     # of the tensors behind it, where scan_inputs made it


class DeltaInputs(ctypes.Structure):
    """Mirror of ``precog_delta_inputs`` (include/precog.h)."""
    _fields_ = [("n_qk_heads", ctypes.c_int32), ("n_v_heads", ctypes.c_int32), ("dk", ctypes.c_int32),
                ("dv", ctypes.c_int32), ("in_dtype", ctypes.c_int32), ("scale", ctypes.c_float),
                ("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("g", ctypes.c_void_p), ("beta", ctypes.c_void_p), ("q_stride", ctypes.c_int64),
                ("k_stride", ctypes.c_int64), ("v_stride", ctypes.c_int64)]


class QkNormArgs(ctypes.Structure):
    """Mirror of ``precog_qk_norm_args`` (include/precog.h)."""
    _fields_ = [("n_q_heads", ctypes.c_int32), ("n_k_heads", ctypes.c_int32), ("dim", ctypes.c_int32),
                ("rot_dim", ctypes.c_int32), ("dtype", ctypes.c_int32), ("norm", ctypes.c_int32),
                ("interleaved", ctypes.c_int32), ("eps", ctypes.c_float), ("q", ctypes.c_void_p),
                ("k", ctypes.c_void_p), ("q_out", ctypes.c_void_p), ("k_out", ctypes.c_void_p),
                ("q_stride", ctypes.c_int64), ("k_stride", ctypes.c_int64), ("q_out_stride", ctypes.c_int64),
                ("k_out_stride", ctypes.c_int64), ("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p),
                ("cos", ctypes.c_void_p), ("sin", ctypes.c_void_p), ("n_positions", ctypes.c_int64),
                ("d_positions", ctypes.c_void_p)]


class ConvArgs(ctypes.Structure):
    """Mirror of ``precog_conv_args`` (include/precog.h)."""
    _fields_ = [("dtype", ctypes.c_int32), ("dim", ctypes.c_int32), ("kernel", ctypes.c_int32),
                ("silu", ctypes.c_int32), ("x", ctypes.c_void_p), ("y", ctypes.c_void_p),
                ("x_stride", ctypes.c_int64), ("y_stride", ctypes.c_int64), ("weight", ctypes.c_void_p),
                ("bias", ctypes.c_void_p)]


class ScanStepArgs(ctypes.Structure):
    """Mirror of ``precog_scan_step_args`` (include/precog.h)."""
    _fields_ = [("states", ctypes.c_void_p), ("n_slots", ctypes.c_int64), ("d_slots", ctypes.c_void_p),
                ("layer0", ctypes.c_int32), ("L_total", ctypes.c_int32), ("skip", ctypes.c_void_p),
                ("gate", ctypes.c_void_p), ("gate_stride", ctypes.c_int64), ("gate_layer_stride", ctypes.c_int64),
                ("y_out", ctypes.c_void_p), ("y_dtype", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class BlockNormArgs(ctypes.Structure):
    """Mirror of ``precog_block_norm_args`` (include/precog.h)."""
    _fields_ = [("dtype", ctypes.c_int32), ("residual_dtype", ctypes.c_int32), ("dim", ctypes.c_int32),
                ("groups", ctypes.c_int32), ("norm", ctypes.c_int32), ("gate_first", ctypes.c_int32),
                ("scale", ctypes.c_float), ("eps", ctypes.c_float), ("x", ctypes.c_void_p),
                ("skip_input", ctypes.c_void_p), ("gate", ctypes.c_void_p), ("residual", ctypes.c_void_p),
                ("residual_out", ctypes.c_void_p), ("out", ctypes.c_void_p), ("x_stride", ctypes.c_int64),
                ("skip_stride", ctypes.c_int64), ("gate_stride", ctypes.c_int64), ("residual_stride", ctypes.c_int64),
                ("residual_out_stride", ctypes.c_int64), ("out_stride", ctypes.c_int64), ("skip", ctypes.c_void_p),
                ("weight", ctypes.c_void_p), ("scale_weight", ctypes.c_void_p), ("out_weight", ctypes.c_void_p)]


class AdjustArgs(ctypes.Structure):
    """Mirror of ``precog_adjust_args`` (include/precog.h)."""
    _fields_ = [("dtype", ctypes.c_int32), ("reserved", ctypes.c_int32), ("vocab", ctypes.c_int64),
                ("stride", ctypes.c_int64), ("out_stride", ctypes.c_int64), ("logits", ctypes.c_void_p),
                ("out", ctypes.c_void_p), ("d_history", ctypes.c_void_p), ("d_history_offsets", ctypes.c_void_p),
                ("d_count_from", ctypes.c_void_p), ("n_history", ctypes.c_int64), ("d_repetition", ctypes.c_void_p),
                ("d_frequency", ctypes.c_void_p), ("d_presence", ctypes.c_void_p), ("d_bias_idx", ctypes.c_void_p),
                ("d_bias", ctypes.c_void_p), ("d_bias_offsets", ctypes.c_void_p), ("n_bias", ctypes.c_int64),
                ("d_mask", ctypes.c_void_p), ("n_masks", ctypes.c_int64), ("d_mask_rows", ctypes.c_void_p)]


def _packer(cls) -> struct.Struct:
    """Packs what a Structure of ``cls`` would hold (pointers as numbers, 0 for NULL)."""
    codes = {ctypes.c_int32: "i", ctypes.c_float: "f", ctypes.c_int64: "q", ctypes.c_void_p: "P"}
    return struct.Struct("@" + "".join(codes[kind] for _, kind in cls._fields_))


# A Structure of 24 fields takes 1.0 us to fill on the Arm cores beside a GB300 and 0.5 to pass, a packed one 0.2
# and 0.3; the launches that follow are of 2 to 3 us.
_packed_calls = {}
_lib = None


def load_library(path: str = LIB_PATH):
    """Load ``libprecog.so`` (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise ImportError(f"libprecog.so not found at {path}; build it with "
                          "`python -m paper_2608_02560_gb300.build`")
    lib = ctypes.CDLL(path)
    i32, i64, vp, sz = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t
    lib.precog_encode_chunks.restype = i32
    lib.precog_encode_chunks.argtypes = [ctypes.POINTER(ScanInputs), vp, i64, i64, vp, i32, i32,
                                         i32, vp, i32, vp]
    lib.precog_encode_chunks_ordered.restype = i32
    lib.precog_encode_chunks_ordered.argtypes = [ctypes.POINTER(ScanInputs), vp, i64, i64, vp, vp, i32, i32,
                                                 i32, vp, i32, vp]
    lib.precog_retrieve.restype = i32
    lib.precog_retrieve.argtypes = [vp, i32, i64, i32, vp, i32, vp, vp, vp, sz, vp]
    lib.precog_retrieve_keys.restype = i32
    lib.precog_retrieve_keys.argtypes = [vp, i32, i64, i32, vp, i32, i64, vp, vp, sz, vp]
    lib.precog_decode_keys.restype = i32
    lib.precog_decode_keys.argtypes = [vp, i32, vp, vp, vp]
    lib.precog_retrieve_workspace_size.restype = sz
    lib.precog_retrieve_workspace_size.argtypes = [i64, i32, i32]
    lib.precog_prefill_from_state.restype = i32
    lib.precog_prefill_from_state.argtypes = [ctypes.POINTER(ScanInputs), i32, i32, vp, i32, i64,
                                              i32, i32, vp, vp, i32, vp, i32, vp]
    lib.precog_encode_trajectory.restype = i32
    lib.precog_encode_trajectory.argtypes = [ctypes.POINTER(ScanInputs), vp, i64, i64, i64, vp, vp,
                                             i32, i32, i32, vp]
    lib.precog_smc_route.restype = i32
    lib.precog_smc_route.argtypes = [vp, i32, i64, i32, vp, i32, vp, i32, vp, vp, vp, vp, vp]
    lib.precog_smc_consolidate.restype = i32
    lib.precog_smc_consolidate.argtypes = [vp, i64, i64, vp, i32, vp, i64, ctypes.c_float, vp]
    lib.precog_retrieve_topk.restype = i32
    lib.precog_retrieve_topk.argtypes = [vp, i32, i64, i32, vp, i32, i32, vp, vp, vp, sz, vp]
    lib.precog_retrieve_topk_workspace_size.restype = sz
    lib.precog_retrieve_topk_workspace_size.argtypes = [i64, i32, i32]
    lib.precog_prefill_composed.restype = i32
    lib.precog_prefill_composed.argtypes = [ctypes.POINTER(ScanInputs), i32, i32, vp, i32, i64, i32,
                                            i32, i32, vp, vp, ctypes.c_float, vp, i32, vp, i32, vp]
    lib.precog_delta_scan.restype = i32
    lib.precog_delta_scan.argtypes = [ctypes.POINTER(DeltaInputs), vp, i64, i64, vp, i32, i64, vp, vp, i32, i32,
                                      i32, vp, i32, vp, sz, vp]
    lib.precog_delta_scan_workspace_size.restype = sz
    lib.precog_delta_scan_workspace_size.argtypes = [ctypes.POINTER(DeltaInputs), i64, i64]
    lib.precog_delta_step.restype = i32
    lib.precog_delta_step.argtypes = [ctypes.POINTER(DeltaInputs), i64, vp, i64, vp, i32, i32, vp, i32, vp]
    lib.precog_qk_norm_rope.restype = i32
    lib.precog_qk_norm_rope.argtypes = [ctypes.POINTER(QkNormArgs), i64, vp]
    lib.precog_token_logprobs.restype = i32
    lib.precog_token_logprobs.argtypes = [vp, i32, i64, i64, i64, vp, ctypes.c_float, i32, vp, vp, vp, vp, vp]
    lib.precog_causal_conv.restype = i32
    lib.precog_causal_conv.argtypes = [ctypes.POINTER(ConvArgs), vp, i64, i64, vp, i64, vp, vp, i32, i32, vp]
    lib.precog_conv_step.restype = i32
    lib.precog_conv_step.argtypes = [ctypes.POINTER(ConvArgs), i64, vp, i64, vp, i32, i32, vp]
    lib.precog_scan_step.restype = i32
    lib.precog_scan_step.argtypes = [ctypes.POINTER(ScanInputs), ctypes.POINTER(ScanStepArgs), i64, vp]
    lib.precog_block_norm.restype = i32
    lib.precog_block_norm.argtypes = [ctypes.POINTER(BlockNormArgs), i64, vp]
    lib.precog_adjust_logits.restype = i32
    lib.precog_adjust_logits.argtypes = [ctypes.POINTER(AdjustArgs), i64, vp]
    lib.precog_selftest_wait_timeout.restype = i32
    lib.precog_selftest_wait_timeout.argtypes = [ctypes.c_uint32, vp]
    lib.precog_device_status.restype = i32
    lib.precog_device_status.argtypes = [vp, ctypes.POINTER(ctypes.c_uint32)]
    lib.precog_status_string.restype = ctypes.c_char_p
    lib.precog_status_string.argtypes = [i32]
    lib.precog_last_error.restype = ctypes.c_char_p
    lib.precog_last_error.argtypes = []
    lib.precog_abi_version.restype = i32
    lib.precog_abi_version.argtypes = []
    lib.precog_retrieve_noalloc.restype = i32
    lib.precog_retrieve_noalloc.argtypes = [vp, i32, i64, i32, vp, i32, vp, vp, vp]
    lib.precog_launch_count.restype = ctypes.c_uint64
    lib.precog_launch_count.argtypes = []
    for name, cls in (("precog_causal_conv", ConvArgs), ("precog_conv_step", ConvArgs), ("precog_scan_step", ScanStepArgs),
                      ("precog_block_norm", BlockNormArgs), ("precog_adjust_logits", AdjustArgs)):
        call = lib[name]        # the same function, with its arguments' struct as packed bytes
        call.restype = i32
        call.argtypes = [ctypes.c_char_p if t is ctypes.POINTER(cls) else t for t in getattr(lib, name).argtypes]
        _packed_calls[name] = (call, _packer(cls).pack)
    _lib = lib
    return lib


def _check(status: int):
    if status:
        raise PrecogError(status, load_library().precog_last_error().decode())


# ------------------------------------------------------------------------------- marshalling


# Marshalling runs on every call, next to launches of a few microseconds: the dtype table and
# torch's raw stream getter are looked up once (a torch.cuda.Stream object per call took 3 of
# the 8 us that a retrieval spent here; now 1.4 us on the same Arm core).
_torch_module = None
_dtype_codes = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


def _row_code(t) -> int:
    """The code of real rows."""
    global _dtype_codes
    if _dtype_codes is None:
        torch = _torch()
        _dtype_codes = {torch.float32: PRECOG_F32, torch.bfloat16: PRECOG_BF16, torch.float16: PRECOG_F16}
    code = _dtype_codes.get(t.dtype)
    if code is None:
        raise TypeError(f"unsupported dtype {t.dtype}")
    return code


def _dtype_code(t) -> int:
    """The code of a buffer or bank of the scans' states: complex64 ones are (re, im) fp32 pairs, F32 as stored."""
    if t.dtype is _torch().complex64:
        _resolved(t)
        return PRECOG_F32
    return _row_code(t)


def _resolved(t):
    """Refuses a complex tensor whose memory does not hold its values: ``t.conj()`` is contiguous and has t's pointer."""
    if t.is_conj() or t.is_neg():
        raise ValueError("tensors passed to libprecog must hold their values: call resolve_conj() and resolve_neg() "
                         "on a lazily conjugated or negated one")


def _ptr(t):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("tensors passed to libprecog must live on the GPU")
    if not t.is_contiguous():
        raise ValueError("tensors passed to libprecog must be contiguous")
    return t.data_ptr()


def _ptr_on(t, device: int):
    """:func:`_ptr` of a tensor that has to be on GPU ``device``."""
    if t is None:
        return None
    if t.get_device() != device or device < 0:
        raise ValueError("tensors passed to libprecog must live on the GPU, and on the same one")
    if not t.is_contiguous():
        raise ValueError("tensors passed to libprecog must be contiguous")
    return t.data_ptr()


_raw_stream = None


def _stream(stream):
    global _raw_stream
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None:
        torch = _torch()
        raw, device = (getattr(torch._C, n, None) for n in ("_cuda_getCurrentRawStream", "_cuda_getDevice"))
        if raw is None or device is None or not torch.cuda.is_initialized():
            return torch.cuda.current_stream().cuda_stream
        _raw_stream = lambda: raw(device())  # noqa: E731
    return _raw_stream()


def _workspace(need: int, device, stream):
    """``need`` bytes of the stream that will work on them: the allocator may hand a freed block to that
    stream's next tensor at once, and to no other's."""
    torch = _torch()
    if stream is None:
        return torch.empty(need, dtype=torch.uint8, device=device)
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(stream.cuda_stream, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(need, dtype=torch.uint8, device=device)


def scan_inputs(x, dt, B, A, C=None, a_kind: int = PRECOG_A_GENERAL) -> ScanInputs:
    """Describe x, dt ``[L, T, D]`` (or ``[T, D]``), B, C ``[L, T, N]``, A ``[L, D, N]``.

    ``a_kind=PRECOG_A_POWER`` states that A[d, n] == (n + 1) * A[d, 0] <= 0 (verified on
    the device); it selects the one-exponential update forms. ``a_kind=PRECOG_A_COMPLEX``
    takes a complex64 A (Eq. 1's complex diagonal) and complex states."""
    shape = x.shape
    if len(shape) == 2:
        x, dt, B = x.unsqueeze(0), dt.unsqueeze(0), B.unsqueeze(0)
        C = None if C is None else C.unsqueeze(0)
        shape = x.shape
    if A.dim() == 2:
        A = A.unsqueeze(0)
    L, T, D = shape
    rows = B.shape
    N = rows[-1]
    if dt.shape != shape or rows != (L, T, N) or (C is not None and C.shape != rows):
        raise ValueError("x/dt/B/C shapes disagree")
    torch = _torch_module or _torch()
    if a_kind == PRECOG_A_COMPLEX:
        if A.shape != (L, D, N) or A.dtype != torch.complex64:
            raise ValueError("complex A must be complex64 [L, D, N]")
        _resolved(A)
    elif A.shape != (L, D, N) or A.dtype != torch.float32:
        raise ValueError("A must be float32 [L, D, N]")
    kind, device = x.dtype, x.get_device()
    if dt.dtype is not kind or B.dtype is not kind or (C is not None and C.dtype is not kind):
        raise TypeError("x, dt, B and C must have one dtype")
    s = ScanInputs(L, D, N, _row_code(x), a_kind, 0, _ptr_on(x, device), _ptr_on(dt, device), _ptr_on(B, device),
                   _ptr_on(C, device), _ptr_on(A, device), T * D, T * N)
    # the struct holds raw device pointers: keep the tensors alive as long as it lives
    s._keepalive = (x, dt, B, C, A)
    s.rows, s.device = T, device
    return s


def _rows(t, what: str):
    """(pointer, elements between rows) of a GPU tensor whose rows are contiguous."""
    if t is None:
        return None, 0
    if not t.is_cuda:
        raise ValueError("tensors passed to libprecog must live on the GPU")
    shape, strides = t.shape, t.stride()
    inner = 1
    for i in range(len(shape) - 1, 0, -1):
        if strides[i] != inner and shape[i] > 1:
            raise ValueError(f"the rows of {what} must be contiguous")
        inner *= shape[i]
    return t.data_ptr(), (strides[0] if shape[0] > 1 else inner)


def _of(t, dtype, shape, what: str):
    """The pointer of a contiguous GPU tensor of this dtype and shape (None stays None)."""
    if t is None:
        return None
    if t.dtype is not dtype or t.shape != shape:
        raise ValueError(f"{what} must be {dtype} {tuple(shape)}, got {t.dtype} {tuple(t.shape)}")
    return _ptr(t)


def delta_inputs(q, k, v, g, beta, scale: float | None = None) -> DeltaInputs:
    """Describe the gated delta rule's q, k ``[T, Hk, dk]``, v ``[T, Hv, dv]`` (rows may be
    strided: slices of one projection) and the fp32 gates g (log decay), beta ``[T, Hv]``.
    ``q`` may be None without a readout; ``scale`` (default dk**-0.5) multiplies the readout."""
    torch = _torch()
    T, hk, dk = k.shape
    hv, dv = v.shape[1], v.shape[2]
    if v.shape[0] != T or (q is not None and q.shape != k.shape):
        raise ValueError("q/k/v shapes disagree")
    if v.dtype != k.dtype or (q is not None and q.dtype != k.dtype):
        raise TypeError("q, k and v must have one dtype")
    (qp, qs), (kp, ks), (vp, vs) = _rows(q, "q"), _rows(k, "k"), _rows(v, "v")
    s = DeltaInputs(hk, hv, dk, dv, _row_code(k), dk ** -0.5 if scale is None else scale, qp, kp, vp,
                    _of(g, torch.float32, (T, hv), "g"), _of(beta, torch.float32, (T, hv), "beta"), qs, ks, vs)
    # the struct holds raw device pointers: keep the tensors alive as long as it lives
    s._keepalive = (q, k, v, g, beta)
    s.rows = T
    return s


# ------------------------------------------------------------------------------- the C calls


def precog_encode_chunks(inputs: ScanInputs, offsets, T_tot: int, states_out=None,
                         layer0: int = 0, L_total: int | None = None, y_out=None, stream=None):
    """Scan every chunk (rows ``offsets[c]..offsets[c+1]``) from zero; capture final states
    into ``states_out [n_chunks, L_total, D, N]`` and/or readouts into ``y_out [L, T_tot, D]``."""
    lib = load_library()
    n_chunks = offsets.numel() - 1
    if L_total is None:
        L_total = inputs.n_layers
    _check(lib.precog_encode_chunks(
        ctypes.byref(inputs), _ptr(offsets), n_chunks, T_tot, _ptr(states_out),
        _dtype_code(states_out) if states_out is not None else PRECOG_F32, layer0, L_total,
        _ptr(y_out), _row_code(y_out) if y_out is not None else PRECOG_F32, _stream(stream)))


def precog_encode_chunks_ordered(inputs: ScanInputs, offsets, T_tot: int, order, states_out=None,
                                 layer0: int = 0, L_total: int | None = None, y_out=None, stream=None):
    """:func:`precog_encode_chunks` taking chunks up in the order of ``order`` (device
    int64 ``[n_chunks]``, a permutation, e.g. longest first); identical outputs."""
    lib = load_library()
    n_chunks = offsets.numel() - 1
    if L_total is None:
        L_total = inputs.n_layers
    if order.numel() != n_chunks or order.dtype != _torch().int64:
        raise ValueError("order must be int64 with one entry per chunk")
    _check(lib.precog_encode_chunks_ordered(
        ctypes.byref(inputs), _ptr(offsets), n_chunks, T_tot, _ptr(order), _ptr(states_out),
        _dtype_code(states_out) if states_out is not None else PRECOG_F32, layer0, L_total,
        _ptr(y_out), _row_code(y_out) if y_out is not None else PRECOG_F32, _stream(stream)))


def precog_encode_trajectory(inputs: ScanInputs, offsets, T_tot: int, stride: int, entry_offsets,
                             traj_out, layer0: int = 0, L_total: int | None = None, stream=None):
    """Keep the state after every ``stride``-th token and the last token of each chunk in
    ``traj_out [entries, L_total, D, N]`` (K-dial trajectory, Sec. 5.2)."""
    lib = load_library()
    if L_total is None:
        L_total = inputs.n_layers
    _check(lib.precog_encode_trajectory(
        ctypes.byref(inputs), _ptr(offsets), offsets.numel() - 1, T_tot, stride, _ptr(entry_offsets),
        _ptr(traj_out), _dtype_code(traj_out), layer0, L_total, _stream(stream)))


def precog_retrieve_workspace_size(M: int, dim: int, n_queries: int) -> int:
    return int(load_library().precog_retrieve_workspace_size(M, dim, n_queries))


def precog_retrieve(index, queries, best_idx, best_score=None, workspace=None, stream=None):
    """Exact top-1 of ``queries [Q, dim]`` against ``index [M, dim]`` into int64 ``best_idx``
    and fp32 ``best_score``. ``workspace`` is allocated with torch when not given."""
    lib = load_library()
    M, dim = index.shape
    Q = queries.shape[0]
    if workspace is None:
        workspace = _workspace(max(precog_retrieve_workspace_size(M, dim, Q), 16), index.device, stream)
    _check(lib.precog_retrieve(
        _ptr(index), _row_code(index), M, dim, _ptr(queries), Q, _ptr(best_idx),
        _ptr(best_score), _ptr(workspace), workspace.numel() * workspace.element_size(),
        _stream(stream)))


def precog_retrieve_noalloc(index, queries, best_idx, best_score=None, stream=None):
    """precog_retrieve without a caller workspace: the partial keys go to a fixed device
    array inside the library (at most about 430 queries per call; overlapping calls race)."""
    lib = load_library()
    M, dim = index.shape
    _check(lib.precog_retrieve_noalloc(
        _ptr(index), _row_code(index), M, dim, _ptr(queries), queries.shape[0], _ptr(best_idx),
        _ptr(best_score), _stream(stream)))


def precog_retrieve_keys(index_shard, queries, row_offset: int, keys, workspace=None, stream=None):
    """Best row of ``queries [Q, dim]`` in ``index_shard [M, dim]`` (rows ``row_offset ..``
    of a row-partitioned index) as one signed-order int64 key per query in ``keys``; the
    maximum over shards is the key of the whole index's top-1 (see precog.h)."""
    lib = load_library()
    M, dim = index_shard.shape
    Q = queries.shape[0]
    if workspace is None:
        workspace = _workspace(max(precog_retrieve_workspace_size(M, dim, Q), 16), queries.device, stream)
    _check(lib.precog_retrieve_keys(
        _ptr(index_shard), _row_code(index_shard), M, dim, _ptr(queries), Q, int(row_offset), _ptr(keys),
        _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream)))


def precog_decode_keys(keys, best_idx, best_score=None, stream=None):
    """Rows (-1: none) and scores (NaN: none) of int64 keys from precog_retrieve_keys."""
    lib = load_library()
    _check(lib.precog_decode_keys(_ptr(keys), keys.shape[0], _ptr(best_idx), _ptr(best_score),
                                  _stream(stream)))


def precog_prefill_from_state(inputs: ScanInputs, n_queries: int, T_q: int, bank, idx=None,
                              layer0: int = 0, y_out=None, state_out=None, stream=None):
    """Inject ``bank[idx[q]]`` (``[entries, L_bank, D, N]``) and scan each query's T_q tokens."""
    lib = load_library()
    entries, L_bank = bank.shape[0], bank.shape[1]
    _check(lib.precog_prefill_from_state(
        ctypes.byref(inputs), n_queries, T_q, _ptr(bank), _dtype_code(bank), entries, L_bank,
        layer0, _ptr(idx), _ptr(y_out), _row_code(y_out) if y_out is not None else PRECOG_F32,
        _ptr(state_out), _dtype_code(state_out) if state_out is not None else PRECOG_F32,
        _stream(stream)))


def precog_retrieve_topk_workspace_size(M: int, dim: int, n_queries: int) -> int:
    return int(load_library().precog_retrieve_topk_workspace_size(M, dim, n_queries))


def precog_retrieve_topk(index, queries, k, best_idx, best_score=None, workspace=None, stream=None):
    """The k best rows per query into ``best_idx [Q, k]`` (int64) and ``best_score [Q, k]``."""
    lib = load_library()
    M, dim = index.shape
    Q = queries.shape[0]
    if workspace is None:
        workspace = _workspace(max(int(lib.precog_retrieve_topk_workspace_size(M, dim, Q)), 16), index.device, stream)
    _check(lib.precog_retrieve_topk(
        _ptr(index), _row_code(index), M, dim, _ptr(queries), Q, k, _ptr(best_idx),
        _ptr(best_score), _ptr(workspace), workspace.numel() * workspace.element_size(),
        _stream(stream)))


def precog_prefill_composed(inputs: ScanInputs, n_queries: int, T_q: int, bank, idx, scores, k: int,
                            temperature: float = 1.0, layer0: int = 0, y_out=None, state_out=None,
                            stream=None):
    """Inject sum_j softmax(scores/temperature)_j bank[idx[q, j]] and prefill each query."""
    lib = load_library()
    entries, L_bank = bank.shape[0], bank.shape[1]
    _check(lib.precog_prefill_composed(
        ctypes.byref(inputs), n_queries, T_q, _ptr(bank), _dtype_code(bank), entries, L_bank, layer0,
        k, _ptr(idx), _ptr(scores), temperature, _ptr(y_out),
        _row_code(y_out) if y_out is not None else PRECOG_F32, _ptr(state_out),
        _dtype_code(state_out) if state_out is not None else PRECOG_F32, _stream(stream)))


def precog_smc_route(embeddings, domain_protos, sub_protos, J, out_domain, out_sub, out_slot=None,
                     stream=None):
    """Two-level routing (Sec. 5.1): ``sub_protos [M, J_max, dim]``, ``J`` int32 [M]."""
    lib = load_library()
    n, dim = embeddings.shape
    M, J_max = sub_protos.shape[0], sub_protos.shape[1]
    _check(lib.precog_smc_route(
        _ptr(embeddings), _row_code(embeddings), n, dim, _ptr(domain_protos), M, _ptr(sub_protos),
        J_max, _ptr(J), _ptr(out_domain), _ptr(out_sub), _ptr(out_slot), _stream(stream)))


def precog_smc_consolidate(semantic, states, slots, alpha: float, stream=None):
    """EMA of deposited states into the fp32 semantic table, in deposit order (Sec. 5.3)."""
    lib = load_library()
    n_slots = semantic.shape[0]
    elems = semantic[0].numel() if n_slots else 0
    if semantic.is_complex():   # pairs
        _resolved(semantic)
        elems *= 2
    _check(lib.precog_smc_consolidate(
        _ptr(semantic), n_slots, elems, _ptr(states), _dtype_code(states), _ptr(slots),
        states.shape[0], alpha, _stream(stream)))


def precog_delta_scan_workspace_size(inputs: DeltaInputs, n_seqs: int, T_tot: int) -> int:
    return int(load_library().precog_delta_scan_workspace_size(ctypes.byref(inputs), n_seqs, T_tot))


def _delta_states(inputs: DeltaInputs, t, what: str):
    if t is not None and (t.dim() != 5 or tuple(t.shape[2:]) != (inputs.n_v_heads, inputs.dv, inputs.dk)):
        raise ValueError(f"{what} must be [entries, layers, Hv, dv, dk], got {tuple(t.shape)}")
    return t


def precog_delta_scan(inputs: DeltaInputs, offsets, T_tot: int, bank=None, idx=None, layer: int = 0,
                      states_out=None, y_out=None, workspace=None, stream=None):
    """Roll the gated delta rule over the sequences of int64 ``offsets [n + 1]``, from zero states
    or from ``bank[idx[c], layer]`` (``[entries, layers, Hv, dv, dk]``; -1: the zero state), into
    ``states_out[c, layer]`` and/or ``y_out [T_tot, Hv, dv]``. ``workspace`` is allocated with
    torch when one is needed and none is given."""
    lib = load_library()
    torch = _torch()
    n = offsets.numel() - 1
    if T_tot > inputs.rows:
        raise ValueError("T_tot exceeds the inputs' rows")
    _delta_states(inputs, bank, "bank")
    _delta_states(inputs, states_out, "states_out")
    if states_out is not None and states_out.shape[0] != n:
        raise ValueError("states_out must have one entry per sequence")
    if bank is not None and states_out is not None and bank.shape[1] != states_out.shape[1]:
        raise ValueError("bank and states_out must have the same number of layers")
    if y_out is not None and tuple(y_out.shape) != (T_tot, inputs.n_v_heads, inputs.dv):
        raise ValueError("y_out must be [T_tot, Hv, dv]")
    # (an empty bank has no address: the C call would see none)
    if bank is not None and ((idx is None and bank.shape[0] < n) or not 0 <= layer < bank.shape[1]):
        raise ValueError("bank has no entry for every sequence, or no such layer")
    holder = states_out if states_out is not None else bank
    if workspace is None and T_tot >= 1024:   # below, none is needed
        need = int(lib.precog_delta_scan_workspace_size(ctypes.byref(inputs), n, T_tot))
        workspace = _workspace(need, offsets.device, stream) if need else None
    _check(lib.precog_delta_scan(
        ctypes.byref(inputs), _of(offsets, torch.int64, (n + 1,), "offsets"), n, T_tot, _ptr(bank),
        _row_code(bank) if bank is not None else PRECOG_F32, bank.shape[0] if bank is not None else 0,
        _of(idx, torch.int64, (n,), "idx"), _ptr(states_out),
        _row_code(states_out) if states_out is not None else PRECOG_F32, layer,
        holder.shape[1] if holder is not None else 1, _ptr(y_out),
        _row_code(y_out) if y_out is not None else PRECOG_F32, _ptr(workspace),
        workspace.numel() * workspace.element_size() if workspace is not None else 0, _stream(stream)))


def precog_delta_step(inputs: DeltaInputs, states, slots=None, y_out=None, layer: int = 0, stream=None):
    """One token of the gated delta rule for each row of ``inputs``, on the fp32 table ``states
    [slots, layers, Hv, dv, dk]`` (updated in place) at the rows' int64 ``slots`` (-1: an idle
    row), into ``y_out [n, Hv, dv]``."""
    torch = _torch()
    n = inputs.rows
    _delta_states(inputs, states, "states")
    if states.dtype != torch.float32:
        raise ValueError("states must be float32")
    if y_out is None or tuple(y_out.shape) != (n, inputs.n_v_heads, inputs.dv):
        raise ValueError("y_out must be [n, Hv, dv]")
    _check(load_library().precog_delta_step(
        ctypes.byref(inputs), n, _ptr(states), states.shape[0], _of(slots, torch.int64, (n,), "slots"), layer,
        states.shape[1], _ptr(y_out), _row_code(y_out), _stream(stream)))


_NORMS = {"none": PRECOG_NORM_NONE, "l2": PRECOG_NORM_L2, "rms": PRECOG_NORM_RMS}


def precog_qk_norm_rope(q, k, q_out, k_out, norm: str = "l2", q_weight=None, k_weight=None, eps: float = 1e-6,
                        cos=None, sin=None, positions=None, interleaved: bool = False, stream=None):
    """Norm (``"l2"``, ``"rms"`` or ``"none"``) of every head of q ``[T, Hq, d]`` and k ``[T, Hk, d]``
    (rows may be strided), times fp32 weights ``[d]``, its first ``2 * cos.shape[1]`` entries
    rotated by row ``positions[t]`` (int64; default t) of the fp32 tables cos and sin, into
    ``q_out`` and ``k_out`` (which may be q and k)."""
    torch = _torch()
    if norm not in _NORMS:
        raise ValueError(f"norm must be one of {sorted(_NORMS)}")
    T, hq, d = q.shape
    hk = k.shape[1]
    if k.shape != (T, hk, d) or q_out.shape != q.shape or k_out.shape != k.shape:
        raise ValueError("q/k/q_out/k_out shapes disagree")
    if not (q.dtype == k.dtype == q_out.dtype == k_out.dtype):
        raise TypeError("q, k and their outputs must have one dtype")
    if (cos is None) != (sin is None) or (cos is not None and cos.shape != sin.shape):
        raise ValueError("cos and sin must be given together, with one shape")
    (qp, qs), (kp, ks) = _rows(q, "q"), _rows(k, "k")
    (qo, qos), (ko, kos) = _rows(q_out, "q_out"), _rows(k_out, "k_out")
    n_pos, half = cos.shape if cos is not None else (0, 0)
    args = QkNormArgs(hq, hk, d, 2 * half, _row_code(q), _NORMS[norm], int(interleaved), eps, qp, kp, qo, ko, qs,
                      ks, qos, kos, _of(q_weight, torch.float32, (d,), "q_weight"),
                      _of(k_weight, torch.float32, (d,), "k_weight"), _of(cos, torch.float32, (n_pos, half), "cos"),
                      _of(sin, torch.float32, (n_pos, half), "sin"), n_pos,
                      _of(positions, torch.int64, (T,), "positions") if half else None)
    _check(load_library().precog_qk_norm_rope(ctypes.byref(args), T, _stream(stream)))


def precog_token_logprobs(logits, tokens, logprob, entropy=None, top_idx=None, top_logprob=None,
                          temperature: float = 1.0, stream=None):
    """Log probabilities of int64 ``tokens [R]`` (-1: none) under ``softmax(logits / temperature)``
    (``[R, V]``, rows may be strided) into fp32 ``logprob [R]``, with the distribution's
    ``entropy [R]`` and its k best entries ``top_idx [R, k]`` (int64), ``top_logprob [R, k]``."""
    torch = _torch()
    R, V = logits.shape
    if (top_idx is None) != (top_logprob is None):
        raise ValueError("top_idx and top_logprob must be given together")
    k = top_idx.shape[1] if top_idx is not None else 0
    lp, stride = _rows(logits, "logits")
    _check(load_library().precog_token_logprobs(
        lp, _row_code(logits), R, V, stride, _of(tokens, torch.int64, (R,), "tokens"), temperature, k,
        _of(logprob, torch.float32, (R,), "logprob"), _of(entropy, torch.float32, (R,), "entropy"),
        _of(top_idx, torch.int64, (R, k), "top_idx"), _of(top_logprob, torch.float32, (R, k), "top_logprob"),
        _stream(stream)))


# The current device and its stream, once CUDA has begun (each call asks for both: 0.2 us of 7).
_device_getter = _stream_getter = None


def _current_device() -> int:
    global _device_getter, _stream_getter
    if _device_getter is None:
        torch = _torch()
        get, raw = (getattr(torch._C, n, None) for n in ("_cuda_getDevice", "_cuda_getCurrentRawStream"))
        if get is None or raw is None or not torch.cuda.is_initialized():
            return torch.cuda.current_device()
        _device_getter, _stream_getter = get, raw
    return _device_getter()


def _stream_on(device: int, stream):
    if stream is None and _stream_getter is not None:
        return _stream_getter(device)
    return _stream(stream)


def _elsewhere(t, what: str, device: int):
    if not t.is_cuda:
        raise ValueError("tensors passed to libprecog must live on the GPU")
    raise ValueError(f"{what} must live on the current device, cuda:{device}, where the library launches")


def _no_matrix(t, what: str):
    raise ValueError(f"{what} must be a matrix, got {tuple(t.shape)}")


def _matrix(t, shape, dtype, device: int, what: str):
    """(pointer, elements between rows) of a tensor ``[rows, n]`` whose rows are contiguous; None: (0, 0)."""
    if t is None:
        return 0, 0
    if t.shape != shape:
        raise ValueError(f"{what} must be {tuple(shape)}, got {tuple(t.shape)}")
    if t.dtype is not dtype:
        raise TypeError(f"{what} must be {dtype}, got {t.dtype}")
    return _first_matrix(t, shape, device, what)


def _first_matrix(t, shape, device: int, what: str):
    """The same of the tensor that the others' shape and dtype come from."""
    if t.get_device() != device:
        _elsewhere(t, what, device)
    between, one = t.stride()
    if one != 1 and shape[1] > 1:
        raise ValueError(f"the rows of {what} must be contiguous")
    return t.data_ptr(), between


def _dense(t, shape, dtype, device: int, what: str) -> int:
    """The pointer of a contiguous tensor of this shape and dtype; None: 0."""
    if t is None:
        return 0
    if t.shape != shape:
        raise ValueError(f"{what} must be {tuple(shape)}, got {tuple(t.shape)}")
    if t.dtype is not dtype:
        raise TypeError(f"{what} must be {dtype}, got {t.dtype}")
    if t.get_device() != device:
        _elsewhere(t, what, device)
    if not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    return t.data_ptr()


def _table(t, rows: int, n: int, dtype, device: int, what: str):
    """(pointer, entries, layers) of a contiguous table ``[entries, layers, rows, n]``; None: zeros."""
    if t is None:
        return 0, 0, 0
    shape = t.shape
    if len(shape) != 4 or shape[2] != rows or shape[3] != n:
        raise ValueError(f"{what} must be [entries, layers, {rows}, {n}], got {tuple(shape)}")
    if t.dtype is not dtype:
        raise TypeError(f"{what} must be {dtype}, got {t.dtype}")
    if dtype.is_complex:
        _resolved(t)
    if t.get_device() != device:
        _elsewhere(t, what, device)
    if not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    return t.data_ptr(), shape[0], shape[1]


def precog_causal_conv(x, weight, offsets, bias=None, silu: bool = True, bank=None, idx=None, layer: int = 0,
                       windows_out=None, y_out=None, stream=None):
    """The causal convolution with fp32 ``weight [D, K]`` (K = 2, 3 or 4) and ``bias [D]``, then SiLU, of
    the sequences (rows ``offsets[c]..offsets[c + 1]``) of x ``[T, D]`` (rows may be strided) into ``y_out``.
    The inputs before a sequence are ``bank[idx[c], layer]`` (``[entries, layers, K - 1, D]``; -1 or no bank:
    zeros); ``windows_out[c, layer]`` receives those that its next token needs."""
    if y_out is None:
        raise ValueError("y_out is required")
    if idx is not None and bank is None:
        raise ValueError("idx is given without bank")
    load_library()
    torch, device, dtype, shape, taps = _torch(), _current_device(), x.dtype, x.shape, weight.shape
    if len(shape) != 2 or len(taps) != 2:
        _no_matrix(*((x, "x") if len(shape) != 2 else (weight, "weight")))
    (T, D), K, n = shape, taps[1], offsets.numel() - 1
    xp, xs = _first_matrix(x, shape, device, "x")
    yp, ys = _matrix(y_out, shape, dtype, device, "y_out")
    bp, entries, layers = _table(bank, K - 1, D, dtype, device, "bank")
    wp, outs, out_layers = _table(windows_out, K - 1, D, dtype, device, "windows_out")
    if windows_out is not None and outs != n:
        raise ValueError("windows_out must have one entry per sequence")
    if bank is not None and windows_out is not None and layers != out_layers:
        raise ValueError("bank and windows_out must have the same number of layers")
    if bank is not None and idx is None and entries < n:   # (an empty bank has no address: the C call would see none)
        raise ValueError("idx is None but bank has fewer rows than sequences")
    L_total = out_layers if windows_out is not None else layers if bank is not None else layer + 1
    call, pack = _packed_calls["precog_causal_conv"]
    _check(call(pack(_row_code(x), D, K, 1 if silu else 0, xp, yp, xs, ys,
                     _dense(weight, (D, K), torch.float32, device, "weight"),
                     _dense(bias, (D,), torch.float32, device, "bias")),
                _dense(offsets, (n + 1,), torch.int64, device, "offsets"), n, T, bp, entries,
                _dense(idx, (n,), torch.int64, device, "idx"), wp, layer, L_total,
                _stream_on(device, stream)))


def precog_conv_step(x, weight, windows, slots=None, bias=None, silu: bool = True, layer: int = 0, y_out=None,
                     stream=None):
    """One token of :func:`precog_causal_conv` for each row of x ``[n, D]``, on the table ``windows [slots,
    layers, K - 1, D]`` (updated in place) at the rows' int64 ``slots`` (-1: an idle row), into ``y_out``
    (which may be x)."""
    if y_out is None:
        raise ValueError("y_out is required")
    load_library()
    torch, device, dtype, shape, taps = _torch(), _current_device(), x.dtype, x.shape, weight.shape
    if len(shape) != 2 or len(taps) != 2:
        _no_matrix(*((x, "x") if len(shape) != 2 else (weight, "weight")))
    (n, D), K = shape, taps[1]
    xp, xs = _first_matrix(x, shape, device, "x")
    yp, ys = _matrix(y_out, shape, dtype, device, "y_out")
    wp, n_slots, layers = _table(windows, K - 1, D, dtype, device, "windows")
    call, pack = _packed_calls["precog_conv_step"]
    _check(call(pack(_row_code(x), D, K, 1 if silu else 0, xp, yp, xs, ys,
                     _dense(weight, (D, K), torch.float32, device, "weight"),
                     _dense(bias, (D,), torch.float32, device, "bias")),
                n, wp, n_slots, _dense(slots, (n,), torch.int64, device, "slots"), layer, layers, _stream_on(device, stream)))


def precog_scan_step(inputs: ScanInputs, states, slots=None, layer0: int = 0, skip=None, gate=None, y_out=None,
                     stream=None):
    """One token of the diagonal scan for each of the n rows that ``inputs`` (x, dt ``[L, n, D]``) has, on the
    fp32 (complex A: complex64) table ``states [slots, layers, D, N]``, updated in place, at the rows' int64
    ``slots`` (-1: an idle row), into ``y_out [L, n, D]``: the readout, plus fp32 ``skip [L, D]`` times x,
    times SiLU of ``gate [L, n, D]`` (each row contiguous). Inputs that were filled field by field do not know
    their rows; ``y_out`` says how many there are."""
    if y_out is None:
        raise ValueError("y_out is required")
    torch, device = _torch(), _current_device()
    L, D, N, n = inputs.n_layers, inputs.D, inputs.N, inputs.rows
    if L == 1:   # [n, D] stands for one layer's [1, n, D]
        y_out = y_out.unsqueeze(0) if y_out.dim() == 2 else y_out
        gate = gate.unsqueeze(0) if gate is not None and gate.dim() == 2 else gate
        skip = skip.unsqueeze(0) if skip is not None and skip.dim() == 1 else skip
    sp, n_slots, layers = _table(states, D, N, torch.complex64 if inputs.a_kind == PRECOG_A_COMPLEX else torch.float32,
                                 device, "states")
    if n is None:
        if y_out.dim() != 3:
            raise ValueError(f"y_out must be [L, n, D], got {tuple(y_out.shape)}")
        n = y_out.shape[1]
    elif inputs.device != device:
        _elsewhere(inputs._keepalive[0], "the inputs", device)
    gp = gs = gls = 0
    if gate is not None:
        if gate.shape != (L, n, D):
            raise ValueError("gate must be [L, n, D]")
        if _row_code(gate) != inputs.in_dtype:
            raise TypeError("gate and x must have one dtype")
        if gate.get_device() != device:
            _elsewhere(gate, "gate", device)
        gls, gs, one = gate.stride()
        if one != 1 and D > 1:
            raise ValueError("the rows of gate must be contiguous")
        gp = gate.data_ptr()
    load_library()
    call, pack = _packed_calls["precog_scan_step"]
    _check(call(
        ctypes.byref(inputs),
        pack(sp, n_slots, _dense(slots, (n,), torch.int64, device, "slots"), layer0, layers,
             _dense(skip, (L, D), torch.float32, device, "skip"), gp, gs, gls,
             _dense(y_out, (L, n, D), y_out.dtype, device, "y_out"), _row_code(y_out), 0), n, _stream_on(device, stream)))


def precog_block_norm(x, out=None, skip=None, skip_input=None, gate=None, gate_first: bool = True, weight=None,
                      groups: int = 1, residual=None, scale=1.0, residual_out=None, out_weight=None, eps: float = 1e-6,
                      norm: str | None = None, stream=None):
    """The end of a block over the rows of x ``[T, D]`` (all rows may be strided): ``a = x + skip *
    skip_input``, times SiLU of ``gate`` (before the norm, or behind it), the RMS norm of each of ``groups``
    with ``weight`` (``norm``: ``"rms"`` or ``"none"``; default: ``"rms"`` where there is a weight). Without
    a residual ``out`` is a; with one, ``residual_out = residual + scale * a`` (``scale`` a number or fp32
    ``[D]``) and ``out``, if given, the RMS norm of that with ``out_weight``. Weights are fp32 ``[D]``; outputs
    may be inputs of their type."""
    load_library()
    torch, device, dtype, shape = _torch(), _current_device(), x.dtype, x.shape
    if norm is None:
        kind = PRECOG_NORM_NONE if weight is None else PRECOG_NORM_RMS
    elif norm == "none" or norm == "rms":
        kind = _NORMS[norm]
    else:
        raise ValueError('norm must be "none" or "rms"')
    if len(shape) != 2:
        _no_matrix(x, "x")
    T, D = shape
    f32, vec, scale_weight = torch.float32, (D,), 0
    if isinstance(scale, torch.Tensor):
        scale, scale_weight = 1.0, _dense(scale, vec, f32, device, "scale")
    xp, xs = _first_matrix(x, shape, device, "x")
    sp = ss = gp = gs = rp = rs = rop = ros = op = os_ = 0
    if skip_input is not None:
        sp, ss = _matrix(skip_input, shape, dtype, device, "skip_input")
    if gate is not None:
        gp, gs = _matrix(gate, shape, dtype, device, "gate")
    res_dtype, res_code = f32, PRECOG_F32
    if residual is not None:
        res_dtype, res_code = residual.dtype, _row_code(residual)
        rp, rs = _matrix(residual, shape, res_dtype, device, "residual")
    if residual_out is not None:
        rop, ros = _matrix(residual_out, shape, res_dtype, device, "residual_out")
    if out is not None:
        op, os_ = _matrix(out, shape, dtype, device, "out")
    call, pack = _packed_calls["precog_block_norm"]
    _check(call(pack(_row_code(x), res_code, D, groups, kind, 1 if gate_first else 0, scale, eps, xp, sp, gp, rp, rop,
                     op, xs, ss, gs, rs, ros, os_, _dense(skip, vec, f32, device, "skip"),
                     _dense(weight, vec, f32, device, "weight"), scale_weight,
                     _dense(out_weight, vec, f32, device, "out_weight")), T, _stream_on(device, stream)))


def precog_adjust_logits(logits, out, history=None, history_offsets=None, count_from=None, repetition=None,
                         frequency=None, presence=None, bias_idx=None, bias=None, bias_offsets=None, mask=None,
                         mask_rows=None, stream=None):
    """Logits ``[R, V]`` (rows may be strided) before a token is chosen, into ``out`` (which may be logits):
    fp32 ``repetition``, ``frequency`` and ``presence`` penalties ``[R]`` for the tokens of each row's int64
    ``history`` (entries ``history_offsets[r]..history_offsets[r + 1]``; counted from entry ``count_from[r]``
    on), fp32 ``bias`` of the tokens ``bias_idx`` (lists by ``bias_offsets``), and -infinity where row
    ``mask_rows[r]`` (-1: none) of the int32 bit ``mask [masks, ceil(V / 32)]`` has a token's bit clear."""
    if (bias is None) != (bias_idx is None) or (bias is None) != (bias_offsets is None):
        raise ValueError("bias_idx, bias and bias_offsets must be given together")
    if history is not None and history_offsets is None:
        raise ValueError("history needs history_offsets")
    if history is None and not (repetition is None and frequency is None and presence is None):
        raise ValueError("penalties need a history")
    if mask_rows is not None and mask is None:
        raise ValueError("mask_rows is given without mask")
    load_library()
    torch, device, dtype, shape = _torch(), _current_device(), logits.dtype, logits.shape
    if len(shape) != 2:
        _no_matrix(logits, "logits")
    R, V = shape
    lp, ls = _first_matrix(logits, shape, device, "logits")
    op, os_ = _matrix(out, shape, dtype, device, "out")
    i64, f32, row, ends = torch.int64, torch.float32, (R,), (R + 1,)
    nh = history.numel() if history is not None else 0
    nb = bias.numel() if bias is not None else 0
    if mask is not None and mask.dim() != 2:
        _no_matrix(mask, "mask")
    nm = mask.shape[0] if mask is not None else 0
    mp = _dense(mask, (nm, (V + 31) // 32), torch.int32, device, "mask")
    if mask is not None and mask_rows is None and nm < R:   # (an empty mask has no address: the C call would see none)
        raise ValueError("mask_rows is None but there are fewer masks than rows")
    call, pack = _packed_calls["precog_adjust_logits"]
    _check(call(pack(_row_code(logits), 0, V, ls, os_, lp, op, _dense(history, (nh,), i64, device, "history"),
                     _dense(history_offsets, ends, i64, device, "history_offsets"),
                     _dense(count_from, row, i64, device, "count_from"), nh,
                     _dense(repetition, row, f32, device, "repetition"),
                     _dense(frequency, row, f32, device, "frequency"), _dense(presence, row, f32, device, "presence"),
                     _dense(bias_idx, (nb,), i64, device, "bias_idx"), _dense(bias, (nb,), f32, device, "bias"),
                     _dense(bias_offsets, ends, i64, device, "bias_offsets"), nb,
                     mp, nm, _dense(mask_rows, row, i64, device, "mask_rows")), R, _stream_on(device, stream)))


def precog_selftest_wait_timeout(iterations: int = 4096, stream=None):
    """Run the bounded-wait failure path on purpose (a wait that nothing completes): the
    next precog_device_status reports PRECOG_ERR_TIMEOUT. Diagnostic only."""
    _check(load_library().precog_selftest_wait_timeout(iterations, _stream(stream)))


def precog_device_status(stream=None):
    """Synchronise the stream and return (status, bits) of the device status word (cleared)."""
    lib = load_library()
    bits = ctypes.c_uint32(0)
    st = lib.precog_device_status(_stream(stream), ctypes.byref(bits))
    return st, bits.value


def precog_status_string(status: int) -> str:
    """The name of a precog_status code."""
    return load_library().precog_status_string(int(status)).decode()


def precog_last_error() -> str:
    """The message of the last failed call on this host thread (empty if none)."""
    return load_library().precog_last_error().decode()


def precog_abi_version() -> int:
    return int(load_library().precog_abi_version())


def precog_launch_count() -> int:
    """Kernels this process has launched through the library so far."""
    return int(load_library().precog_launch_count())
