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
* :func:`precog_retrieve_noalloc`  -- top-1 retrieval without a caller workspace
* :func:`precog_device_status`    -- device-side status word; :func:`precog_status_string`,
  :func:`precog_last_error`, :func:`precog_abi_version`, :func:`precog_launch_count`
"""
from __future__ import annotations

import ctypes
import os

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
    _lib = lib
    return lib


def _check(status: int):
    if status != PRECOG_OK:
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


def _dtype_code(t) -> int:
    global _dtype_codes
    if _dtype_codes is None:
        torch = _torch()
        # complex64 state/bank buffers are (re, im) fp32 pairs: the F32 storage code
        _dtype_codes = {torch.float32: PRECOG_F32, torch.bfloat16: PRECOG_BF16, torch.float16: PRECOG_F16,
                        torch.complex64: PRECOG_F32}
    code = _dtype_codes.get(t.dtype)
    if code is None:
        raise TypeError(f"unsupported dtype {t.dtype}")
    return code


def _ptr(t):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("tensors passed to libprecog must live on the GPU")
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
    if x.dim() == 2:
        x, dt, B = x.unsqueeze(0), dt.unsqueeze(0), B.unsqueeze(0)
        C = None if C is None else C.unsqueeze(0)
    if A.dim() == 2:
        A = A.unsqueeze(0)
    L, T, D = x.shape
    N = B.shape[-1]
    if dt.shape != x.shape or B.shape != (L, T, N) or (C is not None and C.shape != B.shape):
        raise ValueError("x/dt/B/C shapes disagree")
    torch = _torch()
    if a_kind == PRECOG_A_COMPLEX:
        if A.shape != (L, D, N) or A.dtype != torch.complex64:
            raise ValueError("complex A must be complex64 [L, D, N]")
    elif A.shape != (L, D, N) or A.dtype != torch.float32:
        raise ValueError("A must be float32 [L, D, N]")
    s = ScanInputs(L, D, N, _dtype_code(x), a_kind, 0, _ptr(x), _ptr(dt), _ptr(B), _ptr(C), _ptr(A), T * D, T * N)
    # the struct holds raw device pointers: keep the tensors alive as long as it lives
    s._keepalive = (x, dt, B, C, A)
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
    s = DeltaInputs(hk, hv, dk, dv, _dtype_code(k), dk ** -0.5 if scale is None else scale, qp, kp, vp,
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
        _ptr(y_out), _dtype_code(y_out) if y_out is not None else PRECOG_F32, _stream(stream)))


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
        _ptr(y_out), _dtype_code(y_out) if y_out is not None else PRECOG_F32, _stream(stream)))


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
        _ptr(index), _dtype_code(index), M, dim, _ptr(queries), Q, _ptr(best_idx),
        _ptr(best_score), _ptr(workspace), workspace.numel() * workspace.element_size(),
        _stream(stream)))


def precog_retrieve_noalloc(index, queries, best_idx, best_score=None, stream=None):
    """precog_retrieve without a caller workspace: the partial keys go to a fixed device
    array inside the library (at most about 430 queries per call; overlapping calls race)."""
    lib = load_library()
    M, dim = index.shape
    _check(lib.precog_retrieve_noalloc(
        _ptr(index), _dtype_code(index), M, dim, _ptr(queries), queries.shape[0], _ptr(best_idx),
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
        _ptr(index_shard), _dtype_code(index_shard), M, dim, _ptr(queries), Q, int(row_offset), _ptr(keys),
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
        layer0, _ptr(idx), _ptr(y_out), _dtype_code(y_out) if y_out is not None else PRECOG_F32,
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
        _ptr(index), _dtype_code(index), M, dim, _ptr(queries), Q, k, _ptr(best_idx),
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
        _dtype_code(y_out) if y_out is not None else PRECOG_F32, _ptr(state_out),
        _dtype_code(state_out) if state_out is not None else PRECOG_F32, _stream(stream)))


def precog_smc_route(embeddings, domain_protos, sub_protos, J, out_domain, out_sub, out_slot=None,
                     stream=None):
    """Two-level routing (Sec. 5.1): ``sub_protos [M, J_max, dim]``, ``J`` int32 [M]."""
    lib = load_library()
    n, dim = embeddings.shape
    M, J_max = sub_protos.shape[0], sub_protos.shape[1]
    _check(lib.precog_smc_route(
        _ptr(embeddings), _dtype_code(embeddings), n, dim, _ptr(domain_protos), M, _ptr(sub_protos),
        J_max, _ptr(J), _ptr(out_domain), _ptr(out_sub), _ptr(out_slot), _stream(stream)))


def precog_smc_consolidate(semantic, states, slots, alpha: float, stream=None):
    """EMA of deposited states into the fp32 semantic table, in deposit order (Sec. 5.3)."""
    lib = load_library()
    n_slots = semantic.shape[0]
    elems = semantic[0].numel() if n_slots else 0
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
    holder = states_out if states_out is not None else bank
    if workspace is None and T_tot >= 1024:   # below, none is needed
        need = int(lib.precog_delta_scan_workspace_size(ctypes.byref(inputs), n, T_tot))
        workspace = _workspace(need, offsets.device, stream) if need else None
    _check(lib.precog_delta_scan(
        ctypes.byref(inputs), _of(offsets, torch.int64, (n + 1,), "offsets"), n, T_tot, _ptr(bank),
        _dtype_code(bank) if bank is not None else PRECOG_F32, bank.shape[0] if bank is not None else 0,
        _of(idx, torch.int64, (n,), "idx"), _ptr(states_out),
        _dtype_code(states_out) if states_out is not None else PRECOG_F32, layer,
        holder.shape[1] if holder is not None else 1, _ptr(y_out),
        _dtype_code(y_out) if y_out is not None else PRECOG_F32, _ptr(workspace),
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
        states.shape[1], _ptr(y_out), _dtype_code(y_out), _stream(stream)))


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
    args = QkNormArgs(hq, hk, d, 2 * half, _dtype_code(q), _NORMS[norm], int(interleaved), eps, qp, kp, qo, ko, qs,
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
        lp, _dtype_code(logits), R, V, stride, _of(tokens, torch.int64, (R,), "tokens"), temperature, k,
        _of(logprob, torch.float32, (R,), "logprob"), _of(entropy, torch.float32, (R,), "entropy"),
        _of(top_idx, torch.int64, (R, k), "top_idx"), _of(top_logprob, torch.float32, (R, k), "top_logprob"),
        _stream(stream)))


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
