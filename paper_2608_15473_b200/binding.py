"""Thin ctypes binding over the C ABI in ``include/qf.h``.

Covers ``include/qf.h`` and the test hooks of ``include/qf_testing.h``.
Argument marshalling only: every step of the path runs in the CUDA library.
Functions carry the same names as the C entry points (without the ``qf_``
prefix).  Tensor arguments may be torch tensors (their ``data_ptr()`` is
taken), integers (raw addresses) or ``None`` (NULL).

There is no fallback: if ``libqf.so`` has not been built, loading raises.
"""
from __future__ import annotations

import ctypes
from pathlib import Path
from typing import Optional

_PKG = Path(__file__).resolve().parent
LIB_PATH = _PKG / "libqf.so"

QF_OK = 0
QF_ERR_NULL = -1
QF_ERR_BAD_SHAPE = -2
QF_ERR_UNSUPPORTED = -3
QF_ERR_WORKSPACE = -4
QF_ERR_CUDA = -5
QF_ERR_DEVICE = -6
QF_ERR_STATIC_SCRATCH = -7
QF_STATIC_SCRATCH_BYTES = 8 << 20

QF_FLAG_CHECK_BOUNDS = 1
QF_FLAG_SIMPLE_KERNEL = 2
QF_FLAG_DRAW_ALWAYS = 8
QF_FLAG_KV_NHD = 16
QF_FLAG_NO_SMALL_MERGE = 32

QF_KV_E4M3 = 1      # how a scaled cache holds its numbers
QF_KV_INT8 = 2

QF_STATUS_BAD_PAGE = 1
QF_STATUS_TIMEOUT = 2

# every symbol include/qf.h declares
EXPORTS = (
    "qf_version", "qf_strerror", "qf_workspace_bytes", "qf_decode_partial", "qf_combine",
    "qf_step_scratch_bytes", "qf_decode_step_host", "qf_read_status", "qf_last_launch_count",
    "qf_set_profile_events", "qf_decode_partial_static", "qf_static_scratch_error",
    "qf_combine_self", "qf_append_kv", "qf_selftest_bounded_wait", "qf_plan_pieces",
    "qf_project_workspace_bytes", "qf_project_pair", "qf_project_status", "qf_fold_append",
    "qf_static_scratch_status", "qf_project_status_inject", "qf_enable_peer_access", "qf_decode_step",
    "qf_host_pipe_scratch_bytes", "qf_host_pipe_create", "qf_host_pipe_submit", "qf_host_pipe_wait",
    "qf_host_pipe_destroy",
    "qf_rope_frequencies", "qf_rope_append", "qf_prompt_workspace_bytes", "qf_prompt_attend", "qf_prompt_status",
    "qf_prefix_workspace_bytes", "qf_prefix_partial", "qf_prefix_step", "qf_prefix_status",
    "qf_rows_schedule",
    "qf_rope_append_axes", "qf_rope_pair_axes", "qf_rope_append_scaled", "qf_decode_partial_scaled", "qf_decode_step_scaled",
    "qf_prompt_attend_scaled",
)


class QFParams(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32),
        ("num_q_heads", ctypes.c_int32),
        ("num_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("page_size", ctypes.c_int32),
        ("max_pages_per_req", ctypes.c_int32),
        ("max_shards", ctypes.c_int32),
        ("flags", ctypes.c_int32),
        ("num_pages", ctypes.c_int64),
        ("sm_scale", ctypes.c_float),
        ("out_shards", ctypes.c_int32),
        ("out_shard_offset", ctypes.c_int32),
        ("max_seq_len", ctypes.c_int32),
    ]


class QFRopeParams(ctypes.Structure):
    _fields_ = [
        ("total_tokens", ctypes.c_int32),
        ("rotary_dim", ctypes.c_int32),
        ("interleaved", ctypes.c_int32),
        ("eps", ctypes.c_float),
        ("rot_scale", ctypes.c_float),
        ("reserved", ctypes.c_int32),
        ("q_stride", ctypes.c_int64),
        ("k_stride", ctypes.c_int64),
        ("v_stride", ctypes.c_int64),
    ]


ROPE_SCALINGS = {"plain": 0, "linear": 1, "ntk": 2, "yarn": 3}


class QFError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where} failed with status {status}: {strerror(status)}")


_lib = None


def lib() -> ctypes.CDLL:
    """Load libqf.so (built by ``paper_2608_15473_b200.build``).  Raises if it is missing."""
    global _lib
    if _lib is None:
        if not LIB_PATH.exists():
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2608_15473_b200.build` "
                "(there is no CPU fallback)")
        L = ctypes.CDLL(str(LIB_PATH))
        vp, i32p = ctypes.c_void_p, ctypes.c_void_p
        pp = ctypes.POINTER(QFParams)
        L.qf_version.restype = ctypes.c_int
        L.qf_strerror.restype = ctypes.c_char_p
        L.qf_strerror.argtypes = [ctypes.c_int]
        L.qf_workspace_bytes.restype = ctypes.c_size_t
        L.qf_workspace_bytes.argtypes = [pp]
        L.qf_step_scratch_bytes.restype = ctypes.c_size_t
        L.qf_step_scratch_bytes.argtypes = [pp]
        L.qf_decode_partial.restype = ctypes.c_int
        L.qf_decode_partial.argtypes = [vp, vp, vp, i32p, i32p, i32p, vp, vp, vp, pp, vp, ctypes.c_size_t, vp]
        L.qf_decode_step.restype = ctypes.c_int
        L.qf_decode_step.argtypes = [vp, vp, vp, i32p, i32p, i32p, i32p, vp, vp, vp, vp, vp, pp, vp, ctypes.c_size_t, vp]
        L.qf_combine.restype = ctypes.c_int
        L.qf_combine.argtypes = [vp, vp, i32p, vp, vp, pp, vp]
        L.qf_decode_step_host.restype = ctypes.c_int
        L.qf_decode_step_host.argtypes = [vp, vp, vp, i32p, i32p, i32p, i32p, vp, vp, pp, vp, ctypes.c_size_t, vp]
        L.qf_read_status.restype = ctypes.c_int
        L.qf_read_status.argtypes = [vp, ctypes.POINTER(ctypes.c_int32), vp]
        L.qf_last_launch_count.restype = ctypes.c_int
        L.qf_set_profile_events.restype = ctypes.c_int
        L.qf_set_profile_events.argtypes = [vp, vp]
        L.qf_combine_self.restype = ctypes.c_int
        L.qf_combine_self.argtypes = [vp, vp, i32p, vp, vp, vp, vp, vp, pp, vp]
        L.qf_append_kv.restype = ctypes.c_int
        L.qf_append_kv.argtypes = [vp, vp, i32p, i32p, vp, vp, pp, vp]
        L.qf_selftest_bounded_wait.restype = ctypes.c_int
        L.qf_selftest_bounded_wait.argtypes = [vp, vp]
        L.qf_decode_partial_static.restype = ctypes.c_int
        L.qf_decode_partial_static.argtypes = [vp, vp, vp, i32p, i32p, i32p, vp, vp, vp, pp, vp]
        L.qf_static_scratch_error.restype = ctypes.c_char_p
        L.qf_static_scratch_status.restype = ctypes.c_int
        L.qf_static_scratch_status.argtypes = [ctypes.POINTER(ctypes.c_int32), vp]
        L.qf_host_pipe_scratch_bytes.restype = ctypes.c_size_t
        L.qf_host_pipe_scratch_bytes.argtypes = [pp, ctypes.c_int]
        L.qf_host_pipe_create.restype = ctypes.c_int
        L.qf_host_pipe_create.argtypes = [ctypes.POINTER(ctypes.c_void_p), pp, vp, ctypes.c_size_t, ctypes.c_int]
        L.qf_host_pipe_submit.restype = ctypes.c_longlong
        L.qf_host_pipe_submit.argtypes = [vp, vp, vp, vp, i32p, i32p, i32p, i32p, vp, vp, vp]
        L.qf_host_pipe_wait.restype = ctypes.c_int
        L.qf_host_pipe_wait.argtypes = [vp, ctypes.c_longlong]
        L.qf_host_pipe_destroy.restype = ctypes.c_int
        L.qf_host_pipe_destroy.argtypes = [vp]
        L.qf_enable_peer_access.restype = ctypes.c_int
        L.qf_enable_peer_access.argtypes = [ctypes.c_int]
        L.qf_project_status_inject.restype = ctypes.c_int
        L.qf_project_status_inject.argtypes = [vp, ctypes.c_int32, vp]
        L.qf_fold_append.restype = ctypes.c_int
        L.qf_fold_append.argtypes = [vp, vp, i32p, vp, vp, vp, vp, vp, vp, vp, i32p, i32p, ctypes.c_int, pp, vp]
        L.qf_project_workspace_bytes.restype = ctypes.c_size_t
        L.qf_project_workspace_bytes.argtypes = [ctypes.c_int, ctypes.c_int, ctypes.c_int]
        L.qf_project_pair.restype = ctypes.c_int
        L.qf_project_pair.argtypes = [vp, vp, vp, vp, vp, vp, vp, ctypes.c_int, ctypes.c_int, ctypes.c_int,
                                      ctypes.c_float, vp, ctypes.c_size_t, vp]
        L.qf_project_status.restype = ctypes.c_int
        L.qf_project_status.argtypes = [vp, ctypes.POINTER(ctypes.c_int32), vp]
        L.qf_plan_pieces.restype = ctypes.c_int
        L.qf_plan_pieces.argtypes = [ctypes.c_int, ctypes.c_int, ctypes.c_int, i32p, i32p, ctypes.c_int]
        rp = ctypes.POINTER(QFRopeParams)
        dbl = ctypes.c_double
        L.qf_rope_frequencies.restype = ctypes.c_int
        L.qf_rope_frequencies.argtypes = [vp, ctypes.POINTER(ctypes.c_float), ctypes.c_int, dbl, ctypes.c_int, dbl, dbl, dbl, dbl]
        L.qf_rope_append.restype = ctypes.c_int
        L.qf_rope_append.argtypes = [vp] * 7 + [i32p] * 4 + [vp] * 3 + [pp, rp, vp]
        L.qf_prompt_workspace_bytes.restype = ctypes.c_size_t
        L.qf_prompt_workspace_bytes.argtypes = [pp, ctypes.c_int]
        L.qf_prompt_attend.restype = ctypes.c_int
        L.qf_prompt_attend.argtypes = [vp, vp, vp, i32p, i32p, i32p, vp, vp, pp, ctypes.c_int, ctypes.c_int64, vp,
                                       ctypes.c_size_t, vp]
        L.qf_prompt_status.restype = ctypes.c_int
        L.qf_prompt_status.argtypes = [vp, ctypes.POINTER(ctypes.c_int32), vp]
        L.qf_prefix_workspace_bytes.restype = ctypes.c_size_t
        L.qf_prefix_workspace_bytes.argtypes = [pp]
        L.qf_prefix_partial.restype = ctypes.c_int
        L.qf_prefix_partial.argtypes = [vp, vp, vp, i32p, i32p, i32p, vp, vp, vp, pp, ctypes.c_int, ctypes.c_int, vp,
                                        ctypes.c_size_t, vp]
        L.qf_prefix_step.restype = ctypes.c_int
        L.qf_prefix_step.argtypes = [vp, vp, vp, i32p, i32p, i32p, i32p, i32p, i32p, vp, vp, vp, vp, vp, pp,
                                     ctypes.c_int, ctypes.c_int, vp, ctypes.c_size_t, vp]
        L.qf_prefix_status.restype = ctypes.c_int
        L.qf_prefix_status.argtypes = [vp, pp, ctypes.POINTER(ctypes.c_int32), vp]
        L.qf_rows_schedule.restype = ctypes.c_int
        L.qf_rows_schedule.argtypes = [ctypes.c_int, i32p, i32p] + [ctypes.c_int] * 6 + [i32p, ctypes.c_int]
        L.qf_rope_append_axes.restype = ctypes.c_int
        L.qf_rope_append_axes.argtypes = [vp] * 7 + [i32p] * 5 + [ctypes.c_int] + [vp] * 3 + [pp, rp, vp]
        L.qf_rope_pair_axes.restype = ctypes.c_int
        L.qf_rope_pair_axes.argtypes = [i32p, ctypes.c_int, i32p, ctypes.c_int, ctypes.c_int]
        L.qf_rope_append_scaled.restype = ctypes.c_int
        L.qf_rope_append_scaled.argtypes = [vp] * 9 + [i32p] * 6 + [ctypes.c_int] + [vp] * 3 + [ctypes.c_int, pp, rp, vp]
        L.qf_decode_partial_scaled.restype = ctypes.c_int
        L.qf_decode_partial_scaled.argtypes = [vp] * 5 + [i32p] * 3 + [vp] * 3 + [ctypes.c_int, pp, vp, ctypes.c_size_t, vp]
        L.qf_decode_step_scaled.restype = ctypes.c_int
        L.qf_decode_step_scaled.argtypes = [vp] * 5 + [i32p] * 4 + [vp] * 5 + [ctypes.c_int, pp, vp, ctypes.c_size_t, vp]
        L.qf_prompt_attend_scaled.restype = ctypes.c_int
        L.qf_prompt_attend_scaled.argtypes = [vp] * 5 + [i32p] * 3 + [vp, vp, ctypes.c_int, pp, ctypes.c_int, ctypes.c_int64, vp,
                                              ctypes.c_size_t, vp]
        _lib = L
    return _lib


def _ptr(x) -> Optional[int]:
    if x is None or isinstance(x, int):
        return x
    try:
        return x.data_ptr()
    except AttributeError:
        pass
    if hasattr(x, "ctypes"):  # numpy (host buffers of decode_step_host)
        return int(x.ctypes.data)
    raise TypeError(f"cannot take the address of {type(x)}")


_raw_stream = None      # () -> the current device's current stream, once CUDA is up


def _current_stream() -> int:
    """torch.cuda.current_stream().cuda_stream without the object around it (3.4 us of a 12 us call)."""
    global _raw_stream
    if _raw_stream is None:
        import torch
        stream_of, device = (getattr(torch._C, name, None) for name in ("_cuda_getCurrentRawStream", "_cuda_getDevice"))
        if stream_of is None or device is None or not torch.cuda.is_initialized():
            return int(torch.cuda.current_stream().cuda_stream)
        _raw_stream = lambda: int(stream_of(device()))      # noqa: E731
    return _raw_stream()


def _stream(stream) -> Optional[int]:
    if stream is None:
        return _current_stream()
    if isinstance(stream, int):
        return stream
    return int(stream.cuda_stream)


def params(batch: int, num_q_heads: int, num_kv_heads: int, max_pages_per_req: int, max_shards: int,
           num_pages: int, head_dim: int = 128, page_size: int = 16, flags: int = 0,
           sm_scale: float = 0.0, out_shards: int = 0, out_shard_offset: int = 0, max_seq_len: int = 0) -> QFParams:
    return QFParams(batch, num_q_heads, num_kv_heads, head_dim, page_size, max_pages_per_req, max_shards,
                    flags, num_pages, sm_scale, out_shards, out_shard_offset, max_seq_len)


def version() -> int:
    return int(lib().qf_version())


def strerror(status: int) -> str:
    return lib().qf_strerror(int(status)).decode()


def workspace_bytes(p: QFParams) -> int:
    return int(lib().qf_workspace_bytes(ctypes.byref(p)))


def step_scratch_bytes(p: QFParams) -> int:
    return int(lib().qf_step_scratch_bytes(ctypes.byref(p)))


def last_launch_count() -> int:
    return int(lib().qf_last_launch_count())


def set_profile_events(start_event, stop_event) -> None:
    """cudaEvent_t handles (ints) recorded around the sweep kernel; (None, None) switches it off."""
    lib().qf_set_profile_events(start_event, stop_event)


def decode_partial(q, k_cache, v_cache, block_table, seq_lens, shard_ranges, o_part, m_part, lse_part,
                   p: QFParams, workspace, workspace_bytes: int, stream=None, check: bool = True) -> int:
    rc = lib().qf_decode_partial(_ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(block_table), _ptr(seq_lens),
                                 _ptr(shard_ranges), _ptr(o_part), _ptr(m_part), _ptr(lse_part),
                                 ctypes.byref(p), _ptr(workspace), int(workspace_bytes), _stream(stream))
    if check and rc != QF_OK:
        raise QFError(rc, "qf_decode_partial")
    return rc


def decode_partial_static(q, k_cache, v_cache, block_table, seq_lens, shard_ranges, o_part, m_part, lse_part,
                          p: QFParams, stream=None, check: bool = True) -> int:
    """The sweep with the library's built-in scratch array: for callers that cannot allocate."""
    rc = lib().qf_decode_partial_static(_ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(block_table),
                                        _ptr(seq_lens), _ptr(shard_ranges), _ptr(o_part), _ptr(m_part),
                                        _ptr(lse_part), ctypes.byref(p), _stream(stream))
    if check and rc != QF_OK:
        detail = lib().qf_static_scratch_error().decode()
        raise QFError(rc, "qf_decode_partial_static" + (f" ({detail})" if detail else ""))
    return rc


def decode_step(q, k_cache, v_cache, block_table, seq_lens, shard_ranges, shard_counts, o_part, m_part, lse_part,
                out, lse, p: QFParams, workspace, workspace_bytes: int, stream=None, check: bool = True) -> int:
    """Sweep and merge as one call (a small sweep is followed by one merging kernel instead of two)."""
    rc = lib().qf_decode_step(_ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(block_table), _ptr(seq_lens),
                              _ptr(shard_ranges), _ptr(shard_counts), _ptr(o_part), _ptr(m_part), _ptr(lse_part),
                              _ptr(out), _ptr(lse), ctypes.byref(p), _ptr(workspace), int(workspace_bytes),
                              _stream(stream))
    if check and rc != QF_OK:
        raise QFError(rc, "qf_decode_step")
    return rc


def static_scratch_status(stream=None) -> int:
    """Status bits of the last decode_partial_static on the current device (synchronises the stream)."""
    st = ctypes.c_int32(0)
    rc = lib().qf_static_scratch_status(ctypes.byref(st), _stream(stream))
    if rc != QF_OK:
        raise QFError(rc, "qf_static_scratch_status")
    return int(st.value)


def enable_peer_access(peer_device: int, check: bool = True) -> int:
    """Let the current device's kernels store into memory of ``peer_device`` (shard states left in the merging
    GPU's arrays)."""
    rc = lib().qf_enable_peer_access(int(peer_device))
    if check and rc != QF_OK:
        raise QFError(rc, "qf_enable_peer_access")
    return rc


def project_status_inject(workspace, bits: int, stream=None) -> None:
    """Test hook: OR status bits into the projection pair's status word as a timed-out kernel would."""
    rc = lib().qf_project_status_inject(_ptr(workspace), int(bits), _stream(stream))
    if rc != QF_OK:
        raise QFError(rc, "qf_project_status_inject")


def combine(o_part, lse_part, shard_counts, out, lse, p: QFParams, stream=None, check: bool = True) -> int:
    rc = lib().qf_combine(_ptr(o_part), _ptr(lse_part), _ptr(shard_counts), _ptr(out), _ptr(lse),
                          ctypes.byref(p), _stream(stream))
    if check and rc != QF_OK:
        raise QFError(rc, "qf_combine")
    return rc


def combine_self(o_part, lse_part, shard_counts, q, k_new, v_new, out, lse, p: QFParams, stream=None,
                 check: bool = True) -> int:
    """Shard merge with the current token (k_new, v_new) folded in."""
    rc = lib().qf_combine_self(_ptr(o_part), _ptr(lse_part), _ptr(shard_counts), _ptr(q), _ptr(k_new),
                               _ptr(v_new), _ptr(out), _ptr(lse), ctypes.byref(p), _stream(stream))
    if check and rc != QF_OK:
        raise QFError(rc, "qf_combine_self")
    return rc


def append_kv(k_cache, v_cache, block_table, seq_lens, k_new, v_new, p: QFParams, stream=None,
              check: bool = True) -> int:
    """Write the current token's key and value at position seq_lens[b] of every request."""
    rc = lib().qf_append_kv(_ptr(k_cache), _ptr(v_cache), _ptr(block_table), _ptr(seq_lens), _ptr(k_new),
                            _ptr(v_new), ctypes.byref(p), _stream(stream))
    if check and rc != QF_OK:
        raise QFError(rc, "qf_append_kv")
    return rc


def fold_append(o_part, lse_part, shard_counts, q, k_new, v_new, out, lse, k_cache, v_cache, block_table, seq_lens,
                p: QFParams, advance_lengths: bool = True, stream=None, check: bool = True) -> int:
    """combine_self and append_kv in one launch; advance_lengths also adds one to the stored requests' lengths."""
    rc = lib().qf_fold_append(_ptr(o_part), _ptr(lse_part), _ptr(shard_counts), _ptr(q), _ptr(k_new), _ptr(v_new),
                              _ptr(out), _ptr(lse), _ptr(k_cache), _ptr(v_cache), _ptr(block_table), _ptr(seq_lens),
                              1 if advance_lengths else 0, ctypes.byref(p), _stream(stream))
    if check and rc != QF_OK:
        raise QFError(rc, "qf_fold_append")
    return rc


def decode_step_host(q_host, k_cache, v_cache, block_table, seq_lens_host, shard_ranges_host,
                     shard_counts_host, out_host, lse_host, p: QFParams, dev_scratch, dev_scratch_bytes: int,
                     stream=None, check: bool = True) -> int:
    rc = lib().qf_decode_step_host(_ptr(q_host), _ptr(k_cache), _ptr(v_cache), _ptr(block_table),
                                   _ptr(seq_lens_host), _ptr(shard_ranges_host), _ptr(shard_counts_host),
                                   _ptr(out_host), _ptr(lse_host), ctypes.byref(p), _ptr(dev_scratch),
                                   int(dev_scratch_bytes), _stream(stream))
    if check and rc != QF_OK:
        raise QFError(rc, "qf_decode_step_host")
    return rc


def host_pipe_scratch_bytes(p: QFParams, depth: int) -> int:
    return int(lib().qf_host_pipe_scratch_bytes(ctypes.byref(p), int(depth)))


def host_pipe_create(p: QFParams, dev_scratch, dev_scratch_bytes: int, depth: int) -> int:
    """A pipelined host-buffer stepper; returns its handle (an integer address)."""
    h = ctypes.c_void_p(None)
    rc = lib().qf_host_pipe_create(ctypes.byref(h), ctypes.byref(p), _ptr(dev_scratch), int(dev_scratch_bytes), int(depth))
    if rc != QF_OK:
        raise QFError(rc, "qf_host_pipe_create")
    return int(h.value)


def host_pipe_submit(pipe: int, q_host, k_cache, v_cache, block_table, seq_lens_host, shard_ranges_host,
                     shard_counts_host, out_host, lse_host, stream=None) -> int:
    """Enqueue one step; returns its ticket."""
    t = lib().qf_host_pipe_submit(pipe, _ptr(q_host), _ptr(k_cache), _ptr(v_cache), _ptr(block_table),
                                  _ptr(seq_lens_host), _ptr(shard_ranges_host), _ptr(shard_counts_host),
                                  _ptr(out_host), _ptr(lse_host), _stream(stream))
    if t < 0:
        raise QFError(int(t), "qf_host_pipe_submit")
    return int(t)


def host_pipe_wait(pipe: int, ticket: int) -> None:
    rc = lib().qf_host_pipe_wait(pipe, int(ticket))
    if rc != QF_OK:
        raise QFError(rc, "qf_host_pipe_wait")


def host_pipe_destroy(pipe: int) -> None:
    lib().qf_host_pipe_destroy(pipe)


def selftest_bounded_wait(workspace, stream=None) -> None:
    """Enqueue the kernel whose wait can never be satisfied; read_status must then report a timeout."""
    rc = lib().qf_selftest_bounded_wait(_ptr(workspace), _stream(stream))
    if rc != QF_OK:
        raise QFError(rc, "qf_selftest_bounded_wait")


def project_workspace_bytes(batch: int, d_model: int, n_q: int) -> int:
    return int(lib().qf_project_workspace_bytes(int(batch), int(d_model), int(n_q)))


def project_pair(a, z, w_o, g, w_q, u_out, q_out, eps, workspace, stream=None, check=True) -> int:
    """u' = z + W_o a, q = W_q N_1(u') for a batch of co-resident requests (device tensors; marshalling only)."""
    batch, n_q = int(a.shape[0]), int(a.shape[1])
    d_model = int(z.shape[1])
    rc = lib().qf_project_pair(_ptr(a), _ptr(z), _ptr(w_o), _ptr(g), _ptr(w_q), _ptr(u_out), _ptr(q_out), batch,
                               d_model, n_q, float(eps), _ptr(workspace),
                               int(workspace.numel() * workspace.element_size()), _stream(stream))
    if check and rc != QF_OK:
        raise QFError(rc, "qf_project_pair")
    return rc


def project_status(workspace, stream=None) -> int:
    st = ctypes.c_int32(0)
    rc = lib().qf_project_status(_ptr(workspace), ctypes.byref(st), _stream(stream))
    if rc != QF_OK:
        raise QFError(rc, "qf_project_status")
    return int(st.value)


_many_gpus: Optional[bool] = None
_kinds = {}      # a call's letters -> the element types of its arrays


def _kinds_of(letters):
    """The element types of every array: b bf16 (or 16-bit integers that hold its bits), i int32, f fp32, c one-byte codes, * any."""
    global _many_gpus
    import torch
    _many_gpus = torch.cuda.device_count() > 1
    anything = (torch.uint8, *{x for x in vars(torch).values() if isinstance(x, torch.dtype)})
    types = {"b": (torch.bfloat16, torch.int16, torch.uint16), "i": (torch.int32,), "f": (torch.float32,), "*": anything,
             "c": (torch.uint8, torch.int8, torch.float8_e4m3fn)}
    _kinds[letters] = tuple(types[x] for x in letters)
    return _kinds[letters]


def _address(x, kinds) -> Optional[int]:
    """_arrays for one array, with the reason of a refusal."""
    if x is None or isinstance(x, int):
        return x
    if not hasattr(x, "is_cuda"):
        raise ValueError(f"expected a CUDA tensor, got {type(x).__module__}.{type(x).__qualname__}")
    if not x.is_cuda:
        raise ValueError(f"expected a CUDA tensor, got one on {x.device}")
    if _many_gpus:
        import torch
        if x.get_device() != torch.cuda.current_device():
            raise ValueError(f"expected a tensor on the current device (cuda:{torch.cuda.current_device()}), got one on {x.device}")
    if x.dtype not in kinds:
        raise ValueError(f"expected elements of {kinds[0]}, got {x.dtype}")
    return x.data_ptr()


def _arrays(letters, *args):
    """The arrays' addresses.  The calls below launch on the current device and read each array as what the library
    expects: whatever is not None, an address or a tensor of that device (host tensors, NumPy arrays such as
    rope_frequencies', tensors of another device) is refused, not dereferenced there, and so is a tensor of other elements,
    which would be misread.  (One pass in one expression: a dozen calls of _address would be a third of a small call.)"""
    kinds = _kinds.get(letters) or _kinds_of(letters)
    if not _many_gpus:
        try:
            return [x if x is None or type(x) is int else x.data_ptr() if x.is_cuda and x.dtype in kind else _address(x, kind)
                    for x, kind in zip(args, kinds)]
        except AttributeError:
            pass
    return [_address(x, kind) for x, kind in zip(args, kinds)]


def rope_frequencies(rotary_dim: int = 128, theta: float = 1e6, scaling: str = "plain", factor: float = 1.0,
                     original_len: float = 0.0, beta_fast: float = 32.0, beta_slow: float = 1.0):
    """(inverse frequencies as a float32 array [rotary_dim / 2], factor of every sine and cosine).  Host arithmetic:
    no GPU is touched."""
    import numpy as np
    if scaling not in ROPE_SCALINGS:
        raise ValueError(f"scaling must be one of {sorted(ROPE_SCALINGS)}, not {scaling!r}")
    inv, scale = np.zeros(max(int(rotary_dim), 2) // 2, np.float32), ctypes.c_float(0)
    rc = lib().qf_rope_frequencies(inv.ctypes.data, ctypes.byref(scale), int(rotary_dim), float(theta),
                                   ROPE_SCALINGS[scaling], float(factor), float(original_len), float(beta_fast),
                                   float(beta_slow))
    if rc != QF_OK:
        raise QFError(rc, "qf_rope_frequencies")
    return inv, float(scale.value)


def rope_params(total_tokens: int, rotary_dim: int = 128, interleaved: bool = False, eps: float = 1e-6,
                rot_scale: float = 1.0, q_stride: int = 0, k_stride: int = 0, v_stride: int = 0) -> QFRopeParams:
    return QFRopeParams(total_tokens, rotary_dim, 1 if interleaved else 0, eps, rot_scale, 0, q_stride, k_stride, v_stride)


def rope_append(q, k, v, q_out, k_out, k_cache, v_cache, block_table, cu_tokens, seq_lens, pos_base, q_gain, k_gain,
                inv_freq, p: QFParams, r: QFRopeParams, stream=None, check: bool = True) -> int:
    """Norms, rotary positions and the cache write of packed tokens in one launch; any of q, (k, v), k_out, the
    caches, pos_base and the gains may be None (see qf_rope_append).  Arrays: CUDA tensors of the current device with the
    library's element types, or addresses."""
    at = _arrays("bbbbbbbiiiibbf", q, k, v, q_out, k_out, k_cache, v_cache, block_table, cu_tokens, seq_lens, pos_base, q_gain,
                 k_gain, inv_freq)
    rc = lib().qf_rope_append(*at, ctypes.byref(p), ctypes.byref(r), _stream(stream))
    if check and rc != QF_OK:
        raise QFError(rc, "qf_rope_append")
    return rc


def rope_pair_axes(rotary_dim: int, sections, interleaved: bool = False):
    """Which axis turns each pair, as an int32 array [rotary_dim / 2]: sections[a] pairs belong to axis a, in stretches or
    in turn (see qf_rope_pair_axes).  Host arithmetic: no GPU is touched."""
    import numpy as np
    sec = np.ascontiguousarray([int(x) for x in sections], np.int32)
    out = np.zeros(max(int(rotary_dim), 2) // 2, np.int32)
    rc = lib().qf_rope_pair_axes(out.ctypes.data, int(rotary_dim), sec.ctypes.data, len(sec), 1 if interleaved else 0)
    if rc != QF_OK:
        raise QFError(rc, "qf_rope_pair_axes")
    return out


def _num_axes(positions, num_axes: Optional[int], total_tokens: int) -> int:
    """Axes of a [num_axes, total_tokens] tensor, or what the caller, who may pass an address, says."""
    if positions is None:
        return 0 if num_axes is None else int(num_axes)
    if isinstance(positions, int):
        if num_axes is None:
            raise ValueError("num_axes is needed: an address does not tell")
        return int(num_axes)
    if positions.dim() != 2 or not positions.is_contiguous() or positions.shape[1] != total_tokens or \
            num_axes not in (None, positions.shape[0]):
        raise ValueError(f"positions: expected a contiguous [{num_axes or 'num_axes'}, {total_tokens}] tensor, got {tuple(positions.shape)}")
    return int(positions.shape[0])


def rope_append_axes(q, k, v, q_out, k_out, k_cache, v_cache, block_table, cu_tokens, seq_lens, positions, pair_axis, q_gain,
                     k_gain, inv_freq, p: QFParams, r: QFRopeParams, num_axes: Optional[int] = None, stream=None,
                     check: bool = True) -> int:
    """rope_append with rotary positions of several axes: positions int32 [num_axes, tokens], pair_axis int32
    [rotary_dim / 2] (rope_pair_axes makes it)."""
    at = _arrays("bbbbbbbiiiiibbf", q, k, v, q_out, k_out, k_cache, v_cache, block_table, cu_tokens, seq_lens, positions,
                 pair_axis, q_gain, k_gain, inv_freq)
    rc = lib().qf_rope_append_axes(*at[:12], _num_axes(positions, num_axes, r.total_tokens), *at[12:], ctypes.byref(p), ctypes.byref(r), _stream(stream))
    if check and rc != QF_OK:
        raise QFError(rc, "qf_rope_append_axes")
    return rc


_code_types = {}      # element types that tell what their codes are


def _kv_type(kv_type: Optional[int], *pools) -> int:
    """The code type of a scaled cache: what the caller says, or what the pools' elements say; they must not differ."""
    if not _code_types:
        import torch
        _code_types.update({torch.float8_e4m3fn: QF_KV_E4M3, torch.int8: QF_KV_INT8})
    said = kv_type
    for x in pools:
        of = _code_types.get(getattr(x, "dtype", None))
        if of is None:
            continue
        if said is not None and said != of:
            raise ValueError(f"a pool of {x.dtype} does not hold codes of kv_type {said}")
        said = of
    if said is None and all(x is None for x in pools):
        said = QF_KV_E4M3      # no cache, no codes
    if said is None:
        raise ValueError("kv_type is needed: the pools' element type does not tell e4m3 from int8")
    return int(said)


def rope_append_scaled(q, k, v, q_out, k_out, k_cache, v_cache, k_scale, v_scale, block_table, cu_tokens, seq_lens, pos_base,
                       positions, pair_axis, q_gain, k_gain, inv_freq, p: QFParams, r: QFRopeParams,
                       kv_type: Optional[int] = None, num_axes: Optional[int] = None, stream=None, check: bool = True) -> int:
    """rope_append (rope_append_axes with positions) into a scaled cache: one byte per number, a scale per page and KV head,
    which the call keeps up to date."""
    at = _arrays("bbbbbccffiiiiiibbf", q, k, v, q_out, k_out, k_cache, v_cache, k_scale, v_scale, block_table, cu_tokens, seq_lens,
                 pos_base, positions, pair_axis, q_gain, k_gain, inv_freq)
    rc = lib().qf_rope_append_scaled(*at[:15], _num_axes(positions, num_axes, r.total_tokens), *at[15:], _kv_type(kv_type, k_cache, v_cache),
                                     ctypes.byref(p), ctypes.byref(r), _stream(stream))
    if check and rc != QF_OK:
        raise QFError(rc, "qf_rope_append_scaled")
    return rc


def decode_partial_scaled(q, k_cache, v_cache, k_scale, v_scale, block_table, seq_lens, shard_ranges, o_part, m_part, lse_part,
                          p: QFParams, workspace, workspace_bytes: int, kv_type: Optional[int] = None, stream=None,
                          check: bool = True) -> int:
    """decode_partial over a scaled cache."""
    *at, ws = _arrays("bccffiiifff*", q, k_cache, v_cache, k_scale, v_scale, block_table, seq_lens, shard_ranges, o_part, m_part,
                      lse_part, workspace)
    rc = lib().qf_decode_partial_scaled(*at, _kv_type(kv_type, k_cache, v_cache), ctypes.byref(p), ws, int(workspace_bytes), _stream(stream))
    if check and rc != QF_OK:
        raise QFError(rc, "qf_decode_partial_scaled")
    return rc


def decode_step_scaled(q, k_cache, v_cache, k_scale, v_scale, block_table, seq_lens, shard_ranges, shard_counts, o_part, m_part,
                       lse_part, out, lse, p: QFParams, workspace, workspace_bytes: int, kv_type: Optional[int] = None,
                       stream=None, check: bool = True) -> int:
    """decode_step over a scaled cache."""
    *at, ws = _arrays("bccffiiiifffff*", q, k_cache, v_cache, k_scale, v_scale, block_table, seq_lens, shard_ranges, shard_counts,
                      o_part, m_part, lse_part, out, lse, workspace)
    rc = lib().qf_decode_step_scaled(*at, _kv_type(kv_type, k_cache, v_cache), ctypes.byref(p), ws, int(workspace_bytes), _stream(stream))
    if check and rc != QF_OK:
        raise QFError(rc, "qf_decode_step_scaled")
    return rc


def prompt_attend_scaled(q, k_cache, v_cache, k_scale, v_scale, block_table, cu_tokens, seq_lens, out, lse, p: QFParams,
                         total_tokens: int, workspace, workspace_bytes: int, q_stride: int = 0, kv_type: Optional[int] = None,
                         stream=None, check: bool = True) -> int:
    """prompt_attend over a scaled cache."""
    *at, ws = _arrays("bccffiiibf*", q, k_cache, v_cache, k_scale, v_scale, block_table, cu_tokens, seq_lens, out, lse, workspace)
    rc = lib().qf_prompt_attend_scaled(*at, _kv_type(kv_type, k_cache, v_cache), ctypes.byref(p), int(total_tokens), int(q_stride), ws,
                                       int(workspace_bytes), _stream(stream))
    if check and rc != QF_OK:
        raise QFError(rc, "qf_prompt_attend_scaled")
    return rc


def prompt_workspace_bytes(p: QFParams, total_tokens: int) -> int:
    return int(lib().qf_prompt_workspace_bytes(ctypes.byref(p), int(total_tokens)))


def prompt_attend(q, k_cache, v_cache, block_table, cu_tokens, seq_lens, out, lse, p: QFParams, total_tokens: int,
                  workspace, workspace_bytes: int, q_stride: int = 0, stream=None, check: bool = True) -> int:
    """Causal attention of packed prompt rows over the paged cache that already holds their keys and values."""
    *at, ws = _arrays("bbbiiibf*", q, k_cache, v_cache, block_table, cu_tokens, seq_lens, out, lse, workspace)
    rc = lib().qf_prompt_attend(*at, ctypes.byref(p), int(total_tokens), int(q_stride), ws, int(workspace_bytes), _stream(stream))
    if check and rc != QF_OK:
        raise QFError(rc, "qf_prompt_attend")
    return rc


def prompt_status(workspace, stream=None) -> int:
    st = ctypes.c_int32(0)
    rc = lib().qf_prompt_status(_ptr(workspace), ctypes.byref(st), _stream(stream))
    if rc != QF_OK:
        raise QFError(rc, "qf_prompt_status")
    return int(st.value)


def prefix_workspace_bytes(p: QFParams) -> int:
    return int(lib().qf_prefix_workspace_bytes(ctypes.byref(p)))


def prefix_partial(q, k_cache, v_cache, prefix_table, prefix_lens, group_offsets, o_part, m_part, lse_part,
                   p: QFParams, num_groups: int, max_prefix_pages: int, workspace, workspace_bytes: int, stream=None,
                   check: bool = True) -> int:
    """States of every request over its group's shared prefix, each prefix swept once."""
    *at, ws = _arrays("bbbiiifff*", q, k_cache, v_cache, prefix_table, prefix_lens, group_offsets, o_part, m_part, lse_part, workspace)
    rc = lib().qf_prefix_partial(*at, ctypes.byref(p), int(num_groups), int(max_prefix_pages), ws, int(workspace_bytes),
                                 _stream(stream))
    if check and rc != QF_OK:
        raise QFError(rc, "qf_prefix_partial")
    return rc


def prefix_step(q, k_cache, v_cache, block_table, seq_lens, shard_ranges, prefix_table, prefix_lens, group_offsets,
                o_part, m_part, lse_part, out, lse, p: QFParams, num_groups: int, max_prefix_pages: int, workspace,
                workspace_bytes: int, stream=None, check: bool = True) -> int:
    """One decode step behind shared prefixes: prefix sweep, own pages' sweep and the merge of both."""
    *at, ws = _arrays("bbbiiiiiifffff*", q, k_cache, v_cache, block_table, seq_lens, shard_ranges, prefix_table, prefix_lens,
                      group_offsets, o_part, m_part, lse_part, out, lse, workspace)
    rc = lib().qf_prefix_step(*at, ctypes.byref(p), int(num_groups), int(max_prefix_pages), ws, int(workspace_bytes), _stream(stream))
    if check and rc != QF_OK:
        raise QFError(rc, "qf_prefix_step")
    return rc


def prefix_status(workspace, p: QFParams, stream=None) -> int:
    st = ctypes.c_int32(0)
    rc = lib().qf_prefix_status(_ptr(workspace), ctypes.byref(p), ctypes.byref(st), _stream(stream))
    if rc != QF_OK:
        raise QFError(rc, "qf_prefix_status")
    return int(st.value)


def plan_pieces(total_units: int, n_ctas: int, draw_always: bool = False):
    """The sweep's schedule for (total_units, n_ctas): a list of [begin, end) ranges, one per piece
    (static slices first, then the drawn chunks).  Host arithmetic only: no GPU is touched."""
    cap = n_ctas + 4096
    b = (ctypes.c_int32 * cap)()
    e = (ctypes.c_int32 * cap)()
    n = lib().qf_plan_pieces(int(total_units), int(n_ctas), int(bool(draw_always)), b, e, cap)
    if n < 0:
        raise QFError(n, "qf_plan_pieces")
    return [(int(b[i]), int(e[i])) for i in range(n)]


def rows_schedule(causal: bool, offsets, lens, group: int, num_kv_heads: int, max_tokens: int, n_ctas: int):
    """The schedule of prompt_attend / prefix_partial as an int32 array [stretches, 12] (see qf_testing.h).  Host
    arithmetic only: no GPU is touched."""
    import numpy as np
    off, ln = np.ascontiguousarray(offsets, np.int32), np.ascontiguousarray(lens, np.int32)
    cap = 1 << 12
    while True:
        rec = np.zeros((cap, 12), np.int32)
        n = lib().qf_rows_schedule(int(bool(causal)), off.ctypes.data, ln.ctypes.data, len(ln), int(group),
                                   int(num_kv_heads), int(max_tokens), max(int(off.max()), 1), int(n_ctas),
                                   rec.ctypes.data, cap)
        if n < 0:
            raise QFError(n, "qf_rows_schedule")
        if n <= cap:
            return rec[:n]
        cap = n


def read_status(workspace, stream=None) -> int:
    st = ctypes.c_int32(0)
    rc = lib().qf_read_status(_ptr(workspace), ctypes.byref(st), _stream(stream))
    if rc != QF_OK:
        raise QFError(rc, "qf_read_status")
    return int(st.value)
