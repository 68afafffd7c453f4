from __future__ import annotations

import ctypes
import functools
from ctypes import POINTER, c_char_p, c_float, c_int32, c_int64, c_size_t, c_void_p
from dataclasses import dataclass
from pathlib import Path

import numpy as np

_HERE = Path(__file__).resolve().parent
_LIB_PATH = _HERE / "libpsa.so"
_lib = None

PSA_OUT_BF16, PSA_OUT_F32 = 0, 1

# every symbol include/psa.h declares
EXPORTED_SYMBOLS = [
    "psa_plan_create", "psa_plan_create_cascade", "psa_plan_create_prefill", "psa_prefill", "psa_plan_destroy", "psa_plan_get_info", "psa_plan_workspace_bytes",
    "psa_plan_bind_workspace", "psa_plan_prefix_items", "psa_plan_suffix_items",
    "psa_decode", "psa_decode_static", "psa_static_check_status", "psa_static_selftest_bounded_wait", "psa_decode_prefix", "psa_decode_suffix", "psa_decode_merge",
    "psa_decode_host_staging_bytes", "psa_decode_host", "psa_check_status", "psa_selftest_bounded_wait", "psa_append_kv", "psa_append_kv_alloc", "psa_validate_page_table", "psa_sample_scratch_bytes", "psa_sample_tokens", "psa_sample_tokens_at", "psa_attn_task",
    "psa_page_table_scratch_bytes", "psa_build_page_table", "psa_extend_page_table", "psa_read_status", "psa_kv4_cell_bytes", "psa_store_kv4",
    "psa_load_kv4", "psa_plan_create_kv4", "psa_decode_kv4", "psa_decode_suffix_kv4", "psa_process_logits_scratch_bytes", "psa_process_logits", "psa_mark_tokens",
    "psa_status_string", "psa_last_error_message", "psa_version",
]


class PsaError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"psa status {status} ({status_string(status)}): {message}")
        self.status = status


class _Config(ctypes.Structure):
    _fields_ = [("num_q_heads", c_int32), ("num_kv_heads", c_int32), ("head_dim", c_int32), ("page_size", c_int32),
                ("sm_scale", c_float), ("out_dtype", c_int32), ("num_sms", c_int32), ("suffix_chunk_tokens", c_int32),
                ("prefix_tiles_per_item", c_int32), ("prefix_rows_per_item", c_int32), ("prefix_kernel", c_int32)]


class _Info(ctypes.Structure):
    _fields_ = [("num_sms", c_int32), ("num_samples", c_int32), ("num_prefix_items", c_int32),
                ("num_suffix_items", c_int32), ("prefix_tile_keys", c_int32), ("prefix_tiles_per_item", c_int32),
                ("suffix_chunk_tokens", c_int32), ("kernel_launches", c_int32), ("num_partial_rows", c_int64)]


class _LogitsRules(ctypes.Structure):
    _fields_ = [("repetition", c_void_p), ("frequency", c_void_p), ("presence", c_void_p), ("history", c_void_p),
                ("history_lens", c_void_p), ("history_stride", c_int64), ("history_capacity", c_int32), ("prompt_bits", c_void_p),
                ("prompt_row_words", c_int64), ("num_prompt_bitmaps", c_int32), ("prompt_rows", c_void_p), ("bias_indptr", c_void_p),
                ("bias_ids", c_void_p), ("bias_values", c_void_p), ("num_biases", c_int32), ("mask_bits", c_void_p),
                ("mask_row_words", c_int64), ("num_mask_bitmaps", c_int32), ("mask_rows", c_void_p)]


@dataclass
class PlanInfo:
    num_sms: int
    num_samples: int
    num_prefix_items: int
    num_suffix_items: int
    prefix_tile_keys: int
    prefix_tiles_per_item: int
    suffix_chunk_tokens: int
    kernel_launches: int
    num_partial_rows: int


def library_path() -> Path:
    return _LIB_PATH


def library():
    """Load libpsa.so.  Raises if it has not been built: there is no other implementation."""
    global _lib
    if _lib is None:
        if not _LIB_PATH.exists():
            raise ImportError(f"{_LIB_PATH} is missing: build it with `python -m paper_2502_02534_b200.build`")
        lib = ctypes.CDLL(str(_LIB_PATH))
        P = c_void_p
        lib.psa_plan_create.restype = c_int32
        lib.psa_plan_create.argtypes = [POINTER(_Config), c_int32, P, P, P, POINTER(c_void_p)]
        lib.psa_plan_create_cascade.restype = c_int32
        lib.psa_plan_create_cascade.argtypes = [POINTER(_Config), c_int32, P, P, P, c_int32, P, POINTER(c_void_p)]
        lib.psa_plan_create_prefill.restype = c_int32
        lib.psa_plan_create_prefill.argtypes = [POINTER(_Config), c_int32, P, POINTER(c_void_p)]
        lib.psa_prefill.restype = c_int32
        lib.psa_prefill.argtypes = [P, P, P, P, POINTER(c_int64), P, P, P, c_size_t, P]
        lib.psa_plan_destroy.restype = c_int32
        lib.psa_plan_destroy.argtypes = [P]
        lib.psa_plan_get_info.restype = c_int32
        lib.psa_plan_get_info.argtypes = [P, POINTER(_Info)]
        lib.psa_plan_workspace_bytes.restype = c_size_t
        lib.psa_plan_workspace_bytes.argtypes = [P]
        lib.psa_plan_bind_workspace.restype = c_int32
        lib.psa_plan_bind_workspace.argtypes = [P, P, c_size_t, P]
        lib.psa_plan_prefix_items.restype = c_int32
        lib.psa_plan_prefix_items.argtypes = [P, P]
        lib.psa_plan_suffix_items.restype = c_int32
        lib.psa_plan_suffix_items.argtypes = [P, P]
        lib.psa_decode.restype = c_int32
        lib.psa_decode.argtypes = [P, P, P, P, POINTER(c_int64), P, P, POINTER(c_int64), P, P, P, P, P, P, c_size_t, P]
        lib.psa_decode_static.restype = c_int32
        lib.psa_decode_static.argtypes = [P, P, P, P, POINTER(c_int64), P, P, POINTER(c_int64), P, P, P, P, P, P]
        lib.psa_static_check_status.restype = c_int32
        lib.psa_static_check_status.argtypes = [P]
        lib.psa_static_selftest_bounded_wait.restype = c_int32
        lib.psa_static_selftest_bounded_wait.argtypes = [ctypes.c_uint64, P]
        lib.psa_decode_prefix.restype = c_int32
        lib.psa_decode_prefix.argtypes = [P, P, P, P, POINTER(c_int64), P, c_size_t, P]
        lib.psa_decode_suffix.restype = c_int32
        lib.psa_decode_suffix.argtypes = [P, P, P, P, POINTER(c_int64), P, P, P, P, c_size_t, P]
        lib.psa_decode_merge.restype = c_int32
        lib.psa_decode_merge.argtypes = [P, P, P, P, P, c_size_t, P]
        lib.psa_decode_host_staging_bytes.restype = c_size_t
        lib.psa_decode_host_staging_bytes.argtypes = [P, c_int64, c_int64, c_int64]
        lib.psa_decode_host.restype = c_int32
        lib.psa_decode_host.argtypes = [P, P, P, P, c_int64, P, P, c_int64, P, P, c_int64, P, P, P, P, c_size_t, P, c_size_t, P]
        lib.psa_check_status.restype = c_int32
        lib.psa_check_status.argtypes = [P, P, P]
        lib.psa_append_kv.restype = c_int32
        lib.psa_append_kv.argtypes = [P, P, P, P, P, POINTER(c_int64), P, P, P, P, c_size_t, P]
        lib.psa_append_kv_alloc.restype = c_int32
        lib.psa_append_kv_alloc.argtypes = [P, P, P, P, P, POINTER(c_int64), P, P, P, P, P, P, c_size_t, P]
        lib.psa_sample_tokens_at.restype = c_int32
        lib.psa_sample_tokens_at.argtypes = [P, c_int32, c_int64, c_int32, c_int32, P, P, P, ctypes.c_uint32, P, P, c_size_t, P]
        lib.psa_validate_page_table.restype = c_int32
        lib.psa_validate_page_table.argtypes = [P, P, P, P, c_int64, P, c_size_t, P]
        lib.psa_sample_scratch_bytes.restype = c_size_t
        lib.psa_sample_scratch_bytes.argtypes = [c_int32]
        lib.psa_sample_tokens.restype = c_int32
        lib.psa_sample_tokens.argtypes = [P, c_int32, c_int64, c_int32, c_int32, P, P, ctypes.c_uint32, P, P, c_size_t, P]
        lib.psa_attn_task.restype = c_int32
        lib.psa_attn_task.argtypes = [c_int32, P, P, P, c_int32, c_int32, c_int32, c_float, P, P, P, P]
        lib.psa_selftest_bounded_wait.restype = c_int32
        lib.psa_selftest_bounded_wait.argtypes = [P, c_size_t, ctypes.c_uint64, P]
        lib.psa_page_table_scratch_bytes.restype = c_size_t
        lib.psa_page_table_scratch_bytes.argtypes = [c_int32]
        lib.psa_build_page_table.restype = c_int32
        lib.psa_build_page_table.argtypes = [P, P, c_int32, P, P, P, P, P, c_int64, P, P, c_int64, P, P, P, c_size_t, P]
        lib.psa_extend_page_table.restype = c_int32
        lib.psa_extend_page_table.argtypes = [P, P, P, c_int32, P, P, P, P, P, c_int64, P, P, c_int64, P, P, P, c_size_t, P]
        lib.psa_read_status.restype = c_int32
        lib.psa_read_status.argtypes = [P, P]
        lib.psa_kv4_cell_bytes.restype = c_size_t
        lib.psa_kv4_cell_bytes.argtypes = [c_int32]
        lib.psa_store_kv4.restype = c_int32
        lib.psa_store_kv4.argtypes = [P, P, POINTER(c_int64), P, c_int64, c_int32, c_int32, P, POINTER(c_int64), c_int64, P, P]
        lib.psa_load_kv4.restype = c_int32
        lib.psa_load_kv4.argtypes = [P, POINTER(c_int64), c_int64, P, c_int64, c_int32, c_int32, P, P, POINTER(c_int64), P, P]
        lib.psa_plan_create_kv4.restype = c_int32
        lib.psa_plan_create_kv4.argtypes = [P, POINTER(c_void_p)]
        lib.psa_decode_kv4.restype = c_int32
        lib.psa_decode_kv4.argtypes = [P, P, P, P, POINTER(c_int64), P, POINTER(c_int64), P, P, P, P, P, P, c_size_t, P]
        lib.psa_decode_suffix_kv4.restype = c_int32
        lib.psa_decode_suffix_kv4.argtypes = [P, P, P, POINTER(c_int64), P, P, P, P, c_size_t, P]
        lib.psa_process_logits_scratch_bytes.restype = c_size_t
        lib.psa_process_logits_scratch_bytes.argtypes = [c_int32, c_int32]
        lib.psa_process_logits.restype = c_int32
        lib.psa_process_logits.argtypes = [P, c_int32, c_int64, c_int32, c_int32, POINTER(_LogitsRules), P, c_int32, c_int64, P, c_size_t, P]
        lib.psa_mark_tokens.restype = c_int32
        lib.psa_mark_tokens.argtypes = [P, c_int32, P, c_int32, c_int32, P, c_int64, P]
        lib.psa_status_string.restype = c_char_p
        lib.psa_status_string.argtypes = [c_int32]
        lib.psa_last_error_message.restype = c_char_p
        lib.psa_last_error_message.argtypes = []
        lib.psa_version.restype = c_int32
        lib.psa_version.argtypes = []
        _lib = lib
    return _lib


def status_string(status: int) -> str:
    return library().psa_status_string(int(status)).decode()


def _check(status: int):
    if status != 0:
        raise PsaError(status, library().psa_last_error_message().decode())


def _ptr(t):
    """Address of a torch tensor / numpy array / None."""
    if t is None:
        return None
    if isinstance(t, np.ndarray):
        return t.ctypes.data
    return t.data_ptr()


def _stream_ptr(stream):
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    return stream if isinstance(stream, int) else stream.cuda_stream


def _i32(a):
    return np.ascontiguousarray(np.asarray(a, dtype=np.int32))


class Plan:
    """psa_plan_create / psa_plan_destroy, plus the workspace the plan needs (a torch uint8 tensor)."""

    def __init__(self, prefix_lens, n_samples_per_prefix, suffix_lens, *, num_q_heads, num_kv_heads, head_dim,
                 page_size=16, sm_scale=None, out_dtype="bf16", num_sms=0, suffix_chunk_tokens=0, prefix_tiles_per_item=0,
                 prefix_rows_per_item=0, prefix_kernel=0, groups=None, prefill_prompt_lens=None):
        """``groups`` = (first_sample[], n_samples[], token_len[]) plans a cascade of shared prefixes
        (psa_plan_create_cascade); ``prefix_lens`` / ``n_samples_per_prefix`` are then ignored."""
        lib = library()
        self.prefix_lens, self.n_samples, self.suffix_len_bounds = _i32(prefix_lens), _i32(n_samples_per_prefix), _i32(suffix_lens)
        self.num_q_heads, self.num_kv_heads, self.head_dim, self.page_size = num_q_heads, num_kv_heads, head_dim, page_size
        self.sm_scale = float(sm_scale if sm_scale is not None else head_dim ** -0.5)
        self.out_dtype = {"bf16": PSA_OUT_BF16, "f32": PSA_OUT_F32}[out_dtype]
        cfg = _Config(num_q_heads, num_kv_heads, head_dim, page_size, self.sm_scale, self.out_dtype, num_sms,
                      suffix_chunk_tokens, prefix_tiles_per_item, prefix_rows_per_item, int(prefix_kernel))
        handle = c_void_p()
        self._h = None
        if prefill_prompt_lens is not None:     # causal self-attention of whole prompts (psa_plan_create_prefill)
            self.prompt_lens = _i32(prefill_prompt_lens)
            _check(lib.psa_plan_create_prefill(ctypes.byref(cfg), len(self.prompt_lens), _ptr(self.prompt_lens), ctypes.byref(handle)))
        elif groups is None:
            _check(lib.psa_plan_create(ctypes.byref(cfg), len(self.prefix_lens), _ptr(self.prefix_lens), _ptr(self.n_samples),
                                       _ptr(self.suffix_len_bounds), ctypes.byref(handle)))
        else:
            self.groups = tuple(_i32(a) for a in groups)
            _check(lib.psa_plan_create_cascade(ctypes.byref(cfg), len(self.groups[0]), _ptr(self.groups[0]), _ptr(self.groups[1]),
                                               _ptr(self.groups[2]), len(self.suffix_len_bounds), _ptr(self.suffix_len_bounds),
                                               ctypes.byref(handle)))
        self._h = handle
        self.workspace = None
        self._kv4 = None

    def for_kv4(self) -> "Plan":
        """The plan of the same problem whose pieces are sized for a 4-bit cache (psa_plan_create_kv4), with a workspace of its own.
        decode_kv4 uses it in place of this one; it is made once and kept."""
        if self._kv4 is None:
            handle = c_void_p()
            _check(library().psa_plan_create_kv4(self._h, ctypes.byref(handle)))
            plan = Plan.__new__(Plan)
            plan.__dict__.update(self.__dict__, _h=handle, workspace=None)
            plan._kv4 = plan
            self._kv4 = plan
        return self._kv4

    def __del__(self):
        if getattr(self, "_h", None):
            try:
                library().psa_plan_destroy(self._h)
            except Exception:       # interpreter shutdown: the module globals are already gone
                pass
            self._h = None

    @property
    def handle(self):
        return self._h

    @property
    def info(self) -> PlanInfo:
        i = _Info()
        _check(library().psa_plan_get_info(self._h, ctypes.byref(i)))
        return PlanInfo(*(getattr(i, f[0]) for f in _Info._fields_))

    @property
    def workspace_bytes(self) -> int:
        return int(library().psa_plan_workspace_bytes(self._h))

    def prefix_items(self) -> np.ndarray:
        n = library().psa_plan_prefix_items(self._h, None)
        a = np.zeros((n, 8), dtype=np.int32)
        library().psa_plan_prefix_items(self._h, _ptr(a))
        return a

    def suffix_items(self) -> np.ndarray:
        n = library().psa_plan_suffix_items(self._h, None)
        a = np.zeros((n, 4), dtype=np.int32)
        library().psa_plan_suffix_items(self._h, _ptr(a))
        return a

    def bind_workspace(self, workspace=None, stream=None):
        """Allocate (through torch) or adopt a device workspace and upload the work lists into it."""
        import torch
        if workspace is None:
            workspace = torch.empty(max(256, self.workspace_bytes), dtype=torch.uint8, device="cuda")
        _check(library().psa_plan_bind_workspace(self._h, _ptr(workspace), workspace.numel(), _stream_ptr(stream)))
        self.workspace = workspace
        return workspace

    def validate_page_table(self, page_indptr, page_indices, suffix_lens, num_pool_pages, stream=None):
        """psa_validate_page_table: enqueue the check; check_status() raises PSA_ERR_BOUNDS if the table is bad."""
        if self.workspace is None:
            self.bind_workspace(stream=stream)
        _check(library().psa_validate_page_table(self._h, _ptr(page_indptr), _ptr(page_indices), _ptr(suffix_lens),
                                                 int(num_pool_pages), _ptr(self.workspace), self.workspace.numel(), _stream_ptr(stream)))

    def selftest_bounded_wait(self, limit_ns=2_000_000, stream=None):
        """Enqueue the kernel whose wait can never be satisfied; check_status() must then raise PSA_ERR_TIMEOUT."""
        _check(library().psa_selftest_bounded_wait(_ptr(self.workspace), self.workspace.numel(), int(limit_ns), _stream_ptr(stream)))

    def check_status(self, stream=None):
        """Raise if a step left a device-side error in the workspace (that of for_kv4 included), and clear it."""
        if self._kv4 is not None and self._kv4 is not self and self._kv4.workspace is not None:
            self._kv4.check_status(stream)
            if self.workspace is None:
                return
        _check(library().psa_check_status(self._h, _ptr(self.workspace), _stream_ptr(stream)))


def _strides(values, n):
    arr = (c_int64 * n)(*[int(v) for v in values])
    return arr


def default_prefix_strides(plan: Plan):
    return (plan.num_kv_heads * plan.head_dim, plan.head_dim)


def default_pool_strides(plan: Plan):
    return (plan.num_kv_heads * plan.page_size * plan.head_dim, plan.page_size * plan.head_dim, plan.head_dim)


def decode(plan: Plan, q, prefix_k, prefix_v, suffix_k_pool, suffix_v_pool, page_indptr, page_indices, suffix_lens,
           out, lse, *, prefix_strides=None, pool_strides=None, stream=None, stage="all"):
    """psa_decode (or one of its stages) on torch CUDA tensors.  Only enqueues work."""
    lib = library()
    if plan.workspace is None:
        plan.bind_workspace(stream=stream)
    ws, wsb, st = _ptr(plan.workspace), plan.workspace.numel(), _stream_ptr(stream)
    pst = _strides(prefix_strides or default_prefix_strides(plan), 2)
    qst = _strides(pool_strides or default_pool_strides(plan), 3)
    if stage == "all":
        _check(lib.psa_decode(plan.handle, _ptr(q), _ptr(prefix_k), _ptr(prefix_v), pst, _ptr(suffix_k_pool),
                              _ptr(suffix_v_pool), qst, _ptr(page_indptr), _ptr(page_indices), _ptr(suffix_lens),
                              _ptr(out), _ptr(lse), ws, wsb, st))
    elif stage == "prefix":
        _check(lib.psa_decode_prefix(plan.handle, _ptr(q), _ptr(prefix_k), _ptr(prefix_v), pst, ws, wsb, st))
    elif stage == "suffix":
        _check(lib.psa_decode_suffix(plan.handle, _ptr(q), _ptr(suffix_k_pool), _ptr(suffix_v_pool), qst,
                                     _ptr(page_indptr), _ptr(page_indices), _ptr(suffix_lens), ws, wsb, st))
    elif stage == "merge":
        _check(lib.psa_decode_merge(plan.handle, _ptr(suffix_lens), _ptr(out), _ptr(lse), ws, wsb, st))
    else:
        raise ValueError(stage)


STATIC_WORKSPACE_BYTES = 16 << 20


def decode_static(plan: Plan, q, prefix_k, prefix_v, suffix_k_pool, suffix_v_pool, page_indptr, page_indices,
                  suffix_lens, out, lse, *, prefix_strides=None, pool_strides=None, stream=None):
    """psa_decode_static: the same step with the library's built-in scratch array instead of a
    workspace tensor -- nothing is allocated, here or in the library.  Calls that may overlap on
    the GPU share that array and must be serialised by the caller."""
    pst = _strides(prefix_strides or default_prefix_strides(plan), 2)
    qst = _strides(pool_strides or default_pool_strides(plan), 3)
    _check(library().psa_decode_static(plan.handle, _ptr(q), _ptr(prefix_k), _ptr(prefix_v), pst, _ptr(suffix_k_pool),
                                       _ptr(suffix_v_pool), qst, _ptr(page_indptr), _ptr(page_indices),
                                       _ptr(suffix_lens), _ptr(out), _ptr(lse), _stream_ptr(stream)))


def static_check_status(stream=None):
    """psa_static_check_status: raise if the last psa_decode_static step left a device-side error; clears it."""
    _check(library().psa_static_check_status(_stream_ptr(stream)))


def static_selftest_bounded_wait(limit_ns=2_000_000, stream=None):
    """psa_static_selftest_bounded_wait: the unsatisfiable wait, reporting into the library's own array."""
    _check(library().psa_static_selftest_bounded_wait(int(limit_ns), _stream_ptr(stream)))


def prefill(plan: Plan, q, k, v, out, lse, *, kv_strides=None, stream=None):
    """psa_prefill on torch CUDA tensors: causal attention of every prompt over itself."""
    if plan.workspace is None:
        plan.bind_workspace(stream=stream)
    st = _strides(kv_strides or default_prefix_strides(plan), 2)
    _check(library().psa_prefill(plan.handle, _ptr(q), _ptr(k), _ptr(v), st, _ptr(out), _ptr(lse), _ptr(plan.workspace),
                                 plan.workspace.numel(), _stream_ptr(stream)))


def append_kv(plan: Plan, new_k, new_v, suffix_k_pool, suffix_v_pool, page_indptr, page_indices, suffix_lens, *,
              pool_strides=None, stream=None):
    """psa_append_kv: one new token per sample goes to position suffix_lens[s]; suffix_lens is incremented in place."""
    if plan.workspace is None:
        plan.bind_workspace(stream=stream)
    qst = _strides(pool_strides or default_pool_strides(plan), 3)
    _check(library().psa_append_kv(plan.handle, _ptr(new_k), _ptr(new_v), _ptr(suffix_k_pool), _ptr(suffix_v_pool), qst,
                                   _ptr(page_indptr), _ptr(page_indices), _ptr(suffix_lens), _ptr(plan.workspace),
                                   plan.workspace.numel(), _stream_ptr(stream)))


def append_kv_alloc(plan: Plan, new_k, new_v, suffix_k_pool, suffix_v_pool, page_indptr, page_indices, suffix_lens,
                    free_pages, free_count, *, pool_strides=None, stream=None):
    """psa_append_kv_alloc: like append_kv, but a sample that starts a new page takes it from the stack
    free_pages[0 .. free_count) (int32 device tensors; free_count has one element and is updated in place)."""
    if plan.workspace is None:
        plan.bind_workspace(stream=stream)
    qst = _strides(pool_strides or default_pool_strides(plan), 3)
    _check(library().psa_append_kv_alloc(plan.handle, _ptr(new_k), _ptr(new_v), _ptr(suffix_k_pool), _ptr(suffix_v_pool), qst,
                                         _ptr(page_indptr), _ptr(page_indices), _ptr(suffix_lens), _ptr(free_pages),
                                         _ptr(free_count), _ptr(plan.workspace), plan.workspace.numel(), _stream_ptr(stream)))


def sample_tokens_at(logits, temperature, seeds, step_device, advance=1, tokens=None, scratch=None, *, stream=None):
    """psa_sample_tokens_at: the decode step is read from (and advanced in) the one-element int32 device tensor
    `step_device`, so that a captured graph holding this call can be replayed step after step."""
    import torch
    lib = library()
    B, V = logits.shape
    dtype = {torch.bfloat16: PSA_OUT_BF16, torch.float32: PSA_OUT_F32}[logits.dtype]
    if logits.stride(1) != 1:
        raise ValueError("logits must be contiguous along the vocabulary")
    if tokens is None:
        tokens = torch.empty(B, dtype=torch.int32, device=logits.device)
    if scratch is None:
        scratch = torch.empty(max(8, int(lib.psa_sample_scratch_bytes(B))), dtype=torch.uint8, device=logits.device)
    _check(lib.psa_sample_tokens_at(_ptr(logits), dtype, logits.stride(0), B, V, _ptr(temperature), _ptr(seeds), _ptr(step_device),
                                    int(advance), _ptr(tokens), _ptr(scratch), scratch.numel(), _stream_ptr(stream)))
    return tokens


def sample_tokens(logits, temperature, seeds, step, tokens=None, scratch=None, *, stream=None):
    """psa_sample_tokens on torch CUDA tensors: logits [B, V] (bf16 or f32, rows may be padded: stride(0) >= V),
    temperature [B] f32, seeds [B] int64 (bit pattern of the u64 seed).  Returns the int32 token tensor."""
    import torch
    lib = library()
    B, V = logits.shape
    dtype = {torch.bfloat16: PSA_OUT_BF16, torch.float32: PSA_OUT_F32}[logits.dtype]
    if logits.stride(1) != 1:
        raise ValueError("logits must be contiguous along the vocabulary")
    if tokens is None:
        tokens = torch.empty(B, dtype=torch.int32, device=logits.device)
    need = int(lib.psa_sample_scratch_bytes(B))
    if scratch is None:
        scratch = torch.empty(max(8, need), dtype=torch.uint8, device=logits.device)
    _check(lib.psa_sample_tokens(_ptr(logits), dtype, logits.stride(0), B, V, _ptr(temperature), _ptr(seeds), int(step) & 0xFFFFFFFF,
                                 _ptr(tokens), _ptr(scratch), scratch.numel(), _stream_ptr(stream)))
    return tokens


def attn_task(task, q, k, v, sm_scale, *, stream=None):
    """psa_attn_task on torch CUDA tensors: q [R, D], k / v [M, D] bf16.  Returns (out [R, D] f32, m [R], l [R])."""
    import torch
    R, D = q.shape
    M = k.shape[0]
    out = torch.empty((R, D), dtype=torch.float32, device=q.device)
    m = torch.empty(R, dtype=torch.float32, device=q.device)
    l = torch.empty(R, dtype=torch.float32, device=q.device)
    _check(library().psa_attn_task(int(task), _ptr(q), _ptr(k) if M else None, _ptr(v) if M else None, R, M, D, float(sm_scale),
                                   _ptr(out), _ptr(m), _ptr(l), _stream_ptr(stream)))
    return out, m, l


def decode_host(plan: Plan, q, prefix_k, prefix_v, suffix_k_pool, suffix_v_pool, page_indptr, page_indices, suffix_lens,
                out, lse, staging, *, stream=None):
    """psa_decode_host: every tensor is a host buffer (numpy array or pinned torch CPU tensor)."""
    lib = library()
    if plan.workspace is None:
        plan.bind_workspace(stream=stream)
    n_tok = int(prefix_k.shape[0]) if prefix_k is not None else 0
    n_pages = int(suffix_k_pool.shape[0]) if suffix_k_pool is not None else 0
    n_idx = int(page_indices.shape[0]) if page_indices is not None else 0
    _check(lib.psa_decode_host(plan.handle, _ptr(q), _ptr(prefix_k), _ptr(prefix_v), n_tok, _ptr(suffix_k_pool),
                               _ptr(suffix_v_pool), n_pages, _ptr(page_indptr), _ptr(page_indices), n_idx,
                               _ptr(suffix_lens), _ptr(out), _ptr(lse), _ptr(staging), staging.numel(),
                               _ptr(plan.workspace), plan.workspace.numel(), _stream_ptr(stream)))


def host_staging_bytes(plan: Plan, n_prefix_tokens: int, n_pool_pages: int, n_page_indices: int) -> int:
    return int(library().psa_decode_host_staging_bytes(plan.handle, n_prefix_tokens, n_pool_pages, n_page_indices))


# ---- page tables, the 4-bit cache and rules on logits.  These check the tensors they are given: type, layout, size, and that all of
# ---- them live on the current CUDA device (ValueError otherwise); what the library itself refuses comes back as PsaError.
# ---- The checks are written for the latency of a decode step: a handful of attribute reads per tensor, no per-call imports.

_torch = None


def _bind_torch():
    """Module-level references for the functions below (torch is not needed to import this module)."""
    global _torch, _i32_t, _i64_t, _u8_t, _bf16_t, _f32_t, _current_device, _raw_stream
    import torch
    _i32_t, _i64_t, _u8_t, _bf16_t, _f32_t = torch.int32, torch.int64, torch.uint8, torch.bfloat16, torch.float32
    _current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda dev: torch.cuda.current_stream(dev).cuda_stream)
    _torch = torch


def _flat(t, dtype, name, dev, size=0):
    """Address of a contiguous tensor of at least `size` elements on device `dev` (None passes through)."""
    if t is None:
        return None
    if t.dtype is dtype and t.get_device() == dev and t.is_contiguous() and t.numel() >= size:
        return t.data_ptr()
    if t.dtype is not dtype:
        raise ValueError(f"{name} must be {dtype}, not {t.dtype}")
    if not t.is_contiguous() or t.numel() < size:
        raise ValueError(f"{name} must be contiguous" + (f" and hold at least {size} elements" if size else ""))
    raise ValueError(f"{name} must be on the current CUDA device")


def _device_of(t, name):
    """The device the call runs on: that of tensor `t`, which must be the current one."""
    dev = t.get_device()
    if dev < 0 or dev != _current_device():
        raise ValueError(f"{name} must be on the current CUDA device")
    return dev


def _stream_on(stream, dev):
    return _raw_stream(dev) if stream is None else _stream_ptr(stream)


@functools.lru_cache(maxsize=256)
def _strides2(a, b):
    return (c_int64 * 2)(a, b)


def _outer_strides(t, inner, name):
    """Strides of dimensions 0 and 1 of a 3-d tensor whose last dimension is contiguous; a dimension of one element has none of its own."""
    s0, s1, s2 = t.stride()
    n0, n1, n2 = t.shape
    if n2 != inner or (s2 != 1 and n2 > 1):
        raise ValueError(f"{name} must be [.., .., {inner}] with a contiguous last dimension")
    if n1 <= 1:
        s1 = inner
    if n0 <= 1:
        s0 = max(1, n1) * max(s1, inner)
    return _strides2(s0, s1)


def page_table_scratch(num_samples):
    """Scratch tensor for build_page_table / extend_page_table, to be kept by callers that must not allocate (uint8)."""
    import torch
    return torch.empty(int(library().psa_page_table_scratch_bytes(int(num_samples))), dtype=torch.uint8, device="cuda")


def build_page_table(seq_lens, free_pages, free_count, page_indptr, page_indices, token_indptr, slot_map, *, reserve_lens=None,
                     lens_out=None, free_count_out=None, status=None, scratch=None, stream=None):
    """psa_build_page_table on torch CUDA tensors (int32; slot_map int64): page lists for samples of seq_lens tokens (room for
    reserve_lens), pages from the stack free_pages[0 .. free_count), and the slot of every token.  Outputs: page_indptr [B+1],
    page_indices (any capacity), token_indptr [B+1], slot_map (any capacity), lens_out [B], free_count_out (free_count in place
    when None)."""
    if _torch is None:
        _bind_torch()
    i32, n, dev = _i32_t, seq_lens.numel(), seq_lens.get_device()
    p_seq = _flat(seq_lens, i32, "seq_lens", dev)
    p_indptr = _flat(page_indptr, i32, "page_indptr", dev, n + 1)
    p_tokens = _flat(token_indptr, i32, "token_indptr", dev, n + 1)
    dev = _device_of(seq_lens, "seq_lens")
    if scratch is None:
        scratch = page_table_scratch(n)
    p_count = _flat(free_count, i32, "free_count", dev, 1)
    _check(library().psa_build_page_table(
        p_seq, _flat(reserve_lens, i32, "reserve_lens", dev, n), n, _flat(free_pages, i32, "free_pages", dev), p_count,
        p_count if free_count_out is None else _flat(free_count_out, i32, "free_count_out", dev, 1), p_indptr,
        _flat(page_indices, i32, "page_indices", dev), page_indices.numel(), p_tokens, _flat(slot_map, _i64_t, "slot_map", dev), slot_map.numel(),
        _flat(lens_out, i32, "lens_out", dev, n), _status_ptr(status, dev), _flat(scratch, _u8_t, "scratch", dev), scratch.numel(),
        _stream_on(stream, dev)))


def extend_page_table(held_lens, new_lens, free_pages, free_count, page_indptr, page_indices, token_indptr, slot_map, *, max_lens=None,
                      lens_out=None, free_count_out=None, status=None, scratch=None, stream=None):
    """psa_extend_page_table on torch CUDA tensors: new_lens more tokens for samples that hold held_lens, in existing page lists.
    Outputs as for build_page_table; lens_out and free_count_out may be held_lens and free_count themselves."""
    if _torch is None:
        _bind_torch()
    i32, n, dev = _i32_t, held_lens.numel(), held_lens.get_device()
    p_held = _flat(held_lens, i32, "held_lens", dev)
    p_new = _flat(new_lens, i32, "new_lens", dev, n)
    p_indptr = _flat(page_indptr, i32, "page_indptr", dev, n + 1)
    p_tokens = _flat(token_indptr, i32, "token_indptr", dev, n + 1)
    dev = _device_of(held_lens, "held_lens")
    if scratch is None:
        scratch = page_table_scratch(n)
    p_count = _flat(free_count, i32, "free_count", dev, 1)
    _check(library().psa_extend_page_table(
        p_held, p_new, _flat(max_lens, i32, "max_lens", dev, n), n, _flat(free_pages, i32, "free_pages", dev), p_count,
        p_count if free_count_out is None else _flat(free_count_out, i32, "free_count_out", dev, 1), p_indptr,
        _flat(page_indices, i32, "page_indices", dev), page_indices.numel(), p_tokens, _flat(slot_map, _i64_t, "slot_map", dev), slot_map.numel(),
        _flat(lens_out, i32, "lens_out", dev, n), _status_ptr(status, dev), _flat(scratch, _u8_t, "scratch", dev), scratch.numel(),
        _stream_on(stream, dev)))


def _status_ptr(status, dev):
    """A status word: a one-element int32 tensor, or a Plan (the word Plan.check_status reads)."""
    if status is None:
        return None
    if isinstance(status, Plan):
        if status.workspace is None:
            raise ValueError("status: the plan has no workspace yet")
        return _flat(status.workspace, _u8_t, "status", dev)
    return _flat(status, _i32_t, "status", dev, 1)


def read_status(status, stream=None):
    """psa_read_status: synchronise, raise if the one-element int32 tensor `status` holds an error, and clear it."""
    if _torch is None:
        _bind_torch()
    dev = _device_of(status, "status")
    _check(library().psa_read_status(_flat(status, _i32_t, "status", dev, 1), _stream_on(stream, dev)))


def kv4_cell_bytes(head_dim) -> int:
    """Bytes of one (page, KV head) cell of the 4-bit cache."""
    return int(library().psa_kv4_cell_bytes(int(head_dim)))


def _kv4_args(k, v, slot_map, pool, names):
    shape = k.shape
    if len(shape) != 3 or k.dtype is not _bf16_t or v.dtype is not _bf16_t or v.shape != shape or v.stride() != k.stride():
        raise ValueError(f"{names} must be bf16 [tokens, heads, head_dim] of the same shape and strides")
    tokens, heads, dim = shape
    if pool.dtype is not _u8_t or pool.dim() != 3 or pool.shape[1] != heads:
        raise ValueError("pool must be uint8 [pages, heads, kv4_cell_bytes(head_dim)]")
    if slot_map.dtype is not _i64_t or slot_map.numel() < tokens or not slot_map.is_contiguous():
        raise ValueError(f"slot_map must be contiguous int64 with at least {tokens} elements")
    dev = _device_of(k, names)
    if v.get_device() != dev or slot_map.get_device() != dev or pool.get_device() != dev:
        raise ValueError("all tensors must be on the current CUDA device")
    return tokens, heads, dim, _outer_strides(k, dim, names), _outer_strides(pool, 20 * dim, "pool"), dev


def store_kv4(new_k, new_v, slot_map, pool, *, status=None, stream=None):
    """psa_store_kv4: quantise new_k / new_v [T, Hkv, D] bf16 (any token and head stride) into the slots of a 4-bit pool
    [pages, Hkv, kv4_cell_bytes(D)] uint8."""
    if _torch is None:
        _bind_torch()
    t, h, d, kst, pst, dev = _kv4_args(new_k, new_v, slot_map, pool, "new_k and new_v")
    _check(library().psa_store_kv4(new_k.data_ptr(), new_v.data_ptr(), kst, slot_map.data_ptr(), t, h, d, pool.data_ptr(), pst,
                                   pool.shape[0], _status_ptr(status, dev), _stream_on(stream, dev)))


def load_kv4(pool, slot_map, out_k, out_v, *, status=None, stream=None):
    """psa_load_kv4: the cached tokens of slot_map as bf16 rows out_k / out_v [T, Hkv, D]; rows of negative slots are left alone."""
    if _torch is None:
        _bind_torch()
    t, h, d, kst, pst, dev = _kv4_args(out_k, out_v, slot_map, pool, "out_k and out_v")
    _check(library().psa_load_kv4(pool.data_ptr(), pst, pool.shape[0], slot_map.data_ptr(), t, h, d, out_k.data_ptr(), out_v.data_ptr(),
                                  kst, _status_ptr(status, dev), _stream_on(stream, dev)))


def decode_kv4(plan: Plan, q, prefix_k, prefix_v, pool, page_indptr, page_indices, suffix_lens, out, lse, *, prefix_strides=None,
               stream=None, stage="all"):
    """psa_decode_kv4 (or one of its stages): decode with the samples' own tokens in a 4-bit pool [pages, Hkv, kv4_cell_bytes(D)]
    uint8.  Everything else as for decode; the work lists and the workspace are those of plan.for_kv4()."""
    if _torch is None:
        _bind_torch()
    if stage not in ("all", "prefix", "suffix", "merge"):
        raise ValueError(stage)
    plan = plan._kv4 or plan.for_kv4()
    if stage in ("prefix", "merge"):
        decode(plan, q, prefix_k, prefix_v, None, None, page_indptr, page_indices, suffix_lens, out, lse, prefix_strides=prefix_strides,
               stream=stream, stage=stage)
        return
    if pool.dtype is not _u8_t or pool.dim() != 3 or pool.shape[1] != plan.num_kv_heads:
        raise ValueError("pool must be uint8 [pages, num_kv_heads, kv4_cell_bytes(head_dim)]")
    pst = _outer_strides(pool, 20 * plan.head_dim, "pool")
    rows, i32 = plan.suffix_len_bounds.size, _i32_t
    dev = _device_of(pool, "pool")
    if plan.workspace is None:
        plan.bind_workspace(stream=stream)
    lib, ws, heads = library(), plan.workspace, rows * plan.num_q_heads
    p_q = _flat(q, _bf16_t, "q", dev, heads * plan.head_dim)
    p_indptr = _flat(page_indptr, i32, "page_indptr", dev, rows + 1)
    p_indices = _flat(page_indices, i32, "page_indices", dev)
    p_lens = _flat(suffix_lens, i32, "suffix_lens", dev, rows)
    st = _stream_on(stream, dev)
    if stage == "suffix":
        _check(lib.psa_decode_suffix_kv4(plan._h, p_q, pool.data_ptr(), pst, p_indptr, p_indices, p_lens, ws.data_ptr(), ws.numel(), st))
        return
    for t, name in ((prefix_k, "prefix_k"), (prefix_v, "prefix_v")):
        if t is not None and (t.dtype is not _bf16_t or t.get_device() != dev):
            raise ValueError(f"{name} must be bf16 on the current CUDA device")
    p_out = _flat(out, _f32_t if plan.out_dtype == PSA_OUT_F32 else _bf16_t, "out", dev, heads * plan.head_dim)
    p_lse = _flat(lse, _f32_t, "lse", dev, heads)
    kst = _strides2(plan.num_kv_heads * plan.head_dim, plan.head_dim) if prefix_strides is None else _strides2(*prefix_strides)
    _check(lib.psa_decode_kv4(plan._h, p_q, _ptr(prefix_k), _ptr(prefix_v), kst, pool.data_ptr(), pst, p_indptr, p_indices, p_lens,
                              p_out, p_lse, ws.data_ptr(), ws.numel(), st))


def _dtype_code(t, name):
    if t.dtype is _bf16_t:
        return PSA_OUT_BF16
    if t.dtype is _f32_t:
        return PSA_OUT_F32
    raise ValueError(f"{name} must be bf16 or f32, not {t.dtype}")


def _bitmap_args(bits, rows, words, R, name, dev):
    """(address, row stride in words, number of bitmaps, address of the row numbers) of a set of bitmaps."""
    if bits is None:
        if rows is not None:
            raise ValueError(f"{name}_rows without {name}_bits")
        return None, 0, 0, None
    count, width = bits.shape if bits.dim() == 2 else (0, -1)
    if bits.dtype is not _i32_t or width < words or (bits.stride(1) != 1 and width > 1):
        raise ValueError(f"{name}_bits must be int32 [bitmaps, words >= {words}], contiguous along the second dimension")
    if rows is None and count < R:
        raise ValueError(f"{name}_bits needs one bitmap per row, or {name}_rows")
    if bits.get_device() != dev:
        raise ValueError(f"{name}_bits must be on the current CUDA device")
    return bits.data_ptr(), bits.stride(0) if count > 1 else width, count, _flat(rows, _i32_t, f"{name}_rows", dev, R)


def process_logits(logits, out=None, *, repetition=None, frequency=None, presence=None, history=None, history_lens=None,
                   prompt_bits=None, prompt_rows=None, bias_indptr=None, bias_ids=None, bias_values=None, mask_bits=None,
                   mask_rows=None, scratch=None, stream=None):
    """psa_process_logits on torch CUDA tensors: penalties for repeated tokens, biases and grammar masks.  logits and out [R, V] bf16
    or f32 (rows may be padded; out may be logits; allocated when None); repetition / frequency / presence [R] f32; history
    [R, capacity] int32 with history_lens [R]; prompt_bits / mask_bits [*, >= ceil(V / 32)] int32 bitmaps chosen per row by prompt_rows /
    mask_rows [R] int32; bias_indptr [R+1], bias_ids int32 and bias_values f32; scratch uint8 (psa_process_logits_scratch_bytes, for callers
    that must not allocate).  Returns out."""
    if _torch is None:
        _bind_torch()
    if logits.dim() != 2 or (out is not None and out.shape != logits.shape):
        raise ValueError("logits must be [rows, vocab], and out of the same shape")
    R, V = logits.shape
    in_code = _dtype_code(logits, "logits")
    if out is None:
        out = _torch.empty((R, (V + 7) // 8 * 8), dtype=logits.dtype, device=logits.device)[:, :V]
    out_code = _dtype_code(out, "out")
    in_stride, step = logits.stride()
    out_stride, out_step = out.stride()
    if (step != 1 or out_step != 1) and V > 1:
        raise ValueError("logits and out must be contiguous along the vocabulary")
    if R <= 1:      # one row has no stride of its own
        in_stride = out_stride = (V + 7) // 8 * 8
    dev = logits.get_device()
    h_ptr, h_lens, h_stride, h_cap = None, None, 0, 0
    if history is not None and history_lens is not None:
        if history.dtype is not _i32_t or history.dim() != 2 or history.shape[0] < R or (history.stride(1) != 1 and history.shape[1] > 1):
            raise ValueError("history must be int32 [rows, capacity], contiguous along the second dimension")
        h_cap = history.shape[1]
        h_stride = history.stride(0) if history.shape[0] > 1 else h_cap
        if history.get_device() != dev:
            raise ValueError("history must be on the current CUDA device")
        h_ptr, h_lens = history.data_ptr(), _flat(history_lens, _i32_t, "history_lens", dev, R)
    elif history is not history_lens:
        raise ValueError("history and history_lens go together")
    b_indptr, b_ids, b_values, b_count = None, None, None, 0
    if bias_indptr is not None and bias_ids is not None and bias_values is not None:
        b_count = bias_ids.numel()
        b_indptr = _flat(bias_indptr, _i32_t, "bias_indptr", dev, R + 1)
        b_ids = _flat(bias_ids, _i32_t, "bias_ids", dev)
        b_values = _flat(bias_values, _f32_t, "bias_values", dev, b_count)
    elif not (bias_indptr is bias_ids is bias_values):
        raise ValueError("bias_indptr, bias_ids and bias_values go together")
    words = (V + 31) // 32
    prompt = _bitmap_args(prompt_bits, prompt_rows, words, R, "prompt", dev)
    mask = _bitmap_args(mask_bits, mask_rows, words, R, "mask", dev)
    f32 = _f32_t
    rules = _LogitsRules(_flat(repetition, f32, "repetition", dev, R), _flat(frequency, f32, "frequency", dev, R),
                         _flat(presence, f32, "presence", dev, R), h_ptr, h_lens, h_stride, h_cap, *prompt, b_indptr, b_ids, b_values, b_count, *mask)
    if out.get_device() != _device_of(logits, "logits"):
        raise ValueError("out must be on the current CUDA device")
    lib, need = library(), 0
    if h_cap > 0 or b_count > 0:
        need = lib.psa_process_logits_scratch_bytes(R, V)
        if need and scratch is None:
            scratch = _torch.empty(need, dtype=_u8_t, device=logits.device)
    _check(lib.psa_process_logits(logits.data_ptr(), in_code, in_stride, R, V, ctypes.byref(rules), out.data_ptr(), out_code, out_stride,
                                  _flat(scratch, _u8_t, "scratch", dev, need) if need else None, need, _stream_on(stream, dev)))
    return out


def mark_tokens(ids, indptr, vocab, bits=None, *, stream=None):
    """psa_mark_tokens: bitmaps [rows, >= ceil(vocab / 32)] int32 of the tokens in ids[indptr[m] .. indptr[m + 1]).  Returns bits."""
    if _torch is None:
        _bind_torch()
    vocab = int(vocab)
    rows, words = indptr.numel() - 1, (vocab + 31) // 32
    if rows < 0:
        raise ValueError("indptr must hold rows + 1 elements")
    if bits is None:
        bits = _torch.empty((rows, words), dtype=_i32_t, device=ids.device)
    count, width = bits.shape if bits.dim() == 2 else (0, -1)
    if bits.dtype is not _i32_t or count < rows or width < words or (bits.stride(1) != 1 and width > 1):
        raise ValueError(f"bits must be int32 [rows, words >= {words}], contiguous along the second dimension")
    dev = ids.get_device()
    p_ids = _flat(ids, _i32_t, "ids", dev)
    p_indptr = _flat(indptr, _i32_t, "indptr", dev)
    if bits.get_device() != _device_of(ids, "ids"):
        raise ValueError("bits must be on the current CUDA device")
    _check(library().psa_mark_tokens(p_ids, ids.numel(), p_indptr, rows, vocab, bits.data_ptr(), bits.stride(0) if count > 1 else width,
                                     _stream_on(stream, dev)))
    return bits
