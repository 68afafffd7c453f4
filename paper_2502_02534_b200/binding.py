from __future__ import annotations

import ctypes
from contextlib import nullcontext
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
    "psa_load_kv4", "psa_plan_create_kv4", "psa_decode_kv4", "psa_decode_suffix_kv4", "psa_process_logits", "psa_mark_tokens",
    "psa_store_kv", "psa_attend_paged_scratch_bytes", "psa_attend_paged",
    "psa_accumulate_weights_scratch_bytes", "psa_accumulate_weights", "psa_evict_pages_scratch_bytes", "psa_evict_pages", "psa_token_logprobs",
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
        lib.psa_process_logits.restype = c_int32
        lib.psa_process_logits.argtypes = [P, c_int32, c_int64, c_int32, c_int32, POINTER(_LogitsRules), P, c_int32, c_int64, P]
        lib.psa_mark_tokens.restype = c_int32
        lib.psa_mark_tokens.argtypes = [P, c_int32, P, c_int32, c_int32, P, c_int64, P]
        lib.psa_store_kv.restype = c_int32
        lib.psa_store_kv.argtypes = [P, P, POINTER(c_int64), P, c_int64, c_int32, c_int32, P, P, POINTER(c_int64), c_int64, P, P]
        lib.psa_attend_paged_scratch_bytes.restype = c_size_t
        lib.psa_attend_paged_scratch_bytes.argtypes = [c_int64, c_int32, c_int32, c_int32, c_int32]
        lib.psa_attend_paged.restype = c_int32
        lib.psa_attend_paged.argtypes = [P, POINTER(c_int64), P, c_int64, c_int32, c_int32, c_int32, c_int32, c_float, P, P, POINTER(c_int64), c_int64, P, P,
                                         c_int64, P, P, c_int32, P, P, c_int32, P, P, P, c_size_t, P]
        lib.psa_accumulate_weights_scratch_bytes.restype = c_size_t
        lib.psa_accumulate_weights_scratch_bytes.argtypes = [c_int64, c_int32]
        lib.psa_accumulate_weights.restype = c_int32
        lib.psa_accumulate_weights.argtypes = [P, POINTER(c_int64), P, c_int64, c_int32, c_int32, c_int32, c_int32, c_float, P, P, POINTER(c_int64), c_int64, P,
                                               P, c_int64, P, P, P, P, P, c_size_t, P]
        lib.psa_evict_pages_scratch_bytes.restype = c_size_t
        lib.psa_evict_pages_scratch_bytes.argtypes = [c_int32, c_int64]
        lib.psa_evict_pages.restype = c_int32
        lib.psa_evict_pages.argtypes = [P, c_int64, c_int32, P, P, c_int64, P, P, c_int32, c_int32, P, c_int64, P, P, P, P, P, P, c_size_t, P]
        lib.psa_token_logprobs.restype = c_int32
        lib.psa_token_logprobs.argtypes = [P, c_int32, c_int64, c_int32, c_int32, P, P, P, P, c_int32, P, P, c_int64, P]
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


def _on(stream):
    """The context of a stream, given as torch's, as its handle or as an object that has one (None: the current stream)."""
    if stream is None:
        return nullcontext()
    import torch
    if not isinstance(stream, torch.cuda.Stream):
        handle = _stream_ptr(stream)
        stream = torch.cuda.ExternalStream(handle) if handle else torch.cuda.default_stream()
    return torch.cuda.stream(stream)


_TYPE_CODES = {"int32": 1, "uint8": 2, "float32": 3}


def _new(shape, like, stream, dtype=None):
    """A tensor that a call on `stream` writes and returns, on the device and (dtype None) of the type of `like`.  Allocated for that stream, as
    the native module's `empty` says."""
    if stream is not None:
        return (_calls or _native()).empty(like, _TYPE_CODES.get(dtype, 0), shape, stream, True)
    import torch
    return torch.empty(shape, dtype=getattr(torch, dtype) if dtype else like.dtype, device=like.device)


def _scratch(nbytes, like, stream):
    """A scratch tensor for one call on `stream` (None: the current one)."""
    if stream is not None:
        return (_calls or _native()).empty(like, 2, (int(nbytes),), stream, False)
    import torch
    return torch.empty(int(nbytes), dtype=torch.uint8, device=like.device)


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
        self._kv4 = None            # the plan for_kv4 returns, once made
        self._is_kv4 = False

    def for_kv4(self) -> "Plan":
        """The plan of the same problem whose pieces are sized for a 4-bit cache (psa_plan_create_kv4), with a workspace of its own.
        decode_kv4 uses it in place of this one; it is made once and kept.  `plan.for_kv4().bind_workspace()` makes it ready for a capture or
        gives it a workspace of the caller's."""
        if self._is_kv4:
            return self
        if self._kv4 is None:
            handle = c_void_p()
            _check(library().psa_plan_create_kv4(self._h, ctypes.byref(handle)))
            plan = Plan.__new__(Plan)
            plan.__dict__.update(self.__dict__, _h=handle, workspace=None, _is_kv4=True, _prefix_tokens=self._prefix_tokens_read())
            self._kv4 = plan
        return self._kv4

    def _prefix_tokens_read(self) -> int:
        """Tokens the packed prefix arrays must hold: all of them (a tile of keys reaches into the next prompt's), or none if no sample attends
        over any."""
        samples, lens = self.groups[1:] if hasattr(self, "groups") else (self.n_samples, self.prefix_lens)
        return int(lens.sum(dtype=np.int64)) if ((samples > 0) & (lens > 0)).any() else 0

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
            with _on(stream):
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
        if self._kv4 is not None and self._kv4.workspace is not None:
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
        tokens = _new((B,), logits, stream, "int32")
    if scratch is None:
        scratch = _scratch(max(8, int(lib.psa_sample_scratch_bytes(B))), logits, stream)
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
        tokens = _new((B,), logits, stream, "int32")
    need = int(lib.psa_sample_scratch_bytes(B))
    if scratch is None:
        scratch = _scratch(max(8, need), logits, stream)
    _check(lib.psa_sample_tokens(_ptr(logits), dtype, logits.stride(0), B, V, _ptr(temperature), _ptr(seeds), int(step) & 0xFFFFFFFF,
                                 _ptr(tokens), _ptr(scratch), scratch.numel(), _stream_ptr(stream)))
    return tokens


def attn_task(task, q, k, v, sm_scale, *, stream=None):
    """psa_attn_task on torch CUDA tensors: q [R, D], k / v [M, D] bf16.  Returns (out [R, D] f32, m [R], l [R])."""
    R, D = q.shape
    M = k.shape[0]
    out, m, l = (_new(shape, q, stream, "float32") for shape in ((R, D), (R,), (R,)))  # noqa: E741
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


# ---- page tables, the 4-bit cache and rules on logits.  Their tensors are checked (type, layout, size, and that all of them live on the
# ---- current CUDA device: ValueError otherwise) and marshalled by the native module _torch_calls; what the library itself refuses comes
# ---- back as PsaError.

_CALLS_PATH = _HERE / "_torch_calls.so"
_calls = None


def _native():
    """Load _torch_calls.so.  Raises if it has not been built: there is no other implementation."""
    global _calls
    if _calls is None:
        import importlib.util
        import torch  # noqa: F401  (the module's own libraries)
        library()
        if not _CALLS_PATH.exists():
            raise ImportError(f"{_CALLS_PATH} is missing: build it with `python -m paper_2502_02534_b200.build`")
        spec = importlib.util.spec_from_file_location("_torch_calls", _CALLS_PATH)
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
        module.attach(str(_LIB_PATH))
        _calls = module
    return _calls


def _status_tensor(status):
    """A status word: a one-element int32 tensor, or a Plan (a word that Plan.check_status reads)."""
    if isinstance(status, Plan):
        workspace = status.workspace
        if workspace is None and status._kv4 is not None:
            workspace = status._kv4.workspace
        if workspace is None:
            raise ValueError("status: the plan has no workspace yet")
        return workspace
    return status


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
    if status is not None:
        status = _status_tensor(status)
    if scratch is None:
        scratch = _scratch(library().psa_page_table_scratch_bytes(seq_lens.numel()), seq_lens, stream)
    rc = (_calls or _native()).build_page_table(seq_lens, reserve_lens, free_pages, free_count, free_count_out, page_indptr, page_indices,
                                                token_indptr, slot_map, lens_out, status, scratch, stream)
    if rc:
        _check(rc)


def extend_page_table(held_lens, new_lens, free_pages, free_count, page_indptr, page_indices, token_indptr, slot_map, *, max_lens=None,
                      lens_out=None, free_count_out=None, status=None, scratch=None, stream=None):
    """psa_extend_page_table on torch CUDA tensors: new_lens more tokens for samples that hold held_lens, in existing page lists.
    Outputs as for build_page_table; lens_out and free_count_out may be held_lens and free_count themselves."""
    if status is not None:
        status = _status_tensor(status)
    if scratch is None:
        scratch = _scratch(library().psa_page_table_scratch_bytes(held_lens.numel()), held_lens, stream)
    rc = (_calls or _native()).extend_page_table(held_lens, new_lens, max_lens, free_pages, free_count, free_count_out, page_indptr, page_indices,
                                                 token_indptr, slot_map, lens_out, status, scratch, stream)
    if rc:
        _check(rc)


def read_status(status, stream=None):
    """psa_read_status: synchronise, raise if the one-element int32 tensor `status` holds an error, and clear it."""
    import torch
    if status.dtype is not torch.int32 or status.numel() < 1 or not status.is_cuda:
        raise ValueError("status must be a one-element int32 CUDA tensor")
    _check(library().psa_read_status(status.data_ptr(), _stream_ptr(stream)))


def kv4_cell_bytes(head_dim) -> int:
    """Bytes of one (page, KV head) cell of the 4-bit cache."""
    return int(library().psa_kv4_cell_bytes(int(head_dim)))


def store_kv4(new_k, new_v, slot_map, pool, *, status=None, stream=None):
    """psa_store_kv4: quantise new_k / new_v [T, Hkv, D] bf16 (any token and head stride, the same for both) into the slots of a 4-bit pool
    [pages, Hkv, kv4_cell_bytes(D)] uint8."""
    if status is not None:
        status = _status_tensor(status)
    rc = (_calls or _native()).store_kv4(new_k, new_v, slot_map, pool, status, stream)
    if rc:
        _check(rc)


def load_kv4(pool, slot_map, out_k, out_v, *, status=None, stream=None):
    """psa_load_kv4: the cached tokens of slot_map as bf16 rows out_k / out_v [T, Hkv, D]; rows of negative slots are left alone."""
    if status is not None:
        status = _status_tensor(status)
    rc = (_calls or _native()).load_kv4(out_k, out_v, slot_map, pool, status, stream)
    if rc:
        _check(rc)


def decode_kv4(plan: Plan, q, prefix_k, prefix_v, pool, page_indptr, page_indices, suffix_lens, out, lse, *, prefix_strides=None,
               stream=None, stage="all"):
    """psa_decode_kv4 (or one of its stages): decode with the samples' own tokens in a 4-bit pool [pages, Hkv, kv4_cell_bytes(D)]
    uint8.  prefix_k and prefix_v are [tokens, Hkv, D] of any token and head stride (prefix_strides: those of the packed array in their
    storage, for tensors of another form).  Everything else as for decode; the work lists and the workspace are those of plan.for_kv4(),
    made at the first call unless plan.for_kv4().bind_workspace() has been called before: one of the two has to come before a stream
    capture."""
    plan = plan._kv4 or plan.for_kv4()
    if stage != "all":
        return _decode_kv4_stage(plan, q, prefix_k, prefix_v, pool, page_indptr, page_indices, suffix_lens, out, lse, prefix_strides, stream, stage)
    if plan.workspace is None:
        if not pool.is_cuda:
            raise ValueError("pool must be on the current CUDA device")
        _bind_kv4(plan, stream)
    head_dim = plan.head_dim
    s0, s1 = (None, None) if prefix_strides is None else prefix_strides
    rc = (_calls or _native()).decode_kv4(plan._h.value, plan.suffix_len_bounds.size, plan.num_q_heads, plan.num_kv_heads, head_dim, plan.out_dtype,
                                          plan._prefix_tokens, q, prefix_k, prefix_v, s0, s1, pool, page_indptr, page_indices, suffix_lens, out, lse,
                                          plan.workspace, stream)
    if rc:
        _check(rc)


def _bind_kv4(plan, stream):
    """Bind a workspace to a 4-bit plan outside a capture.  Inside one the upload would run at every replay instead of now, out of memory that
    the plan may have freed by then, and an eager call before the first replay would find no work lists."""
    import torch
    with _on(stream):
        if torch.cuda.is_current_stream_capturing():
            raise ValueError("the 4-bit plan has no workspace yet: call plan.for_kv4().bind_workspace(), or decode_kv4 once, before the capture")
    plan.bind_workspace(stream=stream)


def _decode_kv4_stage(plan, q, prefix_k, prefix_v, pool, page_indptr, page_indices, suffix_lens, out, lse, prefix_strides, stream, stage):
    """One stage of a 4-bit step, for tests and per-kernel timing."""
    if stage in ("prefix", "merge"):
        if plan.workspace is None:
            _bind_kv4(plan, stream)
        if stage == "prefix":
            s0, s1 = (None, None) if prefix_strides is None else prefix_strides
            prefix_strides = (_calls or _native()).prefix_strides(plan._prefix_tokens, plan.num_kv_heads, plan.head_dim, prefix_k, prefix_v, s0, s1, stream)
        return decode(plan, q, prefix_k, prefix_v, None, None, page_indptr, page_indices, suffix_lens, out, lse, prefix_strides=prefix_strides,
                      stream=stream, stage=stage)
    if stage != "suffix":
        raise ValueError(stage)
    if pool.dim() != 3 or pool.element_size() != 1 or pool.stride(2) != 1 or not pool.is_cuda:
        raise ValueError("pool must be uint8 [pages, num_kv_heads, kv4_cell_bytes(head_dim)] on the current CUDA device")
    if plan.workspace is None:
        _bind_kv4(plan, stream)
    _check(library().psa_decode_suffix_kv4(plan.handle, _ptr(q), _ptr(pool), _strides(pool.stride()[:2], 2), _ptr(page_indptr), _ptr(page_indices),
                                           _ptr(suffix_lens), _ptr(plan.workspace), plan.workspace.numel(), _stream_ptr(stream)))


def process_logits(logits, out=None, *, repetition=None, frequency=None, presence=None, history=None, history_lens=None,
                   prompt_bits=None, prompt_rows=None, bias_indptr=None, bias_ids=None, bias_values=None, mask_bits=None,
                   mask_rows=None, stream=None):
    """psa_process_logits on torch CUDA tensors: penalties for repeated tokens, biases and grammar masks.  logits and out [R, V] bf16
    or f32 (rows may be padded; out may be logits; allocated when None); repetition / frequency / presence [R] f32; history
    [R, capacity] int32 with history_lens [R]; prompt_bits / mask_bits [*, >= ceil(V / 32)] int32 bitmaps chosen per row by prompt_rows /
    mask_rows [R] int32; bias_indptr [R+1], bias_ids int32 and bias_values f32.  Returns out."""
    rows, vocab = logits.shape
    if out is None:
        out = _new((rows, (vocab + 7) // 8 * 8), logits, stream)[:, :vocab]
    rc = (_calls or _native()).process_logits(logits, out, repetition, frequency, presence, history, history_lens, prompt_bits, prompt_rows, bias_indptr,
                                              bias_ids, bias_values, mask_bits, mask_rows, stream)
    if rc:
        _check(rc)
    return out


def mark_tokens(ids, indptr, vocab, bits=None, *, stream=None):
    """psa_mark_tokens: bitmaps [rows, >= ceil(vocab / 32)] int32 of the tokens in ids[indptr[m] .. indptr[m + 1]).  Returns bits."""
    if bits is None:
        bits = _new((max(0, indptr.numel() - 1), (int(vocab) + 31) // 32), ids, stream, "int32")
    rc = (_calls or _native()).mark_tokens(ids, indptr, vocab, bits, stream)
    if rc:
        _check(rc)
    return bits


# ---- several new tokens per sample over the bf16 cache, checked and marshalled as above

def store_kv(new_k, new_v, slot_map, k_pool, v_pool, *, status=None, stream=None):
    """psa_store_kv: write new_k / new_v [T, Hkv, D] bf16 (any token and head stride, the same for both) into the slots of the pools
    [pages, Hkv, 16, D] bf16 (any strides, the same for both; the last dimension contiguous)."""
    if status is not None:
        status = _status_tensor(status)
    rc = (_calls or _native()).store_kv(new_k, new_v, slot_map, k_pool, v_pool, status, stream)
    if rc:
        _check(rc)


def attend_paged_scratch(num_tokens, num_samples, num_q_heads, num_kv_heads, head_dim):
    """Scratch tensor for attend_paged, to be kept by callers that must not allocate (uint8)."""
    import torch
    return torch.empty(int(library().psa_attend_paged_scratch_bytes(num_tokens, num_samples, num_q_heads, num_kv_heads, head_dim)), dtype=torch.uint8, device="cuda")


def attend_paged(q, k_pool, v_pool, page_indptr, page_indices, kv_lens, q_indptr=None, out=None, lse=None, *, sm_scale=None, prior_out=None,
                 prior_lse=None, status=None, scratch=None, stream=None):
    """psa_attend_paged on torch CUDA tensors: the new tokens q [T, Hq, D] bf16 (any token and head stride) of every sample, rows
    q_indptr[s] .. q_indptr[s + 1] (one each when None), over the sample's kv_lens[s] tokens in pages, which end with the new ones; each sees
    what stands up to itself.  prior_out / prior_lse: the same rows over other keys, joined with the result.  out [T, Hq, D] bf16 or f32
    (bf16 when None), lse [T, Hq] f32.  Returns (out, lse)."""
    if q.dim() != 3 or k_pool.dim() != 4:
        raise ValueError("q must be [tokens, heads, head_dim] and the pools [pages, heads, 16, head_dim]")
    if status is not None:
        status = _status_tensor(status)
    if out is None:
        out = _new3(q, stream)
    if lse is None:
        lse = _new(tuple(q.shape[:2]), q, stream, "float32")
    if scratch is None:
        nbytes = library().psa_attend_paged_scratch_bytes(q.shape[0], kv_lens.numel(), q.shape[1], k_pool.shape[1], q.shape[2])
        scratch = _scratch(nbytes, q, stream)
    rc = (_calls or _native()).attend_paged(q, k_pool, v_pool, page_indptr, page_indices, kv_lens, q_indptr, out, lse,
                                            q.shape[-1] ** -0.5 if sm_scale is None else sm_scale, prior_out, prior_lse, status, scratch, stream)
    if rc:
        _check(rc)
    return out, lse


def _new3(like, stream):
    """_new of the shape and type of the three-dimensional `like`."""
    T, H, D = like.shape
    return _new((T * H, D), like, stream).view(T, H, D)


def accumulate_weights_scratch(num_tokens, num_samples):
    """Scratch tensor for accumulate_weights, to be kept by callers that must not allocate (uint8)."""
    import torch
    return torch.empty(int(library().psa_accumulate_weights_scratch_bytes(num_tokens, num_samples)), dtype=torch.uint8, device="cuda")


def accumulate_weights(q, lse, k_pool, page_indptr, page_indices, kv_lens, q_indptr, weights, *, weights_out=None, sm_scale=None, status=None,
                       scratch=None, stream=None):
    """psa_accumulate_weights on torch CUDA tensors: add to weights [pages, Hkv, 16] f32 (or write to weights_out) the attention weight that
    the rows q [T, Hq, D] with log-sum-exps lse [T, Hq] f32 gave to every cached token they see; new tokens start from zero.  Rows and
    samples as for attend_paged."""
    if status is not None:
        status = _status_tensor(status)
    if scratch is None:
        scratch = _scratch(library().psa_accumulate_weights_scratch_bytes(q.shape[0], kv_lens.numel()), q, stream)
    rc = (_calls or _native()).accumulate_weights(q, lse, k_pool, page_indptr, page_indices, kv_lens, q_indptr, weights, weights_out,
                                                  q.shape[-1] ** -0.5 if sm_scale is None else sm_scale, status, scratch, stream)
    if rc:
        _check(rc)


def evict_pages_scratch(num_samples, num_entries):
    """Scratch tensor for evict_pages, to be kept by callers that must not allocate (uint8)."""
    import torch
    return torch.empty(int(library().psa_evict_pages_scratch_bytes(num_samples, num_entries)), dtype=torch.uint8, device="cuda")


def evict_pages(weights, page_indptr, page_indices, kv_lens, budgets, recent, free_pages, free_count, *, page_indices_out=None, lens_out=None,
                free_count_out=None, status=None, scratch=None, stream=None):
    """psa_evict_pages on torch CUDA tensors (int32; weights [pages, Hkv, 16] f32): samples of more than budgets[s] pages keep their `recent`
    newest and the heaviest others; ids that leave go onto the stack free_pages[0 .. free_count).  Lists, lengths and count are updated in
    place where no output is given."""
    if status is not None:
        status = _status_tensor(status)
    if scratch is None:
        scratch = _scratch(library().psa_evict_pages_scratch_bytes(kv_lens.numel(), page_indices.numel()), weights, stream)
    rc = (_calls or _native()).evict_pages(weights, page_indptr, page_indices, kv_lens, budgets, recent, free_pages, free_count, page_indices_out,
                                           lens_out, free_count_out, status, scratch, stream)
    if rc:
        _check(rc)


def token_logprobs(logits, tokens, top=0, *, temperature=None, logprobs=None, entropy=None, top_ids=None, top_logprobs=None, stream=None):
    """psa_token_logprobs on torch CUDA tensors: of every row of logits [R, V] (bf16 or f32; rows may be padded) at temperature [R] f32 the
    log probability of tokens [R] int32 (None: left out), the entropy, and the `top` likeliest tokens with theirs.  Returns (logprobs [R],
    entropy [R], top_ids [R, top] int32, top_logprobs [R, top])."""
    rows = logits.shape[0]
    if logprobs is None and tokens is not None:
        logprobs = _new((rows,), logits, stream, "float32")
    if entropy is None:
        entropy = _new((rows,), logits, stream, "float32")
    if top_ids is None:
        top_ids = _new((rows, top), logits, stream, "int32")
    if top_logprobs is None:
        top_logprobs = _new((rows, top), logits, stream, "float32")
    rc = (_calls or _native()).token_logprobs(logits, tokens, top, temperature, logprobs, entropy, top_ids, top_logprobs, stream)
    if rc:
        _check(rc)
    return logprobs, entropy, top_ids, top_logprobs
