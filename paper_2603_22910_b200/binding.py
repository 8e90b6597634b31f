"""ctypes binding of libechokv.so: the same names as include/echokv.h, argument
marshalling only.  Every step of the decode path runs in the library's CUDA
kernels; PyTorch is used by `Context` for device memory and streams.

The library must have been built (python -m paper_2603_22910_b200.build);
loading fails loudly otherwise -- there is no fallback path.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import math
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libechokv.so")

ECHOKV_BF16, ECHOKV_FP32 = 0, 1
ECHOKV_OK = 0
ECHOKV_EINVAL, ECHOKV_ENOTANCHOR, ECHOKV_ENOTCOMPRESSED, ECHOKV_ECAPACITY = -1, -2, -3, -4
ECHOKV_ENOWEIGHTS, ECHOKV_ECUDA, ECHOKV_ETIMEOUT, ECHOKV_EBADPAGE = -5, -6, -7, -8
ECHOKV_EUNSUPPORTED, ECHOKV_ENOTABLE, ECHOKV_EBADLENGTH, ECHOKV_ESCRATCH = -9, -10, -11, -12
ECHOKV_INT8, ECHOKV_E4M3 = 0, 1
ECHOKV_QUANT_BLOCK_TOKENS = 16
ECHOKV_FOURBIT_GROUP, ECHOKV_FOURBIT_MAX_SELECT = 16, 1024
QUANT_FORMATS = {"int8": ECHOKV_INT8, "e4m3": ECHOKV_E4M3}


class echokv_config(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("group_size", C.c_int32), ("n_retained_heads", C.c_int32),
                ("page_tokens", C.c_int32), ("max_batch", C.c_int32), ("max_pages_per_seq", C.c_int32),
                ("dtype", C.c_int32), ("n_pages", C.c_int64), ("softmax_scale", C.c_float),
                ("device", C.c_int32), ("n_retained_dims", C.c_int32), ("save_k", C.c_int32)]


class echokv_sizes(C.Structure):
    _fields_ = [("anchor_pool_bytes", C.c_uint64), ("compressed_pool_bytes", C.c_uint64),
                ("block_table_bytes", C.c_uint64), ("workspace_bytes", C.c_uint64),
                ("max_partials", C.c_int32), ("reserved", C.c_int32)]


class echokv_buffers(C.Structure):
    _fields_ = [("k_pools", C.POINTER(C.c_void_p)), ("v_pools", C.POINTER(C.c_void_p)),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_uint64)]


class echokv_step_plan(C.Structure):
    _fields_ = [("cu_tokens", C.c_void_p), ("positions", C.c_void_p), ("token_seqs", C.c_void_p),
                ("slot_map", C.c_void_p), ("seq_lens", C.c_void_p), ("free_count", C.c_void_p)]


class echokv_quant_cache(C.Structure):
    _fields_ = [("k_codes", C.c_void_p), ("v_codes", C.c_void_p), ("k_scales", C.c_void_p), ("v_scales", C.c_void_p),
                ("k_tail", C.c_void_p), ("v_tail", C.c_void_p), ("format", C.c_int32), ("reserved", C.c_int32)]


class echokv_quant_sizes(C.Structure):
    _fields_ = [("codes_bytes", C.c_uint64), ("scales_bytes", C.c_uint64), ("tail_bytes", C.c_uint64),
                ("workspace_bytes", C.c_uint64)]


class echokv_score_options(C.Structure):
    _fields_ = [("softcap", C.c_float), ("reserved", C.c_int32), ("alibi_slopes", C.c_void_p),
                ("prefix_lens", C.c_void_p)]


class echokv_fourbit_cache(C.Structure):
    _fields_ = [("blocks", C.c_void_p), ("bounds", C.c_void_p), ("bound_scales", C.c_void_p), ("k_unit", C.c_float),
                ("v_unit", C.c_float)]


class echokv_fourbit_sizes(C.Structure):
    _fields_ = [("blocks_bytes", C.c_uint64), ("bounds_bytes", C.c_uint64), ("bound_scales_bytes", C.c_uint64),
                ("workspace_bytes", C.c_uint64)]


class echokv_rotation(C.Structure):
    _fields_ = [("theta", C.c_double), ("sections", C.POINTER(C.c_int32)), ("n_axes", C.c_int32), ("interleaved", C.c_int32),
                ("rot_dim", C.c_int32), ("reserved", C.c_int32)]


EXPORTS = {
    # name: (restype, argtypes)
    "echokv_query_sizes": (C.c_int, [C.POINTER(echokv_config), C.POINTER(echokv_sizes)]),
    "echokv_create": (C.c_int, [C.POINTER(echokv_config), C.POINTER(echokv_buffers), C.POINTER(C.c_void_p)]),
    "echokv_destroy": (None, [C.c_void_p]),
    "echokv_set_weights": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "echokv_set_block_table": (C.c_int, [C.c_void_p, C.c_void_p]),
    "echokv_append_kv": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                   C.c_int, C.c_void_p]),
    "echokv_append_kv_chunk": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                         C.c_int, C.c_int, C.c_void_p]),
    "echokv_compress_layer": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                        C.c_void_p, C.c_int, C.c_void_p]),
    "echokv_decode_attention": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p,
                                          C.c_void_p, C.c_int, C.c_void_p]),
    "echokv_full_attention": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p,
                                        C.c_void_p, C.c_int, C.c_void_p]),
    "echokv_prefill_scratch_bytes": (C.c_int, [C.POINTER(echokv_config), C.POINTER(C.c_uint64)]),
    "echokv_prefill_attention": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p,
                                           C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_uint64,
                                           C.c_void_p]),
    "echokv_layer_step_host": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p,
                                         C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_void_p]),
    "echokv_get_device_status": (C.c_int, [C.c_void_p, C.POINTER(C.c_int32)]),
    "echokv_launch_count": (C.c_int64, [C.c_void_p]),
    "echokv_decode_path": (C.c_int, [C.c_void_p]),
    "echokv_set_decode_path": (C.c_int, [C.c_void_p, C.c_int]),
    "echokv_side_buffer_bytes": (C.c_int, [C.POINTER(echokv_config), C.c_int, C.c_int, C.POINTER(C.c_uint64)]),
    "echokv_set_full_precision_window": (C.c_int, [C.c_void_p, C.c_int, C.c_int, C.POINTER(C.c_void_p),
                                                   C.POINTER(C.c_void_p)]),
    "echokv_rope_table_bytes": (C.c_int, [C.POINTER(echokv_config), C.POINTER(C.c_uint64)]),
    "echokv_set_rope": (C.c_int, [C.c_void_p, C.c_double, C.c_void_p, C.c_uint64, C.c_void_p]),
    "echokv_rope_enabled": (C.c_int, [C.c_void_p]),
    "echokv_absorbed_workspace_bytes": (C.c_int, [C.POINTER(echokv_config), C.POINTER(C.c_uint64)]),
    "echokv_enable_absorbed": (C.c_int, [C.c_void_p, C.c_void_p, C.c_uint64]),
    "echokv_decode_mode": (C.c_int, [C.c_void_p]),
    "echokv_set_decode_mode": (C.c_int, [C.c_void_p, C.c_int]),
    "echokv_stored_path": (C.c_int, [C.c_void_p]),
    "echokv_set_stored_path": (C.c_int, [C.c_void_p, C.c_int]),
    "echokv_set_kernel_timing": (C.c_int, [C.c_void_p, C.c_int]),
    "echokv_read_kernel_timing": (C.c_int, [C.c_void_p, C.POINTER(C.c_double), C.POINTER(C.c_int64)]),
    "echokv_read_kernel_timing_by_kind": (C.c_int, [C.c_void_p, C.POINTER(C.c_double), C.POINTER(C.c_int64)]),
    "echokv_diag_bounded_wait": (C.c_int, [C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p]),
    "echokv_diag_page_order": (C.c_int, [C.c_void_p, C.POINTER(C.c_int32)]),
    "echokv_full_attention_noalloc": (C.c_int, [C.POINTER(echokv_config), C.c_void_p, C.c_void_p, C.c_void_p,
                                                C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int,
                                                C.c_void_p, C.c_void_p]),
    "echokv_noalloc_scratch_bytes": (C.c_uint64, []),
    "echokv_plan_tokens": (C.c_int, [C.POINTER(echokv_config), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                     C.c_void_p, C.c_int, C.c_int, C.POINTER(echokv_step_plan), C.c_void_p, C.c_void_p]),
    "echokv_release_pages": (C.c_int, [C.POINTER(echokv_config), C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p,
                                       C.c_void_p, C.c_void_p, C.c_void_p]),
    "echokv_rotate": (C.c_int, [C.POINTER(echokv_config), C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64,
                                C.c_void_p, C.c_int64, C.c_void_p, C.c_int, C.POINTER(C.c_int32), C.c_int, C.c_int, C.c_double,
                                C.c_int, C.c_int, C.c_void_p]),
    "echokv_query_quant_sizes": (C.c_int, [C.POINTER(echokv_config), C.POINTER(echokv_quant_sizes)]),
    "echokv_quant_append": (C.c_int, [C.POINTER(echokv_config), C.POINTER(echokv_quant_cache), C.c_void_p, C.c_int64, C.c_void_p,
                                      C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_void_p,
                                      C.c_void_p]),
    "echokv_quant_attention": (C.c_int, [C.POINTER(echokv_config), C.POINTER(echokv_quant_cache), C.POINTER(echokv_score_options),
                                         C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int,
                                         C.c_int, C.c_int, C.c_void_p, C.c_uint64, C.c_void_p, C.c_void_p]),
    "echokv_query_fourbit_sizes": (C.c_int, [C.POINTER(echokv_config), C.POINTER(echokv_fourbit_sizes)]),
    "echokv_fourbit_append": (C.c_int, [C.POINTER(echokv_config), C.POINTER(echokv_fourbit_cache), C.POINTER(echokv_rotation), C.c_void_p,
                                    C.c_int64, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p,
                                    C.c_void_p, C.c_int, C.c_void_p, C.c_void_p]),
    "echokv_fourbit_read": (C.c_int, [C.POINTER(echokv_config), C.POINTER(echokv_fourbit_cache), C.c_void_p, C.c_int, C.c_void_p, C.c_int64,
                                  C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p]),
    "echokv_fourbit_attention": (C.c_int, [C.POINTER(echokv_config), C.POINTER(echokv_fourbit_cache), C.POINTER(echokv_score_options),
                                       C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int,
                                       C.c_int, C.c_int, C.c_void_p, C.c_uint64, C.c_void_p, C.c_void_p]),
    "echokv_fourbit_select": (C.c_int, [C.POINTER(echokv_config), C.POINTER(echokv_fourbit_cache), C.c_void_p, C.c_int64, C.c_void_p,
                                    C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_int, C.c_int, C.c_void_p,
                                    C.c_void_p, C.c_uint64, C.c_void_p, C.c_void_p]),
    "echokv_fourbit_sparse_attention": (C.c_int, [C.POINTER(echokv_config), C.POINTER(echokv_fourbit_cache), C.POINTER(echokv_score_options),
                                              C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                              C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_void_p, C.c_uint64, C.c_void_p, C.c_void_p]),
    "echokv_strerror": (C.c_char_p, [C.c_int]),
}

_lib = None


def lib() -> C.CDLL:
    """The loaded shared library (loaded once)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("libechokv.so is not built: run `python -m paper_2603_22910_b200.build` "
                               "(there is no fallback implementation)")
        _lib = C.CDLL(LIB_PATH)
        for name, (res, args) in EXPORTS.items():
            fn = getattr(_lib, name)
            fn.restype = res
            fn.argtypes = args
    return _lib


class EchoKVError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__("%s: %s (%d)" % (where, echokv_strerror(status), status))


def echokv_strerror(status: int) -> str:
    return lib().echokv_strerror(status).decode()


def _check(status: int, where: str) -> None:
    if status != ECHOKV_OK:
        raise EchoKVError(status, where)


def _ptr(t) -> int | None:
    """Device / host address of a torch tensor (None stays NULL)."""
    return None if t is None else t.data_ptr()


def _stream_handle(stream) -> int | None:
    import torch
    s = torch.cuda.current_stream() if stream is None else stream
    return s.cuda_stream or None


_CURRENT = contextlib.nullcontext()


def _memory_of(stream):
    """Where new tensors of a call on `stream` (None: the current one) are allocated: in that stream's memory, since the current
    stream's may still be in use by what is queued there."""
    if stream is None:
        return _CURRENT
    import torch
    return torch.cuda.stream(stream)


def make_config(*, n_layers, n_q_heads, n_kv_heads, head_dim, group_size, n_retained_heads,
                page_tokens, max_batch, max_pages_per_seq, n_pages, dtype, softmax_scale=0.0,
                device=0, n_retained_dims=0, save_k=0) -> echokv_config:
    return echokv_config(n_layers, n_q_heads, n_kv_heads, head_dim, group_size, n_retained_heads,
                         page_tokens, max_batch, max_pages_per_seq, dtype, n_pages, softmax_scale, device,
                         n_retained_dims, save_k)


def echokv_query_sizes(cfg: echokv_config) -> echokv_sizes:
    out = echokv_sizes()
    _check(lib().echokv_query_sizes(C.byref(cfg), C.byref(out)), "echokv_query_sizes")
    return out


class Context:
    """A context plus the torch tensors it borrows (pools, workspace, block table).

    Allocation is the only thing done here that is not a direct C-ABI call.
    """

    def __init__(self, cfg: echokv_config, zero_pools: bool = False):
        import torch
        self.torch = torch
        self.cfg = cfg
        self.device = torch.device("cuda", cfg.device)
        self.sizes = echokv_query_sizes(cfg)
        self.tdtype = torch.bfloat16 if cfg.dtype == ECHOKV_BF16 else torch.float32
        D = cfg.n_kv_heads * cfg.head_dim
        m = cfg.n_retained_dims if cfg.n_retained_dims else cfg.n_retained_heads * cfg.head_dim
        self.D, self.m = D, m
        alloc = torch.zeros if zero_pools else torch.empty
        self.k_pools, self.v_pools = [], []
        self.mk = D if (cfg.save_k and m < D) else m      # K dims a compressed layer stores ("save K": all of them)
        for l in range(cfg.n_layers):
            for pools, width in ((self.k_pools, D if l % cfg.group_size == 0 else self.mk),
                                 (self.v_pools, D if l % cfg.group_size == 0 else m)):
                if width == 0:
                    pools.append(None)
                else:
                    pools.append(alloc((cfg.n_pages, cfg.page_tokens, width), dtype=self.tdtype, device=self.device))
        self.workspace = torch.empty(self.sizes.workspace_bytes, dtype=torch.uint8, device=self.device)
        self.block_table = torch.zeros((cfg.max_batch, cfg.max_pages_per_seq), dtype=torch.int32,
                                       device=self.device)
        n = cfg.n_layers
        self._kp = (C.c_void_p * n)(*[_ptr(t) for t in self.k_pools])
        self._vp = (C.c_void_p * n)(*[_ptr(t) for t in self.v_pools])
        buf = echokv_buffers(C.cast(self._kp, C.POINTER(C.c_void_p)), C.cast(self._vp, C.POINTER(C.c_void_p)),
                             self.workspace.data_ptr(), self.sizes.workspace_bytes)
        self.handle = C.c_void_p()
        _check(lib().echokv_create(C.byref(cfg), C.byref(buf), C.byref(self.handle)), "echokv_create")
        _check(lib().echokv_set_block_table(self.handle, self.block_table.data_ptr()), "echokv_set_block_table")
        self._weights = {}

    # -- direct wrappers -------------------------------------------------------------
    def close(self):
        if self.handle:
            lib().echokv_destroy(self.handle)
            self.handle = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def set_block_table(self, table) -> None:
        """Copy a host/device int32 table into the borrowed device block table."""
        self.block_table[:table.shape[0], :table.shape[1]].copy_(table)

    def set_weights(self, layer: int, Wk, Wv, bk=None, bv=None) -> None:
        self._weights[layer] = (Wk, Wv, bk, bv)   # keep the borrowed tensors alive
        _check(lib().echokv_set_weights(self.handle, layer, _ptr(Wk), _ptr(Wv), _ptr(bk), _ptr(bv)),
               "echokv_set_weights")

    def append_kv(self, layer: int, k_new, v_new, positions, seq_slots=None, stream=None) -> None:
        _check(lib().echokv_append_kv(self.handle, layer, _ptr(k_new), _ptr(v_new), _ptr(seq_slots),
                                      _ptr(positions), k_new.shape[0], _stream_handle(stream)),
               "echokv_append_kv")

    def append_kv_chunk(self, layer: int, k_new, v_new, first_positions, seq_slots=None, stream=None) -> None:
        """k_new, v_new [B][n_tokens][H_kv][d]: n_tokens consecutive new tokens per sequence."""
        _check(lib().echokv_append_kv_chunk(self.handle, layer, _ptr(k_new), _ptr(v_new), _ptr(seq_slots),
                                            _ptr(first_positions), k_new.shape[1], k_new.shape[0],
                                            _stream_handle(stream)), "echokv_append_kv_chunk")

    def compress_layer(self, layer: int, k_full, v_full, seq_lens, seq_begins=None, seq_slots=None, stream=None) -> None:
        """Evict a layer cached at full width ([n_pages][page_tokens][D] pools) down to its retained dims."""
        _check(lib().echokv_compress_layer(self.handle, layer, _ptr(k_full), _ptr(v_full), _ptr(seq_slots),
                                           _ptr(seq_begins), _ptr(seq_lens), seq_lens.shape[0],
                                           _stream_handle(stream)), "echokv_compress_layer")

    def decode_attention(self, layer: int, q, seq_lens, out=None, seq_slots=None, stream=None):
        out = self._out(q, stream) if out is None else out
        _check(lib().echokv_decode_attention(self.handle, layer, _ptr(q), _ptr(out), _ptr(seq_slots),
                                             _ptr(seq_lens), q.shape[0], _stream_handle(stream)),
               "echokv_decode_attention")
        return out

    def prefill_attention(self, layer: int, q, seq_lens, out=None, seq_slots=None, stream=None, k_recent=None,
                          v_recent=None):
        """q [B][n_q][H_q][d]: the last n_q cached tokens of every sequence as causal queries.  The scratch
        for the rebuilt cache rows is allocated on first use and kept.  k_recent, v_recent [B][n_q + n_window - 1][D]:
        whole K / V rows of the chunk and the n_window - 1 tokens before it (needed while a window is set)."""
        if getattr(self, "prefill_scratch", None) is None:
            n = C.c_uint64(0)
            _check(lib().echokv_prefill_scratch_bytes(C.byref(self.cfg), C.byref(n)), "echokv_prefill_scratch_bytes")
            with _memory_of(stream):
                self.prefill_scratch = self.torch.empty(n.value, dtype=self.torch.uint8, device=self.device)
        out = self._out(q, stream) if out is None else out
        _check(lib().echokv_prefill_attention(self.handle, layer, _ptr(q), _ptr(out), q.shape[1], _ptr(seq_slots),
                                              _ptr(seq_lens), q.shape[0], _ptr(k_recent), _ptr(v_recent),
                                              self.prefill_scratch.data_ptr(),
                                              self.prefill_scratch.numel(), _stream_handle(stream)),
               "echokv_prefill_attention")
        return out

    def full_attention(self, layer: int, q, seq_lens, out=None, seq_slots=None, stream=None):
        out = self._out(q, stream) if out is None else out
        _check(lib().echokv_full_attention(self.handle, layer, _ptr(q), _ptr(out), _ptr(seq_slots),
                                           _ptr(seq_lens), q.shape[0], _stream_handle(stream)),
               "echokv_full_attention")
        return out

    def layer_step_host(self, layer: int, q_host, k_new_host, v_new_host, out_host, seq_lens_host,
                        attend: bool = True, stream=None) -> None:
        _check(lib().echokv_layer_step_host(self.handle, layer, _ptr(q_host), _ptr(k_new_host),
                                            _ptr(v_new_host), _ptr(out_host), _ptr(seq_lens_host),
                                            k_new_host.shape[0], 1 if attend else 0,
                                            _stream_handle(stream)),
               "echokv_layer_step_host")

    def device_status(self) -> int:
        v = C.c_int32(0)
        _check(lib().echokv_get_device_status(self.handle, C.byref(v)), "echokv_get_device_status")
        return v.value

    def launch_count(self) -> int:
        return lib().echokv_launch_count(self.handle)

    def decode_path(self) -> int:
        return lib().echokv_decode_path(self.handle)

    def diag_page_order(self) -> int:
        out = C.c_int32(-1)
        _check(lib().echokv_diag_page_order(self.handle, C.byref(out)), "echokv_diag_page_order")
        return out.value

    def set_decode_path(self, path: int) -> None:
        _check(lib().echokv_set_decode_path(self.handle, path), "echokv_set_decode_path")

    def set_full_precision_window(self, n_sink: int, n_window: int) -> None:
        """Keep the first n_sink and the last n_window tokens of every sequence uncompressed: allocates the
        side buffers of the compressed layers ([max_batch][n_sink + n_window][D - m]) and hands them over."""
        cfg, n = self.cfg, self.cfg.n_layers
        self.k_side, self.v_side = [], []
        for l in range(n):
            if l % cfg.group_size == 0 or self.D == self.m or n_sink + n_window == 0:
                self.k_side.append(None)
                self.v_side.append(None)
            else:
                shape = (cfg.max_batch, n_sink + n_window, self.D - self.m)
                self.k_side.append(self.torch.zeros(shape, dtype=self.tdtype, device=self.device))
                self.v_side.append(self.torch.zeros(shape, dtype=self.tdtype, device=self.device))
        self._ks = (C.c_void_p * n)(*[_ptr(t) for t in self.k_side])
        self._vs = (C.c_void_p * n)(*[_ptr(t) for t in self.v_side])
        _check(lib().echokv_set_full_precision_window(self.handle, n_sink, n_window,
                                                      C.cast(self._ks, C.POINTER(C.c_void_p)),
                                                      C.cast(self._vs, C.POINTER(C.c_void_p))),
               "echokv_set_full_precision_window")
        self.n_sink, self.n_window = n_sink, n_window

    def set_rope(self, theta: float, stream=None) -> None:
        """Rotate cached keys to their positions when they are read (the cache holds un-rotated keys):
        allocates the (cos, sin) table and has the library fill it.  theta = 0 switches it off."""
        if not theta:
            _check(lib().echokv_set_rope(self.handle, 0.0, None, 0, None), "echokv_set_rope")
            self.rope_table = None
            return
        n = C.c_uint64(0)
        _check(lib().echokv_rope_table_bytes(C.byref(self.cfg), C.byref(n)), "echokv_rope_table_bytes")
        with _memory_of(stream):
            self.rope_table = self.torch.empty(n.value, dtype=self.torch.uint8, device=self.device)
        _check(lib().echokv_set_rope(self.handle, float(theta), self.rope_table.data_ptr(), n.value,
                                     _stream_handle(stream)), "echokv_set_rope")

    def rope_enabled(self) -> bool:
        return bool(lib().echokv_rope_enabled(self.handle))

    def enable_absorbed(self) -> None:
        """Allocate the absorbed mode's workspace and switch the context to that mode."""
        n = C.c_uint64(0)
        _check(lib().echokv_absorbed_workspace_bytes(C.byref(self.cfg), C.byref(n)), "echokv_absorbed_workspace_bytes")
        self.workspace_absorbed = self.torch.empty(n.value, dtype=self.torch.uint8, device=self.device)
        _check(lib().echokv_enable_absorbed(self.handle, self.workspace_absorbed.data_ptr(), n.value),
               "echokv_enable_absorbed")

    def decode_mode(self) -> int:
        return lib().echokv_decode_mode(self.handle)

    def set_decode_mode(self, mode: int) -> None:
        _check(lib().echokv_set_decode_mode(self.handle, mode), "echokv_set_decode_mode")

    def stored_path(self) -> int:
        return lib().echokv_stored_path(self.handle)

    def set_stored_path(self, path: int) -> None:
        _check(lib().echokv_set_stored_path(self.handle, path), "echokv_set_stored_path")

    def set_kernel_timing(self, enable: bool) -> None:
        _check(lib().echokv_set_kernel_timing(self.handle, 1 if enable else 0), "echokv_set_kernel_timing")

    def read_kernel_timing(self):
        """(total milliseconds, launches) of the dominant kernel since the last read."""
        ms, n = C.c_double(0.0), C.c_int64(0)
        _check(lib().echokv_read_kernel_timing(self.handle, C.byref(ms), C.byref(n)), "echokv_read_kernel_timing")
        return ms.value, n.value

    def read_kernel_timing_by_kind(self):
        """{"stored": (ms, launches), "recon": (ms, launches)} since the last read."""
        ms, n = (C.c_double * 4)(), (C.c_int64 * 4)()
        _check(lib().echokv_read_kernel_timing_by_kind(self.handle, ms, n), "echokv_read_kernel_timing_by_kind")
        return {"stored": (ms[0], n[0]), "recon": (ms[1], n[1]), "absorb_k": (ms[2], n[2]), "absorb_v": (ms[3], n[3])}

    def diag_bounded_wait(self, limit_cycles: int, stream=None):
        """Run the bounded-wait probe; returns the device tensor int32[2] saying how its two warps left."""
        with _memory_of(stream):
            left = self.torch.zeros(2, dtype=self.torch.int32, device=self.device)
        _check(lib().echokv_diag_bounded_wait(self.handle, int(limit_cycles), left.data_ptr(), _stream_handle(stream)),
               "echokv_diag_bounded_wait")
        return left

    def _out(self, q, stream):
        with _memory_of(stream):
            return self.torch.empty(q.shape, dtype=self.torch.float32, device=self.device)


def echokv_full_attention_noalloc(cfg: echokv_config, k_pool, v_pool, block_table, q, out, seq_lens,
                                  seq_slots=None, status_out=None, stream=None) -> None:
    """Full-cache attention without a context or a workspace, for callers that cannot allocate
    device memory: partial results live in a fixed 8 MiB array inside the library.  Tensors are
    only read for their addresses; nothing is allocated here either.  Calls sharing a device must
    not overlap on the GPU, and the first call on a device should precede any stream capture."""
    _check(lib().echokv_full_attention_noalloc(C.byref(cfg), _ptr(k_pool), _ptr(v_pool), _ptr(block_table),
                                               _ptr(q), _ptr(out), _ptr(seq_slots), _ptr(seq_lens),
                                               q.shape[0], _ptr(status_out), _stream_handle(stream)),
           "echokv_full_attention_noalloc")


# ---- a serving step over a cache held in 8 bits ------------------------------------------------------------------
# (A decode step's calls are short: what happens here per call is kept short too.)
# stream: the torch stream that a call runs on, the current one if None.  New tensors are allocated for it.  As with torch's own
# operators the caller orders streams: inputs have to be ready on it, and who uses the outputs elsewhere waits for it.
def _stream_on(device: int, stream) -> int | None:
    if stream is not None:
        return stream.cuda_stream or None
    import torch
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)     # the same handle without a Stream object around it
    return (raw(device) if raw is not None else torch.cuda.current_stream(device).cuda_stream) or None


def _dense(t, dtype, n, name, device):
    """Address of a contiguous tensor of `dtype` with at least n elements on CUDA device `device` (None stays NULL)."""
    if t is None:
        return None
    if t.dtype is not dtype or t.get_device() != device or not t.is_contiguous() or t.numel() < n:
        raise ValueError("%s: a contiguous %s device tensor of at least %d elements is needed, on cuda:%d" % (name, dtype, n, device))
    return t.data_ptr()


def _rows(t, n, heads, d, dtype, name, device):
    """(address, elements from row to row) of a [n][heads][d] tensor on CUDA device `device` whose rows are dense."""
    st = t.stride()
    if t.dtype is not dtype or t.shape != (n, heads, d) or t.get_device() != device or (n > 0 and (st[2] != 1 or (st[1] != d and heads > 1))):
        raise ValueError("%s: a [%d tokens][%d][%d] %s device tensor with dense rows is needed, on cuda:%d" % (name, n, heads, d, dtype, device))
    # (the stride of a single row is anything)
    return t.data_ptr(), st[0] if n > 1 else heads * d


def _dtype(cfg):
    import torch
    return torch.bfloat16 if cfg.dtype == ECHOKV_BF16 else torch.float32


class StepPlan:
    """What plan_tokens writes: cu_tokens [B + 1], positions, token_seqs [n_tokens], seq_lens [B], free_count [1] (int32) and
    slot_map [n_tokens] (int64)."""
    __slots__ = ("cu_tokens", "positions", "token_seqs", "slot_map", "seq_lens", "free_count", "_c", "_held", "_batch", "_tokens", "_device")

    def __init__(self, batch: int, n_tokens: int, device, seq_lens=None, free_count=None):
        import torch
        buf = torch.empty(2 * batch + 2 * n_tokens + 2, dtype=torch.int32, device=device)
        self.cu_tokens, self.positions, self.token_seqs, lens, count = buf.split_with_sizes((batch + 1, n_tokens, n_tokens, batch, 1))
        self.slot_map = buf.new_empty(n_tokens, dtype=torch.int64)
        self.seq_lens = lens if seq_lens is None else seq_lens
        self.free_count = count if free_count is None else free_count
        cu = buf.data_ptr()
        self._c = echokv_step_plan(cu, cu + 4 * (batch + 1), cu + 4 * (batch + 1 + n_tokens), self.slot_map.data_ptr(),
                                   lens.data_ptr() if seq_lens is None else _dense(seq_lens, torch.int32, batch, "seq_lens", buf.get_device()),
                                   count.data_ptr() if free_count is None else _dense(free_count, torch.int32, 1, "free_count", buf.get_device()))
        self._held = buf, self.slot_map, self.seq_lens, self.free_count       # (what _c's addresses are of, whatever becomes of the attributes)
        self._batch, self._tokens, self._device = batch, n_tokens, buf.get_device()

    def _beginning(self, batch: int, n_tokens: int) -> StepPlan:
        """The plan of a smaller step in the same buffers."""
        if batch == self._batch and n_tokens == self._tokens:
            return self
        part = object.__new__(StepPlan)
        part.cu_tokens, part.seq_lens, part.free_count = self.cu_tokens[:batch + 1], self.seq_lens[:batch], self.free_count
        part.positions, part.token_seqs, part.slot_map = self.positions[:n_tokens], self.token_seqs[:n_tokens], self.slot_map[:n_tokens]
        part._c, part._held, part._batch, part._tokens, part._device = self._c, self._held, batch, n_tokens, self._device
        return part


def plan_tokens(cfg: echokv_config, block_table, seq_lens, new_lens, free_pages, free_count, n_tokens: int, seq_slots=None,
                out: StepPlan | None = None, status=None, stream=None) -> StepPlan:
    """Pages for new_lens[b] more tokens of sequences that hold seq_lens[b]: fills block_table ([max_batch][max_pages_per_seq]
    int32) and returns the step's plan for up to n_tokens tokens.  `out` is used again by later (and captured) steps, and may
    hold the buffers seq_lens and free_count themselves, which are then updated in place; for a step smaller than it the returned
    plan holds the beginnings of its tensors (behind them an earlier step's entries remain).  status: optional int32 device tensor
    (see echokv.h)."""
    import torch
    i32, B = torch.int32, seq_lens.shape[0]
    if out is None:
        with _memory_of(stream):
            out = StepPlan(B, n_tokens, seq_lens.device)
    elif out._batch < B or out._tokens < n_tokens:
        raise ValueError("out: too small for %d sequences and %d tokens" % (B, n_tokens))
    elif out._device != cfg.device:
        raise ValueError("out: a plan on cuda:%d is needed" % cfg.device)
    _check(lib().echokv_plan_tokens(C.byref(cfg), _dense(block_table, i32, cfg.max_batch * cfg.max_pages_per_seq, "block_table", cfg.device),
                                    _dense(seq_slots, i32, B, "seq_slots", cfg.device), _dense(seq_lens, i32, B, "seq_lens", cfg.device),
                                    _dense(new_lens, i32, B, "new_lens", cfg.device), _dense(free_pages, i32, cfg.n_pages, "free_pages", cfg.device),
                                    _dense(free_count, i32, 1, "free_count", cfg.device), B, n_tokens, C.byref(out._c),
                                    _dense(status, i32, 1, "status", cfg.device), _stream_on(cfg.device, stream)), "echokv_plan_tokens")
    return out._beginning(B, n_tokens)


def release_pages(cfg: echokv_config, block_table, seq_lens, free_pages, free_count, seq_slots=None, status=None,
                  stream=None) -> None:
    """Put the pages of finished sequences back on the free list (free_pages, free_count are updated)."""
    import torch
    i32, B = torch.int32, seq_lens.shape[0]
    _check(lib().echokv_release_pages(C.byref(cfg), _dense(block_table, i32, cfg.max_batch * cfg.max_pages_per_seq, "block_table", cfg.device),
                                      _dense(seq_slots, i32, B, "seq_slots", cfg.device), _dense(seq_lens, i32, B, "seq_lens", cfg.device), B,
                                      _dense(free_pages, i32, cfg.n_pages, "free_pages", cfg.device), _dense(free_count, i32, 1, "free_count", cfg.device),
                                      _dense(status, i32, 1, "status", cfg.device), _stream_on(cfg.device, stream)), "echokv_release_pages")


def rotate(cfg: echokv_config, q, k, positions, theta: float, sections=None, rot_dim: int = 0, interleaved: bool = False,
           inverse: bool = False, q_out=None, k_out=None, stream=None):
    """Rotary positions on q [T][n_q_heads][d] and k [T][n_kv_heads][d] (either may be None; rows may be slices of a wider
    tensor); positions int32 [T] or [n_axes][T].  Returns (q_out, k_out), new tensors unless given -- they may be q and k.
    inverse = True is the gradient's pass."""
    import torch
    dt, d, n_q, n_kv = _dtype(cfg), cfg.head_dim, cfg.n_q_heads, cfg.n_kv_heads
    if q is None and k is None:
        raise ValueError("rotate: neither q nor k")
    T = (k if q is None else q).shape[0]
    axes = 1 if positions.dim() == 1 else positions.shape[0]
    if positions.shape[-1] != T:
        raise ValueError("rotate: q, k and positions differ in their number of tokens")
    qp = kp = qo = ko = None
    qs = ks = qos = kos = 0
    if q is not None:
        qp, qs = _rows(q, T, n_q, d, dt, "q", cfg.device)
        if q_out is None:
            with _memory_of(stream):
                q_out = q.new_empty((T, n_q, d))
            qo, qos = q_out.data_ptr(), n_q * d
        else:
            qo, qos = _rows(q_out, T, n_q, d, dt, "q_out", cfg.device)
    if k is not None:
        kp, ks = _rows(k, T, n_kv, d, dt, "k", cfg.device)
        if k_out is None:
            with _memory_of(stream):
                k_out = k.new_empty((T, n_kv, d))
            ko, kos = k_out.data_ptr(), n_kv * d
        else:
            ko, kos = _rows(k_out, T, n_kv, d, dt, "k_out", cfg.device)
    sec = None
    if sections is not None:
        if len(sections) != axes:
            raise ValueError("rotate: one section per position axis")
        sec = (C.c_int32 * axes)(*sections)
    _check(lib().echokv_rotate(C.byref(cfg), qp, qs, kp, ks, qo, qos, ko, kos, _dense(positions, torch.int32, axes * T, "positions", cfg.device),
                               axes, sec, 1 if interleaved else 0, rot_dim, theta, 1 if inverse else 0, T,
                               _stream_on(cfg.device, stream)), "echokv_rotate")
    return (q_out if q is not None else None), (k_out if k is not None else None)


def query_quant_sizes(cfg: echokv_config) -> echokv_quant_sizes:
    out = echokv_quant_sizes()
    _check(lib().echokv_query_quant_sizes(C.byref(cfg), C.byref(out)), "echokv_query_quant_sizes")
    return out


class QuantCache:
    """One layer's cache in 8 bits: codes int8 or float8_e4m3fn [n_pages][n_kv_heads][page_tokens][d], a scale for each 16 tokens
    and head [n_pages][n_kv_heads][page_tokens / 16], and the open blocks' rows in the storage type [max_batch][n_kv_heads][16][d].
    Allocates them unless they are given; `workspace` (42 MB in bf16 with heads of 128) is best shared by the layers of a model
    (calls that share one must not overlap on the device).  The other tensors are the cache's for its life."""
    _FIXED = frozenset(("cfg", "k_codes", "v_codes", "k_scales", "v_scales", "k_tail", "v_tail"))

    def __setattr__(self, name, value):
        if name in self._FIXED and name in self.__dict__:
            raise AttributeError("%s: the library holds its address; make a new QuantCache" % name)
        self.__dict__[name] = value

    def __init__(self, cfg: echokv_config, fmt: str, k_codes=None, v_codes=None, k_scales=None, v_scales=None, k_tail=None,
                 v_tail=None, workspace=None):
        import torch
        if fmt not in QUANT_FORMATS:
            raise ValueError("format %r is not one of %s" % (fmt, sorted(QUANT_FORMATS)))
        self.cfg, self.fmt, self.tdtype = cfg, fmt, _dtype(cfg)
        self.sizes = sizes = query_quant_sizes(cfg)
        self._ws_bytes = sizes.workspace_bytes
        dev = torch.device("cuda", cfg.device)
        H, P, d, N = cfg.n_kv_heads, cfg.page_tokens, cfg.head_dim, cfg.n_pages
        code = torch.int8 if fmt == "int8" else torch.float8_e4m3fn

        def held(t, shape, dtype, name):
            if t is None:
                return torch.zeros(shape, dtype=dtype, device=dev)
            if tuple(t.shape) != shape or t.dtype is not dtype or t.get_device() != cfg.device or not t.is_contiguous():
                raise ValueError("%s: a contiguous %s device tensor of shape %s is needed, on cuda:%d" % (name, dtype, shape, cfg.device))
            return t
        self.k_codes = held(k_codes, (N, H, P, d), code, "k_codes")
        self.v_codes = held(v_codes, (N, H, P, d), code, "v_codes")
        self.k_scales = held(k_scales, (N, H, P // ECHOKV_QUANT_BLOCK_TOKENS), torch.float32, "k_scales")
        self.v_scales = held(v_scales, (N, H, P // ECHOKV_QUANT_BLOCK_TOKENS), torch.float32, "v_scales")
        tail = (cfg.max_batch, H, ECHOKV_QUANT_BLOCK_TOKENS, d)
        self.k_tail = held(k_tail, tail, self.tdtype, "k_tail")
        self.v_tail = held(v_tail, tail, self.tdtype, "v_tail")
        self.workspace = torch.empty(sizes.workspace_bytes, dtype=torch.uint8, device=dev) if workspace is None else workspace
        _dense(self.workspace, torch.uint8, self._ws_bytes, "workspace", cfg.device)
        self._c = echokv_quant_cache(self.k_codes.data_ptr(), self.v_codes.data_ptr(), self.k_scales.data_ptr(),
                                     self.v_scales.data_ptr(), self.k_tail.data_ptr(), self.v_tail.data_ptr(),
                                     QUANT_FORMATS[fmt], 0)

    def append(self, k_new, v_new, slot_map, token_seqs, cu_tokens, seq_slots=None, status=None, stream=None) -> None:
        """k_new, v_new [T][n_kv_heads][d] (rows may be slices of a wider tensor); slot_map, token_seqs, cu_tokens: plan_tokens'."""
        import torch
        cfg, T, B = self.cfg, k_new.shape[0], cu_tokens.shape[0] - 1
        kp, ks = _rows(k_new, T, cfg.n_kv_heads, cfg.head_dim, self.tdtype, "k_new", cfg.device)
        vp, vs = _rows(v_new, T, cfg.n_kv_heads, cfg.head_dim, self.tdtype, "v_new", cfg.device)
        _check(lib().echokv_quant_append(C.byref(cfg), C.byref(self._c), kp, ks, vp, vs, _dense(slot_map, torch.int64, T, "slot_map", cfg.device),
                                         _dense(token_seqs, torch.int32, T, "token_seqs", cfg.device),
                                         _dense(cu_tokens, torch.int32, B + 1, "cu_tokens", cfg.device), _dense(seq_slots, torch.int32, B, "seq_slots", cfg.device),
                                         B, T, _dense(status, torch.int32, 1, "status", cfg.device), _stream_on(cfg.device, stream)),
               "echokv_quant_append")

    def attention(self, q, block_table, seq_lens, cu_tokens=None, max_new: int = 1, seq_slots=None, softcap: float = 0.0,
                  alibi_slopes=None, prefix_lens=None, out=None, status=None, stream=None):
        """q [T][n_q_heads][d]: the new tokens of every sequence, which are its last ones and already appended (cu_tokens None:
        one each).  max_new bounds the new tokens of any sequence; one with more gets zeros and a status.  Returns out
        [T][n_q_heads][d] in the storage type, which may be q itself; rows behind the last sequence's stay as they are (in a new
        tensor: anything)."""
        import torch
        cfg, T, B = self.cfg, q.shape[0], seq_lens.shape[0]
        qp, qs = _rows(q, T, cfg.n_q_heads, cfg.head_dim, self.tdtype, "q", cfg.device)
        if out is None:
            with _memory_of(stream):
                out = q.new_empty((T, cfg.n_q_heads, cfg.head_dim))
            op = out.data_ptr()
        else:
            op = _dense(out, self.tdtype, T * cfg.n_q_heads * cfg.head_dim, "out", cfg.device)
        opts = None
        if softcap or alibi_slopes is not None or prefix_lens is not None:
            opts = C.byref(echokv_score_options(softcap, 0, _dense(alibi_slopes, torch.float32, cfg.n_q_heads, "alibi_slopes", cfg.device),
                                                _dense(prefix_lens, torch.int32, B, "prefix_lens", cfg.device)))
        _check(lib().echokv_quant_attention(C.byref(cfg), C.byref(self._c), opts, qp, qs, op,
                                            _dense(block_table, torch.int32, cfg.max_batch * cfg.max_pages_per_seq, "block_table", cfg.device),
                                            _dense(seq_slots, torch.int32, B, "seq_slots", cfg.device), _dense(seq_lens, torch.int32, B, "seq_lens", cfg.device),
                                            _dense(cu_tokens, torch.int32, B + 1, "cu_tokens", cfg.device), B, T, max_new,
                                            _dense(self.workspace, torch.uint8, self._ws_bytes, "workspace", cfg.device),
                                            self._ws_bytes, _dense(status, torch.int32, 1, "status", cfg.device),
                                            _stream_on(cfg.device, stream)), "echokv_quant_attention")
        return out


# ---- the same step over a cache held in 4 bits ---------------------------------------------------------------------
class Rotation:
    """Rotary positions for Fp4Cache.append: theta, and as in rotate() the sections of several position axes and rot_dim (a multiple of
    16; 0: the whole head)."""
    __slots__ = ("_c", "_sections", "n_axes")

    def __init__(self, cfg: echokv_config, theta: float, n_axes: int = 1, sections=None, rot_dim: int = 0, interleaved: bool = False):
        if sections is not None and len(sections) != n_axes:
            raise ValueError("Rotation: one section per position axis")
        half = (rot_dim or cfg.head_dim) // 2
        if not 0 <= rot_dim <= cfg.head_dim or rot_dim % 16 or n_axes < 1 or (n_axes > 1 if sections is None else sum(sections) != half):
            raise ValueError("Rotation: rot_dim is a multiple of 16 up to the head's, the sections sum to half of it")
        self.n_axes = n_axes
        self._sections = None if sections is None else (C.c_int32 * n_axes)(*sections)
        self._c = echokv_rotation(theta, self._sections, n_axes, 1 if interleaved else 0, rot_dim, 0)


def query_fourbit_sizes(cfg: echokv_config) -> echokv_fourbit_sizes:
    out = echokv_fourbit_sizes()
    _check(lib().echokv_query_fourbit_sizes(C.byref(cfg), C.byref(out)), "echokv_query_fourbit_sizes")
    return out


class Fp4Cache:
    """One layer's cache in 4 bits: blocks uint8 [n_pages][n_kv_heads][page_tokens / 16][18 d] and, for select_pages, the bounds of
    every page's keys, int8 [n_pages][n_kv_heads][2][d] around fp32 scales [n_pages][n_kv_heads] (`selection` False: none are kept).
    Allocates them unless they are given; `workspace` is best shared by the layers of a model (calls that share one must not overlap
    on the device).  k_unit, v_unit: the magnitudes of keys and values are held around them (see echokv.h).  The other tensors
    are the cache's for its life."""
    _FIXED = frozenset(("cfg", "blocks", "bounds", "bound_scales", "k_unit", "v_unit"))

    def __setattr__(self, name, value):
        if name in self._FIXED and name in self.__dict__:
            raise AttributeError("%s: the library holds it; make a new Fp4Cache" % name)
        self.__dict__[name] = value

    def __init__(self, cfg: echokv_config, k_unit: float = 1.0, v_unit: float = 1.0, blocks=None, bounds=None, bound_scales=None,
                 selection: bool = True, workspace=None):
        import torch
        self.cfg, self.tdtype, self.k_unit, self.v_unit = cfg, _dtype(cfg), k_unit, v_unit
        self.sizes = sizes = query_fourbit_sizes(cfg)
        if not all(2.0 ** -60 <= u <= 2.0 ** 60 for u in (k_unit, v_unit)):
            raise ValueError("k_unit, v_unit: between 2^-60 and 2^60")
        if (bounds is None) != (bound_scales is None) or (bounds is not None and not selection):
            raise ValueError("bounds and bound_scales go together, and with selection")
        self._ws_bytes = sizes.workspace_bytes
        dev = torch.device("cuda", cfg.device)
        H, P, d, N = cfg.n_kv_heads, cfg.page_tokens, cfg.head_dim, cfg.n_pages

        def held(t, shape, dtype, name):
            if t is None:
                return torch.zeros(shape, dtype=dtype, device=dev)
            if tuple(t.shape) != shape or t.dtype is not dtype or t.get_device() != cfg.device or not t.is_contiguous():
                raise ValueError("%s: a contiguous %s device tensor of shape %s is needed, on cuda:%d" % (name, dtype, shape, cfg.device))
            return t
        self.blocks = held(blocks, (N, H, P // 16, 18 * d), torch.uint8, "blocks")
        self.bounds = held(bounds, (N, H, 2, d), torch.int8, "bounds") if selection else None
        self.bound_scales = held(bound_scales, (N, H), torch.float32, "bound_scales") if selection else None
        self.workspace = torch.empty(sizes.workspace_bytes, dtype=torch.uint8, device=dev) if workspace is None else workspace
        _dense(self.workspace, torch.uint8, self._ws_bytes, "workspace", cfg.device)
        self._c = echokv_fourbit_cache(self.blocks.data_ptr(), _ptr(self.bounds), _ptr(self.bound_scales), k_unit, v_unit)

    def append(self, k_new, v_new, slot_map, q=None, rotation: Rotation | None = None, positions=None, q_out=None, status=None,
               stream=None):
        """k_new, v_new [T][n_kv_heads][d] (rows may be slices of a wider tensor) into the pool rows slot_map (plan_tokens').  With a
        rotation, keys are turned to positions (int32 [T] or [n_axes][T]) on their way, and q [T][n_q_heads][d], if given, into the
        returned q_out (which may be q)."""
        import torch
        cfg, T, d = self.cfg, k_new.shape[0], self.cfg.head_dim
        if q is not None and rotation is None:
            raise ValueError("append: queries are turned, so a rotation is needed")
        if (rotation is None) != (positions is None):
            raise ValueError("append: rotation and positions go together")
        kp, ks = _rows(k_new, T, cfg.n_kv_heads, d, self.tdtype, "k_new", cfg.device)
        vp, vs = _rows(v_new, T, cfg.n_kv_heads, d, self.tdtype, "v_new", cfg.device)
        qp = qo = rot = pos = None
        qs = qos = 0
        if rotation is not None:
            if (1 if positions.dim() == 1 else positions.shape[0]) != rotation.n_axes or positions.shape[-1] != T:
                raise ValueError("append: positions are [n_axes][n_tokens]")
            rot, pos = C.byref(rotation._c), _dense(positions, torch.int32, rotation.n_axes * T, "positions", cfg.device)
        if q is not None:
            qp, qs = _rows(q, T, cfg.n_q_heads, d, self.tdtype, "q", cfg.device)
            if q_out is None:
                with _memory_of(stream):
                    q_out = q.new_empty((T, cfg.n_q_heads, d))
                qo, qos = q_out.data_ptr(), cfg.n_q_heads * d
            else:
                qo, qos = _rows(q_out, T, cfg.n_q_heads, d, self.tdtype, "q_out", cfg.device)
        _check(lib().echokv_fourbit_append(C.byref(cfg), C.byref(self._c), rot, qp, qs, qo, qos, kp, ks, vp, vs, pos,
                                       _dense(slot_map, torch.int64, T, "slot_map", cfg.device), T,
                                       _dense(status, torch.int32, 1, "status", cfg.device), _stream_on(cfg.device, stream)), "echokv_fourbit_append")
        return q_out if q is not None else None

    def read(self, slot_map, k_out=None, v_out=None, status=None, stream=None):
        """The rows that the cache holds in the pool rows slot_map: (k, v) [T][n_kv_heads][d] in the storage type, new tensors unless
        given."""
        import torch
        cfg, T, H, d = self.cfg, slot_map.shape[0], self.cfg.n_kv_heads, self.cfg.head_dim
        with _memory_of(stream):
            if k_out is None:
                k_out = slot_map.new_empty((T, H, d), dtype=self.tdtype)
                kp, ks = k_out.data_ptr(), H * d
            else:
                kp, ks = _rows(k_out, T, H, d, self.tdtype, "k_out", cfg.device)
            if v_out is None:
                v_out = slot_map.new_empty((T, H, d), dtype=self.tdtype)
                vp, vs = v_out.data_ptr(), H * d
            else:
                vp, vs = _rows(v_out, T, H, d, self.tdtype, "v_out", cfg.device)
        _check(lib().echokv_fourbit_read(C.byref(cfg), C.byref(self._c), _dense(slot_map, torch.int64, T, "slot_map", cfg.device), T, kp, ks, vp, vs,
                                     _dense(status, torch.int32, 1, "status", cfg.device), _stream_on(cfg.device, stream)), "echokv_fourbit_read")
        return k_out, v_out

    def _queries(self, q, out, stream):
        cfg, T = self.cfg, q.shape[0]
        qp, qs = _rows(q, T, cfg.n_q_heads, cfg.head_dim, self.tdtype, "q", cfg.device)
        if out is None:
            with _memory_of(stream):
                out = q.new_empty((T, cfg.n_q_heads, cfg.head_dim))
            return qp, qs, out, out.data_ptr()
        return qp, qs, out, _dense(out, self.tdtype, T * cfg.n_q_heads * cfg.head_dim, "out", cfg.device)

    def attention(self, q, block_table, seq_lens, cu_tokens=None, max_new: int = 1, seq_slots=None, softcap: float = 0.0,
                  alibi_slopes=None, prefix_lens=None, out=None, status=None, stream=None):
        """As QuantCache.attention: q [T][n_q_heads][d], the new tokens of every sequence, attend the whole of it."""
        import torch
        cfg, T, B = self.cfg, q.shape[0], seq_lens.shape[0]
        qp, qs, out, op = self._queries(q, out, stream)
        opts = None
        if softcap or alibi_slopes is not None or prefix_lens is not None:
            opts = C.byref(echokv_score_options(softcap, 0, _dense(alibi_slopes, torch.float32, cfg.n_q_heads, "alibi_slopes", cfg.device),
                                                _dense(prefix_lens, torch.int32, B, "prefix_lens", cfg.device)))
        _check(lib().echokv_fourbit_attention(C.byref(cfg), C.byref(self._c), opts, qp, qs, op,
                                          _dense(block_table, torch.int32, cfg.max_batch * cfg.max_pages_per_seq, "block_table", cfg.device),
                                          _dense(seq_slots, torch.int32, B, "seq_slots", cfg.device), _dense(seq_lens, torch.int32, B, "seq_lens", cfg.device),
                                          _dense(cu_tokens, torch.int32, B + 1, "cu_tokens", cfg.device), B, T, max_new,
                                          _dense(self.workspace, torch.uint8, self._ws_bytes, "workspace", cfg.device), self._ws_bytes,
                                          _dense(status, torch.int32, 1, "status", cfg.device), _stream_on(cfg.device, stream)),
               "echokv_fourbit_attention")
        return out

    def _batch(self, n_seqs, seq_slots):
        return n_seqs if n_seqs is not None else self.cfg.max_batch if seq_slots is None else seq_slots.shape[0]

    def select_pages(self, q, block_table, token_seqs, positions, n_select: int, n_first: int = 1, n_recent: int = 1, seq_slots=None,
                     out=None, status=None, stream=None, n_seqs: int | None = None):
        """The n_select pages of its sequence that each token reads, per KV head: int32 [T][n_kv_heads][n_select], ascending, -1 behind
        the last one -- the first n_first, the last n_recent, and those with the largest scores (see echokv.h).  token_seqs, positions:
        plan_tokens'.  n_seqs: how many sequences the tokens are of, all ids below it (None: as many as seq_slots has, or max_batch);
        a prompt's tokens are taken together, as many as there are to a sequence, so a bound far above it costs time."""
        import torch
        cfg, T, B = self.cfg, q.shape[0], self._batch(n_seqs, seq_slots)
        if self.bounds is None:
            raise ValueError("select_pages: a cache made without selection has no bounds")
        qp, qs = _rows(q, T, cfg.n_q_heads, cfg.head_dim, self.tdtype, "q", cfg.device)
        if out is None:
            with _memory_of(stream):
                out = torch.empty((T, cfg.n_kv_heads, n_select), dtype=torch.int32, device=q.device)
        _check(lib().echokv_fourbit_select(C.byref(cfg), C.byref(self._c), qp, qs,
                                       _dense(block_table, torch.int32, cfg.max_batch * cfg.max_pages_per_seq, "block_table", cfg.device),
                                       _dense(seq_slots, torch.int32, B, "seq_slots", cfg.device),
                                       _dense(token_seqs, torch.int32, T, "token_seqs", cfg.device),
                                       _dense(positions, torch.int32, T, "positions", cfg.device), B, T, n_select, n_first, n_recent,
                                       _dense(out, torch.int32, T * cfg.n_kv_heads * n_select, "out", cfg.device),
                                       _dense(self.workspace, torch.uint8, self._ws_bytes, "workspace", cfg.device), self._ws_bytes,
                                       _dense(status, torch.int32, 1, "status", cfg.device), _stream_on(cfg.device, stream)),
               "echokv_fourbit_select")
        return out

    def sparse_attention(self, q, block_table, token_seqs, positions, pages, seq_slots=None, softcap: float = 0.0, alibi_slopes=None,
                         out=None, status=None, stream=None, n_seqs: int | None = None):
        """q [T][n_q_heads][d]: every token attends the pages that pages [T][n_kv_heads][n_select] lists of its sequence (select_pages', or
        any others), keys up to its own position.  Rows of tokens with sequence -1 stay as they are (in a new tensor: anything).  n_seqs: as
        for select_pages."""
        import torch
        cfg, T, B = self.cfg, q.shape[0], self._batch(n_seqs, seq_slots)
        if pages.dim() != 3 or pages.shape[0] != T or pages.shape[1] != cfg.n_kv_heads:
            raise ValueError("pages: [%d tokens][%d][n_select] is needed" % (T, cfg.n_kv_heads))
        qp, qs, out, op = self._queries(q, out, stream)
        opts = None
        if softcap or alibi_slopes is not None:
            opts = C.byref(echokv_score_options(softcap, 0, _dense(alibi_slopes, torch.float32, cfg.n_q_heads, "alibi_slopes", cfg.device), None))
        _check(lib().echokv_fourbit_sparse_attention(C.byref(cfg), C.byref(self._c), opts, qp, qs, op,
                                                 _dense(block_table, torch.int32, cfg.max_batch * cfg.max_pages_per_seq, "block_table", cfg.device),
                                                 _dense(seq_slots, torch.int32, B, "seq_slots", cfg.device),
                                                 _dense(token_seqs, torch.int32, T, "token_seqs", cfg.device),
                                                 _dense(positions, torch.int32, T, "positions", cfg.device),
                                                 _dense(pages, torch.int32, pages.numel(), "pages", cfg.device), pages.shape[2], B, T,
                                                 _dense(self.workspace, torch.uint8, self._ws_bytes, "workspace", cfg.device), self._ws_bytes,
                                                 _dense(status, torch.int32, 1, "status", cfg.device), _stream_on(cfg.device, stream)),
               "echokv_fourbit_sparse_attention")
        return out


def config_for(w, n_pages: int | None = None, device: int = 0, max_batch: int | None = None) -> echokv_config:
    """echokv_config of a synth.Workload."""
    pages = w.pages_per_seq
    return make_config(n_layers=w.n_layers, n_q_heads=w.n_q_heads, n_kv_heads=w.n_kv_heads,
                       head_dim=w.head_dim, group_size=w.group_size,
                       n_retained_heads=w.n_retained_heads, page_tokens=w.page_tokens,
                       max_batch=max_batch or w.batch, max_pages_per_seq=pages,
                       n_pages=n_pages or w.batch * pages,
                       dtype=ECHOKV_BF16 if w.dtype == "bf16" else ECHOKV_FP32,
                       softmax_scale=1.0 / math.sqrt(w.head_dim), device=device,
                       n_retained_dims=w.n_retained_dims, save_k=1 if w.save_k else 0)
