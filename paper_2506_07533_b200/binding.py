"""ctypes binding of libmoqae.so: argument marshalling only.

Function names follow the C ABI (`include/moqae.h`); tensors are torch CUDA tensors whose
`data_ptr()` is handed to the library, work runs on torch's current stream.  There is no
CPU path: loading fails loudly if the CUDA library has not been built.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass, field

import torch

from . import build as _build

EXPERT_BITS = (2, 4, 8, 16)
N_CACHE_BUFFERS = 12
DT_FP16, DT_BF16 = 0, 1

OK = 0
ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_MISALIGNED, ERR_POOL_FULL = -1, -2, -3, -4
ERR_WORKSPACE_TOO_SMALL, ERR_CUDA, ERR_TIMEOUT = -5, -6, -7
ERR_CORRUPT_TABLE = -8

EXPORTS = ["moqae_version", "moqae_last_cuda_error", "moqae_error_string", "moqae_cache_bytes",
           "moqae_cache_bind", "moqae_route", "moqae_quantize_kv", "moqae_append_kv",
           "moqae_decode_attn_workspace", "moqae_decode_attn", "moqae_poll_status",
           "moqae_decode_attn_static", "moqae_decode_attn_static_max_bytes", "moqae_flush_tail", "moqae_prefill_attn",
           "moqae_prefill_attn_workspace", "moqae_decode_attn_ex", "moqae_project_quantize_kv",
           "moqae_validate_tables", "moqae_validate_tables_host", "moqae_decode_attn_step",
           "moqae_norm_rope", "moqae_paged_append", "moqae_paged_decode_attn_workspace", "moqae_paged_decode_attn",
           "moqae_paged_prefill_attn_workspace", "moqae_paged_prefill_attn", "moqae_paged_validate_host",
           "moqae_paged_validate", "moqae_paged_poll_status", "moqae_paged_plan", "moqae_paged4_append", "moqae_paged4_read",
           "moqae_paged4_decode_attn_workspace", "moqae_paged4_decode_attn", "moqae_paged4_prefill_attn_workspace",
           "moqae_paged4_prefill_attn", "moqae_paged4_validate", "moqae_paged4_poll_status"]


class MoqaeConfig(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("chunk", C.c_int32), ("group", C.c_int32),
                ("dtype", C.c_int32), ("n_experts", C.c_int32), ("expert_bits", C.c_int32 * 4),
                ("rs_group", C.c_int32), ("rf_first_chunk", C.c_int32), ("d_in", C.c_int32),
                ("max_tokens", C.c_int32), ("tail_capacity", C.c_int32), ("batch", C.c_int32),
                ("per_head_routing", C.c_int32)]


class MoqaeCache(C.Structure):
    _fields_ = [("pool", C.c_void_p * 4), ("capacity", C.c_int64 * 4), ("map", C.c_void_p),
                ("slot", C.c_void_p), ("count", C.c_void_p), ("votes", C.c_void_p),
                ("tail_k", C.c_void_p), ("tail_v", C.c_void_p), ("tail_len", C.c_void_p),
                ("status", C.c_void_p)]


class MoqaePagedCache(C.Structure):
    _fields_ = [("k_pages", C.c_void_p), ("v_pages", C.c_void_p), ("k_stride", C.c_int64 * 3), ("v_stride", C.c_int64 * 3),
                ("block_table", C.c_void_p), ("kv_len", C.c_void_p), ("status", C.c_void_p), ("n_pages", C.c_int32),
                ("page_size", C.c_int32), ("n_kv_heads", C.c_int32), ("dtype", C.c_int32), ("batch", C.c_int32),
                ("max_pages", C.c_int32)]


class MoqaePaged4Cache(C.Structure):
    _fields_ = [("pages", C.c_void_p), ("page_stride", C.c_int64), ("head_stride", C.c_int64), ("block_table", C.c_void_p),
                ("kv_len", C.c_void_p), ("status", C.c_void_p), ("n_pages", C.c_int32), ("page_size", C.c_int32),
                ("n_kv_heads", C.c_int32), ("dtype", C.c_int32), ("batch", C.c_int32), ("max_pages", C.c_int32)]


class MoqaePagePool(C.Structure):
    _fields_ = [("ring", C.c_void_p), ("state", C.c_void_p), ("n_pages", C.c_int32)]


class MoqaeRows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("token_stride", C.c_int64), ("head_stride", C.c_int64), ("n_heads", C.c_int32)]


class MoqaeRope(C.Structure):
    _fields_ = [("cos_sin", C.c_void_p), ("q_weight", C.c_void_p), ("k_weight", C.c_void_p), ("n_positions", C.c_int32),
                ("rot_dim", C.c_int32), ("interleaved", C.c_int32), ("eps", C.c_float)]


class MoqaeAttnOptions(C.Structure):
    _fields_ = [("slopes", C.c_void_p), ("prefix_len", C.c_void_p), ("scale", C.c_float), ("cap", C.c_float),
                ("window", C.c_int32), ("max_new", C.c_int32)]


class MoqaeError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        msg = lib().moqae_error_string(code).decode()
        if code == ERR_CUDA:
            msg += f" [cuda error {lib().moqae_last_cuda_error()}]"
        super().__init__(f"{where}: {msg} ({code})")


_LIB = None


def lib_path() -> str:
    return _build.LIB


def lib() -> C.CDLL:
    """The loaded C-ABI library.  Raises if it has not been built (no fallback exists)."""
    global _LIB
    if _LIB is None:
        path = lib_path()
        if not os.path.exists(path):
            raise RuntimeError(f"{path} is missing: run `python -m paper_2506_07533_b200.build` "
                               "(the CUDA library is the only implementation)")
        L = C.CDLL(path)
        L.moqae_version.restype = C.c_int
        L.moqae_last_cuda_error.restype = C.c_int
        L.moqae_error_string.restype = C.c_char_p
        L.moqae_error_string.argtypes = [C.c_int]
        L.moqae_cache_bytes.argtypes = [C.POINTER(MoqaeConfig), C.POINTER(C.c_int64), C.POINTER(C.c_int64)]
        L.moqae_cache_bind.argtypes = [C.POINTER(MoqaeConfig), C.POINTER(C.c_int64), C.POINTER(C.c_void_p),
                                       C.POINTER(MoqaeCache)]
        L.moqae_route.argtypes = [C.POINTER(MoqaeConfig), C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p,
                                  C.c_void_p, C.c_void_p, C.c_int32, C.POINTER(MoqaeCache), C.c_void_p,
                                  C.c_void_p]
        L.moqae_quantize_kv.argtypes = [C.POINTER(MoqaeConfig), C.c_void_p, C.c_void_p, C.c_int32, C.c_int32,
                                        C.c_void_p, C.POINTER(MoqaeCache), C.c_void_p]
        L.moqae_project_quantize_kv.argtypes = [C.POINTER(MoqaeConfig), C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32,
                                                C.c_int32, C.c_void_p, C.POINTER(MoqaeCache), C.c_void_p, C.c_void_p,
                                                C.c_void_p]
        L.moqae_append_kv.argtypes = [C.POINTER(MoqaeConfig), C.c_void_p, C.c_void_p, C.c_int32,
                                      C.POINTER(MoqaeCache), C.c_void_p]
        L.moqae_flush_tail.argtypes = [C.POINTER(MoqaeConfig), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                       C.c_void_p, C.c_int32, C.POINTER(MoqaeCache), C.c_void_p]
        L.moqae_prefill_attn.argtypes = [C.POINTER(MoqaeConfig), C.c_void_p, C.c_int32, C.c_int32,
                                         C.POINTER(MoqaeCache), C.c_void_p, C.c_float, C.c_void_p, C.c_int64, C.c_void_p]
        L.moqae_prefill_attn_workspace.argtypes = [C.POINTER(MoqaeConfig), C.c_int32, C.POINTER(C.c_int64)]
        L.moqae_decode_attn_workspace.argtypes = [C.POINTER(MoqaeConfig), C.POINTER(C.c_int64)]
        L.moqae_decode_attn.argtypes = [C.POINTER(MoqaeConfig), C.c_void_p, C.c_int32, C.POINTER(MoqaeCache),
                                        C.c_void_p, C.c_float, C.c_void_p, C.c_int64, C.c_void_p]
        L.moqae_decode_attn_ex.argtypes = [C.POINTER(MoqaeConfig), C.c_void_p, C.c_int32, C.POINTER(MoqaeCache),
                                           C.c_void_p, C.c_float, C.c_void_p, C.c_int64, C.c_int32, C.c_void_p]
        L.moqae_decode_attn_step.argtypes = [C.POINTER(MoqaeConfig), C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32,
                                             C.POINTER(MoqaeCache), C.c_void_p, C.c_float, C.c_void_p, C.c_int64,
                                             C.c_int32, C.c_void_p]
        L.moqae_poll_status.argtypes = [C.POINTER(MoqaeCache), C.c_void_p, C.POINTER(C.c_int32)]
        L.moqae_validate_tables.argtypes = [C.POINTER(MoqaeConfig), C.POINTER(MoqaeCache), C.c_int32, C.c_int32,
                                            C.c_void_p, C.POINTER(C.c_int32), C.POINTER(C.c_int32)]
        L.moqae_validate_tables_host.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32,
                                                 C.POINTER(C.c_int64), C.POINTER(C.c_int32), C.POINTER(C.c_int32)]
        L.moqae_decode_attn_static.argtypes = [C.POINTER(MoqaeConfig), C.c_void_p, C.c_int32,
                                               C.POINTER(MoqaeCache), C.c_void_p, C.c_float, C.c_void_p]
        L.moqae_decode_attn_static_max_bytes.argtypes = []
        pc, rows, opts = C.POINTER(MoqaePagedCache), C.POINTER(MoqaeRows), C.POINTER(MoqaeAttnOptions)
        L.moqae_norm_rope.argtypes = [C.POINTER(MoqaeRope), C.c_int32, rows, rows, rows, rows, C.c_void_p, C.c_int32,
                                      C.c_void_p, C.c_void_p]
        L.moqae_paged_append.argtypes = [pc, C.POINTER(MoqaeRope), rows, rows, rows, rows, C.c_void_p, C.c_void_p,
                                         C.c_int32, C.c_void_p]
        L.moqae_paged_decode_attn_workspace.argtypes = [pc, C.c_int32, C.POINTER(C.c_int64)]
        L.moqae_paged_decode_attn.argtypes = [pc, rows, rows, opts, C.c_void_p, C.c_int64, C.c_void_p]
        L.moqae_paged_prefill_attn_workspace.argtypes = [pc, C.c_int32, C.c_int32, C.POINTER(C.c_int64)]
        L.moqae_paged_prefill_attn.argtypes = [pc, rows, C.c_void_p, C.c_int32, rows, opts, C.c_void_p, C.c_int64, C.c_void_p]
        L.moqae_paged_validate_host.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int32,
                                                C.POINTER(C.c_int32), C.POINTER(C.c_int32)]
        L.moqae_paged_validate.argtypes = [pc, C.c_void_p, C.POINTER(C.c_int32), C.POINTER(C.c_int32)]
        L.moqae_paged_poll_status.argtypes = [pc, C.c_void_p, C.POINTER(C.c_int32)]
        L.moqae_paged_plan.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p,
                                       C.POINTER(MoqaePagePool), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32,
                                       C.c_void_p, C.c_void_p]
        pc4 = C.POINTER(MoqaePaged4Cache)
        L.moqae_paged4_append.argtypes = [pc4, C.POINTER(MoqaeRope), rows, rows, rows, rows, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p]
        L.moqae_paged4_read.argtypes = [pc4, rows, rows, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p]
        L.moqae_paged4_decode_attn_workspace.argtypes = [pc4, C.c_int32, C.POINTER(C.c_int64)]
        L.moqae_paged4_decode_attn.argtypes = [pc4, rows, rows, opts, C.c_void_p, C.c_int64, C.c_void_p]
        L.moqae_paged4_prefill_attn_workspace.argtypes = [pc4, C.c_int32, C.c_int32, C.POINTER(C.c_int64), C.POINTER(C.c_int64)]
        L.moqae_paged4_prefill_attn.argtypes = [pc4, rows, C.c_void_p, C.c_int32, rows, opts, C.c_void_p, C.c_int64, C.c_void_p]
        L.moqae_paged4_validate.argtypes = [pc4, C.c_void_p, C.POINTER(C.c_int32), C.POINTER(C.c_int32)]
        L.moqae_paged4_poll_status.argtypes = [pc4, C.c_void_p, C.POINTER(C.c_int32)]
        for name in EXPORTS:
            if name not in ("moqae_error_string",):
                getattr(L, name).restype = C.c_int
        L.moqae_decode_attn_static_max_bytes.restype = C.c_int64
        _LIB = L
    return _LIB


def _check(rc: int, where: str):
    if rc != OK:
        raise MoqaeError(rc, where)


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def make_config(*, n_layers, n_q_heads, n_kv_heads, chunk, dtype, d_in, max_tokens, batch, rs_group=1,
                rf_first_chunk=1, tail_capacity=None, per_head_routing=False) -> MoqaeConfig:
    cfg = MoqaeConfig()
    cfg.n_layers, cfg.n_q_heads, cfg.n_kv_heads = n_layers, n_q_heads, n_kv_heads
    cfg.head_dim, cfg.chunk, cfg.group, cfg.dtype, cfg.n_experts = 128, chunk, 32, dtype, 4
    cfg.expert_bits = (C.c_int32 * 4)(*EXPERT_BITS)
    cfg.rs_group, cfg.rf_first_chunk, cfg.d_in = rs_group, int(rf_first_chunk), d_in
    cfg.max_tokens, cfg.batch = max_tokens, batch
    cfg.tail_capacity = chunk if tail_capacity is None else tail_capacity
    cfg.per_head_routing = int(bool(per_head_routing))
    return cfg


def moqae_version() -> int:
    return lib().moqae_version()


def moqae_cache_bytes(cfg: MoqaeConfig, capacity) -> list:
    cap = (C.c_int64 * 4)(*[int(c) for c in capacity])
    out = (C.c_int64 * N_CACHE_BUFFERS)()
    _check(lib().moqae_cache_bytes(C.byref(cfg), cap, out), "moqae_cache_bytes")
    return list(out)


@dataclass
class Cache:
    """Device buffers of one cache plus the C view handed to the library."""
    cfg: MoqaeConfig
    capacity: list
    buffers: list = field(default_factory=list)      # 12 torch uint8 tensors
    view: MoqaeCache = None

    @property
    def n_groups(self):
        return (self.cfg.n_layers + self.cfg.rs_group - 1) // self.cfg.rs_group

    @property
    def max_chunks(self):
        return self.cfg.max_tokens // self.cfg.chunk

    @property
    def table_rows(self):
        """Rows of the map / slot / count / votes tables per group: one per sequence, or one per
        (sequence, kv head) with per-head routing."""
        return self.cfg.batch * (self.cfg.n_kv_heads if self.cfg.per_head_routing else 1)

    def table(self, idx, dtype, shape):
        n = 1
        for d in shape:
            n *= d
        nbytes = n * torch.empty(0, dtype=dtype).element_size()
        return self.buffers[idx][:nbytes].view(dtype).view(*shape)

    @property
    def map(self):
        return self.table(4, torch.uint8, (self.n_groups, self.table_rows, self.max_chunks))

    @property
    def slot(self):
        return self.table(5, torch.int32, (self.n_groups, self.table_rows, self.max_chunks))

    @property
    def count(self):
        return self.table(6, torch.int32, (self.n_groups, self.table_rows, 4))

    @property
    def votes(self):
        return self.table(7, torch.int32, (self.n_groups, self.table_rows, self.max_chunks, 4))

    @property
    def tail_len(self):
        return self.table(10, torch.int32, (self.cfg.n_layers, self.cfg.batch))

    def pool(self, w):
        """uint8 view [n_layers, batch, n_kv_heads, capacity_w, slot_bytes_w]."""
        tb = 16384 if w == 3 else 1024 + 1024 * EXPERT_BITS[w]
        sb = max(1, self.cfg.chunk // 32) * tb      # a chunk of 8 or 16 tokens is one (padded) tile
        n = self.cfg.n_layers * self.cfg.batch * self.cfg.n_kv_heads * self.capacity[w] * sb
        return self.buffers[w][:n].view(self.cfg.n_layers, self.cfg.batch, self.cfg.n_kv_heads,
                                        self.capacity[w], sb)

    def tail(self, which):
        n = self.cfg.n_layers * self.cfg.batch * self.cfg.n_kv_heads * self.cfg.tail_capacity * 256
        t = self.buffers[8 if which == "k" else 9][:n].view(torch.int16)
        return t.view(self.cfg.n_layers, self.cfg.batch, self.cfg.n_kv_heads, self.cfg.tail_capacity, 128)


def moqae_cache_bind(cfg: MoqaeConfig, capacity, device="cuda", zero_pools=False) -> Cache:
    """Allocate the twelve buffers with torch and bind them (the library allocates nothing)."""
    sizes = moqae_cache_bytes(cfg, capacity)
    bufs = []
    for i, n in enumerate(sizes):
        n_alloc = max(16, (n + 15) // 16 * 16)
        if i < 4 and not zero_pools:
            bufs.append(torch.empty(n_alloc, dtype=torch.uint8, device=device))
        else:
            bufs.append(torch.zeros(n_alloc, dtype=torch.uint8, device=device))
    cap = (C.c_int64 * 4)(*[int(c) for c in capacity])
    ptrs = (C.c_void_p * N_CACHE_BUFFERS)(*[b.data_ptr() for b in bufs])
    view = MoqaeCache()
    _check(lib().moqae_cache_bind(C.byref(cfg), cap, ptrs, C.byref(view)), "moqae_cache_bind")
    return Cache(cfg=cfg, capacity=[int(c) for c in capacity], buffers=bufs, view=view)


def moqae_route(cfg, hidden, T, W1, W2, W3, bias, layer_group, cache: Cache, votes_out=None):
    _check(lib().moqae_route(C.byref(cfg), _ptr(hidden), int(T), _ptr(W1), _ptr(W2), _ptr(W3), _ptr(bias),
                             int(layer_group), C.byref(cache.view), _ptr(votes_out), _stream()), "moqae_route")


def moqae_quantize_kv(cfg, K, V, T, layer, cache: Cache, forced_map=None):
    _check(lib().moqae_quantize_kv(C.byref(cfg), _ptr(K), _ptr(V), int(T), int(layer), _ptr(forced_map),
                                   C.byref(cache.view), _stream()), "moqae_quantize_kv")


def moqae_project_quantize_kv(cfg, hidden, Wk, Wv, T, layer, cache: Cache, forced_map=None, k_rounded=None, v_rounded=None):
    _check(lib().moqae_project_quantize_kv(C.byref(cfg), _ptr(hidden), _ptr(Wk), _ptr(Wv), int(T), int(layer),
                                           _ptr(forced_map), C.byref(cache.view), _ptr(k_rounded), _ptr(v_rounded),
                                           _stream()), "moqae_project_quantize_kv")


def moqae_append_kv(cfg, k_new, v_new, layer, cache: Cache):
    _check(lib().moqae_append_kv(C.byref(cfg), _ptr(k_new), _ptr(v_new), int(layer), C.byref(cache.view),
                                 _stream()), "moqae_append_kv")


def moqae_flush_tail(cfg, hidden_tail, W1, W2, W3, bias, layer_group, cache: Cache):
    _check(lib().moqae_flush_tail(C.byref(cfg), _ptr(hidden_tail), _ptr(W1), _ptr(W2), _ptr(W3), _ptr(bias),
                                  int(layer_group), C.byref(cache.view), _stream()), "moqae_flush_tail")


def moqae_prefill_attn_workspace(cfg, T) -> int:
    out = C.c_int64(0)
    _check(lib().moqae_prefill_attn_workspace(C.byref(cfg), int(T), C.byref(out)), "moqae_prefill_attn_workspace")
    return int(out.value)


def moqae_prefill_attn(cfg, q, T, layer, cache: Cache, out, scale=0.0, workspace=None):
    nbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().moqae_prefill_attn(C.byref(cfg), _ptr(q), int(T), int(layer), C.byref(cache.view), _ptr(out),
                                    C.c_float(scale), _ptr(workspace), C.c_int64(nbytes), _stream()), "moqae_prefill_attn")


def moqae_decode_attn_workspace(cfg) -> int:
    out = C.c_int64(0)
    _check(lib().moqae_decode_attn_workspace(C.byref(cfg), C.byref(out)), "moqae_decode_attn_workspace")
    return int(out.value)


DECODE_OVERLAP_PREVIOUS = 1


def moqae_decode_attn(cfg, q, layer, cache: Cache, out, workspace, scale=0.0):
    _check(lib().moqae_decode_attn(C.byref(cfg), _ptr(q), int(layer), C.byref(cache.view), _ptr(out),
                                   C.c_float(scale), _ptr(workspace), int(workspace.numel() * workspace.element_size()),
                                   _stream()), "moqae_decode_attn")


def moqae_decode_attn_ex(cfg, q, layer, cache: Cache, out, workspace, flags=0, scale=0.0):
    """moqae_decode_attn with flags; DECODE_OVERLAP_PREVIOUS lets the launch start while the
    previous kernel on the stream is finishing (see include/moqae.h for the caller's promise)."""
    _check(lib().moqae_decode_attn_ex(C.byref(cfg), _ptr(q), int(layer), C.byref(cache.view), _ptr(out),
                                      C.c_float(scale), _ptr(workspace), int(workspace.numel() * workspace.element_size()),
                                      int(flags), _stream()), "moqae_decode_attn_ex")


def moqae_decode_attn_step(cfg, q, k_new, v_new, layer, cache: Cache, out, workspace, flags=0, scale=0.0):
    """Decode attention that also attends to the current token's own rows k_new / v_new (not yet in the
    cache); append them afterwards with moqae_append_kv."""
    _check(lib().moqae_decode_attn_step(C.byref(cfg), _ptr(q), _ptr(k_new), _ptr(v_new), int(layer), C.byref(cache.view),
                                        _ptr(out), C.c_float(scale), _ptr(workspace),
                                        int(workspace.numel() * workspace.element_size()), int(flags), _stream()),
           "moqae_decode_attn_step")


def moqae_decode_attn_static_max_bytes() -> int:
    return int(lib().moqae_decode_attn_static_max_bytes())


def moqae_decode_attn_static(cfg, q, layer, cache: Cache, out, scale=0.0):
    """moqae_decode_attn without a caller-provided workspace: for callers that cannot allocate
    device memory, the split partials live in a fixed array inside the library."""
    _check(lib().moqae_decode_attn_static(C.byref(cfg), _ptr(q), int(layer), C.byref(cache.view), _ptr(out),
                                          C.c_float(scale), _stream()), "moqae_decode_attn_static")


def moqae_validate_tables(cfg, cache: Cache, T, layer_group=0):
    """(code, bad_row, bad_chunk): OK, or ERR_CORRUPT_TABLE with the first offending position."""
    r, c = C.c_int32(-1), C.c_int32(-1)
    rc = lib().moqae_validate_tables(C.byref(cfg), C.byref(cache.view), int(T), int(layer_group), _stream(),
                                     C.byref(r), C.byref(c))
    if rc not in (OK, ERR_CORRUPT_TABLE):
        raise MoqaeError(rc, "moqae_validate_tables")
    return rc, int(r.value), int(c.value)


def moqae_validate_tables_host(map_u8, slot_i32, count_i32, n_chunks, capacity):
    """The same check on host numpy arrays map / slot [rows, max_chunks] and count [rows, 4]."""
    import numpy as np
    m = np.ascontiguousarray(map_u8, dtype=np.uint8)
    s = np.ascontiguousarray(slot_i32, dtype=np.int32)
    k = np.ascontiguousarray(count_i32, dtype=np.int32)
    cap = (C.c_int64 * 4)(*[int(x) for x in capacity])
    r, c = C.c_int32(-1), C.c_int32(-1)
    rc = lib().moqae_validate_tables_host(m.ctypes.data_as(C.c_void_p), s.ctypes.data_as(C.c_void_p),
                                          k.ctypes.data_as(C.c_void_p), m.shape[0], m.shape[1], int(n_chunks), cap,
                                          C.byref(r), C.byref(c))
    return rc, int(r.value), int(c.value)


def moqae_poll_status(cache: Cache) -> int:
    out = C.c_int32(0)
    _check(lib().moqae_poll_status(C.byref(cache.view), _stream(), C.byref(out)), "moqae_poll_status")
    return int(out.value)


# ---- paged 16-bit cache ---------------------------------------------------------------------------

_DTYPE_CODE = {torch.float16: DT_FP16, torch.bfloat16: DT_BF16}


# The calls below are made once per layer and generated token; their arguments are taken apart in csrc/marshal.cpp.
_MARSHAL = None


def _native():
    """The marshalling module, bound to the loaded library.  Raises if it has not been built."""
    global _MARSHAL
    if _MARSHAL is None:
        names = ("moqae_norm_rope", "moqae_paged_append", "moqae_paged_decode_attn", "moqae_paged_prefill_attn", "moqae_paged_plan",
                 "moqae_paged4_append", "moqae_paged4_read", "moqae_paged4_decode_attn", "moqae_paged4_prefill_attn")
        addresses = [C.cast(getattr(lib(), n), C.c_void_p).value for n in names]
        missing = f"{_build.MARSHAL} is missing or was built for another torch: run `python -m paper_2506_07533_b200.build`"
        try:
            from . import _marshal
        except ImportError as e:
            raise RuntimeError(missing) from e
        if getattr(_marshal, "built_for", None) != _build.marshal_key():
            raise RuntimeError(missing)
        _marshal.bind(*addresses[:4])
        _marshal.bind4(*addresses[4:])
        _MARSHAL = _marshal
    return _MARSHAL


def _need(ok: bool, where: str, code: int = ERR_INVALID_ARG):
    if not ok:
        raise MoqaeError(code, where)


def _vector(t, dtype, n, index, where):
    """Address of a contiguous tensor of `n` values on device `index`; None stays None."""
    if t is None:
        return None
    _need(t.dtype is dtype and t.get_device() == index and t.numel() == n and t.is_contiguous(), where)
    return t.data_ptr()


@dataclass
class Rope:
    """A moqae_rope and the tensors it points to."""
    view: MoqaeRope
    code: int                    # dtype of the rows, -1 without weights
    device: int                  # device index, -1 without tensors
    tensors: tuple
    address: int = 0

    def __post_init__(self):
        self.address = C.addressof(self.view)


def rope_table(n_positions, rot_dim, base=10000.0, device="cuda"):
    """float32 [n_positions, rot_dim]: cosines, then sines, of p * base^(-2 i / rot_dim), angles taken in 64 bits."""
    freq = base ** (-torch.arange(0, rot_dim, 2, dtype=torch.float64, device=device) / max(rot_dim, 1))
    angle = torch.arange(n_positions, dtype=torch.float64, device=device)[:, None] * freq
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def make_rope(cos_sin, rot_dim, *, interleaved=False, q_weight=None, k_weight=None, eps=1e-6) -> Rope:
    """Norm and rotation of moqae_norm_rope / moqae_paged_append.  cos_sin float32 [n_positions, rot_dim]
    (rope_table), or None with rot_dim = 0; weights [128] in the rows' dtype, or None for no norm."""
    where = "make_rope"
    given = [t for t in (cos_sin, q_weight, k_weight) if t is not None]
    _need(all(t.is_cuda and t.is_contiguous() and t.get_device() == given[0].get_device() for t in given), where)
    _need((cos_sin is None) == (rot_dim == 0), where)
    if cos_sin is not None:
        _need(cos_sin.dtype == torch.float32 and cos_sin.dim() == 2 and cos_sin.shape[1] == rot_dim, where)
    weights = [w for w in (q_weight, k_weight) if w is not None]
    _need(all(w.shape == (128,) and w.dtype == weights[0].dtype and w.dtype in _DTYPE_CODE for w in weights), where)
    ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    view = MoqaeRope(ptr(cos_sin), ptr(q_weight), ptr(k_weight), 0 if cos_sin is None else cos_sin.shape[0], int(rot_dim),
                     int(bool(interleaved)), float(eps))
    return Rope(view, _DTYPE_CODE[weights[0].dtype] if weights else -1, given[0].get_device() if given else -1, (cos_sin, q_weight, k_weight))


def moqae_norm_rope(rope: Rope, q, k, positions, q_out=None, k_out=None, status=None):
    """Norm and rotate query rows q [n, heads, 128] and key rows k (either may be None) into q_out / k_out, which
    default to q and k themselves.  positions int32 [n], negative = padding; status int32 [4] or None."""
    rc = (_MARSHAL or _native()).norm_rope(rope.address, rope.code, rope.device, q, k, positions, q_out, k_out, status)
    if rc:
        raise MoqaeError(rc, "moqae_norm_rope")


@dataclass
class PagedCache:
    """The tensors of a paged 16-bit cache and the C view handed to the library."""
    k_pages: torch.Tensor        # [n_pages, n_kv_heads, page_size, 128], any strides of whole rows
    v_pages: torch.Tensor
    block_table: torch.Tensor    # int32 [batch, max_pages]
    kv_len: torch.Tensor         # int32 [batch]
    status: torch.Tensor         # int32 [4]
    view: MoqaePagedCache
    code: int                    # MOQAE_DTYPE_*
    device: int                  # device index
    batch: int
    address: int = 0

    def __post_init__(self):
        self.address = C.addressof(self.view)


def moqae_paged_bind(k_pages, v_pages, block_table, kv_len, status=None) -> PagedCache:
    """A paged cache over the caller's tensors.  k_pages, v_pages [n_pages, n_kv_heads, page_size, 128] with
    contiguous rows (a [n_pages, page_size, n_kv_heads, 128] buffer is given transposed); block_table int32
    [batch, max_pages]; kv_len int32 [batch].  The contents of all of them may change between calls."""
    where = "moqae_paged_bind"
    _need(k_pages.is_cuda and k_pages.dtype in _DTYPE_CODE and k_pages.dim() == 4 and k_pages.shape[3] == 128, where)
    index = k_pages.get_device()
    _need(v_pages.shape == k_pages.shape and v_pages.dtype == k_pages.dtype and v_pages.get_device() == index, where)
    _need(k_pages.stride(3) == 1 and v_pages.stride(3) == 1, where)
    _need(block_table.dim() == 2 and block_table.dtype == torch.int32 and block_table.is_contiguous() and block_table.get_device() == index, where)
    if status is None:
        status = torch.zeros(4, dtype=torch.int32, device=k_pages.device)
    view = MoqaePagedCache(k_pages.data_ptr(), v_pages.data_ptr(), (C.c_int64 * 3)(*k_pages.stride()[:3]),
                           (C.c_int64 * 3)(*v_pages.stride()[:3]), block_table.data_ptr(),
                           _vector(kv_len, torch.int32, block_table.shape[0], index, where), _vector(status, torch.int32, 4, index, where),
                           k_pages.shape[0], k_pages.shape[2], k_pages.shape[1], _DTYPE_CODE[k_pages.dtype],
                           block_table.shape[0], block_table.shape[1])
    return PagedCache(k_pages, v_pages, block_table, kv_len, status, view, _DTYPE_CODE[k_pages.dtype], index, block_table.shape[0])


def moqae_paged_append(cache: PagedCache, k, v, positions, *, seq=None, rope: Rope = None, q=None, q_out=None):
    """Put key and value rows k, v [n, n_kv_heads, 128] into their pages: token t is token positions[t] (negative =
    padding) of sequence seq[t] (None: sequence t).  With `rope` keys, and queries q into q_out (default: in
    place), are normalised and rotated on the way."""
    r = (0, -1, -1) if rope is None else (rope.address, rope.code, rope.device)
    rc = (_MARSHAL or _native()).append(cache.address, cache.code, cache.device, *r, k, v, positions, seq, q, q_out)
    if rc:
        raise MoqaeError(rc, "moqae_paged_append")


@dataclass
class AttnOptions:
    """A moqae_attn_options and the tensors it points to."""
    view: MoqaeAttnOptions
    slopes: torch.Tensor
    prefix_len: torch.Tensor
    address: int = 0

    def __post_init__(self):
        self.address = C.addressof(self.view)


def make_attn_options(*, scale=0.0, cap=0.0, window=0, slopes=None, prefix_len=None, max_new=0) -> AttnOptions:
    """Options of the paged attention calls: scale (<= 0: 1/sqrt(128)), tanh cap of the scores (0: none), sliding
    window (0: none), slopes float32 [n_q_heads] of the distance bias, prefix_len int32 [batch].  max_new: no sequence of the
    call brings more new tokens (0: not known), which spares moqae_paged4_prefill_attn two launches where all bring few."""
    ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    window = max(min(int(window), 1 << 30), -1)              # no sequence is longer; numbers past 32 bits would lose their upper ones
    return AttnOptions(MoqaeAttnOptions(ptr(slopes), ptr(prefix_len), float(scale), float(cap), window, max(min(int(max_new), 1 << 30), 0)), slopes, prefix_len)


def _options(options, cache, q, where):
    if options is None:
        return 0
    if options.slopes is not None:
        _vector(options.slopes, torch.float32, q.shape[1], cache.device, where)
    if options.prefix_len is not None:
        _vector(options.prefix_len, torch.int32, cache.batch, cache.device, where)
    return options.address


def moqae_paged_decode_attn_workspace(cache: PagedCache, n_q_heads) -> int:
    out = C.c_int64(0)
    _check(lib().moqae_paged_decode_attn_workspace(C.byref(cache.view), int(n_q_heads), C.byref(out)), "moqae_paged_decode_attn_workspace")
    return int(out.value)


def moqae_paged_decode_attn(cache: PagedCache, q, out, workspace, options: AttnOptions = None):
    """Attention of one new token per sequence: q, out [batch, n_q_heads, 128] in the cache's dtype; workspace a
    tensor of moqae_paged_decode_attn_workspace bytes, zeroed once."""
    where = "moqae_paged_decode_attn"
    rc = (_MARSHAL or _native()).decode(cache.address, cache.code, cache.device, cache.batch, q, out, workspace, _options(options, cache, q, where))
    if rc:
        raise MoqaeError(rc, where)


def moqae_paged_prefill_attn_workspace(cache: PagedCache, n_q_heads, n_tokens) -> int:
    """Bytes for every call of up to n_tokens tokens over up to as many sequences as `cache` has, one-token calls included."""
    out = C.c_int64(0)
    _check(lib().moqae_paged_prefill_attn_workspace(C.byref(cache.view), int(n_q_heads), int(n_tokens), C.byref(out)),
           "moqae_paged_prefill_attn_workspace")
    return int(out.value)


def moqae_paged_prefill_attn(cache: PagedCache, q, cu_q, out, workspace=None, options: AttnOptions = None):
    """Attention of the last cu_q[b + 1] - cu_q[b] tokens of every sequence: q, out [n_tokens, n_q_heads, 128] in the
    cache's dtype, cu_q int32 [batch + 1]; workspace None, or moqae_paged_prefill_attn_workspace bytes zeroed once."""
    where = "moqae_paged_prefill_attn"
    rc = (_MARSHAL or _native()).prefill(cache.address, cache.code, cache.device, cache.batch, q, cu_q, out, workspace,
                                         _options(options, cache, q, where))
    if rc:
        raise MoqaeError(rc, where)


def moqae_paged_validate(cache):
    """(code, bad_seq, bad_entry): OK, or ERR_CORRUPT_TABLE with the first offending table entry (-1: the length).  Of
    a PagedCache or a Paged4Cache."""
    b, e = C.c_int32(-1), C.c_int32(-1)
    call = lib().moqae_paged4_validate if isinstance(cache, Paged4Cache) else lib().moqae_paged_validate
    with torch.cuda.device(cache.device):
        rc = call(C.byref(cache.view), torch.cuda.current_stream().cuda_stream, C.byref(b), C.byref(e))
    if rc not in (OK, ERR_CORRUPT_TABLE):
        raise MoqaeError(rc, "moqae_paged_validate")
    return rc, int(b.value), int(e.value)


def moqae_paged_validate_host(block_table, kv_len, n_pages, page_size):
    """The same check on host numpy arrays block_table [batch, max_pages] and kv_len [batch]."""
    import numpy as np
    t = np.ascontiguousarray(block_table, dtype=np.int32)
    n = np.ascontiguousarray(kv_len, dtype=np.int32)
    b, e = C.c_int32(-1), C.c_int32(-1)
    rc = lib().moqae_paged_validate_host(t.ctypes.data_as(C.c_void_p), n.ctypes.data_as(C.c_void_p), t.shape[0], t.shape[1],
                                         int(n_pages), int(page_size), C.byref(b), C.byref(e))
    return rc, int(b.value), int(e.value)


def moqae_paged_poll_status(cache) -> int:
    """MOQAE_OK or the first device-side error of a PagedCache or a Paged4Cache."""
    out = C.c_int32(0)
    call = lib().moqae_paged4_poll_status if isinstance(cache, Paged4Cache) else lib().moqae_paged_poll_status
    with torch.cuda.device(cache.device):
        _check(call(C.byref(cache.view), torch.cuda.current_stream().cuda_stream, C.byref(out)), "moqae_paged_poll_status")
    return int(out.value)


# ---- plan of a step -------------------------------------------------------------------------------

@dataclass
class PagePool:
    """The free pages of a cache: ring[(first + i) % n], i < free, of page numbers.  state int32 [4]: first, free, 0, 0."""
    ring: torch.Tensor           # int32 [n_pages]
    state: torch.Tensor          # int32 [4]


def make_page_pool(n_pages, device="cuda") -> PagePool:
    """A pool that holds the pages 0 .. n_pages - 1."""
    return PagePool(torch.arange(n_pages, dtype=torch.int32, device=device), torch.tensor([0, n_pages, 0, 0], dtype=torch.int32, device=device))


def moqae_paged_plan(cache, pool: PagePool, n_new, cu_q, positions, seq, *, past_len=None, pool_state=None):
    """Block table and lengths of a step of `cache` (PagedCache or Paged4Cache), pages taken from and given back to `pool`.
    n_new int32 [batch]: tokens that each sequence gets (negative: loses).  Written: cache.block_table, cache.kv_len, cu_q int32
    [batch + 1], positions and seq int32 [rows] (-1 behind the last row).  past_len, the lengths before, and pool_state, the
    pool's state before, default to cache.kv_len and pool.state.  Errors are recorded in cache.status."""
    rc = (_MARSHAL or _native()).plan(cache.device, cache.batch, cache.block_table.shape[1], cache.view.page_size, cache.block_table,
                                      cache.kv_len, cache.status, pool.ring, pool.state, n_new, past_len, pool_state, cu_q, positions, seq)
    if rc:
        raise MoqaeError(rc, "moqae_paged_plan")


# ---- paged 4-bit cache ----------------------------------------------------------------------------

TOKEN_BYTES4 = 160               # of a token and kv head


@dataclass
class Paged4Cache:
    """The tensors of a paged 4-bit cache and the C view handed to the library."""
    pages: torch.Tensor          # uint8 [n_pages, n_kv_heads, page_size * 160], any strides of whole pages and heads
    block_table: torch.Tensor    # int32 [batch, max_pages]
    kv_len: torch.Tensor         # int32 [batch]
    status: torch.Tensor         # int32 [4]
    view: MoqaePaged4Cache
    code: int                    # MOQAE_DTYPE_* of rows
    device: int                  # device index
    batch: int
    address: int = 0

    def __post_init__(self):
        self.address = C.addressof(self.view)


def moqae_paged4_bind(pages, block_table, kv_len, dtype, status=None) -> Paged4Cache:
    """A paged 4-bit cache over the caller's tensors.  pages uint8 [n_pages, n_kv_heads, page_size * 160] (contents need not be
    initialised); block_table int32 [batch, max_pages]; kv_len int32 [batch]; dtype of the rows that the calls take and give.
    The contents of all of them may change between calls."""
    where = "moqae_paged4_bind"
    _need(pages.is_cuda and pages.dtype == torch.uint8 and pages.dim() == 3 and pages.shape[2] % TOKEN_BYTES4 == 0, where)
    _need(pages.stride(2) == 1 and dtype in _DTYPE_CODE, where)
    index = pages.get_device()
    _need(block_table.dim() == 2 and block_table.dtype == torch.int32 and block_table.is_contiguous() and block_table.get_device() == index, where)
    if status is None:
        status = torch.zeros(4, dtype=torch.int32, device=pages.device)
    head_stride = pages.stride(1) if pages.shape[1] > 1 else pages.shape[2]      # (a stride along one element may be anything)
    page_stride = pages.stride(0) if pages.shape[0] > 1 else max(pages.shape[1], 1) * pages.shape[2]
    view = MoqaePaged4Cache(pages.data_ptr(), page_stride, head_stride, block_table.data_ptr(),
                            _vector(kv_len, torch.int32, block_table.shape[0], index, where), _vector(status, torch.int32, 4, index, where),
                            pages.shape[0], pages.shape[2] // TOKEN_BYTES4, pages.shape[1], _DTYPE_CODE[dtype], block_table.shape[0],
                            block_table.shape[1])
    return Paged4Cache(pages, block_table, kv_len, status, view, _DTYPE_CODE[dtype], index, block_table.shape[0])


def moqae_paged4_append(cache: Paged4Cache, k, v, positions, *, seq=None, rope: Rope = None, q=None, q_out=None):
    """moqae_paged_append into a 4-bit cache: keys (normalised and rotated with `rope`) and values are quantised on their way."""
    r = (0, -1, -1) if rope is None else (rope.address, rope.code, rope.device)
    rc = (_MARSHAL or _native()).append4(cache.address, cache.code, cache.device, *r, k, v, positions, seq, q, q_out)
    if rc:
        raise MoqaeError(rc, "moqae_paged4_append")


def moqae_paged4_read(cache: Paged4Cache, k_out, v_out, positions, *, seq=None):
    """Keys and values of tokens positions[t] (negative: left out) of sequences seq[t] (None: sequence t) as the values they
    stand for, into rows k_out, v_out [n, n_kv_heads, 128] (one of them may be None)."""
    rc = (_MARSHAL or _native()).read4(cache.address, cache.code, cache.device, k_out, v_out, positions, seq)
    if rc:
        raise MoqaeError(rc, "moqae_paged4_read")


def moqae_paged4_decode_attn_workspace(cache: Paged4Cache, n_q_heads) -> int:
    out = C.c_int64(0)
    _check(lib().moqae_paged4_decode_attn_workspace(C.byref(cache.view), int(n_q_heads), C.byref(out)), "moqae_paged4_decode_attn_workspace")
    return int(out.value)


def moqae_paged4_decode_attn(cache: Paged4Cache, q, out, workspace, options: AttnOptions = None):
    """Attention of one new token per sequence: q, out [batch, n_q_heads, 128] in the cache's dtype; workspace a
    tensor of moqae_paged4_decode_attn_workspace bytes, zeroed once."""
    where = "moqae_paged4_decode_attn"
    rc = (_MARSHAL or _native()).decode4(cache.address, cache.code, cache.device, cache.batch, q, out, workspace, _options(options, cache, q, where))
    if rc:
        raise MoqaeError(rc, where)


def moqae_paged4_prefill_attn_workspace(cache: Paged4Cache, n_q_heads, n_tokens, *, least=False) -> int:
    """Bytes for every call of up to n_tokens tokens over up to as many sequences as `cache` has, one-token calls included.
    They hold the sequences' blocks at 16 bits, as far as 1 GiB goes; least=True leaves these out (slower calls)."""
    out, low = C.c_int64(0), C.c_int64(0)
    _check(lib().moqae_paged4_prefill_attn_workspace(C.byref(cache.view), int(n_q_heads), int(n_tokens), C.byref(out), C.byref(low)),
           "moqae_paged4_prefill_attn_workspace")
    return int(low.value if least else out.value)


def moqae_paged4_prefill_attn(cache: Paged4Cache, q, cu_q, out, workspace, options: AttnOptions = None):
    """Attention of the last cu_q[b + 1] - cu_q[b] tokens of every sequence: q, out [n_tokens, n_q_heads, 128] in the
    cache's dtype, cu_q int32 [batch + 1]; workspace of moqae_paged4_prefill_attn_workspace bytes, zeroed once."""
    where = "moqae_paged4_prefill_attn"
    rc = (_MARSHAL or _native()).prefill4(cache.address, cache.code, cache.device, cache.batch, q, cu_q, out, workspace,
                                          _options(options, cache, q, where))
    if rc:
        raise MoqaeError(rc, where)
