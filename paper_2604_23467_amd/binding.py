"""Thin ctypes binding of ``libll.so`` (declarations: ``include/ll.h``).

Argument marshalling only: every step of the decode / prefill path runs in the
HIP kernels behind the C ABI.  PyTorch appears here solely as the owner of
device memory (weights, workspace) and of the HIP stream.  There is no CPU
fallback: a missing library raises.
"""
import ctypes as C
import os

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libll.so")

LL_OK = 0
LL_E_NOT_INIT, LL_E_BAD_CONFIG, LL_E_BAD_ARG, LL_E_CAPACITY = -1, -2, -3, -4
LL_E_WORKSPACE, LL_E_STATE, LL_E_HIP, LL_E_ALREADY_INIT = -5, -6, -7, -8
LL_FLAG_EAGER = 1
LL_FLAG_MULTIKERNEL = 2
LL_FLAG_PERSISTENT = 4
LL_FLAG_PER_LENGTH_GRAPHS = 8
LL_FLAG_FUSED_ATTN_OPROJ = 16
LL_FLAG_LEAN_WORKSPACE = 32
LL_F16, LL_BF16 = 0, 1
LL_MODE_PERSISTENT_GRAPH, LL_MODE_MULTIKERNEL_GRAPH, LL_MODE_EAGER, LL_MODE_PER_LENGTH_GRAPHS = 0, 1, 2, 3
KERNEL_CLASSES = ("embed", "qkv", "attn", "oproj", "gateup", "down", "lmhead", "sample")
LAYER_KEYS = ("attn_norm", "wq", "wk", "wv", "wo", "ffn_norm", "w_gate", "w_up", "w_down")

EXPORTS = ("ll_workspace_bytes", "ll_init", "ll_prefill", "ll_prefill_static", "ll_decode_step", "ll_decode_n", "ll_reset",
           "ll_set_sampling", "ll_shutdown", "ll_max_prompt", "ll_position", "ll_decode_mode", "ll_last_error", "ll_dbg_get_logits",
           "ll_batch_pool_bytes", "ll_batch_open", "ll_batch_add", "ll_batch_step", "ll_batch_remove", "ll_batch_close",
           "ll_kv4_pool_bytes", "ll_kv4_write", "ll_kv4_read", "ll_kv4_attention_workspace_bytes", "ll_kv4_attention",
           "ll_batch_pool_bytes_kv", "ll_batch_open_kv", "ll_batch_dbg_get_kv",
           "ll_batch_dbg_get_logits", "ll_batch_dbg_force_next_token", "ll_batch_dbg_time_steps",
           "ll_dbg_get_hidden", "ll_dbg_set_spin_limit", "ll_dbg_give_up_at", "ll_dbg_small_plan", "ll_dbg_graph_stats", "ll_dbg_gemm_plan", "ll_dbg_gemm_slice_count", "ll_dbg_tile_plan", "ll_dbg_batch_order", "ll_dbg_force_next_token", "ll_dbg_get_kv", "ll_dbg_profile_decode",
           "ll_dbg_time_decode", "ll_dbg_time_kernel_class", "ll_dbg_stream_copy", "ll_dbg_stream_read", "ll_dbg_poison_scratch", "ll_dbg_trace_decode")


class LLConfig(C.Structure):
    _fields_ = [(k, C.c_int32) for k in
                ("n_layers", "d_model", "n_heads", "head_dim", "ffn_hidden", "vocab", "max_seq")] + \
               [("rope_theta", C.c_float), ("rms_eps", C.c_float), ("flags", C.c_int32)]


class LLLayerWeights(C.Structure):
    _fields_ = [(k, C.c_void_p) for k in LAYER_KEYS]


class LLWeights(C.Structure):
    _fields_ = [("tok_emb", C.c_void_p), ("layers", C.POINTER(LLLayerWeights)),
                ("final_norm", C.c_void_p), ("lm_head", C.c_void_p)]


class LLKV4Cache(C.Structure):
    _fields_ = [("pool", C.c_void_p), ("pool_bytes", C.c_size_t)] + \
               [(k, C.c_int32) for k in ("n_kv_heads", "head_dim", "page_tokens", "n_pages")]


class LLKV4Rows(C.Structure):
    _fields_ = [(k, C.c_void_p) for k in ("row_start", "len", "page_table")] + \
               [(k, C.c_int32) for k in ("n_seqs", "max_rows", "n_rows", "table_stride", "max_len")]


class LLKV4View(C.Structure):
    _fields_ = [("data", C.c_void_p), ("row_stride", C.c_int64), ("head_stride", C.c_int64)]


class LLError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__("ll error %d: %s" % (code, msg))
        self.code = code


_lib = None


def load():
    """Loads libll.so (built beforehand by ``paper_2604_23467_amd.build``)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError("HIP library %s is missing: run `python -m paper_2604_23467_amd.build` "
                           "(there is no CPU fallback)" % LIB_PATH)
    L = C.CDLL(LIB_PATH)
    L.ll_workspace_bytes.restype = C.c_size_t
    L.ll_workspace_bytes.argtypes = [C.POINTER(LLConfig)]
    L.ll_init.restype = C.c_int
    L.ll_init.argtypes = [C.POINTER(LLConfig), C.POINTER(LLWeights), C.c_void_p, C.c_size_t, C.c_void_p]
    L.ll_prefill.restype = C.c_int32
    L.ll_prefill.argtypes = [C.POINTER(C.c_int32), C.c_int32]
    L.ll_prefill_static.restype = C.c_int32
    L.ll_prefill_static.argtypes = [C.POINTER(C.c_int32), C.c_int32]
    L.ll_decode_step.restype = C.c_int32
    L.ll_decode_step.argtypes = []
    L.ll_decode_n.restype = C.c_int32
    L.ll_decode_n.argtypes = [C.c_int32, C.POINTER(C.c_int32)]
    for name in ("ll_reset", "ll_shutdown", "ll_dbg_poison_scratch"):
        getattr(L, name).restype = C.c_int
        getattr(L, name).argtypes = []
    for name in ("ll_max_prompt", "ll_position", "ll_decode_mode"):
        getattr(L, name).restype = C.c_int32
        getattr(L, name).argtypes = []
    L.ll_set_sampling.restype = C.c_int
    L.ll_set_sampling.argtypes = [C.c_float, C.c_int32, C.c_float, C.c_uint64]
    L.ll_last_error.restype = C.c_char_p
    L.ll_last_error.argtypes = []
    L.ll_dbg_get_logits.restype = C.c_int
    L.ll_dbg_get_logits.argtypes = [C.POINTER(C.c_float)]
    L.ll_batch_pool_bytes.restype = C.c_size_t
    L.ll_batch_pool_bytes.argtypes = [C.c_int32, C.c_int32]
    L.ll_batch_open.restype = C.c_int
    L.ll_batch_open.argtypes = [C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_size_t]
    L.ll_batch_pool_bytes_kv.restype = C.c_size_t
    L.ll_batch_pool_bytes_kv.argtypes = [C.c_int32] * 3
    L.ll_batch_open_kv.restype = C.c_int
    L.ll_batch_open_kv.argtypes = [C.c_int32] * 4 + [C.c_void_p, C.c_size_t]
    L.ll_batch_dbg_get_kv.restype = C.c_int
    L.ll_batch_dbg_get_kv.argtypes = [C.c_int32] * 4 + [C.POINTER(C.c_float)]
    L.ll_batch_add.restype = C.c_int32
    L.ll_batch_add.argtypes = [C.POINTER(C.c_int32), C.c_int32, C.POINTER(C.c_int32)]
    L.ll_batch_step.restype = C.c_int
    L.ll_batch_step.argtypes = [C.POINTER(C.c_int32)]
    L.ll_batch_remove.restype = C.c_int
    L.ll_batch_remove.argtypes = [C.c_int32]
    L.ll_batch_close.restype = C.c_int
    L.ll_batch_close.argtypes = []
    L.ll_batch_dbg_get_logits.restype = C.c_int
    L.ll_batch_dbg_get_logits.argtypes = [C.c_int32, C.POINTER(C.c_float)]
    L.ll_batch_dbg_force_next_token.restype = C.c_int
    L.ll_batch_dbg_force_next_token.argtypes = [C.c_int32, C.c_int32]
    L.ll_batch_dbg_time_steps.restype = C.c_int
    L.ll_batch_dbg_time_steps.argtypes = [C.c_int32, C.POINTER(C.c_float)]
    L.ll_dbg_batch_order.restype = C.c_int
    L.ll_dbg_batch_order.argtypes = [C.POINTER(C.c_int32)] * 2 + [C.c_int32] * 2 + [C.POINTER(C.c_int32)]
    L.ll_dbg_tile_plan.restype = C.c_int
    L.ll_dbg_tile_plan.argtypes = [C.c_int32] * 4 + [C.POINTER(C.c_int32)]
    L.ll_dbg_gemm_plan.restype = C.c_int
    L.ll_dbg_gemm_plan.argtypes = [C.c_int32] * 4 + [C.POINTER(C.c_int32)]
    L.ll_dbg_gemm_slice_count.restype = C.c_int
    L.ll_dbg_gemm_slice_count.argtypes = [C.c_int32] * 5
    L.ll_dbg_set_spin_limit.restype = C.c_int
    L.ll_dbg_set_spin_limit.argtypes = [C.c_int32]
    L.ll_dbg_give_up_at.restype = C.c_int
    L.ll_dbg_give_up_at.argtypes = [C.c_int32]
    L.ll_dbg_small_plan.restype = C.c_int
    L.ll_dbg_small_plan.argtypes = [C.POINTER(LLConfig), C.c_int32, C.c_int32, C.POINTER(C.c_int32)]
    L.ll_dbg_graph_stats.restype = C.c_int
    L.ll_dbg_graph_stats.argtypes = [C.POINTER(C.c_int64)]
    L.ll_dbg_get_hidden.restype = C.c_int
    L.ll_dbg_get_hidden.argtypes = [C.POINTER(C.c_float)]
    L.ll_dbg_force_next_token.restype = C.c_int
    L.ll_dbg_force_next_token.argtypes = [C.c_int32]
    L.ll_dbg_get_kv.restype = C.c_int
    L.ll_dbg_get_kv.argtypes = [C.c_int32, C.c_int32, C.c_int32, C.POINTER(C.c_float)]
    L.ll_dbg_profile_decode.restype = C.c_int
    L.ll_dbg_profile_decode.argtypes = [C.c_int32, C.POINTER(C.c_float), C.POINTER(C.c_int32)]
    L.ll_dbg_time_kernel_class.restype = C.c_int
    L.ll_dbg_time_kernel_class.argtypes = [C.c_int32, C.c_int32, C.POINTER(C.c_float)]
    L.ll_dbg_trace_decode.restype = C.c_int
    L.ll_dbg_trace_decode.argtypes = [C.POINTER(C.c_uint64), C.c_int32]
    L.ll_dbg_stream_copy.restype = C.c_int
    L.ll_dbg_stream_copy.argtypes = [C.c_void_p, C.c_void_p, C.c_size_t]
    L.ll_dbg_stream_read.restype = C.c_int
    L.ll_dbg_stream_read.argtypes = [C.c_void_p, C.c_size_t, C.c_int32, C.c_void_p, C.POINTER(C.c_float)]
    L.ll_dbg_time_decode.restype = C.c_int
    L.ll_dbg_time_decode.argtypes = [C.c_int32, C.POINTER(C.c_float)]
    cache, rows, view = C.POINTER(LLKV4Cache), C.POINTER(LLKV4Rows), C.POINTER(LLKV4View)
    L.ll_kv4_pool_bytes.restype = C.c_size_t
    L.ll_kv4_pool_bytes.argtypes = [cache]
    for name in ("ll_kv4_write", "ll_kv4_read"):
        getattr(L, name).restype = C.c_int
        getattr(L, name).argtypes = [cache, rows, C.c_int32, view, view, C.c_void_p]
    L.ll_kv4_attention_workspace_bytes.restype = C.c_size_t
    L.ll_kv4_attention_workspace_bytes.argtypes = [cache, rows, C.c_int32]
    L.ll_kv4_attention.restype = C.c_int
    L.ll_kv4_attention.argtypes = [cache, rows, C.c_int32, C.c_int32, C.c_float] + [view] * 4 + [C.c_void_p, C.c_size_t, C.c_void_p]
    _lib = L
    return L


def _check(rc):
    if rc < 0:
        raise LLError(rc, load().ll_last_error().decode())
    return rc


def make_config(cfg, flags=0):
    return LLConfig(**{k: int(cfg[k]) for k in ("n_layers", "d_model", "n_heads", "head_dim",
                                                  "ffn_hidden", "vocab", "max_seq")},
                    rope_theta=float(cfg["rope_theta"]), rms_eps=float(cfg["rms_eps"]), flags=flags)


def ll_workspace_bytes(cfg, flags=0):
    c = make_config(cfg, flags)
    return int(load().ll_workspace_bytes(C.byref(c)))


def ll_dbg_stream_copy(dst, src):
    """Copies one contiguous CUDA tensor into another of the same byte size."""
    nbytes = src.numel() * src.element_size()
    assert dst.numel() * dst.element_size() == nbytes
    return _check(load().ll_dbg_stream_copy(C.c_void_p(dst.data_ptr()), C.c_void_p(src.data_ptr()),
                                            C.c_size_t(nbytes)))


def ll_dbg_stream_read(src, reps=4):
    """GB/s of a read-only streaming pass over one contiguous CUDA tensor."""
    import torch
    sink = torch.zeros(4096, dtype=torch.int32, device=src.device)
    out = C.c_float(0.0)
    _check(load().ll_dbg_stream_read(C.c_void_p(src.data_ptr()), C.c_size_t(src.numel() * src.element_size()),
                                     reps, C.c_void_p(sink.data_ptr()), C.byref(out)))
    return float(out.value)


def ll_set_sampling_raw(temperature, top_k, top_p, seed):
    """ll_set_sampling on whatever instance the library holds (an error without one)."""
    return _check(load().ll_set_sampling(C.c_float(temperature), C.c_int32(top_k), C.c_float(top_p),
                                         C.c_uint64(seed)))


def ll_dbg_gemm_plan(N, K, nmat, rows):
    """Work distribution of the prefill projection GEMM (host arithmetic, no GPU needed)."""
    out = (C.c_int32 * 6)()
    _check(load().ll_dbg_gemm_plan(N, K, nmat, rows, out))
    return dict(zip(("row_tile", "row_tiles", "runs", "quota", "tile_slabs", "max_slices"), out))


def ll_dbg_tile_plan(kind, N, K, rows):
    """Tiles of a prefill projection that reads the weight copy (host arithmetic, no GPU needed)."""
    out = (C.c_int32 * 6)()
    _check(load().ll_dbg_tile_plan(kind, N, K, rows, out))
    return dict(zip(("row_tiles", "col_tiles", "blocks", "pieces", "stage_steps", "workgroups"), out))


def ll_dbg_batch_order(pos, active, per_round):
    """Slots in the order in which a batched step's attention takes them (host arithmetic, no GPU needed)."""
    n = len(pos)
    arr = C.c_int32 * n
    out = arr()
    _check(load().ll_dbg_batch_order(arr(*pos), arr(*active), n, per_round, out))
    return list(out)


def ll_dbg_small_plan(cfg, pos, steps, flags=0):
    """How a small model's decode steps run in one kernel (host arithmetic, no GPU needed)."""
    out = (C.c_int32 * 4)()
    _check(load().ll_dbg_small_plan(C.byref(make_config(cfg, flags)), pos, steps, out))
    return dict(zip(("workgroups", "first_pos", "greedy_keys", "sampled_keys"), out))


def ll_dbg_gemm_slice_count(N, K, nmat, rows, col):
    return _check(load().ll_dbg_gemm_slice_count(N, K, nmat, rows, col))


def ll_last_error():
    return load().ll_last_error().decode()


# ---- a key/value cache held in 4 bits ----

def ll_kv4_pool_bytes(n_kv_heads, head_dim, page_tokens, n_pages):
    """Bytes of one layer's pool (host arithmetic, no GPU needed); 0 for a shape that is not supported."""
    return int(load().ll_kv4_pool_bytes(C.byref(LLKV4Cache(None, 0, n_kv_heads, head_dim, page_tokens, n_pages))))


class KV4Cache:
    """One layer's pool, a contiguous uint8 CUDA tensor of ll_kv4_pool_bytes() bytes on a 256-byte border, and its shape."""

    def __init__(self, pool, n_kv_heads, head_dim, page_tokens, n_pages):
        if not pool.is_cuda or not pool.is_contiguous():
            raise ValueError("the pool must be a contiguous CUDA tensor")
        self.pool, self.n_kv_heads, self.head_dim = pool, n_kv_heads, head_dim
        self.device, self.index = pool.device, pool.get_device()
        self.c = LLKV4Cache(pool.data_ptr(), pool.numel() * pool.element_size(), n_kv_heads, head_dim, page_tokens, n_pages)


class KV4Rows:
    """Which rows a call has: int32 CUDA tensors ``lens`` [n_seqs], ``page_table`` [n_seqs, pages] and, unless every sequence
    has ``max_rows`` rows, ``row_start`` [n_seqs + 1]; see ll_kv4_rows in include/ll.h."""

    def __init__(self, lens, page_table, max_rows=1, row_start=None, max_len=0):
        import torch
        index, shape, int32 = lens.get_device(), page_table.shape, torch.int32
        for t in (lens, page_table) if row_start is None else (lens, page_table, row_start):
            if t.dtype is not int32 or not t.is_contiguous() or not t.is_cuda or t.get_device() != index:
                raise ValueError("lens, page_table and row_start must be contiguous int32 tensors of one CUDA device")
        n = lens.shape[0]
        if lens.dim() != 1 or len(shape) != 2 or shape[0] != n or (row_start is not None and row_start.shape != (n + 1,)):
            raise ValueError("lens [n_seqs], page_table [n_seqs, pages] and row_start [n_seqs + 1] do not fit together")
        self.lens, self.page_table, self.row_start, self.index = lens, page_table, row_start, index
        self.c = LLKV4Rows(None if row_start is None else row_start.data_ptr(), lens.data_ptr(), page_table.data_ptr(),
                           n, max_rows, 0, shape[1], max_len)


def _kv4_view(t, name, cache, heads, n_rows, dtype):
    shape, strides = t.shape, t.stride()
    if len(shape) != 3 or shape[0] != n_rows or shape[1] != heads or shape[2] != cache.head_dim:
        raise ValueError("%s must be [%d, %d, %d], is %s" % (name, n_rows, heads, cache.head_dim, list(shape)))
    if t.dtype is not dtype or strides[2] != 1 or t.get_device() != cache.index:
        raise ValueError("%s must be a %s tensor on the pool's device with a contiguous last dimension" % (name, dtype))
    return LLKV4View(t.data_ptr(), strides[0], strides[1])


def _kv4_enter(torch, cache, rows, n_rows, dtype, stream):
    """Checks of every call: the row type's code, the handle of the stream to work on, and what has to be entered for the call so
    that the pool's device and a given ``stream`` are torch's current ones (and own what the call allocates): None mostly."""
    if rows.index != cache.index:
        raise ValueError("lens and page_table must be on the pool's device")
    if dtype is not torch.float16 and dtype is not torch.bfloat16:
        raise ValueError("rows are float16 or bfloat16, not %s" % dtype)
    rows.c.n_rows = n_rows
    kind = LL_F16 if dtype is torch.float16 else LL_BF16
    if stream is not None:
        if stream.device.index != cache.index:
            raise ValueError("the stream must be one of the pool's device")
        return kind, stream.cuda_stream, torch.cuda.stream(stream)
    on = None if torch._C._cuda_getDevice() == cache.index else torch.cuda.device(cache.index)
    return kind, torch._C._cuda_getCurrentRawStream(cache.index), on


def ll_kv4_write(cache, rows, k, v, stream=None):
    """Quantises rows of k and v, [rows, n_kv_heads, head_dim] float16 or bfloat16, into the cache."""
    import torch
    n, dtype, heads = k.shape[0], k.dtype, cache.n_kv_heads
    kind, s, on = _kv4_enter(torch, cache, rows, n, dtype, stream)
    if on is not None:
        with on:
            return ll_kv4_write(cache, rows, k, v)
    rc = load().ll_kv4_write(cache.c, rows.c, kind, _kv4_view(k, "k", cache, heads, n, dtype), _kv4_view(v, "v", cache, heads, n, dtype), s)
    if rc < 0:
        _check(rc)


def ll_kv4_read(cache, rows, k=None, v=None, n_rows=0, dtype=None, stream=None):
    """The rows out of the cache into k and v, or into new tensors of n_rows rows."""
    import torch
    if k is not None:
        n_rows, dtype = k.shape[0], k.dtype
    kind, s, on = _kv4_enter(torch, cache, rows, n_rows, dtype, stream)
    if on is not None:
        with on:
            return ll_kv4_read(cache, rows, k, v, n_rows, dtype)
    heads = cache.n_kv_heads
    if k is None:
        k = torch.empty((n_rows, heads, cache.head_dim), dtype=dtype, device=cache.device)
        v = torch.empty_like(k)
    rc = load().ll_kv4_read(cache.c, rows.c, kind, _kv4_view(k, "k", cache, heads, n_rows, dtype),
                            _kv4_view(v, "v", cache, heads, n_rows, dtype), s)
    if rc < 0:
        _check(rc)
    return k, v


def ll_kv4_attention_workspace_bytes(cache, rows, n_heads, n_rows):
    """Bytes of workspace of such an attention call (host arithmetic)."""
    rows.c.n_rows = n_rows
    return load().ll_kv4_attention_workspace_bytes(cache.c, rows.c, n_heads)


def ll_kv4_attention(cache, rows, q, k=None, v=None, scale=0.0, out=None, workspace=None, stream=None):
    """Causal attention of rows q [rows, heads, head_dim] over the cache; k and v: these rows' own, written first.
    Without ``workspace`` (a CUDA tensor on a 256-byte border) the call takes one from torch's allocator where it needs any."""
    import torch
    shape, dtype = q.shape, q.dtype
    if len(shape) != 3:
        raise ValueError("q must be [rows, heads, %d]" % cache.head_dim)
    n, heads = shape[0], shape[1]
    kind, s, on = _kv4_enter(torch, cache, rows, n, dtype, stream)
    if on is not None:
        with on:
            return ll_kv4_attention(cache, rows, q, k, v, scale, out, workspace)
    qv = _kv4_view(q, "q", cache, heads, n, dtype)
    kv = None if k is None else _kv4_view(k, "k", cache, cache.n_kv_heads, n, dtype)
    vv = None if v is None else _kv4_view(v, "v", cache, cache.n_kv_heads, n, dtype)
    if out is None:
        out = q.new_empty(shape)
    ov = _kv4_view(out, "out", cache, heads, n, dtype)
    lib = load()
    if workspace is None:
        nbytes = lib.ll_kv4_attention_workspace_bytes(cache.c, rows.c, heads)
        if nbytes:
            workspace = torch.empty(nbytes, dtype=torch.uint8, device=cache.device)
    elif workspace.get_device() != cache.index or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous tensor on the pool's device")
    else:
        nbytes = workspace.numel() * workspace.element_size()
    rc = lib.ll_kv4_attention(cache.c, rows.c, kind, heads, scale, qv, kv, vv, ov, workspace.data_ptr() if nbytes else None, nbytes, s)
    if rc < 0:
        _check(rc)
    return out


class Session:
    """Owns the torch tensors the library points into, for the life of one ll_init()."""

    def __init__(self, cfg, weights, flags=0, stream=None, device="cuda:0"):
        """``weights``: dict of fp16 torch tensors on ``device`` (see workloads.weight_shapes)."""
        import torch
        self.torch = torch
        self.cfg = dict(cfg)
        self.lib = load()
        self.device = torch.device(device)
        self.stream = stream if stream is not None else torch.cuda.Stream(device=self.device)
        self._weights = weights
        for name, t in self._iter_weights(weights):
            if t.dtype != torch.float16 or not t.is_contiguous() or t.device.type != "cuda":
                raise ValueError("weight %s must be a contiguous fp16 CUDA tensor" % name)
        self._layers = (LLLayerWeights * cfg["n_layers"])()
        for i, Lw in enumerate(weights["layers"]):
            for k in LAYER_KEYS:
                setattr(self._layers[i], k, Lw[k].data_ptr())
        self._w = LLWeights(tok_emb=weights["tok_emb"].data_ptr(),
                            layers=C.cast(self._layers, C.POINTER(LLLayerWeights)),
                            final_norm=weights["final_norm"].data_ptr(),
                            lm_head=weights["lm_head"].data_ptr())
        self._cfg = make_config(cfg, flags)
        nbytes = int(self.lib.ll_workspace_bytes(C.byref(self._cfg)))
        if nbytes == 0:
            raise LLError(LL_E_BAD_CONFIG, "ll_workspace_bytes rejected the configuration")
        self.workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
        base = self.workspace.data_ptr()
        self._ws_ptr = (base + 255) // 256 * 256
        torch.cuda.synchronize(self.device)
        _check(self.lib.ll_init(C.byref(self._cfg), C.byref(self._w), C.c_void_p(self._ws_ptr),
                                C.c_size_t(nbytes), C.c_void_p(self.stream.cuda_stream)))
        self.open = True

    @staticmethod
    def _iter_weights(w):
        for k, v in w.items():
            if k == "layers":
                for i, Lw in enumerate(v):
                    for kk, vv in Lw.items():
                        yield "layers[%d].%s" % (i, kk), vv
            else:
                yield k, v

    # ---- the four calls ------------------------------------------------
    def ll_prefill(self, tokens):
        arr = np.ascontiguousarray(tokens, dtype=np.int32)
        return _check(self.lib.ll_prefill(arr.ctypes.data_as(C.POINTER(C.c_int32)), arr.shape[0]))

    def ll_prefill_static(self, tokens):
        arr = np.ascontiguousarray(tokens, dtype=np.int32)
        return _check(self.lib.ll_prefill_static(arr.ctypes.data_as(C.POINTER(C.c_int32)), arr.shape[0]))

    def ll_decode_step(self):
        return _check(self.lib.ll_decode_step())

    def ll_decode_n(self, k):
        out = np.empty(k, dtype=np.int32)
        _check(self.lib.ll_decode_n(k, out.ctypes.data_as(C.POINTER(C.c_int32))))
        return out

    def ll_reset(self):
        return _check(self.lib.ll_reset())

    def ll_set_sampling(self, temperature, top_k=0, top_p=1.0, seed=0):
        return ll_set_sampling_raw(temperature, top_k, top_p, seed)

    def ll_shutdown(self):
        if self.open:
            self.open = False
            rc = _check(self.lib.ll_shutdown())
            self.workspace = None          # the library is done with it
            self.pool = None
            return rc
        return 0

    close = ll_shutdown

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def ll_max_prompt(self):
        return _check(self.lib.ll_max_prompt())

    def ll_decode_mode(self):
        return _check(self.lib.ll_decode_mode())

    def ll_position(self):
        return _check(self.lib.ll_position())

    # ---- hooks ---------------------------------------------------------
    def ll_dbg_get_logits(self):
        out = np.empty(self.cfg["vocab"], dtype=np.float32)
        _check(self.lib.ll_dbg_get_logits(out.ctypes.data_as(C.POINTER(C.c_float))))
        return out

    # ---- batched decoding over a paged KV cache ----
    def ll_batch_open(self, max_batch, page_tokens, n_pages, kv_bits=16):
        """kv_bits: what an element of the paged cache is held in, 16 or 4 (see ll_batch_open_kv)."""
        nbytes = int(self.lib.ll_batch_pool_bytes_kv(page_tokens, n_pages, kv_bits))
        if nbytes == 0:
            raise LLError(LL_E_BAD_ARG, "ll_batch_pool_bytes rejected the arguments")
        self.pool = self.torch.empty(nbytes + 256, dtype=self.torch.uint8, device=self.device)
        ptr = (self.pool.data_ptr() + 255) // 256 * 256
        self.max_batch = max_batch
        return _check(self.lib.ll_batch_open_kv(max_batch, page_tokens, n_pages, kv_bits, C.c_void_p(ptr), C.c_size_t(nbytes)))

    def ll_batch_add(self, tokens):
        arr = (C.c_int32 * len(tokens))(*[int(t) for t in tokens])
        first = C.c_int32(-1)
        slot = _check(self.lib.ll_batch_add(arr, len(tokens), C.byref(first)))
        return slot, int(first.value)

    def ll_batch_step(self):
        out = (C.c_int32 * self.max_batch)()
        _check(self.lib.ll_batch_step(out))
        return list(out)

    def ll_batch_remove(self, slot):
        return _check(self.lib.ll_batch_remove(slot))

    def ll_batch_close(self):
        rc = _check(self.lib.ll_batch_close())
        self.pool = None
        return rc

    def ll_batch_dbg_get_logits(self, slot):
        out = np.empty(self.cfg["vocab"], dtype=np.float32)
        _check(self.lib.ll_batch_dbg_get_logits(slot, out.ctypes.data_as(C.POINTER(C.c_float))))
        return out

    def ll_batch_dbg_get_kv(self, slot, layer, which, n_pos):
        out = np.empty((n_pos, self.cfg["d_model"]), dtype=np.float32)
        _check(self.lib.ll_batch_dbg_get_kv(slot, layer, which, n_pos, out.ctypes.data_as(C.POINTER(C.c_float))))
        return out

    def ll_batch_dbg_force_next_token(self, slot, tok):
        return _check(self.lib.ll_batch_dbg_force_next_token(slot, int(tok)))

    def ll_batch_dbg_time_steps(self, k):
        ms = C.c_float(0)
        _check(self.lib.ll_batch_dbg_time_steps(k, C.byref(ms)))
        return float(ms.value)

    def ll_dbg_set_spin_limit(self, polls):
        return bool(_check(self.lib.ll_dbg_set_spin_limit(polls)))

    def ll_dbg_give_up_at(self, token):
        return bool(_check(self.lib.ll_dbg_give_up_at(token)))

    def ll_dbg_graph_stats(self):
        out = (C.c_int64 * 4)()
        _check(self.lib.ll_dbg_graph_stats(out))
        return dict(buffered_replays=out[0], blocking_captures=out[1], overlapped_captures=out[2],
                    capture_ms=out[3] / 1e6)

    def ll_dbg_get_hidden(self):
        out = np.empty(self.cfg["d_model"], dtype=np.float32)
        _check(self.lib.ll_dbg_get_hidden(out.ctypes.data_as(C.POINTER(C.c_float))))
        return out

    def ll_dbg_poison_scratch(self):
        return _check(self.lib.ll_dbg_poison_scratch())

    def ll_dbg_force_next_token(self, tok):
        return _check(self.lib.ll_dbg_force_next_token(int(tok)))

    def ll_dbg_get_kv(self, layer, which, n_pos):
        out = np.empty((n_pos, self.cfg["d_model"]), dtype=np.float32)
        _check(self.lib.ll_dbg_get_kv(layer, which, n_pos, out.ctypes.data_as(C.POINTER(C.c_float))))
        return out

    def ll_dbg_profile_decode(self, steps):
        us = np.zeros(len(KERNEL_CLASSES), dtype=np.float32)
        n = np.zeros(len(KERNEL_CLASSES), dtype=np.int32)
        _check(self.lib.ll_dbg_profile_decode(steps, us.ctypes.data_as(C.POINTER(C.c_float)),
                                              n.ctypes.data_as(C.POINTER(C.c_int32))))
        return {k: (float(us[i]), int(n[i])) for i, k in enumerate(KERNEL_CLASSES)}

    def ll_dbg_time_kernel_class(self, name, reps):
        us = C.c_float(0.0)
        _check(self.lib.ll_dbg_time_kernel_class(KERNEL_CLASSES.index(name), reps, C.byref(us)))
        return float(us.value)

    def ll_dbg_trace_decode(self):
        """[phases][5] timestamps in microseconds relative to the first one."""
        n = 5 * self.cfg["n_layers"] + 1
        buf = np.zeros((n, 8), dtype=np.uint64)
        _check(self.lib.ll_dbg_trace_decode(buf.ctypes.data_as(C.POINTER(C.c_uint64)), n))
        return (buf.astype(np.int64) - np.int64(buf[0, 0])) / 100.0

    def ll_dbg_time_decode(self, k):
        ms = C.c_float(0.0)
        _check(self.lib.ll_dbg_time_decode(k, C.byref(ms)))
        return float(ms.value)
