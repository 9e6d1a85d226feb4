"""ctypes binding of libst3.so: argument marshalling only, one Python function per C entry point.

Every step of the method runs inside the library's CUDA kernels; torch is used by callers for
device memory and streams, never for the computation.  There is no CPU fallback: if the shared
library is missing or does not load, `load()` raises.
"""
from __future__ import annotations

import ctypes as C
import functools
import os

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libst3.so")

ST3_OK = 0
STATUS_NAMES = ["ST3_OK", "ST3_ERR_INVALID_ARG", "ST3_ERR_WORKSPACE_TOO_SMALL", "ST3_ERR_BAD_STATE",
                "ST3_ERR_CAPACITY", "ST3_ERR_CUDA", "ST3_ERR_DEVICE_CHECK", "ST3_ERR_UNSUPPORTED"]
ST3_F32, ST3_BF16 = 0, 1
ST3_ANNEAL_COSINE, ST3_ANNEAL_NONE, ST3_ANNEAL_LINEAR, ST3_ANNEAL_EXP = 0, 1, 2, 3
DEV_COUNT_MISMATCH, DEV_NONFINITE, DEV_COPY_TIMEOUT, DEV_RANGE = 1, 2, 4, 8

EXPORTS = ["st3_schedule_count", "st3_workspace_size", "st3_create", "st3_prefill_select",
           "st3_prefill_select_scored", "st3_decode_step",
           "st3_decode_step_host", "st3_prefill_select_host", "st3_host_sync", "st3_get_kept", "st3_get_rows", "st3_get_status", "st3_rows_held",
           "st3_set_overlap", "st3_profile_enable", "st3_profile_read", "st3_launch_count", "st3_status_string", "st3_destroy",
           "st3_attend_noalloc", "st3_prefill_attend", "st3_prefill_attend_kept",
           "st3_packed_attend", "st3_packed_weights", "st3_cache_store", "st3_cache_attend_workspace", "st3_cache_attend", "st3_cache_evict_workspace",
           "st3_cache_evict", "st3_cache_rows"]


class Config(C.Structure):
    """Mirror of `st3_config` (include/st3.h)."""
    _fields_ = [(n, C.c_int32) for n in (
        "num_layers", "num_heads", "head_dim", "dtype", "batch", "sys_len", "num_visual", "max_text_len",
        "max_decode_steps", "first_prune_layer", "stride", "first_ratio_bp", "step_ratio_bp", "anneal",
        "disable_trim", "rows_per_chunk", "static_rank", "stage_shared", "host_prefill")] + [("lazy_mask", C.c_uint64), ("tau", C.c_double), ("sigma", C.c_double)]


class PackedDesc(C.Structure):
    """Mirror of `st3_packed` (include/st3.h)."""
    _fields_ = [(n, C.c_int32) for n in ("num_seqs", "total", "num_heads", "num_kv_heads", "head_dim", "dtype")] + [
        (f"{t}_{n}_stride", C.c_int64) for t in ("q", "k", "v", "out") for n in ("token", "head")]


class CacheDesc(C.Structure):
    """Mirror of `st3_cache` (include/st3.h)."""
    _fields_ = [(n, C.c_int32) for n in ("batch", "num_kv_heads", "head_dim", "capacity")] + [
        (n, C.c_void_p) for n in ("k", "v", "k_scale", "v_scale", "ids", "weights")]


class St3Error(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        name = STATUS_NAMES[code] if 0 <= code < len(STATUS_NAMES) else str(code)
        super().__init__(f"{where}: {name}")


_lib = None


def load():
    """Loads libst3.so (once) and declares the prototypes.  Raises if it is not there."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it first (python -m paper_2412_20105_b200.build); "
                           "there is no fallback path")
    lib = C.CDLL(LIB_PATH)
    vp, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
    cfgp = C.POINTER(Config)
    lib.st3_schedule_count.argtypes = [cfgp, i32, i32]
    lib.st3_schedule_count.restype = i32
    lib.st3_workspace_size.argtypes = [cfgp, C.POINTER(C.c_size_t)]
    lib.st3_create.argtypes = [cfgp, vp, C.c_size_t, C.POINTER(vp)]
    lib.st3_prefill_select.argtypes = [vp, i32, i32, vp, vp, vp, C.POINTER(i32), vp, vp]
    lib.st3_prefill_select_scored.argtypes = [vp, i32, i32, vp, vp, vp, C.POINTER(i32), vp, vp, vp]
    lib.st3_decode_step.argtypes = [vp, i32, i32, i32, vp, vp, vp, vp, vp]
    lib.st3_decode_step_host.argtypes = [vp, i32, i32, i32, vp, vp, vp, vp, vp]
    lib.st3_prefill_select_host.argtypes = [vp, i32, i32, vp, vp, vp, C.POINTER(i32), vp, vp]
    lib.st3_host_sync.argtypes = [vp, vp]
    lib.st3_get_kept.argtypes = [vp, i32, vp, vp, vp, vp]
    lib.st3_get_rows.argtypes = [vp, i32, i32, i32, vp, vp, vp, vp, vp]
    lib.st3_get_status.argtypes = [vp, C.POINTER(i32)]
    lib.st3_rows_held.argtypes = [vp, C.POINTER(i64), C.POINTER(i64)]
    lib.st3_set_overlap.argtypes = [vp, i32]
    lib.st3_profile_enable.argtypes = [vp, i32]
    lib.st3_profile_read.argtypes = [vp, C.POINTER(C.c_double), C.POINTER(C.c_double), C.POINTER(i64),
                                     C.POINTER(i64)]
    lib.st3_launch_count.argtypes = [vp]
    lib.st3_launch_count.restype = i64
    lib.st3_status_string.argtypes = [C.c_int]
    lib.st3_status_string.restype = C.c_char_p
    lib.st3_destroy.argtypes = [vp]
    lib.st3_attend_noalloc.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, vp]
    lib.st3_prefill_attend.argtypes = [vp, vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, i32, vp]
    lib.st3_prefill_attend_kept.argtypes = [vp, vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, i32, vp, i32, vp]
    cp, szp = C.POINTER(CacheDesc), C.POINTER(C.c_size_t)
    pp = C.POINTER(PackedDesc)
    lib.st3_packed_attend.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.st3_packed_weights.argtypes = [pp, vp, vp, vp, vp, vp, i32, i32, vp, vp]
    lib.st3_cache_store.argtypes = [cp, vp, vp, i32, i64, i64, i64, i64, vp, i32, vp, vp, vp, vp]
    lib.st3_cache_attend_workspace.argtypes = [cp, i32, i32, szp]
    lib.st3_cache_attend.argtypes = [cp, vp, vp, i32, i32, vp, vp, vp, vp, C.c_size_t, vp, vp]
    lib.st3_cache_evict_workspace.argtypes = [cp, szp]
    lib.st3_cache_evict.argtypes = [cp, cp, vp, vp, i32, i32, vp, vp, C.c_size_t, vp, vp]
    lib.st3_cache_rows.argtypes = [cp, vp, vp, i32, vp, vp, i32, vp, vp, vp]
    for name in EXPORTS:
        if name not in ("st3_schedule_count", "st3_launch_count", "st3_status_string"):
            getattr(lib, name).restype = C.c_int
    _lib = lib
    return lib


def _check(code: int, where: str):
    if code != ST3_OK:
        raise St3Error(code, where)


def make_config(*, num_layers, num_heads, head_dim, dtype, batch, sys_len, num_visual, max_text_len,
                max_decode_steps, stride, step_ratio_bp, tau, first_prune_layer=3, first_ratio_bp=5000,
                anneal=ST3_ANNEAL_COSINE, disable_trim=0, rows_per_chunk=0, sigma=20.0, static_rank=0, stage_shared=0, lazy_mask=0,
                host_prefill=0) -> Config:
    dt = {"f32": ST3_F32, "bf16": ST3_BF16}.get(dtype, dtype)
    return Config(num_layers, num_heads, head_dim, dt, batch, sys_len, num_visual, max_text_len,
                  max_decode_steps, first_prune_layer, stride, first_ratio_bp, step_ratio_bp, anneal,
                  int(disable_trim), rows_per_chunk, int(static_rank), int(stage_shared), int(host_prefill), int(lazy_mask),
                  float(tau), float(sigma))


def st3_schedule_count(cfg: Config, layer: int, step: int) -> int:
    return load().st3_schedule_count(C.byref(cfg), layer, step)


def st3_workspace_size(cfg: Config) -> int:
    n = C.c_size_t(0)
    _check(load().st3_workspace_size(C.byref(cfg), C.byref(n)), "st3_workspace_size")
    return n.value


def st3_create(cfg: Config, workspace_ptr: int, nbytes: int) -> int:
    h = C.c_void_p(None)
    _check(load().st3_create(C.byref(cfg), workspace_ptr, nbytes, C.byref(h)), "st3_create")
    return h.value


def st3_prefill_select(ctx, layer_begin, layer_count, q_last, k, v, text_len, out, stream=0):
    """q_last/k/v/out are device addresses (ints); text_len is a host sequence of ints."""
    arr = (C.c_int32 * len(text_len))(*[int(x) for x in text_len])
    _check(load().st3_prefill_select(ctx, layer_begin, layer_count, q_last, k, v, arr, out, stream),
           "st3_prefill_select")


def st3_prefill_select_scored(ctx, layer_begin, layer_count, q_last, k, v, text_len, scores, out, stream=0):
    """As st3_prefill_select, but the kept set comes from `scores` (device address, fp32
    [layer_count][B][num_visual]) and the layer attends over the kept rows only."""
    arr = (C.c_int32 * len(text_len))(*[int(x) for x in text_len])
    _check(load().st3_prefill_select_scored(ctx, layer_begin, layer_count, q_last, k, v, arr, scores, out, stream),
           "st3_prefill_select_scored")


def st3_decode_step(ctx, step, layer_begin, layer_count, q, k_new, v_new, out, stream=0):
    _check(load().st3_decode_step(ctx, step, layer_begin, layer_count, q, k_new, v_new, out, stream),
           "st3_decode_step")


def st3_decode_step_host(ctx, step, layer_begin, layer_count, q, k_new, v_new, out, stream=0):
    _check(load().st3_decode_step_host(ctx, step, layer_begin, layer_count, q, k_new, v_new, out, stream),
           "st3_decode_step_host")


def st3_prefill_select_host(ctx, layer_begin, layer_count, q_last, k, v, text_len, out, stream=0):
    """As st3_prefill_select with pinned HOST addresses; needs a config with host_prefill=1."""
    arr = (C.c_int32 * len(text_len))(*[int(x) for x in text_len])
    _check(load().st3_prefill_select_host(ctx, layer_begin, layer_count, q_last, k, v, arr, out, stream),
           "st3_prefill_select_host")


def st3_host_sync(ctx, stream=0):
    _check(load().st3_host_sync(ctx, stream), "st3_host_sync")


def st3_get_kept(ctx, layer, ids, count, mass=None, stream=0):
    _check(load().st3_get_kept(ctx, layer, ids, count, mass, stream), "st3_get_kept")


def st3_get_rows(ctx, layer, b, h, k_vis=None, v_vis=None, k_txt=None, v_txt=None, stream=0):
    _check(load().st3_get_rows(ctx, layer, b, h, k_vis, v_vis, k_txt, v_txt, stream), "st3_get_rows")


def st3_get_status(ctx, raise_on_error=True) -> int:
    w = C.c_int32(0)
    code = load().st3_get_status(ctx, C.byref(w))
    if raise_on_error and code != ST3_OK:
        raise St3Error(code, f"st3_get_status (device word {w.value})")
    return w.value


def st3_rows_held(ctx):
    a, b = C.c_int64(0), C.c_int64(0)
    _check(load().st3_rows_held(ctx, C.byref(a), C.byref(b)), "st3_rows_held")
    return a.value, b.value


def st3_set_overlap(ctx, on: bool):
    _check(load().st3_set_overlap(ctx, int(on)), "st3_set_overlap")


def st3_profile_enable(ctx, on: bool):
    _check(load().st3_profile_enable(ctx, int(on)), "st3_profile_enable")


def st3_profile_read(ctx):
    a, f = C.c_double(0), C.c_double(0)
    na, nf = C.c_int64(0), C.c_int64(0)
    _check(load().st3_profile_read(ctx, C.byref(a), C.byref(f), C.byref(na), C.byref(nf)), "st3_profile_read")
    return a.value, f.value, na.value, nf.value


def st3_launch_count(ctx) -> int:
    return load().st3_launch_count(ctx)


def st3_status_string(code: int) -> str:
    return load().st3_status_string(code).decode()


def st3_destroy(ctx):
    _check(load().st3_destroy(ctx), "st3_destroy")


def st3_prefill_attend(q, k, v, out, head_probs, scores, dev_status, num_inst, num_heads, seq_len, head_dim, dtype,
                       sys_len, num_visual, stream=0):
    """Causal attention of a whole prompt on the tensor cores (device addresses; see st3.h)."""
    dt = {"f32": ST3_F32, "bf16": ST3_BF16}.get(dtype, dtype)
    _check(load().st3_prefill_attend(q, k, v, out, head_probs, scores, dev_status, num_inst, num_heads, seq_len,
                                     head_dim, dt, sys_len, num_visual, stream), "st3_prefill_attend")


def st3_prefill_attend_kept(q, k, v, out, head_probs, scores, dev_status, num_inst, num_heads, seq_len, head_dim,
                            dtype, sys_len, num_visual, ids, num_visual_total, stream=0):
    """The same for a prompt that holds only the visual tokens `ids` names; scores come out by original index."""
    dt = {"f32": ST3_F32, "bf16": ST3_BF16}.get(dtype, dtype)
    _check(load().st3_prefill_attend_kept(q, k, v, out, head_probs, scores, dev_status, num_inst, num_heads, seq_len,
                                          head_dim, dt, sys_len, num_visual, ids, num_visual_total, stream),
           "st3_prefill_attend_kept")


def st3_attend_noalloc(q, k, v, out, num_heads, num_rows, head_dim, dtype, stream=0):
    """Workspace-free attention for callers that may not allocate device memory: q/k/v/out are
    device addresses, the split partials live in a fixed array inside the library (see st3.h for
    the size limit and the sharing rules)."""
    dt = {"f32": ST3_F32, "bf16": ST3_BF16}.get(dtype, dtype)
    _check(load().st3_attend_noalloc(q, k, v, out, num_heads, num_rows, head_dim, dt, stream), "st3_attend_noalloc")


def st3_packed_attend(desc, q, k, v, cu, out, lse=None, dev_status=None, stream=0):
    """desc is a PackedDesc; the rest device addresses."""
    _check(load().st3_packed_attend(C.byref(desc), q, k, v, cu, out, lse, dev_status, stream), "st3_packed_attend")


def st3_packed_weights(desc, q, k, lse, cu, weights, capacity, window=0, dev_status=None, stream=0):
    _check(load().st3_packed_weights(C.byref(desc), q, k, lse, cu, weights, capacity, window, dev_status, stream),
           "st3_packed_weights")


def st3_cache_store(cache, k, v, dtype, k_strides, v_strides, cu, total, start=None, pos=None, dev_status=None, stream=0):
    """cache is a CacheDesc; k_strides and v_strides are (token, head) strides in elements; the rest device addresses."""
    _check(load().st3_cache_store(C.byref(cache), k, v, dtype, *k_strides, *v_strides, cu, total, start, pos, dev_status,
                                  stream), "st3_cache_store")


def st3_cache_attend_workspace(cache, num_heads, with_weights) -> int:
    n = C.c_size_t(0)
    _check(load().st3_cache_attend_workspace(C.byref(cache), num_heads, int(with_weights), C.byref(n)),
           "st3_cache_attend_workspace")
    return n.value


def st3_cache_attend(cache, q, out, dtype, num_heads, held, weights_in, weights_out, workspace, nbytes, dev_status=None,
                     stream=0):
    _check(load().st3_cache_attend(C.byref(cache), q, out, dtype, num_heads, held, weights_in, weights_out, workspace,
                                   nbytes, dev_status, stream), "st3_cache_attend")


def st3_cache_evict_workspace(cache) -> int:
    n = C.c_size_t(0)
    _check(load().st3_cache_evict_workspace(C.byref(cache), C.byref(n)), "st3_cache_evict_workspace")
    return n.value


def st3_cache_evict(cache, to, held, seen, keep, recent, held_out, workspace, nbytes, dev_status=None, stream=0):
    _check(load().st3_cache_evict(C.byref(cache), C.byref(to), held, seen, keep, recent, held_out, workspace, nbytes,
                                  dev_status, stream), "st3_cache_evict")


def st3_cache_rows(cache, first, held, num_rows, k, v, dtype, ids, weights, stream=0):
    _check(load().st3_cache_rows(C.byref(cache), first, held, num_rows, k, v, dtype, ids, weights, stream),
           "st3_cache_rows")


_DTYPES = {}     # torch dtype -> st3_dtype


def _dtype_of(t) -> int:
    if not _DTYPES:
        import torch
        _DTYPES.update({torch.bfloat16: ST3_BF16, torch.float32: ST3_F32})
    if t.dtype not in _DTYPES:
        raise TypeError(f"bfloat16 or float32 is needed, not {t.dtype}")
    return _DTYPES[t.dtype]


def _stream_of(index: int) -> int:
    """The current stream of that device, which has to be the current one."""
    import torch
    try:   # without the public functions around them (a Stream object alone takes 2.2 us a call), where torch offers that
        current, stream = torch._C._cuda_getDevice(), torch._C._cuda_getCurrentRawStream
    except AttributeError:
        current, stream = torch.cuda.current_device(), lambda i: torch.cuda.current_stream(i).cuda_stream
    if index != current:
        raise ValueError(f"the tensors are on cuda:{index}, the current device is cuda:{current}")
    return stream(index)


def _int32(x, what):
    """x, which ctypes would cut to its low 32 bits."""
    if not -2 ** 31 <= x < 2 ** 31:
        raise ValueError(f"{what}: {x} does not fit into 32 bits")
    return x


def _dense(t, shape, dtype, index, what):
    """Address of a dense tensor on CUDA device `index`."""
    if t.shape == shape and t.dtype is dtype and t.is_contiguous() and t.get_device() == index:
        return t.data_ptr()
    raise ValueError(f"{what}: a contiguous {dtype} tensor of {tuple(shape)} on cuda:{index} is needed, "
                     f"not {t.dtype} {tuple(t.shape)} on {t.device}")


def _rows_view(t, heads, dim, dtype, index, what):
    """Address and (token, head) strides of a [tokens, heads, dim] tensor whose last dimension is dense."""
    shape = t.shape
    if len(shape) != 3 or shape[1] != heads or shape[2] != dim or t.dtype is not dtype or t.get_device() != index:
        raise ValueError(f"{what}: a {dtype} tensor of [tokens, {heads}, {dim}] on cuda:{index} is needed, "
                         f"not {t.dtype} {tuple(shape)} on {t.device}")
    token, head, one = t.stride()
    if one != 1:
        raise ValueError(f"{what}: the elements of a head have to lie side by side")
    return t.data_ptr(), token, head


def _packed_shape(q, k):
    """(total, heads, kv heads, dim, device index) of packed queries and keys."""
    if q.dim() != 3 or k.dim() != 3 or not q.is_cuda:
        raise ValueError("q and k: CUDA tensors of [tokens, heads, dim] are needed")
    total, heads, dim = q.shape
    if k.shape[0] != total:
        raise ValueError("q and k have different numbers of tokens")
    return total, heads, k.shape[1], dim, q.get_device()


def _starts_of(cu, index):
    import torch
    if cu.dim() != 1 or cu.numel() < 1:
        raise ValueError("cu: [sequences + 1] is needed")
    return _dense(cu, cu.shape, torch.int32, index, "cu")


def packed_attend(q, k, v, cu, out, lse=None, status=None):
    """Causal attention of packed prompts: q, out [tokens, heads, dim], k, v [tokens, kv heads, dim], lse [heads, tokens]."""
    import torch
    total, heads, kv, dim, index = _packed_shape(q, k)
    dtype = q.dtype
    qp, *qs = _rows_view(q, heads, dim, dtype, index, "q")
    kp, *ks = _rows_view(k, kv, dim, dtype, index, "k")
    vp, *vs = _rows_view(v, kv, dim, dtype, index, "v")
    op, *os_ = _rows_view(out, heads, dim, dtype, index, "out")
    if v.shape[0] != total or out.shape[0] != total:
        raise ValueError("q, v and out have different numbers of tokens")
    cup = _starts_of(cu, index)
    desc = PackedDesc(cu.numel() - 1, total, heads, kv, dim, _dtype_of(q), *qs, *ks, *vs, *os_)
    st3_packed_attend(desc, qp, kp, vp, cup, op,
                      None if lse is None else _dense(lse, (heads, total), torch.float32, index, "lse"),
                      None if status is None else _dense(status, (1,), torch.int32, index, "status"), _stream_of(index))


def packed_weights(q, k, lse, cu, weights, window=0, status=None):
    """What each token has received from all queries, or from the last `window`: weights [sequences, kv heads, capacity]."""
    import torch
    total, heads, kv, dim, index = _packed_shape(q, k)
    qp, *qs = _rows_view(q, heads, dim, q.dtype, index, "q")
    kp, *ks = _rows_view(k, kv, dim, q.dtype, index, "k")
    cup = _starts_of(cu, index)
    if weights.dim() != 3:
        raise ValueError("weights: [sequences, kv heads, capacity] is needed")
    seqs, capacity = cu.numel() - 1, weights.shape[2]
    desc = PackedDesc(seqs, total, heads, kv, dim, _dtype_of(q), *qs, *ks, *ks, *qs)
    st3_packed_weights(desc, qp, kp, _dense(lse, (heads, total), torch.float32, index, "lse"), cup,
                       _dense(weights, (seqs, kv, capacity), torch.float32, index, "weights"), capacity, _int32(window, "window"),
                       None if status is None else _dense(status, (1,), torch.int32, index, "status"), _stream_of(index))


class Cache:
    """One layer's cache of grouped heads held in 8 bits (st3_cache), over tensors of the caller's or its own.

    `Cache(k, v, k_scale, v_scale, ids, weights)` wraps existing tensors, `Cache.empty(...)` allocates them.  `status` is
    the device status word that the calls report into.  How many rows each sequence holds is the caller's to keep: an
    int32 tensor [batch] that goes into the calls.  The workspaces are kept between calls (one for each number of query
    heads, with and without weights, and one for evictions): use a Cache on one stream at a time, order replays of
    graphs that hold its calls against them and each other, and keep it as long as such graphs, or calls on another
    stream than it was made on, may run."""

    def __init__(self, k, v, k_scale, v_scale, ids, weights):
        import torch
        n, heads, cap, dim = k.shape
        if not k.is_cuda:
            raise ValueError("a CUDA device is required: this library has no CPU path")
        self.torch, self.device = torch, k.device
        index = self._index = k.get_device()
        self.k, self.v, self.k_scale, self.v_scale, self.ids, self.weights = k, v, k_scale, v_scale, ids, weights
        codes, blocks = (n, heads, cap, dim), (n, heads, cap // 64)
        f32, i32 = torch.float32, torch.int32
        self.desc = CacheDesc(n, heads, dim, cap, _dense(k, codes, torch.int8, index, "k"),
                              _dense(v, codes, torch.int8, index, "v"), _dense(k_scale, blocks, f32, index, "k_scale"),
                              _dense(v_scale, blocks, f32, index, "v_scale"), _dense(ids, codes[:3], i32, index, "ids"),
                              _dense(weights, codes[:3], f32, index, "weights"))
        self.batch, self.num_kv_heads, self.capacity, self.head_dim = n, heads, cap, dim
        self.status = torch.zeros(1, dtype=i32, device=k.device)
        self._workspaces = {}     # what for -> (tensor, address, bytes); never let go, as a captured graph may hold its address

    @classmethod
    def empty(cls, batch, num_kv_heads, head_dim, capacity, device="cuda:0"):
        import torch
        if not torch.cuda.is_available():
            raise RuntimeError("a CUDA device is required: this library has no CPU path")
        cap = (capacity + 63) // 64 * 64
        new = functools.partial(torch.empty, device=device)
        codes = (batch, num_kv_heads, cap, head_dim)
        return cls(new(codes, dtype=torch.int8), new(codes, dtype=torch.int8), new(*codes[:2], cap // 64),
                   new(*codes[:2], cap // 64), new(codes[:3], dtype=torch.int32), new(codes[:3]))

    def _count(self, t, what):
        return None if t is None else _dense(t, (self.batch,), self.torch.int32, self._index, what)

    def _workspace(self, key, size):
        if key not in self._workspaces:
            nbytes = size()
            ws = self.torch.empty(nbytes + 256, dtype=self.torch.uint8, device=self.device)
            self._workspaces[key] = ws, (ws.data_ptr() + 255) // 256 * 256, nbytes
        return self._workspaces[key][1:]

    def store(self, k, v, cu, start=None, pos=None):
        """Rows cu[s] .. cu[s+1]-1 of k and v ([tokens, kv heads, dim]) go behind the start[s] rows of sequence s."""
        dt = _dtype_of(k)
        kp, *ks = _rows_view(k, self.num_kv_heads, self.head_dim, k.dtype, self._index, "k")
        vp, *vs = _rows_view(v, self.num_kv_heads, self.head_dim, k.dtype, self._index, "v")
        if v.shape[0] != k.shape[0]:
            raise ValueError("k and v have different numbers of rows")
        st3_cache_store(self.desc, kp, vp, dt, ks, vs, _dense(cu, (self.batch + 1,), self.torch.int32, self._index, "cu"),
                        k.shape[0], self._count(start, "start"), self._count(pos, "pos"), self.status.data_ptr(),
                        _stream_of(self._index))

    def attend(self, q, held, out, weights_out=None, weights_in=None):
        """q and out [batch, heads, dim]; weights_out (e.g. this cache's `weights`) gets weights_in (None: this cache's)
        plus the probabilities."""
        heads, dt = q.shape[1], _dtype_of(q)
        shape = (self.batch, heads, self.head_dim)
        wi = wo = None
        if weights_out is not None:
            wi = _dense(self.weights if weights_in is None else weights_in, self.weights.shape, self.torch.float32, self._index, "weights_in")
            wo = _dense(weights_out, self.weights.shape, self.torch.float32, self._index, "weights_out")
        key = (heads, wo is not None)
        ws, nbytes = self._workspace(key, lambda: st3_cache_attend_workspace(self.desc, *key))
        st3_cache_attend(self.desc, _dense(q, shape, q.dtype, self._index, "q"), _dense(out, shape, q.dtype, self._index, "out"),
                         dt, heads, self._count(held, "held"), wi, wo, ws, nbytes, self.status.data_ptr(), _stream_of(self._index))

    def evict(self, held, seen, keep, recent=0, into=None, held_out=None):
        """Cuts every head to `keep` rows, in place or into another Cache; returns the new numbers of rows held."""
        to = self if into is None else into
        if to._index != self._index:
            raise ValueError(f"the target is on cuda:{to._index}, the cache on cuda:{self._index}")
        keep, recent = _int32(keep, "keep"), _int32(recent, "recent")
        if held_out is None:
            held_out = self.torch.empty_like(held)
        ws, nbytes = self._workspace("evict", lambda: st3_cache_evict_workspace(self.desc))
        st3_cache_evict(self.desc, to.desc, self._count(held, "held"), self._count(seen, "seen"), keep, recent,
                        self._count(held_out, "held_out"), ws, nbytes, self.status.data_ptr(), _stream_of(self._index))
        return held_out

    def rows(self, held, num_rows, first=None, dtype=None):
        """(k, v, ids, weights) of rows first[s] .. first[s] + num_rows - 1 as values; rows that are not held read as 0."""
        t = self.torch
        shape = (self.batch, self.num_kv_heads, num_rows)
        like = self.weights.new_empty
        k, v = like((2,) + shape + (self.head_dim,), dtype=dtype or t.bfloat16).unbind(0)
        ids, weights = self.ids.new_empty(shape), like(shape)
        st3_cache_rows(self.desc, self._count(first, "first"), self._count(held, "held"), num_rows, k.data_ptr(),
                       v.data_ptr(), _dtype_of(k), ids.data_ptr(), weights.data_ptr(), _stream_of(self._index))
        return k, v, ids, weights


class Context:
    """Owns a torch-allocated workspace and a library context; forwards to the C entry points.

    Torch supplies device memory and the current stream only.  Tensors passed in must be CUDA,
    contiguous and of the configured dtype.
    """

    def __init__(self, cfg: Config, device="cuda:0"):
        import torch
        if not torch.cuda.is_available():
            raise RuntimeError("a CUDA device is required: this library has no CPU path")
        self._decode_step = load().st3_decode_step
        self.torch = torch
        self.cfg = cfg
        self.device = torch.device(device)
        self.dtype = torch.bfloat16 if cfg.dtype == ST3_BF16 else torch.float32
        nbytes = st3_workspace_size(cfg)
        with torch.cuda.device(self.device):
            self.workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
            base = self.workspace.data_ptr()
            self._ws_ptr = (base + 255) // 256 * 256
            self.handle = st3_create(cfg, self._ws_ptr, nbytes)
        self.workspace_bytes = nbytes
        # the current stream's handle without a Stream object around it (2.2 us a call), where torch offers that
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None) if self.device.index is not None else None
        self._raw_stream = functools.partial(raw, self.device.index) if raw else None

    def _stream(self):
        if self._raw_stream:
            return self._raw_stream()
        return self.torch.cuda.current_stream(self.device).cuda_stream

    def _ptr(self, t):
        assert t.is_cuda and t.is_contiguous() and t.dtype == self.dtype, (t.device, t.dtype, t.is_contiguous())
        return t.data_ptr()

    def io_shape(self, layer_count=None):
        c = self.cfg
        return (c.num_layers if layer_count is None else layer_count, c.batch, c.num_heads, c.head_dim)

    def prefill_select(self, q_last, k, v, text_len, out, layer_begin=0):
        st3_prefill_select(self.handle, layer_begin, q_last.shape[0], self._ptr(q_last), self._ptr(k), self._ptr(v),
                           text_len, self._ptr(out), self._stream())

    def prefill_select_scored(self, q_last, k, v, text_len, scores, out, layer_begin=0):
        assert scores.is_cuda and scores.is_contiguous() and scores.dtype == self.torch.float32
        st3_prefill_select_scored(self.handle, layer_begin, q_last.shape[0], self._ptr(q_last), self._ptr(k),
                                  self._ptr(v), text_len, scores.data_ptr(), self._ptr(out), self._stream())

    def decode_step(self, step, q, k_new, v_new, out, layer_begin=0):
        # called once per token, or once per token and layer: the entry point itself, 10.1 -> 6.7 us of host time a call
        code = self._decode_step(self.handle, step, layer_begin, q.size(0), self._ptr(q), self._ptr(k_new),
                                 self._ptr(v_new), self._ptr(out), self._stream())
        if code != ST3_OK:
            raise St3Error(code, "st3_decode_step")

    def decode_step_host(self, step, q, k_new, v_new, out, layer_begin=0):
        """q/k_new/v_new/out are pinned HOST tensors."""
        st3_decode_step_host(self.handle, step, layer_begin, q.shape[0], q.data_ptr(), k_new.data_ptr(),
                             v_new.data_ptr(), out.data_ptr(), self._stream())

    def prefill_select_host(self, q_last, k, v, text_len, out, layer_begin=0):
        """q_last/k/v/out are pinned HOST tensors."""
        st3_prefill_select_host(self.handle, layer_begin, q_last.shape[0], q_last.data_ptr(), k.data_ptr(),
                                v.data_ptr(), text_len, out.data_ptr(), self._stream())

    def host_sync(self):
        st3_host_sync(self.handle, self._stream())

    def get_kept(self, layer, with_mass=True):
        t, c = self.torch, self.cfg
        ids = t.empty((c.batch, max(1, c.num_visual)), dtype=t.int32, device=self.device)
        cnt = t.empty((c.batch,), dtype=t.int32, device=self.device)
        mass = t.empty((c.batch, max(1, c.num_visual)), dtype=t.float32, device=self.device) if with_mass else None
        st3_get_kept(self.handle, layer, ids.data_ptr(), cnt.data_ptr(), mass.data_ptr() if with_mass else None,
                     self._stream())
        return ids, cnt, mass

    def get_rows(self, layer, b, h):
        t, c = self.torch, self.cfg
        cap = c.sys_len + c.max_text_len + c.max_decode_steps
        kv = [t.empty((max(1, c.num_visual), c.head_dim), dtype=self.dtype, device=self.device) for _ in range(2)]
        tx = [t.empty((cap, c.head_dim), dtype=self.dtype, device=self.device) for _ in range(2)]
        st3_get_rows(self.handle, layer, b, h, kv[0].data_ptr(), kv[1].data_ptr(), tx[0].data_ptr(), tx[1].data_ptr(),
                     self._stream())
        return kv[0], kv[1], tx[0], tx[1]

    def status(self, raise_on_error=True):
        return st3_get_status(self.handle, raise_on_error)

    def rows_held(self):
        return st3_rows_held(self.handle)

    def launch_count(self):
        return st3_launch_count(self.handle)

    def close(self):
        if self.handle:
            self.torch.cuda.synchronize(self.device)
            st3_destroy(self.handle)
            self.handle = None
            self.workspace = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def config_from_workload(wl, **overrides) -> Config:
    """Config for one of the synthetic workloads (any object with the Workload fields)."""
    kw = dict(num_layers=wl.num_layers, num_heads=wl.num_heads, head_dim=wl.head_dim, dtype=wl.dtype,
              batch=wl.batch, sys_len=wl.sys_len, num_visual=wl.num_visual, max_text_len=wl.text_len_max,
              max_decode_steps=wl.decode_steps, stride=wl.stride, step_ratio_bp=wl.step_ratio_bp, tau=wl.tau,
              first_prune_layer=wl.first_prune_layer, first_ratio_bp=wl.first_ratio_bp)
    kw.update(overrides)
    return make_config(**kw)
