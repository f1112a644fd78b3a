"""ctypes binding of the HeadKV C-ABI (include/hkv.h, include/hkv_serve.h,
include/hkv_prompt.h).

Argument marshalling only: every function has the name of the C entry point
it forwards to, accepts integers (device addresses) or objects with a
`data_ptr()` method for pointer arguments, and raises HkvError on a status
other than HKV_OK. There is no fallback: if libheadkv.so is missing the
import of a function fails loudly.
"""
from __future__ import annotations

import ctypes
import os
from ctypes import (POINTER, Structure, c_char_p, c_double, c_float, c_int, c_int32, c_int64, c_size_t,
                    c_uint64, c_void_p)
from fractions import Fraction

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libheadkv.so")

HKV_OK = 0
HKV_ERR_INVALID_ARG = 1
HKV_ERR_SHAPE = 2
HKV_ERR_CAPACITY = 3
HKV_ERR_STATE = 4
HKV_ERR_BOUNDS = 5
HKV_ERR_TIMEOUT = 6
HKV_ERR_CUDA = 7
HKV_ERR_ALIGN = 8

HKV_FP32, HKV_BF16 = 0, 1
HKV_STEP_PREFETCH = 1
HKV_LOCAL, HKV_GLOBAL, HKV_DENSE = 0, 1, 255
HKV_BUDGET_PAPER, HKV_BUDGET_REDISTRIBUTE = 0, 1
HKV_DIST_RASTER, HKV_DIST_GRID2D = 0, 1
HKV_Q8, HKV_Q4 = 8, 4
HKV_ALL_LAYERS = -1
HKV_PACK_SKIP_COND = 1
HKV_ROPE_HALF, HKV_ROPE_PAIRS = 0, 1
HKV_ROPE_PLAIN, HKV_ROPE_LINEAR, HKV_ROPE_BASE, HKV_ROPE_PARTS = 0, 1, 2, 3
HKV_ROPE_BACK = 1
HKV_NORM_RMS, HKV_NORM_LAYER = 1, 2
HKV_ATTN_CAUSAL = 1


class hkv_config(Structure):
    _fields_ = [
        ("n_layers", c_int32), ("n_seqs", c_int32), ("n_heads", c_int32), ("head_dim", c_int32),
        ("dtype", c_int32), ("n_cond", c_int32), ("n_image", c_int32), ("row_len", c_int32),
        ("recent_w", c_int32), ("local_w", c_int32), ("period", c_int32), ("group_at", c_int32),
        ("global_budget", c_int32), ("budget_mode", c_int32), ("distance_mode", c_int32),
        ("reserved", c_int32), ("tau", c_double), ("r_s", c_double),
    ]


class hkv_cache(Structure):
    _fields_ = [
        ("k", c_void_p), ("v", c_void_p), ("pos", c_void_p), ("off", c_void_p), ("cap", c_void_p),
        ("len", c_void_p), ("nbuf", c_void_p), ("ntok", c_void_p), ("label", c_void_p),
        ("qbuf", c_void_p), ("err", c_void_p), ("capacity_tokens", c_int64),
    ]


class hkv_qcache(Structure):
    _fields_ = [
        ("k", c_void_p), ("v", c_void_p), ("ks", c_void_p), ("vs", c_void_p), ("pos", c_void_p),
        ("off", c_void_p), ("cap", c_void_p), ("len", c_void_p), ("nbuf", c_void_p),
        ("ntok", c_void_p), ("label", c_void_p), ("qbuf", c_void_p), ("err", c_void_p),
        ("capacity_tokens", c_int64), ("format", c_int32), ("reserved", c_int32),
    ]


class hkv_prefix(Structure):
    of = None   # (dtype, heads, head_dim) of the rows, where make_prefix knows them
    _fields_ = [
        ("k", c_void_p), ("v", c_void_p), ("len", c_void_p), ("err", c_void_p),
        ("group_stride", c_int64), ("head_stride", c_int64), ("token_stride", c_int64),
        ("n_groups", c_int32), ("max_len", c_int32),
    ]


class hkv_rope_params(Structure):
    _fields_ = [
        ("head_dim", c_int32), ("rot_dim", c_int32), ("layout", c_int32), ("n_axes", c_int32),
        ("section", c_int32 * 3), ("joint", c_int32), ("scaling", c_int32), ("reserved", c_int32),
        ("base", c_double), ("factor", c_double), ("original", c_double), ("low", c_double),
        ("high", c_double), ("amplitude", c_double),
    ]


class hkv_rope(Structure):
    _fields_ = [
        ("head_dim", c_int32), ("rot_dim", c_int32), ("layout", c_int32), ("n_axes", c_int32),
        ("section", c_int32 * 3), ("amplitude", c_float), ("turns", c_uint64 * 64),
    ]


class hkv_rows(Structure):
    of = None   # (sequences, tokens, head_dim) of the rows, where make_rows knows them
    on = None   # the device's number, -1 for the host, where it is known (as of the following)
    _fields_ = [
        ("data", c_void_p), ("seq_stride", c_int64), ("token_stride", c_int64),
        ("head_stride", c_int64), ("n_heads", c_int32), ("dtype", c_int32),
    ]


class hkv_tokens(Structure):
    of = None   # (sequences or None, axes, rows of positions), where make_tokens knows them
    on = None
    _fields_ = [
        ("n_tokens", c_int32), ("reserved", c_int32), ("len", c_void_p), ("pos", c_void_p),
        ("pos_axis_stride", c_int64), ("pos_seq_stride", c_int64), ("err", c_void_p),
    ]


class hkv_norm(Structure):
    of = None   # (dtype, head_dim, heads of q's and of k's weights or None), where make_norm knows them
    on = None
    _fields_ = [
        ("kind", c_int32), ("eps", c_float), ("q_weight", c_void_p), ("q_bias", c_void_p),
        ("k_weight", c_void_p), ("k_bias", c_void_p), ("q_head_stride", c_int64),
        ("k_head_stride", c_int64),
    ]


class hkv_states(Structure):
    of = None   # (dtype, sequences, head_dim) of the states, where make_states knows them
    on = None
    _fields_ = [
        ("k", c_void_p), ("v", c_void_p), ("len", c_void_p), ("err", c_void_p),
        ("seq_stride", c_int64), ("head_stride", c_int64), ("token_stride", c_int64),
        ("n_heads", c_int32), ("max_len", c_int32),
    ]


class HkvError(RuntimeError):
    def __init__(self, name: str, status: int):
        self.status = status
        super().__init__(f"hkv_{name}: {hkv_status_str(status)} ({status})")


_lib = None

# (name, argtypes, restype)
_SIGNATURES = {
    "hkv_status_str": ([c_int], c_char_p),
    "hkv_validate_config": ([POINTER(hkv_config)], c_int),
    "hkv_workspace_size": ([POINTER(hkv_config)], c_size_t),
    "hkv_init_dense": ([POINTER(hkv_config), POINTER(hkv_cache), c_void_p], c_int),
    "hkv_prefill": ([POINTER(hkv_config), POINTER(hkv_cache), c_int, c_void_p, c_void_p, c_void_p], c_int),
    "hkv_append_evict": ([POINTER(hkv_config), POINTER(hkv_cache), c_int, c_void_p, c_void_p, c_void_p,
                          c_void_p], c_int),
    "hkv_decode_attention": ([POINTER(hkv_config), POINTER(hkv_cache), c_int, c_void_p, c_void_p, c_void_p,
                              c_size_t, c_void_p], c_int),
    "hkv_decode_step": ([POINTER(hkv_config), POINTER(hkv_cache), c_int, c_void_p, c_void_p, c_void_p,
                         c_void_p, c_void_p, c_size_t, c_int, c_void_p], c_int),
    "hkv_decode_step_identify": ([POINTER(hkv_config), POINTER(hkv_cache), c_int, c_void_p, c_void_p,
                                  c_void_p, c_void_p, c_void_p, c_void_p, c_size_t, c_int, c_void_p],
                                 c_int),
    "hkv_decode_step_launches": ([POINTER(hkv_config)], c_int),
    "hkv_global_budget": ([c_int64, c_int64, c_int32, POINTER(c_int32)], c_int),
    "hkv_update_due": ([POINTER(hkv_config), c_int32, POINTER(c_int32)], c_int),
    "hkv_evict": ([POINTER(hkv_config), POINTER(hkv_cache), c_int, c_void_p], c_int),
    "hkv_evict_all": ([POINTER(hkv_config), POINTER(hkv_cache), c_void_p], c_int),
    "hkv_identify_heads": ([POINTER(hkv_config), POINTER(hkv_cache), c_int, c_void_p, c_void_p, c_void_p,
                            c_void_p], c_int),
    "hkv_identify_heads_multi": ([POINTER(hkv_config), POINTER(hkv_cache), c_int, c_void_p, c_void_p,
                                  c_void_p], c_int),
    "hkv_allocate_budgets": ([POINTER(hkv_config), c_void_p, c_void_p, c_void_p, c_void_p,
                              POINTER(c_int64), c_void_p], c_int),
    "hkv_repack": ([POINTER(hkv_config), POINTER(hkv_cache), POINTER(hkv_cache), c_int, c_void_p], c_int),
    "hkv_check": ([POINTER(hkv_cache), c_void_p], c_int),
    "hkv_export_state": ([POINTER(hkv_config), POINTER(hkv_cache), c_int, c_void_p, c_void_p, c_void_p,
                          c_void_p, c_void_p, c_int64, POINTER(c_int64), c_void_p], c_int),
    "hkv_quant_pack": ([POINTER(hkv_config), POINTER(hkv_cache), POINTER(hkv_qcache), c_int, c_int,
                        c_void_p], c_int),
    "hkv_quant_unpack": ([POINTER(hkv_config), POINTER(hkv_qcache), POINTER(hkv_cache), c_int,
                          c_void_p], c_int),
    "hkv_quant_workspace_size": ([POINTER(hkv_config)], c_size_t),
    "hkv_quant_attention": ([POINTER(hkv_config), POINTER(hkv_qcache), c_int, c_void_p, c_void_p,
                             c_void_p, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p], c_int),
    "hkv_quant_step": ([POINTER(hkv_config), POINTER(hkv_qcache), c_int, c_void_p, c_void_p, c_void_p,
                        c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_size_t, c_int, c_void_p],
                       c_int),
    "hkv_quant_evict": ([POINTER(hkv_config), POINTER(hkv_qcache), c_int, c_void_p], c_int),
    "hkv_quant_evict_all": ([POINTER(hkv_config), POINTER(hkv_qcache), c_void_p], c_int),
    "hkv_quant_check": ([POINTER(hkv_qcache), c_void_p], c_int),
    "hkv_prefix_workspace_size": ([POINTER(hkv_config), POINTER(hkv_prefix)], c_size_t),
    "hkv_prefix_attention": ([POINTER(hkv_config), POINTER(hkv_prefix), c_void_p, c_void_p, c_void_p,
                              c_void_p, c_size_t, c_void_p], c_int),
    # (addresses of structures: a POINTER argument costs several times an integer)
    "hkv_make_rope": ([c_void_p] * 2, c_int),
    "hkv_rope_rotate": ([c_void_p] * 5 + [c_int, c_void_p], c_int),
    "hkv_qk_norm_rope": ([c_void_p] * 11, c_int),
    "hkv_cross_workspace_size": ([c_void_p] * 3, c_size_t),
    "hkv_cross_attention": ([c_void_p] * 7 + [c_size_t, c_int, c_void_p], c_int),
}


def lib():
    """The loaded libheadkv.so (raises if it was not built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with __graft_entry__.build()")
        l = ctypes.CDLL(LIB_PATH)
        for name, (args, res) in _SIGNATURES.items():
            f = getattr(l, name)
            f.argtypes = args
            f.restype = res
        _lib = l
    return _lib


def _p(x) -> int | None:
    if x is None:
        return None
    if isinstance(x, int):
        return x
    return x.data_ptr()


def _call(name: str, *args) -> None:
    st = getattr(_lib or lib(), "hkv_" + name)(*args)
    if st != HKV_OK:
        raise HkvError(name, st)


def hkv_status_str(status: int) -> str:
    return lib().hkv_status_str(status).decode()


def make_config(*, n_layers, n_seqs, n_heads, head_dim, dtype, n_cond, n_image, row_len,
                recent_w, local_w, period, group_at, rho=None, global_budget=None,
                tau=0.9, r_s=0.5, budget_mode=HKV_BUDGET_PAPER,
                distance_mode=HKV_DIST_RASTER) -> hkv_config:
    """Builds an hkv_config; the global budget is the library's
    hkv_global_budget(rho, N) unless given explicitly."""
    if global_budget is None:
        global_budget = hkv_global_budget(rho, n_image)
    return hkv_config(n_layers, n_seqs, n_heads, head_dim,
                      HKV_BF16 if dtype in ("bf16", HKV_BF16) else HKV_FP32,
                      n_cond, n_image, row_len, recent_w, local_w, period, group_at,
                      int(global_budget), int(budget_mode), int(distance_mode), 0, float(tau),
                      float(r_s))


def hkv_global_budget(rho, n_image: int) -> int:
    """B_g for a budget ratio rho (a Fraction, or anything Fraction takes)."""
    r = Fraction(rho)
    out = c_int32(0)
    _call("global_budget", r.numerator, r.denominator, n_image, ctypes.byref(out))
    return int(out.value)


def hkv_update_due(cfg: hkv_config, t: int) -> bool:
    """Whether image token t's decode step starts with the periodic update."""
    out = c_int32(0)
    _call("update_due", ctypes.byref(cfg), t, ctypes.byref(out))
    return bool(out.value)


def hkv_validate_config(cfg: hkv_config) -> None:
    _call("validate_config", ctypes.byref(cfg))


def hkv_workspace_size(cfg: hkv_config) -> int:
    return int(lib().hkv_workspace_size(ctypes.byref(cfg)))


def hkv_init_dense(cfg, cache, stream=0) -> None:
    _call("init_dense", ctypes.byref(cfg), ctypes.byref(cache), stream)


def hkv_prefill(cfg, cache, layer, kc, vc, stream=0) -> None:
    _call("prefill", ctypes.byref(cfg), ctypes.byref(cache), layer, _p(kc), _p(vc), stream)


def hkv_append_evict(cfg, cache, layer, q, k, v, stream=0) -> None:
    _call("append_evict", ctypes.byref(cfg), ctypes.byref(cache), layer, _p(q), _p(k), _p(v), stream)


def hkv_decode_attention(cfg, cache, layer, q, out, workspace, ws_bytes, stream=0) -> None:
    _call("decode_attention", ctypes.byref(cfg), ctypes.byref(cache), layer, _p(q), _p(out),
          _p(workspace), ws_bytes, stream)


def hkv_decode_step(cfg, cache, layer, q, k, v, out, workspace, ws_bytes, flags=0,
                    stream=0) -> None:
    _call("decode_step", ctypes.byref(cfg), ctypes.byref(cache), layer, _p(q), _p(k), _p(v), _p(out),
          _p(workspace), ws_bytes, flags, stream)


def hkv_decode_step_launches(cfg) -> int:
    """Kernel launches of one hkv_decode_step call (1 or 2) on the current
    device; raises on an invalid config."""
    n = int(lib().hkv_decode_step_launches(ctypes.byref(cfg)))
    if n <= 0:
        raise HkvError("decode_step_launches", HKV_ERR_INVALID_ARG)
    return n


def hkv_decode_step_identify(cfg, cache, layer, q, k, v, out, label_out, workspace, ws_bytes,
                             flags=0, stream=0) -> None:
    _call("decode_step_identify", ctypes.byref(cfg), ctypes.byref(cache), layer, _p(q), _p(k), _p(v),
          _p(out), _p(label_out), _p(workspace), ws_bytes, flags, stream)


def hkv_evict(cfg, cache, layer, stream=0) -> None:
    _call("evict", ctypes.byref(cfg), ctypes.byref(cache), layer, stream)


def hkv_evict_all(cfg, cache, stream=0) -> None:
    _call("evict_all", ctypes.byref(cfg), ctypes.byref(cache), stream)


def hkv_identify_heads(cfg, cache, layer, q, label_out, nh_out=None, stream=0) -> None:
    _call("identify_heads", ctypes.byref(cfg), ctypes.byref(cache), layer, _p(q), _p(label_out),
          _p(nh_out), stream)


def hkv_identify_heads_multi(cfg, cache, layer, label_out, nh_out=None, stream=0) -> None:
    _call("identify_heads_multi", ctypes.byref(cfg), ctypes.byref(cache), layer, _p(label_out),
          _p(nh_out), stream)


def hkv_allocate_budgets(cfg, label, budget, cap, off, stream=0) -> int:
    total = c_int64(0)
    _call("allocate_budgets", ctypes.byref(cfg), _p(label), _p(budget), _p(cap), _p(off),
          ctypes.byref(total), stream)
    return int(total.value)


def hkv_repack(cfg, dense, ragged, layer, stream=0) -> None:
    _call("repack", ctypes.byref(cfg), ctypes.byref(dense), ctypes.byref(ragged), layer, stream)


def hkv_check(cache, stream=0) -> None:
    _call("check", ctypes.byref(cache), stream)


def hkv_export_state(cfg, cache, layer, stream=0):
    """One layer's state on the host: numpy arrays label, len, nbuf, ntok
    (S*H each) and the live positions of every head, packed head after head
    (a list of arrays, one per head)."""
    import numpy as np
    n = cfg.n_seqs * cfg.n_heads
    label = np.zeros(n, np.uint8)
    ln = np.zeros(n, np.int32)
    nbuf = np.zeros(n, np.int32)
    ntok = np.zeros(n, np.int32)
    count = c_int64(0)
    _call("export_state", ctypes.byref(cfg), ctypes.byref(cache), layer, label.ctypes.data,
          ln.ctypes.data, nbuf.ctypes.data, ntok.ctypes.data, None, 0, ctypes.byref(count), stream)
    pos = np.zeros(max(int(count.value), 1), np.int32)
    _call("export_state", ctypes.byref(cfg), ctypes.byref(cache), layer, None, None, None, None,
          pos.ctypes.data, pos.size, ctypes.byref(count), stream)
    split = np.cumsum(ln)[:-1]
    return {"label": label, "len": ln, "nbuf": nbuf, "ntok": ntok,
            "pos": np.split(pos[:int(count.value)], split)}


# ---------------------------------------------------------------------------
# the serving cache (include/hkv_serve.h)
# ---------------------------------------------------------------------------
def make_qcache(fmt, k, v, ks, vs, pos, off, cap, length, nbuf, ntok, label, qbuf, err,
                capacity_tokens) -> hkv_qcache:
    """An hkv_qcache over the caller's buffers (kept alive with it); fmt is
    HKV_Q8 or HKV_Q4."""
    arrays = (k, v, ks, vs, pos, off, cap, length, nbuf, ntok, label, qbuf, err)
    c = hkv_qcache(*(_p(x) for x in arrays), int(capacity_tokens), int(fmt), 0)
    c.arrays = arrays
    return c


_PROMPT_DTYPES = {"torch.float32": HKV_FP32, "torch.bfloat16": HKV_BF16}


def make_prefix(k, v, length, err=None) -> hkv_prefix:
    """An hkv_prefix from tensors k and v of [groups][heads][tokens][head_dim],
    fp32 or bf16 (any strides whose last is 1, the same in both), and the
    prompts' lengths, contiguous int32, all on one device; keeps them alive.
    Calls with a config of another dtype, n_heads or head_dim refuse it."""
    if k.dim() != 4 or k.shape != v.shape or k.stride() != v.stride() or k.stride(3) != 1:
        raise HkvError("make_prefix", HKV_ERR_SHAPE)
    if length.numel() != k.shape[0]:
        raise HkvError("make_prefix", HKV_ERR_SHAPE)
    dtype = _PROMPT_DTYPES.get(str(k.dtype))
    if dtype is None or v.dtype != k.dtype or str(length.dtype) != "torch.int32":
        raise HkvError("make_prefix", HKV_ERR_SHAPE)
    if not length.is_contiguous() or not k.device == v.device == length.device:
        raise HkvError("make_prefix", HKV_ERR_INVALID_ARG)
    p = hkv_prefix(k.data_ptr(), v.data_ptr(), length.data_ptr(), _p(err), k.stride(0),
                   k.stride(1), k.stride(2), k.shape[0], k.shape[2])
    p.arrays = (k, v, length, err)
    p.of = (dtype, k.shape[1], k.shape[3])
    return p


def hkv_quant_pack(cfg, src, dst, layer, flags=0, stream=0) -> None:
    _call("quant_pack", ctypes.byref(cfg), ctypes.byref(src), ctypes.byref(dst), layer, flags, stream)


def hkv_quant_unpack(cfg, src, dst, layer, stream=0) -> None:
    _call("quant_unpack", ctypes.byref(cfg), ctypes.byref(src), ctypes.byref(dst), layer, stream)


def hkv_quant_workspace_size(cfg) -> int:
    return int(lib().hkv_quant_workspace_size(ctypes.byref(cfg)))


def hkv_quant_attention(cfg, cache, layer, q, out, workspace, ws_bytes, prior=None, lse=None,
                        stream=0) -> None:
    """prior: None or (out, lse) of the same queries over other keys."""
    po, pl = prior or (None, None)
    _call("quant_attention", ctypes.byref(cfg), ctypes.byref(cache), layer, _p(q), _p(po), _p(pl),
          _p(out), _p(lse), _p(workspace), ws_bytes, stream)


def hkv_quant_step(cfg, cache, layer, q, k, v, out, workspace, ws_bytes, prior=None, lse=None,
                   flags=0, stream=0) -> None:
    po, pl = prior or (None, None)
    _call("quant_step", ctypes.byref(cfg), ctypes.byref(cache), layer, _p(q), _p(k), _p(v), _p(po),
          _p(pl), _p(out), _p(lse), _p(workspace), ws_bytes, flags, stream)


def hkv_quant_evict(cfg, cache, layer, stream=0) -> None:
    _call("quant_evict", ctypes.byref(cfg), ctypes.byref(cache), layer, stream)


def hkv_quant_evict_all(cfg, cache, stream=0) -> None:
    _call("quant_evict_all", ctypes.byref(cfg), ctypes.byref(cache), stream)


def hkv_quant_check(cache, stream=0) -> None:
    _call("quant_check", ctypes.byref(cache), stream)


def hkv_prefix_workspace_size(cfg, prefix) -> int:
    if prefix.of not in (None, (cfg.dtype, cfg.n_heads, cfg.head_dim)):
        return 0
    return int(lib().hkv_prefix_workspace_size(ctypes.byref(cfg), ctypes.byref(prefix)))


def hkv_prefix_attention(cfg, prefix, q, out, lse, workspace, ws_bytes, stream=0) -> None:
    if prefix.of not in (None, (cfg.dtype, cfg.n_heads, cfg.head_dim)):
        raise HkvError("prefix_attention", HKV_ERR_SHAPE)
    _call("prefix_attention", ctypes.byref(cfg), ctypes.byref(prefix), _p(q), _p(out), _p(lse),
          _p(workspace), ws_bytes, stream)


# ---------------------------------------------------------------------------
# around the cache: rotary positions, norms, attention over other states
# (include/hkv_prompt.h)
# ---------------------------------------------------------------------------
_DTYPES = _PROMPT_DTYPES


def _on(name, *given):
    """The device's number (-1: the host) of the tensors among `given`, which
    have to lie together; None without any."""
    where = on = None
    for x in given:
        d = getattr(x, "device", None)   # an address has none
        if d is None:
            continue
        if where is None:
            where, on = d, x.get_device()
        elif d != where:
            raise HkvError(name, HKV_ERR_INVALID_ARG)
    return on


def hkv_make_rope(*, head_dim, rot_dim=None, layout=HKV_ROPE_HALF, sections=None, joint=False,
                  base=10000.0, scaling=HKV_ROPE_PLAIN, factor=1.0, original=1.0, low=1.0, high=32.0,
                  amplitude=1.0) -> hkv_rope:
    """A rotation of the first rot_dim channels (default: all) of a head;
    sections: the pairs of each axis (default: one axis)."""
    rot_dim = head_dim if rot_dim is None else rot_dim
    sections = (rot_dim // 2,) if sections is None else tuple(sections)
    if not 1 <= len(sections) <= 3:
        raise HkvError("make_rope", HKV_ERR_SHAPE)
    p = hkv_rope_params(head_dim, rot_dim, layout, len(sections), (c_int32 * 3)(*sections), int(joint),
                        scaling, 0, base, factor, original, low, high, amplitude)
    rope = hkv_rope()
    _call("make_rope", _addr(p), _addr(rope))
    return rope


def make_rows(x) -> hkv_rows:
    """hkv_rows over a tensor of [sequences][tokens][heads][head_dim], or
    [sequences][heads][head_dim] for one token each, fp32 or bf16 (any strides
    whose last is 1); keeps it alive. Calls of other sizes refuse it."""
    y = x.unsqueeze(1) if x.dim() == 3 else x
    dtype = _DTYPES.get(str(y.dtype))
    if y.dim() != 4 or dtype is None or y.stride(3) != 1:
        raise HkvError("make_rows", HKV_ERR_SHAPE)
    r = hkv_rows(y.data_ptr(), y.stride(0), y.stride(1), y.stride(2), y.shape[2], dtype)
    r.arrays = x
    r.of = (y.shape[0], y.shape[1], y.shape[3])
    r.on = x.get_device()
    return r


def make_tokens(n_tokens, length=None, pos=None, err=None) -> hkv_tokens:
    """hkv_tokens of n_tokens places a sequence; length: None, or contiguous
    int32 [sequences]; pos: None, or int32 positions of [axes][sequences or
    1][n_tokens] or [sequences or 1][n_tokens], the last stride 1; all on the
    device of the call's other views."""
    if length is not None and (str(length.dtype) != "torch.int32" or length.dim() != 1
                               or not length.is_contiguous()):
        raise HkvError("make_tokens", HKV_ERR_SHAPE)
    strides, axes, rows = (0, 0), 0, None
    if pos is not None:
        p = pos.unsqueeze(0) if pos.dim() == 2 else pos
        if p.dim() != 3 or str(p.dtype) != "torch.int32" or p.shape[2] != n_tokens or \
                (n_tokens > 1 and p.stride(2) != 1):
            raise HkvError("make_tokens", HKV_ERR_SHAPE)
        axes, rows = p.shape[0], p.shape[1]
        strides = (p.stride(0) if axes > 1 else 0, p.stride(1) if rows > 1 else 0)
    on = _on("make_tokens", length, pos, err)
    t = hkv_tokens(n_tokens, 0, _p(length), _p(pos), strides[0], strides[1], _p(err))
    t.arrays = (length, pos, err)
    t.of = (None if length is None else length.numel(), axes, rows)
    t.on = on
    return t


def make_norm(kind, eps, q_weight=None, k_weight=None, q_bias=None, k_bias=None) -> hkv_norm:
    """hkv_norm of weights and biases of [head_dim] or [heads][head_dim] in the
    config dtype (any head stride; a weight and its bias alike); keeps them alive."""
    given = [x for x in (q_weight, q_bias, k_weight, k_bias) if x is not None]
    heads, strides = [], []
    for pair in ((q_weight, q_bias), (k_weight, k_bias)):
        have = [x for x in pair if x is not None]
        if any(x.dim() not in (1, 2) or x.stride(-1) != 1 or str(x.dtype) not in _DTYPES for x in have) \
                or len({(tuple(x.shape), x.stride() if x.dim() == 2 and x.shape[0] > 1 else 0)
                        for x in have}) > 1:
            raise HkvError("make_norm", HKV_ERR_SHAPE)
        rows = [x for x in have if x.dim() == 2]
        heads.append(rows[0].shape[0] if rows else None)
        strides.append(rows[0].stride(0) if rows and rows[0].shape[0] > 1 else 0)
    if len({(x.dtype, x.shape[-1]) for x in given}) > 1:
        raise HkvError("make_norm", HKV_ERR_SHAPE)
    n = hkv_norm(kind, eps, _p(q_weight), _p(q_bias), _p(k_weight), _p(k_bias), strides[0], strides[1])
    n.arrays = given
    n.on = _on("make_norm", *given)
    if given:
        n.of = (_DTYPES[str(given[0].dtype)], given[0].shape[-1], heads[0], heads[1])
    return n


def make_states(k, v, length=None, err=None) -> hkv_states:
    """hkv_states from tensors k and v of [sequences][heads][states][head_dim],
    fp32 or bf16 (any strides whose last is 1, the same in both), and the
    sequences' numbers of states, contiguous int32, or None, all on one
    device; keeps them alive. Calls of other sizes refuse it."""
    if k.dim() != 4 or k.shape != v.shape or k.stride() != v.stride() or k.stride(3) != 1:
        raise HkvError("make_states", HKV_ERR_SHAPE)
    dtype = _DTYPES.get(str(k.dtype))
    if dtype is None or v.dtype != k.dtype:
        raise HkvError("make_states", HKV_ERR_SHAPE)
    if length is not None and (length.numel() != k.shape[0] or str(length.dtype) != "torch.int32"
                               or not length.is_contiguous()):
        raise HkvError("make_states", HKV_ERR_SHAPE)
    on = _on("make_states", k, v, length, err)
    s = hkv_states(k.data_ptr(), v.data_ptr(), _p(length), _p(err), k.stride(0), k.stride(1), k.stride(2),
                   k.shape[1], k.shape[2])
    s.arrays = (k, v, length, err)
    s.of = (dtype, k.shape[0], k.shape[3])
    s.on = on
    return s


_addr = ctypes.addressof


def _at(x):
    return None if x is None else _addr(x)


def _fit(name, cfg, tokens, rope, rows):
    """Refuses views whose known sizes are not the call's. The number of their
    device: None where it is not known, -1 for the host's or several."""
    seqs = cfg.n_seqs
    want = (seqs, tokens.n_tokens, cfg.head_dim)
    ok, on = True, tokens.on
    for r in rows:
        if r is not None:
            if r.of != want and r.of is not None:
                ok = False
            if r.on != on and r.on is not None:
                on = r.on if on is None else -1
    if tokens.of is not None:
        len_seqs, axes, pos_rows = tokens.of
        if len_seqs is not None and len_seqs != seqs:
            ok = False
        if rope is not None and axes and (axes < rope.n_axes or pos_rows not in (1, seqs)):
            ok = False
    if not ok:
        raise HkvError(name, HKV_ERR_SHAPE)
    return on


def hkv_rope_rotate(cfg, rope, tokens, x, out, flags=0, stream=0) -> None:
    if _fit("rope_rotate", cfg, tokens, rope, (x, out)) == -1:
        raise HkvError("rope_rotate", HKV_ERR_INVALID_ARG)
    st = (_lib or lib()).hkv_rope_rotate(_addr(cfg), _addr(rope), _addr(tokens), _addr(x), _addr(out),
                                         flags, stream)
    if st != HKV_OK:
        raise HkvError("rope_rotate", st)


def hkv_qk_norm_rope(cfg, norm, rope, tokens, q, k, v, q_out, k_out, v_out, stream=0) -> None:
    """norm and rope may be None, and pairs of q, k, v and their outs."""
    on = _fit("qk_norm_rope", cfg, tokens, rope, (q, k, v, q_out, k_out, v_out))
    if norm is not None and norm.of is not None:
        dtype, dim, q_heads, k_heads = norm.of
        if dtype != cfg.dtype or dim != cfg.head_dim \
                or (q is not None and q_heads is not None and q_heads != q.n_heads) \
                or (k is not None and k_heads is not None and k_heads != k.n_heads):
            raise HkvError("qk_norm_rope", HKV_ERR_SHAPE)
        if norm.on != on and norm.on is not None:
            on = norm.on if on is None else -1
    if on == -1:
        raise HkvError("qk_norm_rope", HKV_ERR_INVALID_ARG)
    st = (_lib or lib()).hkv_qk_norm_rope(_addr(cfg), _at(norm), _at(rope), _addr(tokens), _at(q), _at(k),
                                          _at(v), _at(q_out), _at(k_out), _at(v_out), stream)
    if st != HKV_OK:
        raise HkvError("qk_norm_rope", st)


def _states_fit(cfg, states) -> bool:
    return states.of is None or states.of == (cfg.dtype, cfg.n_seqs, cfg.head_dim)


def hkv_cross_workspace_size(cfg, states, tokens) -> int:
    if not _states_fit(cfg, states):
        return 0
    return int(lib().hkv_cross_workspace_size(_addr(cfg), _addr(states), _addr(tokens)))


_float32 = None   # torch's, once a call has met it


def hkv_cross_attention(cfg, states, tokens, q, out, lse, workspace, ws_bytes, flags=0, stream=0) -> None:
    """lse: None, an address, or a contiguous fp32 tensor of [n_seqs][n_heads]
    [n_tokens] elements at least; workspace: an address, or a tensor of ws_bytes
    bytes at least."""
    on = _fit("cross_attention", cfg, tokens, None, (q, out))
    if not _states_fit(cfg, states):
        raise HkvError("cross_attention", HKV_ERR_SHAPE)
    if states.on != on and states.on is not None:
        on = states.on if on is None else -1
    global _float32
    size = getattr(lse, "nbytes", None)
    if size is not None:
        if lse.dtype is not _float32:
            if str(lse.dtype) != "torch.float32":
                raise HkvError("cross_attention", HKV_ERR_SHAPE)
            _float32 = lse.dtype
        if size < 4 * cfg.n_seqs * cfg.n_heads * tokens.n_tokens or not lse.is_contiguous():
            raise HkvError("cross_attention", HKV_ERR_SHAPE)
        if lse.get_device() != on and on is not None:
            on = -1
    size = getattr(workspace, "nbytes", None)
    if size is not None:
        if size < ws_bytes:
            raise HkvError("cross_attention", HKV_ERR_CAPACITY)
        if workspace.get_device() != on and on is not None:
            on = -1
    if on == -1:
        raise HkvError("cross_attention", HKV_ERR_INVALID_ARG)
    st = (_lib or lib()).hkv_cross_attention(_addr(cfg), _addr(states), _addr(tokens), _addr(q), _addr(out),
                                             _p(lse), _p(workspace), ws_bytes, flags, stream)
    if st != HKV_OK:
        raise HkvError("cross_attention", st)
