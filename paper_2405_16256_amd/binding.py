"""ctypes binding of libhh.so: the same entry points as the headers in include/, argument marshalling only.

Every numeric step runs in the library's HIP kernels.  PyTorch tensors are used
as owners of device memory (``tensor.data_ptr()``) and for the current stream;
there is no fallback path: if the library is missing, importing fails.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Sequence

# PyTorch-ROCm ships its own HIP runtime.  It has to be in the process before libhh.so is
# opened so that the library binds to that same runtime (one runtime per process: streams
# and device pointers are shared with torch).
import torch  # noqa: F401

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libhh.so")

HH_OK = 0
HH_ERR_INVALID_ARG = -1
HH_ERR_UNSUPPORTED_SHAPE = -2
HH_ERR_BUFFER_TOO_SMALL = -3
HH_ERR_MISALIGNED = -4
HH_ERR_DEVICE = -5
HH_F32 = 0
HH_BF16 = 1
HH_STATIC_SCRATCH_BYTES = 128 << 20
HH_CLIP_WORKSPACE_BYTES = 8192
HH_MX_NONE, HH_MX_E4M3, HH_MX_E2M1 = 0, 1, 2
HH_MX_PAD = 256
HH_MX_SUMS_F32, HH_MX_SUMS_FAST = 0, 1

WEIGHT_FIELDS = ("g_attn", "wq", "wk", "wv", "wo", "g_mlp", "w_gate", "w_up", "w_down")
EXPORTS = ("hh_last_error", "hh_ctx_create", "hh_ctx_destroy", "hh_ctx_reserve", "hh_layer_flops", "hh_layer_sizes",
           "hh_saved_layout_of", "hh_layer_fwd", "hh_layer_fwd_noalloc", "hh_layer_bwd", "hh_stage_sizes", "hh_stage_step", "hh_stage_step_1f1b", "hh_layer_profile", "hh_trace_begin",
           "hh_trace_end", "hh_sim_pipeline", "hh_sim_weighted_mean", "hh_plan_layers", "hh_plan_order", "hh_plan_cluster",
           "hh_head_sizes", "hh_head_loss", "hh_head_step", "hh_head_share_fwd", "hh_head_share_bwd", "hh_grad_clip", "hh_adamw_step",
           "hh_dropout", "hh_mx_sizes", "hh_mx_quantise", "hh_mx_values", "hh_add_norm_fwd", "hh_add_norm_sizes", "hh_add_norm_bwd",
           "hh_mx_product_sizes", "hh_mx_product")
TRACE_KINDS = ("gemm_nt", "gemm_nn", "gemm_tn", "attn_fwd", "attn_bwd", "elementwise")


class hh_layer_cfg(C.Structure):
    _fields_ = [("hidden", C.c_int32), ("n_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("ffn", C.c_int32), ("seq", C.c_int32), ("micro_batch", C.c_int32), ("rms_eps", C.c_float),
                ("rope_base", C.c_float), ("dtype", C.c_int32)]


class hh_layer_weights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in WEIGHT_FIELDS]


class hh_layer_grads(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in WEIGHT_FIELDS]


class hh_profile_rec(C.Structure):
    _fields_ = [("layer", C.c_int32), ("fwd_ms", C.c_float), ("bwd_ms", C.c_float), ("fwd_flop", C.c_double),
                ("bwd_flop", C.c_double), ("fwd_tflops", C.c_float), ("bwd_tflops", C.c_float),
                ("weight_bytes", C.c_uint64), ("grad_bytes", C.c_uint64), ("saved_act_bytes", C.c_uint64),
                ("p2p_bytes", C.c_uint64),
                ("workspace_bytes", C.c_uint64)]


class hh_saved_layout(C.Structure):
    _fields_ = [(n, C.c_size_t) for n in ("xn", "qkv", "a", "h", "hn", "gate_up", "lse", "r1", "r2", "total")]


class hh_trace_sum(C.Structure):
    _fields_ = [("kind", C.c_int32), ("launches", C.c_int32), ("ms", C.c_double), ("work", C.c_double)]


class hh_sim_stage(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("n_devices", C.c_int32), ("fwd_ms", C.c_double), ("bwd_ms", C.c_double),
                ("peak_tflops", C.c_double), ("link_gbytes_per_s", C.c_double), ("weight_bytes", C.c_uint64),
                ("grad_bytes", C.c_uint64), ("optimizer_bytes", C.c_uint64), ("saved_act_bytes", C.c_uint64),
                ("memory_bytes", C.c_uint64)]


class hh_sim_result(C.Structure):
    _fields_ = [("iter_ms", C.c_double), ("bubble_fraction", C.c_double), ("tokens_per_s_per_device", C.c_double),
                ("tflops_per_device", C.c_double), ("mean_peak_tflops", C.c_double), ("mfu", C.c_double),
                ("n_devices", C.c_int64), ("search_truncated", C.c_int32), ("reserved_", C.c_int32)]


class hh_cluster_group(C.Structure):
    _fields_ = [("n_nodes", C.c_int32), ("devices_per_node", C.c_int32), ("fwd_ms_tp", C.c_double * 4), ("bwd_ms_tp", C.c_double * 4),
                ("saved_act_bytes_tp", C.c_uint64 * 4), ("peak_tflops", C.c_double), ("link_gbytes_per_s", C.c_double),
                ("dp_gbytes_per_s", C.c_double), ("weight_bytes", C.c_uint64), ("grad_bytes", C.c_uint64),
                ("optimizer_bytes", C.c_uint64), ("memory_bytes", C.c_uint64)]


class hh_cluster_plan(C.Structure):
    _fields_ = [("data_parallel", C.c_int32), ("tensor_parallel", C.c_int32 * 8), ("stages", C.c_int32 * 8), ("order", C.c_int32 * 8),
                ("n_stages", C.c_int32), ("n_micro", C.c_int32), ("strategies_costed", C.c_int32), ("pipeline_ms", C.c_double),
                ("grad_allreduce_ms", C.c_double), ("sim", hh_sim_result)]


class hh_head_cfg(C.Structure):
    _fields_ = [("hidden", C.c_int32), ("vocab", C.c_int32), ("tokens", C.c_int32), ("dtype", C.c_int32)]


class hh_clip_tensor(C.Structure):
    _fields_ = [("g", C.c_void_p), ("out", C.c_void_p), ("count", C.c_int64), ("dtype", C.c_int32), ("reserved", C.c_int32)]


class hh_adamw_tensor(C.Structure):
    _fields_ = [("param", C.c_void_p), ("master", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p), ("g", C.c_void_p),
                ("count", C.c_int64), ("decay", C.c_float), ("param_dtype", C.c_int32), ("grad_dtype", C.c_int32), ("reserved", C.c_int32)]


class hh_adamw_cfg(C.Structure):
    _fields_ = [("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double), ("step", C.c_int64)]


class hh_dropout_cfg(C.Structure):
    _fields_ = [("seed", C.c_uint64), ("offset", C.c_uint64), ("step", C.c_void_p), ("p", C.c_double)]


class hh_mx_tensor(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("scales", C.c_void_p)]


class hh_add_norm_cfg(C.Structure):
    _fields_ = [("rows", C.c_int32), ("hidden", C.c_int32), ("eps", C.c_float), ("dtype", C.c_int32), ("format", C.c_int32)]


class hh_mx_product_cfg(C.Structure):
    _fields_ = [("m", C.c_int32), ("n", C.c_int32), ("k", C.c_int32), ("a_format", C.c_int32), ("b_format", C.c_int32), ("dtype", C.c_int32),
                ("ldc", C.c_int64), ("sums", C.c_int32)]


class HHError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__("hh error %d: %s" % (code, msg))
        self.code = code


def _load() -> C.CDLL:
    if not os.path.exists(_LIB_PATH):
        raise ImportError("%s is missing: build it with `python -m paper_2405_16256_amd.build` "
                          "(there is no fallback path)" % _LIB_PATH)
    lib = C.CDLL(_LIB_PATH)
    vp, i, sz = C.c_void_p, C.c_int, C.POINTER(C.c_size_t)
    i32, i64, mxp, anp = C.c_int32, C.c_int64, C.POINTER(hh_mx_tensor), C.POINTER(hh_add_norm_cfg)
    cfgp, wp, gp = C.POINTER(hh_layer_cfg), C.POINTER(hh_layer_weights), C.POINTER(hh_layer_grads)
    lib.hh_last_error.restype = C.c_char_p
    lib.hh_last_error.argtypes = []
    sigs = {
        "hh_ctx_create": [C.POINTER(vp), i],
        "hh_ctx_destroy": [vp],
        "hh_ctx_reserve": [vp, cfgp],
        "hh_layer_flops": [cfgp, C.POINTER(C.c_double), C.POINTER(C.c_double)],
        "hh_layer_sizes": [cfgp, sz, sz],
        "hh_saved_layout_of": [cfgp, C.POINTER(hh_saved_layout)],
        "hh_layer_fwd": [vp, cfgp, wp, vp, vp, vp, vp, vp],
        "hh_layer_fwd_noalloc": [vp, cfgp, wp, vp, vp, vp],
        "hh_layer_bwd": [vp, cfgp, wp, vp, vp, vp, vp, gp, i, vp, vp],
        "hh_stage_sizes": [cfgp, i, i, sz, sz],
        "hh_stage_step": [vp, cfgp, i, wp, i, C.POINTER(vp), C.POINTER(vp), C.POINTER(vp), C.POINTER(vp), gp, i, vp, vp, vp],
        "hh_stage_step_1f1b": [vp, cfgp, i, wp, i, i, C.POINTER(vp), C.POINTER(vp), C.POINTER(vp), C.POINTER(vp), gp, i, vp, vp,
                               vp],
        "hh_layer_profile": [vp, cfgp, i, wp, gp, vp, vp, i, i, vp, vp, C.POINTER(hh_profile_rec), vp],
        "hh_trace_begin": [vp, i, C.c_uint32],
        "hh_trace_end": [vp, C.POINTER(hh_trace_sum), i],
        "hh_sim_pipeline": [C.POINTER(hh_sim_stage), i, i, i, i, i, i, C.c_double, C.POINTER(hh_sim_result), C.POINTER(C.c_double),
                            C.POINTER(C.c_uint64)],
        "hh_sim_weighted_mean": [C.POINTER(C.c_double), C.POINTER(C.c_int64), i, C.POINTER(C.c_double)],
        "hh_plan_layers": [C.POINTER(hh_sim_stage), i, i, i, i, i, i, i, C.c_double, i, C.POINTER(C.c_int32),
                           C.POINTER(hh_sim_result)],
        "hh_plan_order": [C.POINTER(hh_sim_stage), C.POINTER(C.c_int32), i, C.c_double, i, i, i, i, i, i, C.c_double, i,
                          C.POINTER(C.c_int32), C.POINTER(C.c_int32), C.POINTER(hh_sim_result)],
        "hh_plan_cluster": [C.POINTER(hh_cluster_group), i, C.c_double, i, i, i, i, i, C.c_double, i, C.POINTER(hh_cluster_plan),
                            C.POINTER(C.c_int32), i],
        "hh_head_sizes": [C.POINTER(hh_head_cfg), sz, sz],
        "hh_head_loss": [vp, C.POINTER(hh_head_cfg), vp, vp, vp, vp, vp, vp],
        "hh_head_step": [vp, C.POINTER(hh_head_cfg), vp, vp, vp, vp, C.c_float, vp, vp, vp, i, vp, vp],
        "hh_head_share_fwd": [vp, C.POINTER(hh_head_cfg), vp, vp, vp, C.c_int32, vp, vp, vp, vp],
        "hh_head_share_bwd": [vp, C.POINTER(hh_head_cfg), vp, vp, vp, C.c_int32, vp, vp, C.c_float, vp, vp, i, vp, vp],
        "hh_grad_clip": [vp, i, C.POINTER(hh_clip_tensor), C.c_float, vp, vp, vp],
        "hh_adamw_step": [vp, C.POINTER(hh_adamw_cfg), i, C.POINTER(hh_adamw_tensor), vp, vp],
        "hh_dropout": [vp, C.POINTER(hh_dropout_cfg), i64, i64, i32, vp, i64, vp, i64, vp],
        "hh_mx_sizes": [i32, i64, i64, sz, sz],
        "hh_mx_quantise": [vp, i64, i64, i32, vp, i64, i32, mxp, mxp, vp],
        "hh_mx_values": [vp, i64, i64, i32, mxp, i32, vp, i64, vp],
        "hh_add_norm_fwd": [vp, anp, C.POINTER(hh_dropout_cfg), vp, vp, vp, vp, vp, mxp, vp],
        "hh_add_norm_sizes": [anp, sz],
        "hh_add_norm_bwd": [vp, anp, C.POINTER(hh_dropout_cfg), vp, vp, vp, vp, vp, vp, vp, i, vp, vp],
        "hh_mx_product_sizes": [C.POINTER(hh_mx_product_cfg), sz],
        "hh_mx_product": [vp, C.POINTER(hh_mx_product_cfg), mxp, mxp, vp, i, vp, vp],
    }
    for name, args in sigs.items():
        fn = getattr(lib, name)
        fn.restype = C.c_int
        fn.argtypes = args
    return lib


lib = _load()


def hh_last_error() -> str:
    return lib.hh_last_error().decode()


def _check(rc: int) -> None:
    if rc != HH_OK:
        raise HHError(rc, hh_last_error())


def _ptr(t) -> int | None:
    """Device address of a torch tensor, or an int / None passed through."""
    if t is None or isinstance(t, int):
        return t
    return t.data_ptr()


def make_cfg(hidden, n_heads, head_dim, ffn, seq, micro_batch=1, rms_eps=1e-5, rope_base=10000.0, dtype=HH_BF16,
             n_kv_heads=None) -> hh_layer_cfg:
    return hh_layer_cfg(hidden, n_heads, n_heads if n_kv_heads is None else n_kv_heads, head_dim, ffn, seq,
                        micro_batch, rms_eps, rope_base, dtype)


def make_weights(w: dict) -> hh_layer_weights:
    return hh_layer_weights(*[_ptr(w[n]) for n in WEIGHT_FIELDS])


def make_grads(g: dict) -> hh_layer_grads:
    return hh_layer_grads(*[_ptr(g[n]) for n in WEIGHT_FIELDS])


def hh_ctx_create(device: int = 0) -> int:
    out = C.c_void_p()
    _check(lib.hh_ctx_create(C.byref(out), device))
    return out.value


def hh_ctx_destroy(ctx: int) -> None:
    _check(lib.hh_ctx_destroy(ctx))


def hh_ctx_reserve(ctx: int, cfg: hh_layer_cfg) -> None:
    _check(lib.hh_ctx_reserve(ctx, C.byref(cfg)))


def hh_layer_flops(cfg: hh_layer_cfg) -> tuple[float, float]:
    f, b = C.c_double(), C.c_double()
    _check(lib.hh_layer_flops(C.byref(cfg), C.byref(f), C.byref(b)))
    return f.value, b.value


def hh_layer_sizes(cfg: hh_layer_cfg) -> tuple[int, int]:
    s, w = C.c_size_t(), C.c_size_t()
    _check(lib.hh_layer_sizes(C.byref(cfg), C.byref(s), C.byref(w)))
    return s.value, w.value


def hh_saved_layout_of(cfg: hh_layer_cfg) -> hh_saved_layout:
    out = hh_saved_layout()
    _check(lib.hh_saved_layout_of(C.byref(cfg), C.byref(out)))
    return out


def hh_stage_sizes(cfg: hh_layer_cfg, n_layers: int, n_micro: int) -> tuple[int, int]:
    s, w = C.c_size_t(), C.c_size_t()
    _check(lib.hh_stage_sizes(C.byref(cfg), n_layers, n_micro, C.byref(s), C.byref(w)))
    return s.value, w.value


def hh_layer_fwd(ctx, cfg, weights: hh_layer_weights, x, y, saved, workspace, stream=0) -> None:
    _check(lib.hh_layer_fwd(ctx, C.byref(cfg), C.byref(weights), _ptr(x), _ptr(y), _ptr(saved), _ptr(workspace), stream))


def hh_layer_fwd_noalloc(ctx, cfg, weights: hh_layer_weights, x, y, stream=0) -> None:
    _check(lib.hh_layer_fwd_noalloc(ctx, C.byref(cfg), C.byref(weights), _ptr(x), _ptr(y), stream))


def hh_layer_bwd(ctx, cfg, weights: hh_layer_weights, x, saved, dy, dx, grads: hh_layer_grads, accumulate, workspace,
                 stream=0) -> None:
    _check(lib.hh_layer_bwd(ctx, C.byref(cfg), C.byref(weights), _ptr(x), _ptr(saved), _ptr(dy), _ptr(dx),
                            C.byref(grads), int(accumulate), _ptr(workspace), stream))


def _ptr_array(ts: Sequence):
    return (C.c_void_p * len(ts))(*[_ptr(t) for t in ts])


def hh_stage_step(ctx, cfg, weights: Sequence[hh_layer_weights], x: Sequence, y: Sequence, dy: Sequence, dx: Sequence,
                  grads: Sequence[hh_layer_grads], zero_grads_first, saved_pool, workspace, stream=0) -> None:
    k, m = len(weights), len(x)
    assert len(grads) == k and len(y) == m and len(dy) == m and len(dx) == m
    warr = (hh_layer_weights * k)(*weights)
    garr = (hh_layer_grads * k)(*grads)
    _check(lib.hh_stage_step(ctx, C.byref(cfg), k, warr, m, _ptr_array(x), _ptr_array(y), _ptr_array(dy), _ptr_array(dx),
                             garr, int(zero_grads_first), _ptr(saved_pool), _ptr(workspace), stream))


def hh_stage_step_1f1b(ctx, cfg, weights: Sequence[hh_layer_weights], n_live: int, x: Sequence, y: Sequence, dy: Sequence,
                       dx: Sequence, grads: Sequence[hh_layer_grads], zero_grads_first, saved_pool, workspace, stream=0) -> None:
    k, m = len(weights), len(x)
    assert len(grads) == k and len(y) == m and len(dy) == m and len(dx) == m
    warr = (hh_layer_weights * k)(*weights)
    garr = (hh_layer_grads * k)(*grads)
    _check(lib.hh_stage_step_1f1b(ctx, C.byref(cfg), k, warr, m, int(n_live), _ptr_array(x), _ptr_array(y), _ptr_array(dy),
                                  _ptr_array(dx), garr, int(zero_grads_first), _ptr(saved_pool), _ptr(workspace), stream))


def hh_layer_profile(ctx, cfg, weights: Sequence[hh_layer_weights], grads: Sequence[hh_layer_grads], x, dy, warmup, iters,
                     saved_pool, workspace, stream=0) -> list[hh_profile_rec]:
    k = len(weights)
    warr = (hh_layer_weights * k)(*weights)
    garr = (hh_layer_grads * k)(*grads)
    out = (hh_profile_rec * k)()
    _check(lib.hh_layer_profile(ctx, C.byref(cfg), k, warr, garr, _ptr(x), _ptr(dy), warmup, iters, _ptr(saved_pool),
                                _ptr(workspace), out, stream))
    return list(out)


def hh_trace_begin(ctx, max_launches: int, kinds=None) -> None:
    """kinds: family names from TRACE_KINDS to record (None: all)."""
    mask = 0xFFFFFFFF if kinds is None else sum(1 << TRACE_KINDS.index(k) for k in kinds)
    _check(lib.hh_trace_begin(ctx, max_launches, mask))


def hh_trace_end(ctx) -> dict:
    """{family: (launches, total_ms, total_work)} for the launches since hh_trace_begin."""
    out = (hh_trace_sum * len(TRACE_KINDS))()
    _check(lib.hh_trace_end(ctx, out, len(TRACE_KINDS)))
    return {TRACE_KINDS[r.kind]: (r.launches, r.ms, r.work) for r in out}


# ---------------------------------------------------------------- predictor (host only)
def hh_sim_pipeline(stages: Sequence[hh_sim_stage], n_micro, micro_batch, seq, hidden, data_parallel, flop_per_layer):
    """-> (hh_sim_result, finish_ms per stage, peak bytes per stage)"""
    n = len(stages)
    arr = (hh_sim_stage * max(n, 1))(*stages)
    res = hh_sim_result()
    fin = (C.c_double * max(n, 1))()
    peak = (C.c_uint64 * max(n, 1))()
    _check(lib.hh_sim_pipeline(arr, n, n_micro, micro_batch, seq, hidden, data_parallel, float(flop_per_layer), C.byref(res), fin,
                               peak))
    return res, list(fin)[:n], list(peak)[:n]


def hh_sim_weighted_mean(values, counts) -> float:
    n = len(values)
    v = (C.c_double * max(n, 1))(*values)
    c = (C.c_int64 * max(n, 1))(*[int(t) for t in counts])
    out = C.c_double()
    _check(lib.hh_sim_weighted_mean(v, c, n, C.byref(out)))
    return out.value


def hh_plan_layers(stages: Sequence[hh_sim_stage], total_layers, n_micro, micro_batch, seq, hidden, data_parallel,
                   flop_per_layer, slack=2):
    """-> (layers per stage, hh_sim_result of that split)"""
    n = len(stages)
    arr = (hh_sim_stage * max(n, 1))(*stages)
    out = (C.c_int32 * max(n, 1))()
    res = hh_sim_result()
    _check(lib.hh_plan_layers(arr, n, total_layers, n_micro, micro_batch, seq, hidden, data_parallel, float(flop_per_layer), slack,
                              out, C.byref(res)))
    return list(out)[:n], res


def hh_plan_order(groups: Sequence[hh_sim_stage], counts: Sequence[int], cross_link_gbytes_per_s, total_layers, n_micro,
                  micro_batch, seq, hidden, data_parallel, flop_per_layer, slack=2):
    """-> (group index per pipeline position, layers per stage in pipeline order, hh_sim_result)"""
    n = len(groups)
    assert len(counts) == n
    arr = (hh_sim_stage * max(n, 1))(*groups)
    cnt = (C.c_int32 * max(n, 1))(*counts)
    total = max(sum(c for c in counts if c > 0), 1)
    order = (C.c_int32 * max(n, 1))()
    layers = (C.c_int32 * total)()
    res = hh_sim_result()
    _check(lib.hh_plan_order(arr, cnt, n, float(cross_link_gbytes_per_s), total_layers, n_micro, micro_batch, seq, hidden,
                             data_parallel, float(flop_per_layer), slack, order, layers, C.byref(res)))
    return list(order)[:n], list(layers)[:sum(counts)], res


def hh_plan_cluster(groups: Sequence[hh_cluster_group], cross_link_gbytes_per_s, total_layers, global_batch, micro_batch, seq,
                    hidden, flop_per_layer, slack=2, max_stages=4096):
    """-> (hh_cluster_plan, layers per stage in pipeline order)"""
    n = len(groups)
    arr = (hh_cluster_group * max(n, 1))(*groups)
    plan = hh_cluster_plan()
    layers = (C.c_int32 * max_stages)()
    _check(lib.hh_plan_cluster(arr, n, float(cross_link_gbytes_per_s), total_layers, global_batch, micro_batch, seq, hidden,
                               float(flop_per_layer), slack, C.byref(plan), layers, max_stages))
    return plan, list(layers)[:plan.n_stages]


# ---------------------------------------------------------------- the end of a training step
def make_head_cfg(hidden, vocab, tokens, dtype=HH_BF16) -> hh_head_cfg:
    return hh_head_cfg(hidden, vocab, tokens, dtype)


def hh_head_sizes(cfg: hh_head_cfg) -> tuple[int, int]:
    """-> workspace bytes of (hh_head_loss, hh_head_step)"""
    a, b = C.c_size_t(), C.c_size_t()
    _check(lib.hh_head_sizes(C.byref(cfg), C.byref(a), C.byref(b)))
    return a.value, b.value


def hh_head_loss(ctx, cfg: hh_head_cfg, x, w, labels, loss, workspace, stream=0) -> None:
    """labels: int64, negative where a token does not count."""
    _check(lib.hh_head_loss(ctx, C.byref(cfg), _ptr(x), _ptr(w), _ptr(labels), _ptr(loss), _ptr(workspace), stream))


def hh_head_step(ctx, cfg: hh_head_cfg, x, w, labels, dloss, scale, loss, dx, dw, accumulate, workspace, stream=0) -> None:
    """dloss: fp32 upstream gradients of the tokens' losses (times scale), or None for scale alone."""
    _check(lib.hh_head_step(ctx, C.byref(cfg), _ptr(x), _ptr(w), _ptr(labels), _ptr(dloss), float(scale), _ptr(loss), _ptr(dx), _ptr(dw),
                            int(accumulate), _ptr(workspace), stream))


def hh_head_share_fwd(ctx, cfg: hh_head_cfg, x, w, labels, first, lse, picked, workspace, stream=0) -> None:
    """w: words first .. first + cfg.vocab - 1 of the vocabulary that the labels count in."""
    _check(lib.hh_head_share_fwd(ctx, C.byref(cfg), _ptr(x), _ptr(w), _ptr(labels), int(first), _ptr(lse), _ptr(picked), _ptr(workspace), stream))


def hh_head_share_bwd(ctx, cfg: hh_head_cfg, x, w, labels, first, lse, dloss, scale, dx, dw, accumulate, workspace, stream=0) -> None:
    """lse: of the whole vocabulary; dx: this share's partial sum."""
    _check(lib.hh_head_share_bwd(ctx, C.byref(cfg), _ptr(x), _ptr(w), _ptr(labels), int(first), _ptr(lse), _ptr(dloss), float(scale), _ptr(dx),
                                 _ptr(dw), int(accumulate), _ptr(workspace), stream))


_DTYPES = {torch.float32: HH_F32, torch.bfloat16: HH_BF16}


def _dtype(t) -> int:
    if t.dtype not in _DTYPES:
        raise TypeError("tensors of a list are float32 or bfloat16, not %s" % t.dtype)
    return _DTYPES[t.dtype]


def _flat(*ts) -> int:
    """Elements of tensors that go together; they are walked as they lie in memory."""
    n = ts[0].numel()
    for t in ts:
        if not t.is_contiguous() or t.numel() != n:
            raise ValueError("tensors that go together are contiguous and of one size")
    return n


def make_clip_tensors(pairs: Sequence):
    """(gradient, tensor for the clipped copy or None) each -> the list that hh_grad_clip takes.  It holds addresses: the tensors
    have to stay alive as long as it is used."""
    out = (hh_clip_tensor * len(pairs))()
    for e, (g, o) in zip(out, pairs):
        if o is not None and o.dtype != g.dtype:
            raise TypeError("a clipped copy has its gradient's type")
        e.g, e.out, e.count, e.dtype = _ptr(g), _ptr(o), _flat(g) if o is None else _flat(g, o), _dtype(g)
    return out


def hh_grad_clip(ctx, tensors, max_norm, result, workspace, stream=0) -> None:
    """tensors: of make_clip_tensors; result: two fp32 values (norm, factor) on the device; workspace: HH_CLIP_WORKSPACE_BYTES."""
    _check(lib.hh_grad_clip(ctx, len(tensors), tensors, float(max_norm), _ptr(result), _ptr(workspace), stream))


def make_adamw_tensors(rows: Sequence):
    """(parameter, fp32 master copy or None, m, v, gradient, weight decay) each -> the list that hh_adamw_step takes.  It holds
    addresses: the tensors have to stay alive as long as it is used."""
    out = (hh_adamw_tensor * len(rows))()
    for e, (p, master, m, v, g, decay) in zip(out, rows):
        for t in (m, v) + (() if master is None else (master,)):
            if t.dtype != torch.float32:
                raise TypeError("master copies and moments are float32")
        e.count = _flat(*(t for t in (p, master, m, v, g) if t is not None))
        e.param, e.master, e.m, e.v, e.g, e.decay = _ptr(p), _ptr(master), _ptr(m), _ptr(v), _ptr(g), decay
        e.param_dtype, e.grad_dtype = _dtype(p), _dtype(g)
    return out


def make_adamw_cfg(lr, beta1=0.9, beta2=0.95, eps=1e-8, step=1) -> hh_adamw_cfg:
    return hh_adamw_cfg(lr, beta1, beta2, eps, step)


def hh_adamw_step(ctx, cfg: hh_adamw_cfg, tensors, factor=None, stream=0) -> None:
    """tensors: of make_adamw_tensors; factor: one fp32 value on the device (result[1:] of hh_grad_clip) or None."""
    _check(lib.hh_adamw_step(ctx, C.byref(cfg), len(tensors), tensors, _ptr(factor), stream))


# ---------------------------------------------------------------- residual path and microscaled products
def _ref(struct):
    return None if struct is None else C.byref(struct)


def make_dropout(p, seed, offset=0, step=None) -> hh_dropout_cfg:
    """step: a tensor of one int64 on the device that is added to offset when the kernel runs, or None.  It has to stay alive."""
    return hh_dropout_cfg(seed, offset, _ptr(step), p)


def hh_dropout(ctx, drop: hh_dropout_cfg, rows, cols, dtype, x, ldx, y, ldy, stream=0) -> None:
    _check(lib.hh_dropout(ctx, _ref(drop), rows, cols, dtype, _ptr(x), ldx, _ptr(y), ldy, stream))


def make_mx(codes, scales) -> hh_mx_tensor:
    """A packed tensor in the caller's buffers (of hh_mx_sizes bytes).  It holds addresses: the buffers have to stay alive."""
    return hh_mx_tensor(_ptr(codes), _ptr(scales))


def hh_mx_sizes(format, rows, k) -> tuple[int, int]:
    """-> bytes of (codes, scales)"""
    a, b = C.c_size_t(), C.c_size_t()
    _check(lib.hh_mx_sizes(format, rows, k, C.byref(a), C.byref(b)))
    return a.value, b.value


def hh_mx_quantise(ctx, rows, cols, dtype, x, ldx, format, by_row: hh_mx_tensor | None, by_column: hh_mx_tensor | None, stream=0) -> None:
    _check(lib.hh_mx_quantise(ctx, rows, cols, dtype, _ptr(x), ldx, format, _ref(by_row), _ref(by_column), stream))


def hh_mx_values(ctx, rows, k, format, q: hh_mx_tensor, dtype, y, ldy, stream=0) -> None:
    _check(lib.hh_mx_values(ctx, rows, k, format, _ref(q), dtype, _ptr(y), ldy, stream))


def make_add_norm_cfg(rows, hidden, eps=1e-5, dtype=HH_BF16, format=HH_MX_NONE) -> hh_add_norm_cfg:
    return hh_add_norm_cfg(rows, hidden, eps, dtype, format)


def hh_add_norm_fwd(ctx, cfg: hh_add_norm_cfg, drop: hh_dropout_cfg | None, x, b, g, h, xn, q: hh_mx_tensor | None, stream=0) -> None:
    _check(lib.hh_add_norm_fwd(ctx, C.byref(cfg), _ref(drop), _ptr(x), _ptr(b), _ptr(g), _ptr(h), _ptr(xn), _ref(q), stream))


def hh_add_norm_sizes(cfg: hh_add_norm_cfg) -> int:
    """-> workspace bytes of hh_add_norm_bwd"""
    a = C.c_size_t()
    _check(lib.hh_add_norm_sizes(C.byref(cfg), C.byref(a)))
    return a.value


def hh_add_norm_bwd(ctx, cfg: hh_add_norm_cfg, drop: hh_dropout_cfg | None, h, g, dxn, dh, dx, db, dg, accumulate, workspace, stream=0) -> None:
    _check(lib.hh_add_norm_bwd(ctx, C.byref(cfg), _ref(drop), _ptr(h), _ptr(g), _ptr(dxn), _ptr(dh), _ptr(dx), _ptr(db), _ptr(dg),
                               int(accumulate), _ptr(workspace), stream))


def make_mx_product_cfg(m, n, k, a_format, b_format, dtype=HH_BF16, ldc=None, sums=HH_MX_SUMS_F32) -> hh_mx_product_cfg:
    return hh_mx_product_cfg(m, n, k, a_format, b_format, dtype, n if ldc is None else ldc, sums)


def hh_mx_product_sizes(cfg: hh_mx_product_cfg) -> int:
    """-> workspace bytes"""
    a = C.c_size_t()
    _check(lib.hh_mx_product_sizes(C.byref(cfg), C.byref(a)))
    return a.value


def hh_mx_product(ctx, cfg: hh_mx_product_cfg, a: hh_mx_tensor, b: hh_mx_tensor, c, accumulate, workspace, stream=0) -> None:
    _check(lib.hh_mx_product(ctx, C.byref(cfg), _ref(a), _ref(b), _ptr(c), int(accumulate), _ptr(workspace), stream))
