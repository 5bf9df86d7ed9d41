"""ctypes binding of libbase.so (the C ABI in include/base.h).

Argument marshalling only: torch tensors in, raw device pointers and sizes
out, the caller's current HIP stream, and a Python exception for a negative
status.  Every step of the computation runs in the library's HIP kernels.
The library must be built (``paper_2609_36222_amd.build``); loading fails
loudly otherwise -- there is no fallback.
"""
from __future__ import annotations

import ctypes
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "_lib", "libbase.so")

BASE_F32, BASE_BF16 = 0, 1
W_ROWMAJOR, W_PACKED, W_MXFP4 = 0, 1, 4
GATE_PAPER, GATE_RENORM = 0, 1
FILL_BACKFILL, FILL_DROP = 0, 2
SCORE_BASE, SCORE_TOP1, SCORE_WEIGHT, SCORE_WEIGHT_SQ, SCORE_STATIC = 0, 1, 2, 3, 4

EXPORTS = ("base_workspace_bytes", "base_route", "base_predict_cost",
           "base_select", "base_moe_forward", "base_decode_layer",
           "base_decode_layer_noalloc",
           "base_pack_experts", "base_set_stage_events", "base_layer_stages",
           "base_status_string",
           "base_calib_stats_bytes", "base_calib_ws_bytes", "base_calib_reset",
           "base_calib_accumulate",
           "base_mx_quantize", "base_mx_dequantize", "base_mx_w13_bytes", "base_mx_w2_bytes",
           "base_mx_pack_experts", "base_mx_quantize_experts",
           "base_norm_residual", "base_decode_block",
           "base_head_rope", "base_kv_append", "base_attention_workspace_bytes",
           "base_paged_attention")
CALIB_LIB_PATH = os.path.join(HERE, "_lib", "libbase_calib.so")
N_STAGES = 9     # one kernel each; base_set_stage_events takes 2 events per stage
STAGES = ("scores", "tail", "select", "backfill", "compact", "gather",
          "ffn_gateup", "ffn_down", "combine")

_vp = ctypes.c_void_p
_i32 = ctypes.c_int32
_i64 = ctypes.c_int64


class base_layer(ctypes.Structure):
    _fields_ = [("d", _i32), ("E", _i32), ("K", _i32), ("I", _i32),
                ("dtype", _i32), ("norm_topk", _i32), ("w_layout", _i32),
                ("score_rule", _i32), ("w_router", _vp), ("b_router", _vp), ("pred_a", _vp),
                ("pred_b", _vp), ("w13", _vp), ("w2", _vp),
                ("n_shared", _i32), ("w13_shared", _vp), ("w2_shared", _vp),
                ("shared_gate", _vp)]


_PLAN_FIELDS = ["logits", "topk_ids", "topk_w", "cost", "scores", "counts",
                "sel_ids", "n_sel", "slot_of_expert", "exec_ids", "exec_gates",
                "offsets", "pair_tok", "pair_gate", "pair_of"]


class base_plan(ctypes.Structure):
    _fields_ = [(f, _vp) for f in _PLAN_FIELDS]


class base_norms(ctypes.Structure):
    _fields_ = [("d", _i32), ("dtype", _i32), ("eps", ctypes.c_float),
                ("res_scale", ctypes.c_float), ("post_gain", _vp), ("gate", _vp),
                ("gate_ld", _i64), ("pre_gain", _vp)]


class base_rope(ctypes.Structure):
    _fields_ = [("D", _i32), ("rot", _i32), ("dtype", _i32), ("layout", _i32),
                ("eps", ctypes.c_float), ("rot_scale", ctypes.c_float), ("inv_freq", _vp),
                ("q_gain", _vp), ("k_gain", _vp)]


class base_kv_cache(ctypes.Structure):
    _fields_ = [("Hk", _i32), ("D", _i32), ("dtype", _i32), ("page_size", _i32),
                ("n_pages", _i32), ("k", _vp), ("v", _vp), ("k_page", _i64), ("k_slot", _i64),
                ("k_head", _i64), ("v_page", _i64), ("v_slot", _i64), ("v_head", _i64)]


class base_kv_batch(ctypes.Structure):
    _fields_ = [("n_seq", _i32), ("max_pages", _i32), ("table_ld", _i64), ("max_q", _i32),
                ("table", _vp), ("q_start", _vp), ("kv_len", _vp)]


class BaseError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__(f"{msg} (status {status})")
        self.status = status


_lib = None


def load(path: str = LIB_PATH):
    """Load libbase.so; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    # torch first: libbase.so then binds to the HIP runtime torch loaded
    # (same SONAME), so streams and events are shared with torch
    import torch  # noqa: F401
    if not os.path.exists(path):
        raise ImportError(
            f"{path} is missing: build it with "
            "`python -m paper_2609_36222_amd.build` (no CPU fallback exists)")
    L = ctypes.CDLL(path)
    L.base_workspace_bytes.restype = ctypes.c_size_t
    L.base_workspace_bytes.argtypes = [ctypes.POINTER(base_layer), _i32, _i32]
    L.base_route.restype = _i32
    L.base_route.argtypes = [ctypes.POINTER(base_layer), _vp, _i32, _vp, _vp,
                             _vp, _vp]
    L.base_predict_cost.restype = _i32
    L.base_predict_cost.argtypes = [ctypes.POINTER(base_layer), _vp, _i32,
                                    _vp, _vp, _vp, _vp]
    L.base_select.restype = _i32
    L.base_select.argtypes = [ctypes.POINTER(base_layer), _i32, _vp, _vp,
                              _i32, _vp, _vp, _vp, _vp, _vp, _vp]
    L.base_moe_forward.restype = _i32
    L.base_moe_forward.argtypes = [ctypes.POINTER(base_layer), _vp, _i32, _vp,
                                   _vp, _vp, _vp, _vp, _i32, _i32, _vp, _vp,
                                   ctypes.POINTER(base_plan), _vp,
                                   ctypes.c_size_t, _vp]
    L.base_decode_layer.restype = _i32
    L.base_decode_layer.argtypes = [ctypes.POINTER(base_layer), _vp, _i32,
                                    _i32, _i32, _vp, _vp,
                                    ctypes.POINTER(base_plan), _vp,
                                    ctypes.c_size_t, _vp]
    L.base_decode_layer_noalloc.restype = _i32
    L.base_decode_layer_noalloc.argtypes = [ctypes.POINTER(base_layer), _vp, _i32,
                                            _i32, _i32, _vp, _vp,
                                            ctypes.POINTER(base_plan), _vp]
    L.base_pack_experts.restype = _i32
    L.base_pack_experts.argtypes = [ctypes.POINTER(base_layer), _vp, _vp, _vp]
    L.base_set_stage_events.restype = _i32
    L.base_set_stage_events.argtypes = [ctypes.POINTER(ctypes.c_void_p), _i32]
    L.base_layer_stages.restype = _i32
    L.base_layer_stages.argtypes = [ctypes.POINTER(base_layer), _i32, _i32,
                                    ctypes.POINTER(_i32)]
    L.base_status_string.restype = ctypes.c_char_p
    L.base_status_string.argtypes = [_i32]
    L.base_calib_stats_bytes.restype = ctypes.c_size_t
    L.base_calib_stats_bytes.argtypes = [ctypes.POINTER(base_layer)]
    L.base_calib_ws_bytes.restype = ctypes.c_size_t
    L.base_calib_ws_bytes.argtypes = [ctypes.POINTER(base_layer), _i32]
    L.base_calib_reset.restype = _i32
    L.base_calib_reset.argtypes = [ctypes.POINTER(base_layer), _vp, _vp]
    L.base_calib_accumulate.restype = _i32
    L.base_calib_accumulate.argtypes = [ctypes.POINTER(base_layer), _vp, _i32, _vp, _vp,
                                        ctypes.c_size_t, _vp]
    L.base_mx_quantize.restype = _i32
    L.base_mx_quantize.argtypes = [_i32, _vp, _i64, _i32, _i64, _vp, _vp, _vp]
    L.base_mx_dequantize.restype = _i32
    L.base_mx_dequantize.argtypes = [_vp, _vp, _i64, _i32, _i32, _vp, _i64, _vp]
    for f in (L.base_mx_w13_bytes, L.base_mx_w2_bytes):
        f.restype = ctypes.c_size_t
        f.argtypes = [ctypes.POINTER(base_layer)]
    L.base_mx_pack_experts.restype = _i32
    L.base_mx_pack_experts.argtypes = [ctypes.POINTER(base_layer)] + [_vp] * 7
    L.base_mx_quantize_experts.restype = _i32
    L.base_mx_quantize_experts.argtypes = [ctypes.POINTER(base_layer)] + [_vp] * 3
    L.base_norm_residual.restype = _i32
    L.base_norm_residual.argtypes = [ctypes.POINTER(base_norms), _i64, _vp, _i64, _vp, _i64, _vp,
                                     _i64, _vp, _i64, _vp]
    L.base_decode_block.restype = _i32
    L.base_decode_block.argtypes = [ctypes.POINTER(base_layer), ctypes.POINTER(base_norms), _vp,
                                    _i32, _i32, _i32, _vp, _vp, _vp, ctypes.POINTER(base_plan),
                                    _vp, ctypes.c_size_t, _vp]
    heads = [_vp, _i64, _i64]
    cache, batch = ctypes.POINTER(base_kv_cache), ctypes.POINTER(base_kv_batch)
    L.base_head_rope.restype = _i32
    L.base_head_rope.argtypes = [ctypes.POINTER(base_rope), _i64, _vp, *2 * [_i32, *2 * heads], _vp]
    L.base_kv_append.restype = _i32
    L.base_kv_append.argtypes = [ctypes.POINTER(base_rope), cache, batch, _i64, _vp, _i32, *4 * heads, _vp]
    L.base_attention_workspace_bytes.restype = ctypes.c_size_t
    L.base_attention_workspace_bytes.argtypes = [cache, batch, _i64, _i32]
    L.base_paged_attention.restype = _i32
    L.base_paged_attention.argtypes = [cache, batch, _i64, _i32, *2 * heads, _vp, ctypes.c_float, _i32,
                                       _vp, ctypes.c_size_t, _vp]
    _lib = L
    return L


_calib = None


def load_calib(path: str = CALIB_LIB_PATH):
    """Load libbase_calib.so (the predictor fit, base_calib.h)."""
    global _calib
    if _calib is not None:
        return _calib
    load()
    if not os.path.exists(path):
        raise ImportError(f"{path} is missing: build it with "
                          "`python -m paper_2609_36222_amd.build`")
    L = ctypes.CDLL(path)
    L.base_calib_fit.restype = _i32
    L.base_calib_fit.argtypes = [ctypes.POINTER(base_layer), _vp, _i32,
                                 ctypes.POINTER(ctypes.c_double), _vp, _vp, _vp, _vp]
    _calib = L
    return L


def status_string(status: int) -> str:
    return load().base_status_string(int(status)).decode()


def _check(status):
    if status != 0:
        raise BaseError(status, status_string(status))


def _ptr(t):
    """Device pointer of a tensor (None -> NULL)."""
    if t is None:
        return None
    return t.data_ptr()


def _stream(stream):
    import torch
    if stream is None:
        # the current stream's handle without a Stream object around it (3 us a call)
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return stream.cuda_stream


def _empty(near, shape, dtype, stream):
    """A new tensor on near's device for a kernel on `stream` to write, in that stream's
    memory (as under torch.cuda.stream(stream)): memory of the current stream may still
    be read or written by what was enqueued there before its last tensor was freed."""
    if stream is None:
        return near.new_empty(shape, dtype=dtype)
    import torch
    with torch.cuda.stream(stream if isinstance(stream, torch.cuda.Stream) else None):
        return near.new_empty(shape, dtype=dtype)


class Layer:
    """One MoE layer: torch tensors plus the C descriptor pointing at them.

    w_router, b_router, pred_a, pred_b: fp32; w13 [E,2I,d], w2 [E,d,I]:
    fp32 or bf16 (the layer dtype, also the dtype of x and y).  shared:
    None or (w13_shared [S,2I,d], w2_shared [S,d,I], gate [d] fp32 or
    None), the always-active shared experts."""

    def __init__(self, w_router, b_router, pred_a, pred_b, w13, w2,
                 norm_topk: int = 1, w_layout: int = 0, score_rule: int = 0,
                 shared=None):
        import torch
        E, d = w_router.shape
        I = w2.shape[2]
        K = None
        self.tensors = (w_router, b_router, pred_a, pred_b, w13, w2)
        self.dtype = BASE_BF16 if w13.dtype == torch.bfloat16 else BASE_F32
        self.torch_dtype = w13.dtype
        self.d, self.E, self.I, self.K = d, E, I, K
        self.norm_topk = norm_topk
        self.w_layout = w_layout
        self.score_rule = score_rule
        self.shared = shared
        self._desc = None

    @classmethod
    def mxfp4(cls, w_router, b_router, pred_a, pred_b, w13, w2, I: int, norm_topk: int = 1,
              score_rule: int = 0, shared=None):
        """A layer of 4-bit experts: w13, w2 (and the shared ones) are the byte
        tensors base_mx_pack_experts / base_mx_quantize_experts wrote, whose
        lengths have to be those of the router's experts and I; shared:
        (w13_shared, w2_shared, gate or None, how many)."""
        import torch
        E, d = w_router.shape
        _mx_bytes("w13, w2", w13, w2, E, d, I, w_router)
        if shared is not None and shared[3] != 0:
            _mx_bytes("shared w13, w2", *shared[:2], shared[3], d, I, w_router)
            gate = shared[2]
            if gate is not None and (gate.dtype is not torch.float32 or gate.shape != (d,)
                                     or not gate.is_contiguous()):
                raise ValueError(f"shared gate: fp32, {d} adjacent elements")
        self = cls.__new__(cls)
        self.tensors = (w_router, b_router, pred_a, pred_b, w13, w2)
        self.dtype, self.torch_dtype = BASE_BF16, torch.bfloat16
        self.E, self.d, self.I, self.K = E, d, I, None
        self.norm_topk, self.w_layout, self.score_rule = norm_topk, W_MXFP4, score_rule
        self.shared = shared
        self._desc = None
        return self

    def desc(self, K: int) -> base_layer:
        w_router, b_router, pred_a, pred_b, w13, w2 = self.tensors
        return base_layer(self.d, self.E, K, self.I, self.dtype,
                          self.norm_topk, self.w_layout, self.score_rule,
                          _ptr(w_router), _ptr(b_router),
                          _ptr(pred_a), _ptr(pred_b), _ptr(w13), _ptr(w2),
                          *self._shared_fields())

    def _shared_fields(self):
        if self.shared is None:
            return (0, None, None, None)
        w13s, w2s, gate = self.shared[:3]
        n = self.shared[3] if self.w_layout == W_MXFP4 else w13s.shape[0]
        return (int(n), _ptr(w13s), _ptr(w2s), _ptr(gate))


def base_workspace_bytes(desc: base_layer, B: int, budget: int) -> int:
    return int(load().base_workspace_bytes(ctypes.byref(desc), B, budget))


def base_route(desc, x, B, logits, topk_ids, topk_w, stream=None):
    _check(load().base_route(ctypes.byref(desc), _ptr(x), B, _ptr(logits),
                             _ptr(topk_ids), _ptr(topk_w), _stream(stream)))


def base_predict_cost(desc, x, B, topk_ids, topk_w, cost, stream=None):
    _check(load().base_predict_cost(ctypes.byref(desc), _ptr(x), B,
                                    _ptr(topk_ids), _ptr(topk_w), _ptr(cost),
                                    _stream(stream)))


def base_select(desc, B, topk_ids, cost, budget, scores, counts, sel_ids,
                n_sel, slot_of_expert, stream=None):
    _check(load().base_select(ctypes.byref(desc), B, _ptr(topk_ids),
                              _ptr(cost), budget, _ptr(scores), _ptr(counts),
                              _ptr(sel_ids), _ptr(n_sel),
                              _ptr(slot_of_expert), _stream(stream)))


def base_moe_forward(desc, x, B, logits, topk_ids, sel_ids, n_sel,
                     slot_of_expert, budget, flags, residual, y, ws,
                     plan=None, stream=None):
    """Returns the filled base_plan (device pointers into ws)."""
    plan = base_plan() if plan is None else plan
    _check(load().base_moe_forward(
        ctypes.byref(desc), _ptr(x), B, _ptr(logits), _ptr(topk_ids),
        _ptr(sel_ids), _ptr(n_sel), _ptr(slot_of_expert), budget, flags,
        _ptr(residual), _ptr(y), ctypes.byref(plan), _ptr(ws),
        ws.numel() * ws.element_size(), _stream(stream)))
    return plan


def base_decode_layer(desc, x, B, budget, flags, residual, y, ws, plan=None,
                      stream=None):
    """Returns the filled base_plan (device pointers into ws)."""
    plan = base_plan() if plan is None else plan
    _check(load().base_decode_layer(
        ctypes.byref(desc), _ptr(x), B, budget, flags, _ptr(residual), _ptr(y),
        ctypes.byref(plan), _ptr(ws), ws.numel() * ws.element_size(),
        _stream(stream)))
    return plan


def base_decode_layer_noalloc(desc, x, B, budget, flags, residual, y, plan=None,
                              stream=None):
    """base_decode_layer on the library's own scratch array (no workspace
    argument, nothing allocated); returns the filled base_plan (device
    pointers into that array)."""
    plan = base_plan() if plan is None else plan
    _check(load().base_decode_layer_noalloc(
        ctypes.byref(desc), _ptr(x), B, budget, flags, _ptr(residual), _ptr(y),
        ctypes.byref(plan), _stream(stream)))
    return plan


NOALLOC_SCRATCH_BYTES = 64 << 20


def base_pack_experts(desc, w13_packed, w2_packed, stream=None):
    _check(load().base_pack_experts(ctypes.byref(desc), _ptr(w13_packed),
                                    _ptr(w2_packed), _stream(stream)))


def packed_layer(layer: "Layer", K: int, stream=None) -> "Layer":
    """A Layer sharing router/predictor tensors, with expert weights packed
    into new tensors by base_pack_experts (one-time, on the device)."""
    w_router, b_router, pred_a, pred_b, w13, w2 = layer.tensors
    w13p, w2p = (_empty(t, t.shape, t.dtype, stream) for t in (w13, w2))
    base_pack_experts(layer.desc(K), w13p, w2p, stream)
    shared = None
    if layer.shared is not None:
        w13s, w2s, gate = layer.shared
        d = base_layer(layer.d, int(w13s.shape[0]), 1, layer.I, layer.dtype, layer.norm_topk,
                       W_ROWMAJOR, 0, None, None, None, None, _ptr(w13s), _ptr(w2s),
                       0, None, None, None)
        w13sp, w2sp = (_empty(t, t.shape, t.dtype, stream) for t in (w13s, w2s))
        base_pack_experts(d, w13sp, w2sp, stream)
        shared = (w13sp, w2sp, gate)
    return Layer(w_router, b_router, pred_a, pred_b, w13p, w2p,
                 layer.norm_topk, W_PACKED, layer.score_rule, shared)


def _device():
    """The current GPU, where the launches go and the tensors have to lie."""
    import torch
    return torch._C._cuda_getDevice() if torch.cuda.is_initialized() else 0


def _rows(t, what, dev):
    """(dtype, rows, cols, row stride) of a 2-D tensor with adjacent columns."""
    import torch
    dt = t.dtype
    if t.dim() != 2 or (dt is not torch.bfloat16 and dt is not torch.float32):
        raise ValueError(f"{what}: a 2-D fp32 or bf16 tensor")
    rows, cols = t.shape
    ld, one = t.stride()
    if t.get_device() != dev or (cols > 1 and one != 1):
        raise ValueError(f"{what}: adjacent columns, on the current GPU")
    return BASE_BF16 if dt is torch.bfloat16 else BASE_F32, rows, cols, ld if rows > 1 else cols


# Microscaled 4-bit floating point (E2M1 codes, an E8M0 scale per 32 elements)
def mx_quantize(src, codes=None, scales=None, stream=None):
    """codes [rows, cols / 2] and scales [rows, cols / 32] (uint8) of src
    [rows, cols], into the two tensors given or into new ones; src's rows may
    lie inside wider ones."""
    import torch
    dev = _device()
    dt, rows, cols, ld = _rows(src, "src", dev)
    if codes is None and scales is None:
        codes = _empty(src, (rows, cols // 2), torch.uint8, stream)
        scales = _empty(src, (rows, cols // 32), torch.uint8, stream)
    else:
        _mx_shapes(codes, scales, (rows,), cols, dev)
    _check(load().base_mx_quantize(dt, _ptr(src), rows, cols, ld, _ptr(codes), _ptr(scales),
                                   _stream(stream)))
    return codes, scales


def mx_dequantize(codes, scales, dtype=None, out=None, stream=None):
    """The values [rows, cols] as `dtype` (bf16), or into `out`."""
    import torch
    rows, cols = codes.shape[0], 2 * codes.shape[1]
    dev = _device()
    _mx_shapes(codes, scales, (rows,), cols, dev)
    if out is None:
        dtype = dtype or torch.bfloat16
        if dtype not in (torch.bfloat16, torch.float32):
            raise ValueError("dtype: fp32 or bf16")
        out = _empty(codes, (rows, cols), dtype, stream)
        dt, ld = BASE_BF16 if dtype is torch.bfloat16 else BASE_F32, cols
    else:
        dt, r, c, ld = _rows(out, "out", dev)
        if (r, c) != (rows, cols):
            raise ValueError("out: the codes' rows and columns")
    _check(load().base_mx_dequantize(_ptr(codes), _ptr(scales), rows, cols, dt, _ptr(out), ld,
                                     _stream(stream)))
    return out


def _mx_shapes(codes, scales, lead, cols, dev):
    import torch
    for t, n, what in ((codes, cols // 2, "codes"), (scales, cols // 32, "scales")):
        if (t is None or t.dtype is not torch.uint8 or t.shape != (*lead, n) or not t.is_contiguous()
                or t.get_device() != dev):
            raise ValueError(f"{what}: contiguous uint8 {[*lead, n]} on the current GPU")


def _mx_desc(E, d, I, dtype=BASE_BF16, w13=None, w2=None):
    return base_layer(d, E, 1, I, dtype, 1, W_ROWMAJOR, 0, None, None, None, None, _ptr(w13),
                      _ptr(w2), 0, None, None, None)


def _mx_sizes(desc):
    n13, n2 = (int(f(ctypes.byref(desc))) for f in (load().base_mx_w13_bytes,
                                                    load().base_mx_w2_bytes))
    if n13 == 0:
        raise BaseError(-2, status_string(-2))
    return n13, n2


def _mx_bytes(what, w13, w2, n, d, I, near):
    """Packed experts have the bytes of n experts of this shape, where `near` lies: the
    kernels take their sizes from the shape."""
    import torch
    for t, size in zip((w13, w2), _mx_sizes(_mx_desc(n, d, I))):
        if (t.dtype is not torch.uint8 or t.numel() != size or not t.is_contiguous()
                or t.device != near.device):
            raise ValueError(f"{what}: the packed bytes of {n} experts with d = {d}, I = {I} "
                             f"({size}, not {t.numel()}), on the router's device")


def _mx_same_shape(what, w13, w2, n, d, I):
    """w13 [n, 2I, d] and w2 [n, d, I] by their shapes."""
    if w13 != (n, 2 * I, d) or w2 != (n, d, I):
        raise ValueError(f"{what}: [{n}, {2 * I}, {d}] and [{n}, {d}, {I}], not {list(w13)} and {list(w2)}")


def _mx_out(desc, near, stream):
    import torch
    return tuple(_empty(near, (n,), torch.uint8, stream) for n in _mx_sizes(desc))


def mx_quantize_experts(w13, w2, stream=None):
    """Row-major experts w13 [E, 2I, d], w2 [E, d, I] (bf16 or fp32) as the byte
    tensors of a W_MXFP4 layer."""
    import torch
    E, d, I = w2.shape
    if (w13.shape != (E, 2 * I, d) or w13.dtype != w2.dtype
            or w13.dtype not in (torch.bfloat16, torch.float32)
            or any(not t.is_contiguous() or t.get_device() != _device() for t in (w13, w2))):
        raise ValueError("w13 [E, 2I, d] and w2 [E, d, I], contiguous fp32 or bf16 on the current GPU")
    desc = _mx_desc(E, d, I, BASE_BF16 if w13.dtype == torch.bfloat16 else BASE_F32, w13, w2)
    out = _mx_out(desc, w13, stream)
    _check(load().base_mx_quantize_experts(ctypes.byref(desc), _ptr(out[0]), _ptr(out[1]),
                                           _stream(stream)))
    return out


def mx_pack_experts(w13, w2, stream=None):
    """The same from (codes, scales) pairs: w13 [E, 2I, d / 2] and [E, 2I, d / 32],
    w2 [E, d, I / 2] and [E, d, I / 32]."""
    E, d = w2[0].shape[:2]
    I = 2 * w2[0].shape[2]
    _mx_shapes(*w13, (E, 2 * I), d, _device())
    _mx_shapes(*w2, (E, d), I, _device())
    desc = _mx_desc(E, d, I)
    out = _mx_out(desc, w13[0], stream)
    _check(load().base_mx_pack_experts(ctypes.byref(desc), *(_ptr(t) for t in (*w13, *w2, *out)),
                                       _stream(stream)))
    return out


def mx_layer(layer: "Layer", stream=None) -> "Layer":
    """A W_MXFP4 Layer (bf16 activations) with a row-major layer's experts, fp32 or
    bf16, quantised, sharing its router and predictor tensors (one-time, on the
    device)."""
    w_router, b_router, pred_a, pred_b, w13, w2 = layer.tensors
    if layer.w_layout != W_ROWMAJOR:
        raise ValueError("row-major experts")
    _mx_same_shape("w13, w2", tuple(w13.shape), tuple(w2.shape), layer.E, layer.d, layer.I)
    shared = None
    if layer.shared is not None:
        w13s, w2s, gate = layer.shared
        _mx_same_shape("shared w13, w2", tuple(w13s.shape), tuple(w2s.shape), int(w13s.shape[0]),
                       layer.d, layer.I)
        shared = (*mx_quantize_experts(w13s, w2s, stream), gate, int(w13s.shape[0]))
    return Layer.mxfp4(w_router, b_router, pred_a, pred_b, *mx_quantize_experts(w13, w2, stream),
                       layer.I, layer.norm_topk, layer.score_rule, shared)


def mx_layer_from_codes(w_router, b_router, pred_a, pred_b, w13, w2, norm_topk: int = 1,
                        score_rule: int = 0, shared=None, stream=None) -> "Layer":
    """A W_MXFP4 Layer from experts held as (codes, scales) pairs (mx_pack_experts);
    shared: None or (w13 pair, w2 pair, gate or None)."""
    E, d = w_router.shape
    I = 2 * w2[0].shape[2]
    values = lambda q: (*q[0].shape[:-1], 2 * q[0].shape[-1])  # noqa: E731
    _mx_same_shape("w13, w2", values(w13), values(w2), E, d, I)
    if shared is not None:
        w13s, w2s, gate = shared
        _mx_same_shape("shared w13, w2", values(w13s), values(w2s), int(w13s[0].shape[0]), d, I)
        shared = (*mx_pack_experts(w13s, w2s, stream), gate, int(w13s[0].shape[0]))
    return Layer.mxfp4(w_router, b_router, pred_a, pred_b, *mx_pack_experts(w13, w2, stream),
                       I, norm_topk, score_rule, shared)


class Norms:
    """The parameters of the norms around a block (base_norms): fp32 gains [d], a
    gate [d] (every row's) or [rows, d] (each row its own), the residual scale."""

    def __init__(self, d, dtype, post_gain=None, gate=None, pre_gain=None, res_scale=1.0, eps=1e-6):
        import torch
        if dtype is not torch.bfloat16 and dtype is not torch.float32:
            raise ValueError("dtype: fp32 or bf16")
        self.tensors = (post_gain, gate, pre_gain)
        self.d, self.torch_dtype, self.gate_rows = d, dtype, None
        dev, f32 = _device(), torch.float32
        ptr, ld = [None, None, None], 0
        for i, t in enumerate(self.tensors):
            if t is None:
                continue
            n, s = t.shape, t.stride()
            two = i == 1 and len(n) == 2
            if (t.dtype is not f32 or not (two or len(n) == 1) or n[-1] != d
                    or (s[-1] != 1 and d > 1) or t.get_device() != dev):
                raise ValueError(f"{('post_gain', 'gate', 'pre_gain')[i]}: fp32, {d} adjacent elements "
                                 "a row, on the current GPU")
            if two:
                self.gate_rows = n[0]
                ld = s[0] if n[0] > 1 else d
            ptr[i] = t.data_ptr()
        self.desc = base_norms(d, BASE_BF16 if dtype is torch.bfloat16 else BASE_F32, eps, res_scale,
                               ptr[0], ptr[1], ld, ptr[2])

    def _pointers(self, rows, dev, tensors, block):
        """The row count checked (the gate's where there is a block, else it is not
        read), and (pointer, row stride) of each tensor (of y, h, h_out, x_out, in this
        order)."""
        if block and self.gate_rows is not None and self.gate_rows != rows:
            raise ValueError(f"gate: one row, or {rows}")
        out, d, dt = [], self.d, self.torch_dtype
        shape = (rows, d)
        for i, t in enumerate(tensors):
            if t is None:
                out += (None, 0)
                continue
            if t.dtype is not dt or t.shape != shape or t.get_device() != dev:
                raise ValueError(f"{('y', 'h', 'h_out', 'x_out')[i]}: {dt} {list(shape)} on the current GPU")
            ld, one = t.stride()
            if one != 1 and d > 1:
                raise ValueError(f"{('y', 'h', 'h_out', 'x_out')[i]}: adjacent columns")
            out += (t.data_ptr(), ld if rows > 1 else d)
        return out


def base_norm_residual(norms: Norms, y, h, h_out=None, x_out=None, stream=None):
    """h_out = res_scale h + gate (post_gain n(y)), x_out = pre_gain n(h_out); [rows, d]
    tensors whose rows may lie inside wider ones; y None: x_out = pre_gain n(h)."""
    rows = h.shape[0]
    a = norms._pointers(rows, _device(), (y, h, h_out, x_out), y is not None)
    _check(load().base_norm_residual(norms.desc, rows, *a, _stream(stream)))


def norm_residual(h, y=None, post_gain=None, gate=None, pre_gain=None, res_scale=1.0, eps=1e-6,
                  h_out=None, x_out=None, stream=None):
    """base_norm_residual with the parameters given here; returns (h_out, x_out), new
    tensors where they are not given (None where there is nothing to write)."""
    n = Norms(h.shape[1], h.dtype, post_gain, gate, pre_gain, res_scale, eps)
    if h_out is None and y is not None:
        h_out = _empty(h, h.shape, h.dtype, stream)   # rows d apart
    if x_out is None and pre_gain is not None:
        x_out = _empty(h, h.shape, h.dtype, stream)
    base_norm_residual(n, y, h, h_out, x_out, stream)
    return h_out, x_out


def base_decode_block(desc, norms: Norms, x, B, budget, flags, h, ws, h_out=None, x_out=None,
                      plan=None, stream=None):
    """base_decode_layer, then base_norm_residual on its output, in the layer's
    launches; returns the filled base_plan (device pointers into ws)."""
    plan = base_plan() if plan is None else plan
    norms._pointers(B, _device(), (None, h, h_out, x_out), True)
    for t, what in ((h, "h"), (h_out, "h_out"), (x_out, "x_out")):
        if t is not None and not t.is_contiguous():
            raise ValueError(f"{what}: contiguous rows")
    _check(load().base_decode_block(
        ctypes.byref(desc), ctypes.byref(norms.desc), _ptr(x), B, budget, flags, _ptr(h),
        _ptr(h_out), _ptr(x_out), ctypes.byref(plan), _ptr(ws), ws.numel() * ws.element_size(),
        _stream(stream)))
    return plan


# Heads: rotation by position, a paged cache, attention over it
ROPE_HALF, ROPE_INTERLEAVED = 0, 1


def rope_frequencies(rot, base=10000.0, factor=1.0, trained=None, fast=32.0, slow=1.0):
    """(inv_freq [rot / 2] fp32 on the CPU, rot_scale) of the angles p base^(-2 i / rot),
    for contexts `factor` times as long as the trained one.  trained None: every angle is
    divided by the factor (rot_scale 1).  Else, with the trained length: pairs that turn
    more than `fast` times over it keep their angle, pairs that turn less than `slow`
    times have it divided, those between a mixture linear in the pair's number from the last
    whole one with `fast` turns (or 0) to the first with `slow` (or rot - 1: it may lie behind
    the last pair); rot_scale = 0.1 ln(factor) + 1."""
    import math

    import torch
    if rot < 0 or rot % 2 or not base > 0 or not factor >= 1:
        raise ValueError("rot even, base > 0, factor >= 1")
    i = torch.arange(rot // 2, dtype=torch.float64)
    inv = float(base) ** (-2.0 * i / max(rot, 1))
    if factor == 1 or rot == 0:
        return inv.float(), 1.0
    if trained is None:
        return (inv / factor).float(), 1.0
    if not fast > slow > 0 or trained < 1 or not base > 1:
        raise ValueError("fast > slow > 0, trained >= 1 and base > 1")
    # the pair that turns n times over the trained length
    pair = lambda n: rot * math.log(trained / (n * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
    lo, hi = max(math.floor(pair(fast)), 0), min(math.ceil(pair(slow)), rot - 1)
    far = ((i - lo) / max(hi - lo, 0.001)).clamp(0, 1)
    far[i > pair(slow)] = 1.0   # (pair 0 too, where none turns so often)
    return (inv * (1 - far) + inv / factor * far).float(), 0.1 * math.log(factor) + 1.0


def _heads(t, what, dtype, dev, n, H, D):
    """(pointer, row stride, head stride) of a tensor [n, H, D] with adjacent elements in a
    head."""
    if t.shape == (n, H, D):
        row, head, one = t.stride()
        if one == 1 and t.dtype is dtype and t.get_device() == dev:
            # (a single row or head has no stride to speak of)
            return t.data_ptr(), row if n > 1 else 0, head if H > 1 else 0
    raise ValueError(f"{what}: {dtype} {[n, H, D]}, adjacent elements in a head, on the current GPU")


def _rows_heads(t, what):
    """Rows and heads of a tensor [n, H, D]."""
    try:
        n, H, _ = t.shape
    except ValueError:
        raise ValueError(f"{what}: [rows, heads, D]") from None
    return n, H


def _here(*made):
    """(the library, torch, the current GPU): what a call on heads looks up once.  made: its
    Rope, KVCache and KVBatch, whose tensors have to lie there."""
    import torch
    dev = torch._C._cuda_getDevice() if torch.cuda.is_initialized() else 0
    for m in made:
        if m.dev != dev:
            raise ValueError(f"{type(m).__name__}: made on GPU {m.dev}, the current one is {dev}")
    return load(), torch, dev


def _stream_on(torch, stream, dev):
    """_stream, where the current device is known."""
    return torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream


def _ints(t, what, dev, shape=None):
    import torch
    if t.dtype is not torch.int32 or t.get_device() != dev or (shape is not None and t.shape != shape):
        raise ValueError(f"{what}: int32{'' if shape is None else ' ' + str(list(shape))} on the current GPU")
    return t


def _flat(t, what, dev, shape=None):
    if not _ints(t, what, dev, shape).is_contiguous():
        raise ValueError(f"{what}: adjacent elements")
    return t


class Rope:
    """Norms of query and key heads with the rotation by position (base_rope): inv_freq
    [rot / 2] fp32 (None: no rotation), fp32 gains [D] or None."""

    def __init__(self, D, dtype, inv_freq=None, interleaved=False, rot_scale=1.0, q_gain=None,
                 k_gain=None, eps=1e-6):
        import torch
        if dtype is not torch.bfloat16 and dtype is not torch.float32:
            raise ValueError("dtype: fp32 or bf16")
        self.dev = dev = _device()
        rot = 0 if inv_freq is None else 2 * inv_freq.numel()
        for t, n, what in ((inv_freq, rot // 2, "inv_freq"), (q_gain, D, "q_gain"), (k_gain, D, "k_gain")):
            if t is not None and (t.dtype is not torch.float32 or t.shape != (n,) or not t.is_contiguous()
                                  or t.get_device() != dev):
                raise ValueError(f"{what}: fp32, {n} adjacent elements, on the current GPU")
        self.tensors = (inv_freq, q_gain, k_gain)
        self.D, self.rot, self.torch_dtype = D, rot, dtype
        self.desc = base_rope(D, rot, BASE_BF16 if dtype is torch.bfloat16 else BASE_F32,
                              ROPE_INTERLEAVED if interleaved else ROPE_HALF, eps, rot_scale,
                              _ptr(inv_freq), _ptr(q_gain), _ptr(k_gain))


class KVCache:
    """A paged cache (base_kv_cache): k and v [pages, page size, Hk, D], fp32 or bf16,
    views with any strides of 16 bytes' multiples (pages that hold their tokens head by
    head are such a view) and adjacent elements in a head."""

    def __init__(self, k, v):
        import torch
        self.dev = dev = _device()
        for t, what in ((k, "k"), (v, "v")):
            if (t.dim() != 4 or t.shape != k.shape or t.dtype is not k.dtype or t.get_device() != dev
                    or t.dtype not in (torch.bfloat16, torch.float32) or t.stride(3) != 1):
                raise ValueError(f"{what}: fp32 or bf16 [pages, page size, heads, D], adjacent elements, k's "
                                 "and v's alike, on the current GPU")
        self.tensors = (k, v)
        self.torch_dtype = k.dtype
        self.n_pages, self.page_size, self.Hk, self.D = k.shape
        ld = [t.stride(i) if t.shape[i] > 1 else 0 for t in (k, v) for i in (0, 1, 2)]
        self.desc = base_kv_cache(self.Hk, self.D, BASE_BF16 if k.dtype is torch.bfloat16 else BASE_F32,
                                  self.page_size, self.n_pages, _ptr(k), _ptr(v), *ld)


class KVBatch:
    """The sequences of a batch (base_kv_batch): int32 table [n_seq, pages], q_start
    [n_seq + 1], kv_len [n_seq]; max_q: the most new tokens of a sequence.  The tensors'
    contents may change between calls."""

    def __init__(self, table, q_start, kv_len, max_q):
        self.dev = dev = _device()
        n = kv_len.shape[0] if kv_len.dim() == 1 else -1
        if table.dim() != 2 or table.shape[0] != n or (table.stride(1) != 1 and table.shape[1] > 1):
            raise ValueError("table: int32 [n_seq, pages], adjacent entries")
        _ints(table, "table", dev)
        self.tensors = (table, _flat(q_start, "q_start", dev, (n + 1,)), _flat(kv_len, "kv_len", dev))
        self.n_seq, self.max_q = n, max_q
        self.desc = base_kv_batch(n, table.shape[1], table.stride(0) if n > 1 else table.shape[1], max_q,
                                  *(_ptr(t) for t in self.tensors))


_NO_HEADS = (0, None, 0, 0, None, 0, 0)


def base_head_rope(rope: Rope, positions, q, k, q_out, k_out, stream=None):
    """q_out and k_out [rows, heads, D] from q and k (either pair None) at int32 positions
    [rows] (None where nothing rotates)."""
    if (q is None) != (q_out is None) or (k is None) != (k_out is None) or (q is None and k is None):
        raise ValueError("q and q_out, k and k_out: both or neither, and one of the two")
    lib, torch, dev = _here(rope)
    dt, D = rope.torch_dtype, rope.D
    qa = ka = _NO_HEADS
    n = None
    if q is not None:
        n, H = _rows_heads(q, "q")
        qa = (H, *_heads(q, "q", dt, dev, n, H, D), *_heads(q_out, "q_out", dt, dev, n, H, D))
    if k is not None:
        rows, H = _rows_heads(k, "k")
        n = rows if n is None else n
        ka = (H, *_heads(k, "k", dt, dev, n, H, D), *_heads(k_out, "k_out", dt, dev, n, H, D))
    if positions is not None:
        positions = _positions(torch, positions, n, dev)
    _check(lib.base_head_rope(rope.desc, n, positions, *qa, *ka, _stream_on(torch, stream, dev)))


def _positions(torch, t, n, dev):
    if t.dtype is not torch.int32 or t.shape != (n,) or (t.stride(0) != 1 and n > 1) or t.get_device() != dev:
        raise ValueError(f"positions: int32, {n} adjacent elements, on the current GPU")
    return t.data_ptr()


def head_rope(rope: Rope, positions, q, k=None, stream=None):
    """base_head_rope into new tensors; returns (q_out, k_out or None)."""
    out = [None if t is None else _empty(t, t.shape, t.dtype, stream) for t in (q, k)]
    base_head_rope(rope, positions, q, k, *out, stream)
    return tuple(out)


def base_kv_append(rope: Rope, cache: KVCache, batch: KVBatch, q, k, v, q_out, positions=None, stream=None):
    """The new tokens' k [rows, Hk, D], normalised and rotated, and v into the cache; q
    [rows, Hq, D] the same to q_out.  positions: int32 [rows], or None: the tokens' numbers
    in their sequences."""
    lib, torch, dev = _here(rope, cache, batch)
    dt, D, Hk = rope.torch_dtype, rope.D, cache.Hk
    n, Hq = _rows_heads(q, "q")
    if positions is not None:
        positions = _positions(torch, positions, n, dev)
    _check(lib.base_kv_append(
        rope.desc, cache.desc, batch.desc, n, positions, Hq, *_heads(q, "q", dt, dev, n, Hq, D),
        *_heads(q_out, "q_out", dt, dev, n, Hq, D), *_heads(k, "k", dt, dev, n, Hk, D),
        *_heads(v, "v", dt, dev, n, Hk, D), _stream_on(torch, stream, dev)))


def attention_workspace_bytes(cache: KVCache, batch: KVBatch, rows, Hq) -> int:
    n = int(load().base_attention_workspace_bytes(cache.desc, batch.desc, rows, Hq))
    if n == 0:
        raise BaseError(-2, status_string(-2))
    return n


def base_paged_attention(cache: KVCache, batch: KVBatch, q, out, ws, scale=None, window=0, lse=None,
                         stream=None):
    """out [rows, Hq, D] (and lse [rows, Hq] fp32) of q over the cache; scale None: 1 /
    sqrt(D); ws: a uint8 tensor of attention_workspace_bytes."""
    lib, torch, dev = _here(cache, batch)
    dt, D = cache.torch_dtype, cache.D
    n, Hq = _rows_heads(q, "q")
    if lse is not None:
        if (lse.dtype is not torch.float32 or lse.shape != (n, Hq) or not lse.is_contiguous()
                or lse.get_device() != dev):
            raise ValueError(f"lse: contiguous fp32 {[n, Hq]} on the current GPU")
        lse = lse.data_ptr()
    if ws.get_device() != dev or not ws.is_contiguous():
        raise ValueError("ws: contiguous, on the current GPU")
    _check(lib.base_paged_attention(
        cache.desc, batch.desc, n, Hq, *_heads(q, "q", dt, dev, n, Hq, D), *_heads(out, "out", dt, dev, n, Hq, D),
        lse, D ** -0.5 if scale is None else scale, window, ws.data_ptr(), ws.nbytes, _stream_on(torch, stream, dev)))


def paged_attention(q, cache: KVCache, batch: KVBatch, scale=None, window=0, return_lse=False, stream=None):
    """base_paged_attention into a new tensor, with a workspace of its own; returns out, or
    (out, lse)."""
    import torch
    out = _empty(q, q.shape, q.dtype, stream)
    lse = _empty(q, q.shape[:2], torch.float32, stream) if return_lse else None
    ws = _empty(q, (attention_workspace_bytes(cache, batch, q.shape[0], q.shape[1]),), torch.uint8, stream)
    base_paged_attention(cache, batch, q, out, ws, scale, window, lse, stream)
    return (out, lse) if return_lse else out


def base_set_stage_events(events):
    """events: a sequence of 2 * N_STAGES raw hipEvent_t handles (start and
    end of each stage's kernel), or None."""
    if events is None:
        _check(load().base_set_stage_events(None, 0))
        return None
    arr = (ctypes.c_void_p * len(events))(*events)
    _check(load().base_set_stage_events(arr, len(events)))
    return arr   # keep alive while timing is on


def layer_stages(desc, B, budget):
    """Names of the stages base_decode_layer launches a kernel for."""
    m = _i32()
    _check(load().base_layer_stages(ctypes.byref(desc), B, budget, ctypes.byref(m)))
    return tuple(s for i, s in enumerate(STAGES) if m.value >> i & 1)


# App. A: the ridge's lambdas, 25 values log-spaced over [1e-4, 1e2]
CALIB_LAMBDAS = tuple(10.0 ** (-4.0 + 6.0 * i / 24) for i in range(25))


def calib_stats(desc: base_layer):
    """A zeroed statistics buffer (torch uint8 tensor on the device)."""
    import torch
    n = int(load().base_calib_stats_bytes(ctypes.byref(desc)))
    if n == 0:
        raise BaseError(-2, "shape outside the supported limits")
    stats = torch.empty(n, dtype=torch.uint8, device="cuda")
    _check(load().base_calib_reset(ctypes.byref(desc), _ptr(stats), _stream(None)))
    return stats


def calib_accumulate(desc, z, B, stats, ws=None, stream=None):
    """Adds one batch of calibration hidden states z [B, d] to stats."""
    import torch
    if ws is None:
        ws = _empty(stats, (int(load().base_calib_ws_bytes(ctypes.byref(desc), B)),), torch.uint8, stream)
    _check(load().base_calib_accumulate(ctypes.byref(desc), _ptr(z), B, _ptr(stats),
                                        _ptr(ws), ws.numel(), _stream(stream)))
    return ws


def calib_fit(desc, stats, lambdas, pred_a, pred_b, lam_out=None, stream=None):
    """pred_a [E, d], pred_b [E] (fp32 device tensors) from the statistics;
    lambdas: a sequence of positive floats (host)."""
    lam = (ctypes.c_double * len(lambdas))(*[float(v) for v in lambdas])
    _check(load_calib().base_calib_fit(ctypes.byref(desc), _ptr(stats), len(lambdas), lam,
                                       _ptr(pred_a), _ptr(pred_b), _ptr(lam_out),
                                       _stream(stream)))


def plan_offset(plan: base_plan, field: str, ws) -> int:
    """Byte offset of a plan array inside the workspace tensor."""
    p = getattr(plan, field)
    return None if p is None else p - ws.data_ptr()
