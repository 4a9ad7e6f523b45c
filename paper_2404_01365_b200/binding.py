"""ctypes binding of libgriffin_ff.so: argument marshalling only.

Every function here has the name of the C entry point it calls (include/griffin_ff.h) and
takes torch tensors for device buffers; each step of the path runs in the library's CUDA
kernels.  There is no fallback: if the library is missing or a call fails, an exception is
raised.
"""
from __future__ import annotations

import ctypes as C
import os

import torch

from . import build as _build

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_ALIGNMENT, ERR_WORKSPACE, ERR_CUDA, ERR_TIMEOUT = range(7)
ACT_SWIGLU, ACT_GEGLU_TANH, ACT_REGLU, ACT_GEGLU_ERF = 0, 1, 2, 3
ACT_RELU, ACT_GELU_TANH, ACT_GELU_ERF, ACT_SILU = 4, 5, 6, 7   # blocks without a gate (Eq. 2): w_gate is None
DT_F32, DT_BF16 = 0, 1
DECODE_DEFAULT, DECODE_OVERLAP_WEIGHT_PREFETCH, DECODE_TCGEN05, DECODE_RING, DECODE_STREAM = 0, 1, 2, 4, 8
MAX_BATCH = 32
NORM_NONE, NORM_RMS, NORM_LAYER = range(3)
GATE_LINEAR, GATE_SIGMOID, GATE_TANH = range(3)
ROPE_HALF, ROPE_PAIRS = range(2)
NORM_BY_NAME = {"none": NORM_NONE, "rms": NORM_RMS, "layer": NORM_LAYER}
GATE_BY_NAME = {"linear": GATE_LINEAR, "sigmoid": GATE_SIGMOID, "tanh": GATE_TANH}
ROPE_BY_NAME = {"half": ROPE_HALF, "pairs": ROPE_PAIRS}

ACT_BY_NAME = {"swiglu": ACT_SWIGLU, "geglu_tanh": ACT_GEGLU_TANH, "reglu": ACT_REGLU, "geglu_erf": ACT_GEGLU_ERF,
               "relu": ACT_RELU, "gelu_tanh": ACT_GELU_TANH, "gelu_erf": ACT_GELU_ERF, "silu": ACT_SILU}


def act_is_gated(act):
    act = ACT_BY_NAME[act] if isinstance(act, str) else int(act)
    return ACT_SWIGLU <= act <= ACT_GEGLU_ERF
DTYPE_BY_NAME = {"f32": DT_F32, "bf16": DT_BF16}

EXPORTS = (
    "griffin_status_string", "griffin_version", "griffin_k_from_keep_ratio", "griffin_compact_ldk",
    "griffin_workspace_bytes", "griffin_workspace_init", "griffin_ff_prefill_score", "griffin_select_topk",
    "griffin_combine_scores", "griffin_compact_experts", "griffin_ff_decode", "griffin_check_device_status",
    "griffin_ff_decode_static", "griffin_ff_decode_indexed", "griffin_ff_prefill_score_chunk",
    "griffin_kernel_launches", "griffin_ff_decode_static_status", "griffin_compact_experts_nm",
    "griffin_norm_residual", "griffin_kv_append", "griffin_attn_workspace_bytes", "griffin_attn_prefix",
    "griffin_kv_q4_block_bytes", "griffin_kv_append_q4", "griffin_kv_read_q4", "griffin_attn_prefix_q4",
)


class GriffinError(RuntimeError):
    def __init__(self, status, what):
        self.status = status
        super().__init__(f"{what}: status {status} ({status_string(status)})")


class FFDesc(C.Structure):
    _fields_ = [("d", C.c_int32), ("d_ff", C.c_int32), ("act", C.c_int32), ("dtype", C.c_int32)]


class FFWeights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("w_gate", "w_up", "w_down", "b_gate", "b_up", "b_down")]


class FFWeightsNM(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("w_gate", "w_up", "w_down_t", "b_gate", "b_up", "b_down")]


class FFCompact(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("w_gate_c", "w_up_c", "w_down_c", "b_gate_c", "b_up_c")] + \
               [("k", C.c_int32), ("ldk", C.c_int32)]


class NormDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("d", "dtype", "res_dtype", "pre_norm", "post_norm", "gate_act")] + \
               [(n, C.c_float) for n in ("eps", "weight_offset", "res_scale", "out_scale")]


class NormWeights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("pre_w", "pre_b", "post_w", "post_b")]
    _form = None     # (torch dtype, width) of the tensors it was made of


class AttnDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_q_heads", "n_kv_heads", "head_dim", "page_size", "dtype")] + [("scale", C.c_float)]


class KVCache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("n_pages", C.c_int32)] + \
               [(n, C.c_int64) for n in ("stride_page", "stride_head", "stride_token")]
    _form = None     # (griffin_dtype, heads, page size, head width) of the tensors it was made of


class KVCacheQ4(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("n_pages", C.c_int32)] + [(n, C.c_int64) for n in ("stride_page", "stride_head")]
    _form = None     # (heads, bytes of one head's part of a page) of the tensors it was made of


class AttnBatch(C.Structure):
    _fields_ = [("n_seq", C.c_int32), ("n_tokens", C.c_int32)] + \
               [(n, C.c_void_p) for n in ("q_start", "seq_len", "page_table")] + \
               [("table_stride", C.c_int32), ("prefix_len", C.c_int32), ("prefix_pages", C.c_void_p)]
    _prefix_pages = None     # how many pages the prefix's list has


class Rope(C.Structure):
    _fields_ = [("table", C.c_void_p), ("n_pos", C.c_int32), ("rot_dim", C.c_int32), ("style", C.c_int32)]


_lib = None


def load(path=None):
    """Loads the shared library (once).  Raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    path = path or os.environ.get("GRIFFIN_FF_LIB") or _build.LIB_PATH
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with `python -m paper_2404_01365_b200.build` "
                           "(there is no fallback path)")
    lib = C.CDLL(path)
    vp, i32, u32, sz = C.c_void_p, C.c_int32, C.c_uint32, C.c_size_t
    lib.griffin_status_string.restype = C.c_char_p
    lib.griffin_status_string.argtypes = [C.c_int]
    lib.griffin_version.restype = i32
    lib.griffin_version.argtypes = []
    lib.griffin_kernel_launches.restype = C.c_uint64
    lib.griffin_kernel_launches.argtypes = []
    lib.griffin_k_from_keep_ratio.restype = i32
    lib.griffin_k_from_keep_ratio.argtypes = [i32, C.c_double]
    lib.griffin_compact_ldk.restype = i32
    lib.griffin_compact_ldk.argtypes = [i32]
    lib.griffin_workspace_bytes.restype = sz
    lib.griffin_workspace_bytes.argtypes = [C.POINTER(FFDesc), i32, i32]
    lib.griffin_workspace_init.restype = C.c_int
    lib.griffin_workspace_init.argtypes = [vp, sz, vp]
    lib.griffin_ff_prefill_score.restype = C.c_int
    lib.griffin_ff_prefill_score.argtypes = [C.POINTER(FFDesc), C.POINTER(FFWeights), vp, i32, vp, vp, vp, sz, vp]
    lib.griffin_ff_prefill_score_chunk.restype = C.c_int
    lib.griffin_ff_prefill_score_chunk.argtypes = [C.POINTER(FFDesc), C.POINTER(FFWeights), vp, i32, vp, vp, vp, i32, vp,
                                                   sz, vp]
    lib.griffin_select_topk.restype = C.c_int
    lib.griffin_select_topk.argtypes = [vp, i32, i32, i32, vp, vp]
    lib.griffin_combine_scores.restype = C.c_int
    lib.griffin_combine_scores.argtypes = [vp, C.POINTER(i32), i32, i32, vp, vp]
    lib.griffin_compact_experts.restype = C.c_int
    lib.griffin_compact_experts.argtypes = [C.POINTER(FFDesc), C.POINTER(FFWeights), vp, C.POINTER(FFCompact), vp, vp]
    lib.griffin_compact_experts_nm.restype = C.c_int
    lib.griffin_compact_experts_nm.argtypes = [C.POINTER(FFDesc), C.POINTER(FFWeightsNM), vp, C.POINTER(FFCompact), vp, vp]
    lib.griffin_ff_decode.restype = C.c_int
    lib.griffin_ff_decode.argtypes = [C.POINTER(FFDesc), i32, C.POINTER(FFCompact), vp, vp, vp, vp, sz, u32, vp]
    lib.griffin_ff_decode_indexed.restype = C.c_int
    lib.griffin_ff_decode_indexed.argtypes = [C.POINTER(FFDesc), i32, C.POINTER(FFWeightsNM), vp, i32, vp, vp, vp, sz, u32, vp]
    lib.griffin_ff_decode_static.restype = C.c_int
    lib.griffin_ff_decode_static.argtypes = [C.POINTER(FFDesc), i32, C.POINTER(FFCompact), vp, vp, vp, u32, vp]
    lib.griffin_ff_decode_static_status.restype = C.c_int
    lib.griffin_ff_decode_static_status.argtypes = [vp]
    i64 = C.c_int64
    lib.griffin_norm_residual.restype = C.c_int
    lib.griffin_norm_residual.argtypes = [C.POINTER(NormDesc), C.POINTER(NormWeights), i32, vp, i64, vp, i64, vp, i64, vp, i64,
                                          vp, i64, vp]
    lib.griffin_kv_append.restype = C.c_int
    lib.griffin_kv_append.argtypes = [C.POINTER(AttnDesc), C.POINTER(AttnBatch), C.POINTER(KVCache), C.POINTER(Rope), vp, i64,
                                      vp, i64, vp, i64, vp, i64, vp, vp]
    lib.griffin_attn_workspace_bytes.restype = sz
    lib.griffin_attn_workspace_bytes.argtypes = [C.POINTER(AttnDesc), i32, i32]
    lib.griffin_attn_prefix.restype = C.c_int
    lib.griffin_attn_prefix.argtypes = [C.POINTER(AttnDesc), C.POINTER(AttnBatch), C.POINTER(KVCache), vp, i64, vp, i64, vp, sz,
                                        vp]
    lib.griffin_kv_q4_block_bytes.restype = sz
    lib.griffin_kv_q4_block_bytes.argtypes = [C.POINTER(AttnDesc)]
    lib.griffin_kv_append_q4.restype = C.c_int
    lib.griffin_kv_append_q4.argtypes = [C.POINTER(AttnDesc), C.POINTER(AttnBatch), C.POINTER(KVCacheQ4), C.POINTER(Rope), vp, i64,
                                         vp, i64, vp, i64, vp, i64, vp, vp]
    lib.griffin_kv_read_q4.restype = C.c_int
    lib.griffin_kv_read_q4.argtypes = [C.POINTER(AttnDesc), C.POINTER(AttnBatch), C.POINTER(KVCacheQ4), vp, i64, vp, i64, vp, vp]
    lib.griffin_attn_prefix_q4.restype = C.c_int
    lib.griffin_attn_prefix_q4.argtypes = [C.POINTER(AttnDesc), C.POINTER(AttnBatch), C.POINTER(KVCacheQ4), vp, i64, vp, i64, vp,
                                           sz, vp]
    lib.griffin_check_device_status.restype = C.c_int
    lib.griffin_check_device_status.argtypes = [vp, vp]
    _lib = lib
    return lib


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


# (current_stream() builds a Stream object, 3 us; its handle alone is a tenth of a microsecond)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is not None:
        return _raw_stream(torch.cuda.current_device())
    return torch.cuda.current_stream().cuda_stream


def _check(st, what):
    if st != OK:
        raise GriffinError(st, what)


def status_string(st):
    return load().griffin_status_string(int(st)).decode()


def griffin_version():
    return load().griffin_version()


def griffin_kernel_launches():
    """Kernels launched by the library in this process so far."""
    return int(load().griffin_kernel_launches())


def griffin_k_from_keep_ratio(d_ff, keep):
    return load().griffin_k_from_keep_ratio(int(d_ff), float(keep))


def griffin_compact_ldk(k):
    return load().griffin_compact_ldk(int(k))


def make_desc(d, d_ff, act, dtype):
    act = ACT_BY_NAME[act] if isinstance(act, str) else int(act)
    dtype = DTYPE_BY_NAME[dtype] if isinstance(dtype, str) else int(dtype)
    return FFDesc(int(d), int(d_ff), act, dtype)


def make_weights(w_gate, w_up, w_down, b_gate=None, b_up=None, b_down=None):
    w = FFWeights(_ptr(w_gate), _ptr(w_up), _ptr(w_down), _ptr(b_gate), _ptr(b_up), _ptr(b_down))
    w._keep = (w_gate, w_up, w_down, b_gate, b_up, b_down)  # keep the tensors alive
    return w


def make_weights_nm(w_gate, w_up, w_down_t, b_gate=None, b_up=None, b_down=None):
    """Neuron-major full weights for griffin_ff_decode_indexed: w_down_t is W_2 transposed, [d_ff, d]."""
    w = FFWeightsNM(_ptr(w_gate), _ptr(w_up), _ptr(w_down_t), _ptr(b_gate), _ptr(b_up), _ptr(b_down))
    w._keep = (w_gate, w_up, w_down_t, b_gate, b_up, b_down)
    return w


def make_compact(w_gate_c, w_up_c, w_down_c, k, ldk, b_gate_c=None, b_up_c=None):
    c = FFCompact(_ptr(w_gate_c), _ptr(w_up_c), _ptr(w_down_c), _ptr(b_gate_c), _ptr(b_up_c), int(k), int(ldk))
    c._keep = (w_gate_c, w_up_c, w_down_c, b_gate_c, b_up_c)
    return c


def alloc_compact(desc, k, device, torch_dtype, with_bias=False):
    """Allocates the buffers of one compact expert set (torch owns the memory)."""
    ldk = griffin_compact_ldk(k)
    gated = act_is_gated(desc.act)   # a block without a gate has no W_g_hat
    g = torch.empty((k, desc.d), device=device, dtype=torch_dtype) if gated else None
    u = torch.empty((k, desc.d), device=device, dtype=torch_dtype)
    dn = torch.empty((desc.d, ldk), device=device, dtype=torch_dtype)
    bg = torch.empty((k,), device=device, dtype=torch_dtype) if with_bias and gated else None
    bu = torch.empty((k,), device=device, dtype=torch_dtype) if with_bias else None
    return make_compact(g, u, dn, k, ldk, bg, bu)


def griffin_workspace_bytes(desc, S_max, n_seq_max):
    return load().griffin_workspace_bytes(C.byref(desc), int(S_max), int(n_seq_max))


def alloc_workspace(desc, S_max, n_seq_max, device, stream=None):
    """Allocates and initialises a workspace tensor (uint8) large enough for any call."""
    n = griffin_workspace_bytes(desc, S_max, n_seq_max)
    if n == 0:
        raise GriffinError(ERR_INVALID_ARG, "griffin_workspace_bytes")
    ws = torch.empty((n,), device=device, dtype=torch.uint8)
    griffin_workspace_init(ws, stream)
    return ws


def griffin_workspace_init(ws, stream=None):
    _check(load().griffin_workspace_init(_ptr(ws), ws.numel(), _stream(stream)), "griffin_workspace_init")


def griffin_ff_prefill_score(desc, weights, x, y, score, ws, stream=None):
    S = x.shape[0]
    _check(load().griffin_ff_prefill_score(C.byref(desc), C.byref(weights), _ptr(x), S, _ptr(y), _ptr(score),
                                           _ptr(ws), ws.numel(), _stream(stream)), "griffin_ff_prefill_score")


def griffin_ff_prefill_score_chunk(desc, weights, x, y, sumsq, score, first, ws, stream=None):
    """One piece of a prompt that is fed piece by piece: sumsq carries the statistic's squares."""
    S = x.shape[0]
    _check(load().griffin_ff_prefill_score_chunk(C.byref(desc), C.byref(weights), _ptr(x), S, _ptr(y), _ptr(sumsq),
                                                 _ptr(score), 1 if first else 0, _ptr(ws), ws.numel(), _stream(stream)),
           "griffin_ff_prefill_score_chunk")


def griffin_select_topk(score, k, idx, stream=None):
    n_seq, d_ff = (1, score.shape[0]) if score.dim() == 1 else score.shape
    _check(load().griffin_select_topk(_ptr(score), int(n_seq), int(d_ff), int(k), _ptr(idx), _stream(stream)),
           "griffin_select_topk")


def griffin_combine_scores(score, prompt_len, out, stream=None):
    n_seq, d_ff = score.shape
    arr = (C.c_int32 * n_seq)(*[int(v) for v in prompt_len])
    _check(load().griffin_combine_scores(_ptr(score), arr, int(n_seq), int(d_ff), _ptr(out), _stream(stream)),
           "griffin_combine_scores")


def griffin_compact_experts(desc, weights, idx, out, ws=None, stream=None):
    _check(load().griffin_compact_experts(C.byref(desc), C.byref(weights), _ptr(idx), C.byref(out), _ptr(ws),
                                          _stream(stream)), "griffin_compact_experts")


def griffin_compact_experts_nm(desc, weights_nm, idx, out, ws=None, stream=None):
    """The same compact set from neuron-major full weights (w_down_t = W_2 transposed)."""
    _check(load().griffin_compact_experts_nm(C.byref(desc), C.byref(weights_nm), _ptr(idx), C.byref(out), _ptr(ws),
                                             _stream(stream)), "griffin_compact_experts_nm")


def compact_array(sets):
    """A C array of compact-set structs for griffin_ff_decode (build once, reuse per step)."""
    arr = (FFCompact * len(sets))()
    for i, s in enumerate(sets):
        C.memmove(C.byref(arr[i]), C.byref(s), C.sizeof(FFCompact))
    arr._keep = list(sets)
    return arr


def griffin_ff_decode(desc, sets, b_down, x, y, ws, flags=DECODE_DEFAULT, stream=None):
    arr = sets if isinstance(sets, C.Array) else compact_array(sets)
    _check(load().griffin_ff_decode(C.byref(desc), len(arr), arr, _ptr(b_down), _ptr(x), _ptr(y), _ptr(ws),
                                    ws.numel(), int(flags), _stream(stream)), "griffin_ff_decode")


def griffin_ff_decode_indexed(desc, weights_nm, idx, x, y, ws, flags=DECODE_DEFAULT, stream=None):
    """Pruned FF straight from the full neuron-major weights; idx [B, k] int32 on the device."""
    B, k = (1, idx.shape[0]) if idx.dim() == 1 else idx.shape
    _check(load().griffin_ff_decode_indexed(C.byref(desc), int(B), C.byref(weights_nm), _ptr(idx), int(k), _ptr(x),
                                            _ptr(y), _ptr(ws), ws.numel(), int(flags), _stream(stream)),
           "griffin_ff_decode_indexed")


STATIC_SCRATCH_BYTES = 1 << 20


def griffin_ff_decode_static(desc, sets, b_down, x, y, flags=DECODE_DEFAULT, stream=None):
    """griffin_ff_decode for callers that cannot allocate a workspace: the scratch is a fixed
    array inside the library (see include/griffin_ff.h for its limit and sharing rules)."""
    arr = sets if isinstance(sets, C.Array) else compact_array(sets)
    _check(load().griffin_ff_decode_static(C.byref(desc), len(arr), arr, _ptr(b_down), _ptr(x), _ptr(y), int(flags),
                                           _stream(stream)), "griffin_ff_decode_static")


def griffin_ff_decode_static_status(stream=None):
    """Status of the static-scratch decode calls on the current device (synchronises the stream)."""
    return load().griffin_ff_decode_static_status(_stream(stream))


def griffin_check_device_status(ws, stream=None):
    return load().griffin_check_device_status(_ptr(ws), _stream(stream))


# ---- around the FF block: norms and the residual stream, the paged cache, attention over it ---------------------
_TORCH_DTYPE = {DT_F32: torch.float32, DT_BF16: torch.bfloat16}
_DTYPE_CODE = {t: c for c, t in _TORCH_DTYPE.items()}


def _dtype(v):
    return DTYPE_BY_NAME[v] if isinstance(v, str) else int(v)


def _rows(t, n, heads, d, dtype, what):
    """Token stride of an [n, heads, d] (or [n, heads * d]) tensor whose tokens are rows of heads * d
    consecutive entries."""
    st, shape = t.stride(), t.shape
    if len(st) == 3:
        ok = shape[1] == heads and shape[2] == d and st[2] == 1 and st[1] == d
    else:
        ok = len(st) == 2 and shape[1] == heads * d and st[1] == 1
    if not ok or shape[0] < n or t.dtype != _TORCH_DTYPE[dtype]:
        raise ValueError(f"{what}: expected {_TORCH_DTYPE[dtype]} [{n}, {heads}, {d}] with the heads of a token in one "
                         f"row, got {t.dtype} {tuple(shape)} with strides {st}")
    return st[0] if shape[0] > 1 else heads * d


def make_norm_desc(d, dtype, res_dtype=None, pre="rms", post="none", eps=1e-6, weight_offset=0.0, res_scale=1.0, out_scale=1.0,
                   gate_act="linear"):
    return NormDesc(int(d), _dtype(dtype), _dtype(dtype if res_dtype is None else res_dtype), NORM_BY_NAME[pre], NORM_BY_NAME[post],
                    GATE_BY_NAME[gate_act], float(eps), float(weight_offset), float(res_scale), float(out_scale))


def make_norm_weights(pre_w=None, pre_b=None, post_w=None, post_b=None):
    """Vectors [d] of the descriptor's dtype, consecutive entries (checked against it when the call is made)."""
    w = NormWeights(_ptr(pre_w), _ptr(pre_b), _ptr(post_w), _ptr(post_b))
    w._keep = (pre_w, pre_b, post_w, post_b)
    for t in w._keep:
        if t is None:
            continue
        if t.dim() != 1 or not t.is_contiguous() or w._form not in (None, (t.dtype, t.shape[0])):
            raise ValueError("norm weights: expected vectors of one dtype and width with consecutive entries, got "
                             + ", ".join(f"{x.dtype} {tuple(x.shape)} with strides {x.stride()}" for x in w._keep if x is not None))
        w._form = (t.dtype, t.shape[0])
    return w


def _norm_rows(t, d, dtype, T, what):
    st, shape = t.stride(), t.shape
    if len(st) != 2 or shape[0] != T or shape[1] != d or st[1] != 1 or t.dtype != dtype:
        raise ValueError(f"{what}: expected {dtype} [{T}, {d}] with consecutive entries, got {t.dtype} {tuple(shape)} with "
                         f"strides {st}")
    return st[0] if T > 1 else d


def griffin_norm_residual(desc, weights, res, res_out, h, y=None, gate=None, stream=None):
    """res_out = a res + c act(gate) * post_norm(y), h = pre_norm(res_out) for the rows of res [T, d].  y, gate, res_out
    and h may be None (see include/griffin_ff.h); gate is [d] or [T, d]."""
    T, d = res.shape[0], desc.d
    if T == 0:
        return
    dt, rdt = _TORCH_DTYPE[desc.dtype], _TORCH_DTYPE[desc.res_dtype]
    if weights._form is not None and weights._form != (dt, d):
        raise ValueError(f"norm weights: expected {dt} [{d}], got {weights._form[0]} [{weights._form[1]}]")
    y_p = g_p = ro_p = h_p = None
    ld_y = ld_g = ld_ro = ld_h = 0
    ld_r = _norm_rows(res, d, rdt, T, "res")
    if y is not None:
        ld_y, y_p = _norm_rows(y, d, dt, T, "y"), y.data_ptr()
    if gate is not None:
        g_p = gate.data_ptr()
        if gate.dim() == 2:
            ld_g = _norm_rows(gate, d, dt, T, "gate")
        else:
            _norm_rows(gate[None], d, dt, 1, "gate")
    if res_out is not None:
        ld_ro, ro_p = _norm_rows(res_out, d, rdt, T, "res_out"), res_out.data_ptr()
    if h is not None:
        ld_h, h_p = _norm_rows(h, d, dt, T, "h"), h.data_ptr()
    st = load().griffin_norm_residual(C.byref(desc), C.byref(weights), T, y_p, ld_y, g_p, ld_g, res.data_ptr(), ld_r, ro_p, ld_ro,
                                      h_p, ld_h, _stream(stream))
    if st != OK:
        raise GriffinError(st, "griffin_norm_residual")


def make_attn_desc(n_q_heads, n_kv_heads, head_dim, page_size, dtype, scale=None):
    return AttnDesc(int(n_q_heads), int(n_kv_heads), int(head_dim), int(page_size), _dtype(dtype),
                    float(head_dim ** -0.5 if scale is None else scale))


def make_kv_cache(k, v):
    """A paged cache from two tensors [n_pages, n_kv_heads, page_size, head_dim] of the same strides (any, as long as the
    entries of a head are consecutive: pages laid out [page_size, n_kv_heads, head_dim] go in as a transposed view)."""
    if k.shape != v.shape or k.stride() != v.stride() or k.dim() != 4 or k.stride(3) != 1 or k.dtype != v.dtype:
        raise ValueError(f"k and v must be alike, [pages, heads, tokens, head_dim]: got {k.dtype} {tuple(k.shape)} {k.stride()}, "
                         f"{v.dtype} {tuple(v.shape)} {v.stride()}")
    c = KVCache(_ptr(k), _ptr(v), k.shape[0], k.stride(0), k.stride(1), k.stride(2))
    c._keep = (k, v)
    c._form = (_DTYPE_CODE.get(k.dtype, str(k.dtype)), *k.shape[1:])
    return c


def _check_cache(form, batch, cache):
    """That the cache's pages are the descriptor's (form: dtype, heads, page size, head width), and the prefix's list as
    long as the prefix."""
    if cache._form != form and cache._form is not None:
        raise ValueError("cache: expected pages [{1}, {2}, {3}] of griffin_dtype {0}, got [{5}, {6}, {7}] of {4}"
                         .format(*form, *cache._form))
    _check_prefix(batch, form[2])


def _check_prefix(batch, page_size):
    if batch._prefix_pages is not None and batch.prefix_len > batch._prefix_pages * page_size:
        raise ValueError(f"prefix_pages: {batch._prefix_pages} pages of {page_size} tokens for a prefix of {batch.prefix_len}")


def make_attn_batch(q_start, seq_len, page_table, n_tokens, prefix_pages=None, prefix_len=0):
    """The tokens of a call.  q_start [n_seq + 1], seq_len [n_seq], page_table [n_seq, pages], prefix_pages: int32 on the
    device, read when the call runs (so the same batch serves every step of a generation whose lengths are counted up on
    the device); n_tokens, prefix_len: host numbers."""
    for name, t in (("q_start", q_start), ("seq_len", seq_len), ("page_table", page_table), ("prefix_pages", prefix_pages)):
        if t is not None and (t.dtype != torch.int32 or not t.is_contiguous()):
            raise ValueError(f"{name}: expected contiguous int32, got {t.dtype}")
    n_seq = seq_len.shape[0]
    if q_start.shape != (n_seq + 1,) or page_table.dim() != 2 or page_table.shape[0] != n_seq:
        raise ValueError(f"q_start {tuple(q_start.shape)}, seq_len {tuple(seq_len.shape)}, page_table {tuple(page_table.shape)}")
    b = AttnBatch(n_seq, int(n_tokens), _ptr(q_start), _ptr(seq_len), _ptr(page_table),
                  page_table.shape[1], int(prefix_len), _ptr(prefix_pages))
    b._keep = (q_start, seq_len, page_table, prefix_pages)
    b._prefix_pages = None if prefix_pages is None else prefix_pages.numel()
    return b


def make_rope(table, style="half"):
    """Rotation by the rows of `table` [n_pos, rot_dim], fp32: rot_dim/2 cosines, then the sines."""
    if table.dim() != 2 or table.dtype != torch.float32 or not table.is_contiguous():
        raise ValueError(f"expected contiguous float32 [n_pos, rot_dim], got {table.dtype} {tuple(table.shape)}")
    r = Rope(_ptr(table), table.shape[0], table.shape[1], ROPE_BY_NAME[style])
    r._keep = table
    return r


def rope_table(n_pos, rot_dim, theta=10000.0, device=None):
    """cos and sin of p * theta^(-2j / rot_dim), angles in float64."""
    freq = float(theta) ** (-torch.arange(rot_dim // 2, dtype=torch.float64) * 2 / rot_dim)
    a = torch.arange(n_pos, dtype=torch.float64)[:, None] * freq
    return torch.cat((a.cos(), a.sin()), 1).float().to(device)


def griffin_kv_append(desc, batch, cache, rope, q, k, v, q_out, ws=None, stream=None):
    """New keys and values [n_tokens, n_kv_heads, head_dim] into the cache, keys and queries rotated; q and q_out may be
    None, q_out may be q."""
    n, hq, hk, d, dt = batch.n_tokens, desc.n_q_heads, desc.n_kv_heads, desc.head_dim, desc.dtype
    _check_cache((dt, hk, desc.page_size, d), batch, cache)
    q_p = o_p = None
    ld_q = ld_o = 0
    if q is not None:
        ld_q, q_p = _rows(q, n, hq, d, dt, "q"), q.data_ptr()
    if q_out is not None:
        ld_o, o_p = _rows(q_out, n, hq, d, dt, "q_out"), q_out.data_ptr()
    st = load().griffin_kv_append(C.byref(desc), C.byref(batch), C.byref(cache), None if rope is None else C.byref(rope), q_p, ld_q,
                                  k.data_ptr(), _rows(k, n, hk, d, dt, "k"), v.data_ptr(), _rows(v, n, hk, d, dt, "v"), o_p, ld_o,
                                  None if ws is None else ws.data_ptr(), _stream(stream))
    if st != OK:
        raise GriffinError(st, "griffin_kv_append")


def griffin_attn_workspace_bytes(desc, n_tokens_max, n_seq_max):
    return load().griffin_attn_workspace_bytes(C.byref(desc), int(n_tokens_max), int(n_seq_max))


def alloc_attn_workspace(desc, n_tokens_max, n_seq_max, device, stream=None):
    n = griffin_attn_workspace_bytes(desc, n_tokens_max, n_seq_max)
    if n == 0:
        raise GriffinError(ERR_INVALID_ARG, "griffin_attn_workspace_bytes")
    ws = torch.empty((n,), device=device, dtype=torch.uint8)
    griffin_workspace_init(ws, stream)
    return ws


def griffin_attn_prefix(desc, batch, cache, q, out, ws, stream=None):
    """Attention of the batch's new tokens over the shared prefix and their own sequences; q, out [n_tokens, n_q_heads,
    head_dim]."""
    n, hq, d, dt = batch.n_tokens, desc.n_q_heads, desc.head_dim, desc.dtype
    _check_cache((dt, desc.n_kv_heads, desc.page_size, d), batch, cache)
    st = load().griffin_attn_prefix(C.byref(desc), C.byref(batch), C.byref(cache), q.data_ptr(), _rows(q, n, hq, d, dt, "q"),
                                    out.data_ptr(), _rows(out, n, hq, d, dt, "out"), ws.data_ptr(), ws.numel(), _stream(stream))
    if st != OK:
        raise GriffinError(st, "griffin_attn_prefix")


# ---- the same cache in 4 bits ------------------------------------------------------------------------------------
def griffin_kv_q4_block_bytes(desc):
    """Bytes of one head's part of a page."""
    return int(load().griffin_kv_q4_block_bytes(C.byref(desc)))


def make_kv_cache_q4(k, v):
    """A paged cache in 4 bits from two uint8 tensors [n_pages, n_kv_heads, griffin_kv_q4_block_bytes] of the same strides
    (any, as long as the bytes of a head are consecutive)."""
    if k.shape != v.shape or k.stride() != v.stride() or k.dim() != 3 or k.stride(2) != 1 or k.dtype != torch.uint8 or v.dtype != torch.uint8:
        raise ValueError(f"k and v must be alike, uint8 [pages, heads, bytes]: got {k.dtype} {tuple(k.shape)} {k.stride()}, "
                         f"{v.dtype} {tuple(v.shape)} {v.stride()}")
    c = KVCacheQ4(_ptr(k), _ptr(v), k.shape[0], k.stride(0), k.stride(1))
    c._keep = (k, v)
    c._form = tuple(k.shape[1:])
    return c


def alloc_kv_cache_q4(desc, n_pages, device):
    """A cache in 4 bits for the descriptor's heads and pages (torch owns the memory)."""
    n = griffin_kv_q4_block_bytes(desc)
    if n == 0:
        raise GriffinError(ERR_INVALID_ARG, "griffin_kv_q4_block_bytes")
    return make_kv_cache_q4(*(torch.empty((n_pages, desc.n_kv_heads, n), dtype=torch.uint8, device=device) for _ in range(2)))


def _check_q4(batch, cache, heads, d, page):
    """That the cache's pages are the descriptor's, and the prefix's list as long as the prefix."""
    form, block = cache._form, page * (d // 2 + (d + 63) // 64 * 4)
    if form is not None and form != (heads, block):
        raise ValueError(f"cache: expected pages [{heads}, {block}], got {list(form)}")
    if batch._prefix_pages is not None:
        _check_prefix(batch, page)


# (structures are handed to ctypes as they are, which passes their address)
def griffin_kv_append_q4(desc, batch, cache, rope, q, k, v, q_out, ws=None, stream=None):
    """griffin_kv_append into a cache in 4 bits: keys, rotated, and values are quantised as they are written."""
    n, hq, hk, d, dt = batch.n_tokens, desc.n_q_heads, desc.n_kv_heads, desc.head_dim, desc.dtype
    _check_q4(batch, cache, hk, d, desc.page_size)
    q_p = o_p = None
    ld_q = ld_o = 0
    if q is not None:
        ld_q, q_p = _rows(q, n, hq, d, dt, "q"), q.data_ptr()
    if q_out is not None:
        ld_o, o_p = _rows(q_out, n, hq, d, dt, "q_out"), q_out.data_ptr()
    ld_k, ld_v = _rows(k, n, hk, d, dt, "k"), _rows(v, n, hk, d, dt, "v")
    if n == 0:       # (empty tensors have no address)
        return
    st = load().griffin_kv_append_q4(desc, batch, cache, rope, q_p, ld_q, k.data_ptr(), ld_k, v.data_ptr(), ld_v, o_p, ld_o,
                                     None if ws is None else ws.data_ptr(), _stream(stream))
    if st != OK:
        raise GriffinError(st, "griffin_kv_append_q4")


def griffin_kv_read_q4(desc, batch, cache, k, v, ws=None, stream=None):
    """The batch's tokens out of a cache in 4 bits: k, v [n_tokens, n_kv_heads, head_dim] of the descriptor's dtype."""
    n, hk, d, dt = batch.n_tokens, desc.n_kv_heads, desc.head_dim, desc.dtype
    _check_q4(batch, cache, hk, d, desc.page_size)
    ld_k, ld_v = _rows(k, n, hk, d, dt, "k"), _rows(v, n, hk, d, dt, "v")
    if n == 0:
        return
    st = load().griffin_kv_read_q4(desc, batch, cache, k.data_ptr(), ld_k, v.data_ptr(), ld_v,
                                   None if ws is None else ws.data_ptr(), _stream(stream))
    if st != OK:
        raise GriffinError(st, "griffin_kv_read_q4")


def griffin_attn_prefix_q4(desc, batch, cache, q, out, ws, stream=None):
    """griffin_attn_prefix over a cache in 4 bits."""
    n, hq, d, dt = batch.n_tokens, desc.n_q_heads, desc.head_dim, desc.dtype
    _check_q4(batch, cache, desc.n_kv_heads, d, desc.page_size)
    ld_q, ld_o = _rows(q, n, hq, d, dt, "q"), _rows(out, n, hq, d, dt, "out")
    if n == 0:
        return
    st = load().griffin_attn_prefix_q4(desc, batch, cache, q.data_ptr(), ld_q, out.data_ptr(), ld_o, ws.data_ptr(), ws.numel(),
                                       _stream(stream))
    if st != OK:
        raise GriffinError(st, "griffin_attn_prefix_q4")
