"""ctypes binding of libfocus.so: same names as include/focus.h, argument marshalling only.

PyTorch is used for device memory and streams; every step of the decode path runs in the library's HIP
kernels.  Importing this module fails loudly when the library has not been built
(python -m paper_2601_23278_amd.build, or __graft_entry__.build()).
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Dict, List, Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfocus.so")

FOCUS_OK, FOCUS_EINVAL, FOCUS_ENOMEM, FOCUS_EHIP = 0, -1, -2, -3
FOCUS_F32, FOCUS_BF16, FOCUS_MX4 = 0, 1, 2
FOCUS_SCORE_SOFTMAX, FOCUS_SCORE_SIGMOID = 0, 1
FOCUS_MAX_BLOCK = 64
KC_GEMM, KC_ATTENTION, KC_IMPORTANCE, KC_POINTWISE, KC_DECODE, KC_ROUTE, KC_EXPERTS, KC_SELECT, KC_GATHER, KC_KV_WRITE, KC_COUNT = range(11)
KC_NAMES = ["gemm", "attention", "importance", "pointwise", "decode", "route", "experts", "select", "gather", "kv_write"]


class focus_config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_layers", "hidden", "n_q_heads", "n_kv_heads", "head_dim", "ffn", "vocab",
                                         "dtype")] + \
               [("rms_eps", C.c_float), ("rope_base", C.c_float)] + \
               [(n, C.c_int32) for n in ("block_size", "mask_token_id", "max_batch", "max_prefix_len", "page_size",
                                         "n_pages", "evict_layer", "importance_mode", "maxpool_k", "budget_mode",
                                         "topk")] + \
               [("keep_ratio", C.c_float), ("alpha", C.c_float), ("constraints", C.c_int32),
                ("conf_threshold", C.c_float), ("intra_block_cache", C.c_int32), ("selection", C.c_int32),
                ("selection_seed", C.c_uint32)] + \
               [(n, C.c_int32) for n in ("n_experts", "experts_per_token", "expert_ffn", "shared_ffn", "first_moe_layer")] + \
               [("route_scale", C.c_float)]


class focus_weights(C.Structure):
    _fields_ = [("embed", C.c_void_p), ("lm_head", C.c_void_p), ("final_norm", C.c_void_p)] + \
               [(n, C.POINTER(C.c_void_p)) for n in ("attn_norm", "w_qkv", "w_o", "mlp_norm", "w_gate_up", "w_down",
                                                     "w_router", "w_expert_gate_up", "w_expert_down", "w_shared_gate_up",
                                                     "w_shared_down")]


_OUT_FIELDS = ("tokens", "mask_bits", "n_decoded", "importance_prev", "importance", "delta_I", "K", "keep_bits",
               "cu_seqlens", "row_map", "conf", "argmax", "hidden_full", "hidden_packed", "logits", "route_experts",
               "route_weights")


class focus_step_out(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in _OUT_FIELDS]


class focus_seq_state(C.Structure):
    _fields_ = [("prefix_len", C.c_int32), ("total_steps", C.c_int32), ("token_sum", C.c_int64),
                ("mask_bits", C.c_uint64), ("processed_bits", C.c_uint64), ("cached_bits", C.c_uint64),
                ("tokens", C.c_int32 * FOCUS_MAX_BLOCK)]


class focus_router(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_experts", "experts_per_token", "score", "n_groups", "groups_kept", "group_top", "renormalize")] + \
               [("route_scale", C.c_float)]


class focus_mx(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("scales", C.c_void_p)]


class focus_kv(C.Structure):
    _fields_ = [("pool", C.c_void_p)] + [(n, C.c_int32) for n in ("dtype", "n_layers", "n_pages", "page_size", "n_kv_heads", "head_dim")]


_MX_FIELDS = ("w_gate_up", "w_down", "w_expert_gate_up", "w_expert_down", "w_shared_gate_up", "w_shared_down")


class focus_mx_weights(C.Structure):
    _fields_ = [(n, C.POINTER(focus_mx)) for n in _MX_FIELDS]


class FocusError(RuntimeError):
    def __init__(self, code: int, text: str):
        super().__init__("libfocus error %d: %s" % (code, text))
        self.code = code


def load_library() -> C.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError("libfocus.so is not built (%s): run `python -m paper_2601_23278_amd.build`" % LIB_PATH)
    lib = C.CDLL(LIB_PATH)
    P, I, SZ = C.c_void_p, C.c_int32, C.POINTER(C.c_size_t)
    sig = {
        "focus_workspace_bytes": [C.POINTER(focus_config), SZ],
        "focus_kv_pool_bytes": [C.POINTER(focus_config), SZ],
        "focus_init": [C.POINTER(focus_config), C.POINTER(focus_weights), P, C.c_size_t, P, C.c_size_t, C.POINTER(P)],
        "focus_prefill_kv": [P, P, I, C.POINTER(I), C.POINTER(I), C.POINTER(I), I, C.POINTER(I), I],
        "focus_step": [P, P, I, P, P, P, C.POINTER(focus_step_out)],
        "focus_select_compact": [P, P, I, P, P, P, C.POINTER(focus_step_out)],
        "focus_select_compact_noalloc": [C.POINTER(focus_config), P, I, P, P, P, P, P, P, C.POINTER(focus_step_out)],
        "focus_commit": [P, P, I, P, P, P, P, P, C.POINTER(focus_step_out)],
        "focus_run_layers": [P, P, I, P, P, P, I, I, P],
        "focus_finalize_blocks": [P, P, I, P, P],
        "focus_set_route_override": [P, P],
        "focus_set_row_hint": [P, I, I],
        "focus_run_steps": [P, P, I, P, I, I, P, C.POINTER(focus_step_out)],
        "focus_get_state": [P, I, C.POINTER(focus_seq_state)],
        "focus_set_state": [P, I, C.POINTER(focus_seq_state)],
        "focus_set_timing": [P, I],
        "focus_get_kernel_time": [P, I, C.POINTER(C.c_float), C.POINTER(I)],
        "focus_free": [P],
        "focus_route": [C.POINTER(focus_router), P, I, I, P, C.c_int64, P, P, P],
        "focus_mx_quantize": [P, I, C.c_int64, I, P, C.c_int64, P, P],
        "focus_mx_dequantize": [P, I, C.c_int64, I, C.POINTER(focus_mx), P, C.c_int64],
        "focus_mx_gemm_bytes": [I, I, I, I, SZ],
        "focus_mx_gemm": [P, I, I, I, I, P, P, C.c_int64, C.POINTER(focus_mx), I, P, C.c_int64, P, C.c_size_t],
        "focus_mx_experts_bytes": [I, I, I, I, I, SZ],
        "focus_mx_experts": [P, I, I, I, C.POINTER(focus_mx), C.POINTER(focus_mx), I, I, P, C.c_int64, P, P, I, P, C.c_int64, I, P, C.c_size_t],
        "focus_set_router": [P, C.POINTER(focus_router), C.POINTER(P)],
        "focus_set_mx_weights": [P, C.POINTER(focus_mx_weights)],
        "focus_kv_append": [C.POINTER(focus_kv), P, I, I, I, P, P, P, I, P, C.c_int64, P, C.c_int64],
        "focus_tree_attention_bytes": [C.POINTER(focus_kv), I, I, I, I, I, I, SZ],
        "focus_tree_attention": [C.POINTER(focus_kv), P, I, I, I, I, I, P, P, P, I, P, I, I, C.c_float, P, C.c_int64, P, C.c_int64, P, C.c_size_t],
        "focus_kv_compact": [C.POINTER(focus_kv), P, I, I, P, P, P, P, I, P, I],
        "focus_kv_fork_bytes": [I, SZ],
        "focus_kv_fork": [C.POINTER(focus_kv), P, I, I, P, P, P, I, P, P, P, P, P, C.c_size_t],
        "focus_kv_reserve_bytes": [I, SZ],
        "focus_kv_reserve": [P, I, I, I, P, I, P, I, P, P, P, C.c_size_t],
        "focus_beam_select_bytes": [I, I, I, I, SZ],
        "focus_beam_select": [P, I, I, I, I, I, P, C.c_int64, P, P, I, P, P, P, P, C.c_size_t],
    }
    for name, args in sig.items():
        f = getattr(lib, name)
        f.argtypes, f.restype = args, C.c_int
    lib.focus_last_error.argtypes, lib.focus_last_error.restype = [P], C.c_char_p
    return lib


_lib = load_library()
EXPORTS = ["focus_workspace_bytes", "focus_kv_pool_bytes", "focus_init", "focus_prefill_kv", "focus_step",
           "focus_select_compact", "focus_select_compact_noalloc", "focus_commit", "focus_run_layers", "focus_finalize_blocks", "focus_set_route_override", "focus_set_row_hint", "focus_run_steps", "focus_get_state", "focus_set_state", "focus_set_timing",
           "focus_get_kernel_time", "focus_free", "focus_last_error", "focus_route", "focus_mx_quantize", "focus_mx_dequantize",
           "focus_mx_gemm_bytes", "focus_mx_gemm", "focus_mx_experts_bytes", "focus_mx_experts", "focus_set_router", "focus_set_mx_weights",
           "focus_kv_append", "focus_tree_attention_bytes", "focus_tree_attention", "focus_kv_compact", "focus_kv_fork_bytes", "focus_kv_fork", "focus_kv_reserve_bytes",
           "focus_kv_reserve", "focus_beam_select_bytes", "focus_beam_select"]


def _check(rc: int, ctx=None):
    if rc != FOCUS_OK:
        raise FocusError(rc, (_lib.focus_last_error(ctx) or b"").decode())


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else C.c_void_p(t.data_ptr())


def _i32(xs: Optional[Sequence[int]]):
    return None if xs is None else (C.c_int32 * len(xs))(*xs)


def focus_workspace_bytes(cfg: focus_config) -> int:
    n = C.c_size_t()
    _check(_lib.focus_workspace_bytes(C.byref(cfg), C.byref(n)))
    return n.value


def focus_kv_pool_bytes(cfg: focus_config) -> int:
    n = C.c_size_t()
    _check(_lib.focus_kv_pool_bytes(C.byref(cfg), C.byref(n)))
    return n.value


FOCUS_NOALLOC_MAX_SEQ = 16384


def focus_select_compact_noalloc(cfg: focus_config, n_seq: int, delta_I: torch.Tensor, mask_bits: torch.Tensor,
                                 out: "focus_step_out", cached_bits: Optional[torch.Tensor] = None,
                                 token_sum: Optional[torch.Tensor] = None, total_steps: Optional[torch.Tensor] = None,
                                 k_override: Optional[torch.Tensor] = None, stream=None):
    _check(_lib.focus_select_compact_noalloc(C.byref(cfg), Focus._stream(stream), n_seq, _ptr(delta_I), _ptr(mask_bits),
                                             _ptr(cached_bits), _ptr(token_sum), _ptr(total_steps), _ptr(k_override),
                                             C.byref(out)))


# -- expert routing and MXFP4 (no context) ----------------------------------------------------------
# A matrix in MXFP4 is a pair (codes, scales) of contiguous uint8 tensors, [..., K / 2] and [..., K / 32].  Tensors are checked here, on the host: the
# library sees addresses only.  They live on the current device; the work goes to `stream`, or to torch's current one.  Outputs that are not
# given, and workspaces, are torch tensors made on the call's stream.
_DTYPES = {torch.float32: FOCUS_F32, torch.bfloat16: FOCUS_BF16}


def _bad(text: str, *args):
    raise FocusError(FOCUS_EINVAL, text % args)


def _begin(device, stream) -> int:
    """Address of the stream that a call's work goes to; its tensors live on `device`, which has to be the current one."""
    if device.type != "cuda" or device.index != torch.cuda.current_device():
        _bad("tensors must be on the current device, not on %s", device)
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(device.index)
    if stream.device_index != device.index:
        _bad("the stream belongs to another device than %s", device)
    return stream.cuda_stream


def _new(shape, dtype, device, stream):
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _rows_of(t: torch.Tensor, name: str):
    """(rows, columns, distance of rows, dtype code) of a matrix whose rows are contiguous."""
    if t.dim() != 2:
        _bad("%s must be a matrix", name)
    (rows, cols), (ld, step) = t.shape, t.stride()
    if rows >= 2 ** 31 or cols >= 2 ** 31:
        _bad("%s is too large", name)
    if (cols > 1 and step != 1) or (rows > 1 and ld < cols):
        _bad("%s must be a matrix with contiguous rows that do not overlap", name)
    code = _DTYPES.get(t.dtype)
    if code is None:
        _bad("%s has an unsupported dtype", name)
    return rows, cols, ld if rows > 1 else cols, code


def _int32(*sizes: int):
    """The C entries take 32-bit sizes, and ctypes cuts longer ones off."""
    if max(sizes) >= 2 ** 31 or min(sizes) < -2 ** 31:
        _bad("a size is too large: %s", sizes)


def _plain(t: torch.Tensor, name: str, shape, dtype, device=None):
    if t.shape != shape or t.dtype != dtype or not t.is_contiguous() or (device is not None and t.device != device):
        _bad("%s must be a contiguous %s tensor of shape %s%s", name, dtype, tuple(shape), "" if device is None else " on %s" % device)


def _mx_of(mx, name: str, *lead: int, device=None) -> tuple:
    """(focus_mx, K) of a pair of codes [*lead, K / 2] and scales [*lead, K / 32]."""
    codes, scales = mx
    blocks = scales.shape[-1] if scales.dim() else 0
    if blocks >= 2 ** 26:
        _bad("%s is too large", name)
    _plain(codes, name + " (codes)", (*lead, 16 * blocks), torch.uint8, device)
    _plain(scales, name + " (scales)", (*lead, blocks), torch.uint8, device)
    return focus_mx(codes.data_ptr(), scales.data_ptr()), 32 * blocks


def _scratch(workspace, nbytes: int, device, stream):
    """(address, bytes) of the caller's workspace, or of one made for the call, and the tensor that keeps it alive."""
    if workspace is None:
        if nbytes == 0:
            return None, 0, None
        workspace = _new(nbytes, torch.uint8, device, stream)
    elif workspace.device != device or not workspace.is_contiguous():
        _bad("the workspace must be a contiguous tensor on %s", device)
    return workspace.data_ptr(), workspace.numel() * workspace.element_size(), workspace


def focus_route(router: focus_router, logits: torch.Tensor, bias: Optional[torch.Tensor] = None, experts: Optional[torch.Tensor] = None,
                weights: Optional[torch.Tensor] = None, stream=None):
    """(experts [rows, k] int32, weights [rows, k] fp32) of the rows of logits [rows, E], fp32 or bf16."""
    rows, cols, ld, dtype = _rows_of(logits, "logits")
    dev, k = logits.device, router.experts_per_token
    to = _begin(dev, stream)
    if cols != router.n_experts or not 1 <= k <= 32:
        _bad("logits have %d columns; the router has %d experts, %d of them for a row", cols, router.n_experts, k)
    if bias is not None:
        _plain(bias, "bias", (cols,), torch.float32, dev)
    if experts is None:
        experts = _new((rows, k), torch.int32, dev, stream)
    else:
        _plain(experts, "experts", (rows, k), torch.int32, dev)
    if weights is None:
        weights = _new((rows, k), torch.float32, dev, stream)
    else:
        _plain(weights, "weights", (rows, k), torch.float32, dev)
    rc = _lib.focus_route(router, to, rows, dtype, logits.data_ptr(), ld, None if bias is None else bias.data_ptr(), experts.data_ptr(), weights.data_ptr())
    if rc:
        _check(rc)
    return experts, weights


def focus_mx_quantize(x: torch.Tensor, codes: Optional[torch.Tensor] = None, scales: Optional[torch.Tensor] = None, stream=None):
    """(codes, scales) of the rows of x [rows, cols], fp32 or bf16."""
    rows, cols, ld, dtype = _rows_of(x, "x")
    dev, blocks = x.device, (cols + 31) // 32
    to = _begin(dev, stream)
    if codes is None:
        codes = _new((rows, 16 * blocks), torch.uint8, dev, stream)
    else:
        _plain(codes, "codes", (rows, 16 * blocks), torch.uint8, dev)
    if scales is None:
        scales = _new((rows, blocks), torch.uint8, dev, stream)
    else:
        _plain(scales, "scales", (rows, blocks), torch.uint8, dev)
    rc = _lib.focus_mx_quantize(to, dtype, rows, cols, x.data_ptr(), ld, codes.data_ptr(), scales.data_ptr())
    if rc:
        _check(rc)
    return codes, scales


def focus_mx_dequantize(codes: torch.Tensor, scales: torch.Tensor, out: torch.Tensor, stream=None):
    """The values of codes and scales, into out [rows, cols], fp32 or bf16."""
    rows, cols, ld, dtype = _rows_of(out, "out")
    to = _begin(out.device, stream)
    mx, k = _mx_of((codes, scales), "mx", rows, device=out.device)
    if k != (cols + 31) // 32 * 32:
        _bad("codes have %d elements a row, out %d columns", k, cols)
    rc = _lib.focus_mx_dequantize(to, dtype, rows, cols, mx, out.data_ptr(), ld)
    if rc:
        _check(rc)
    return out


def focus_mx_gemm_bytes(m: int, n: int, k: int, a_type: int) -> int:
    _int32(m, n, k)
    nbytes = C.c_size_t()
    _check(_lib.focus_mx_gemm_bytes(m, n, k, a_type, C.byref(nbytes)))
    return nbytes.value


def focus_mx_gemm(a, w, out: torch.Tensor, workspace: Optional[torch.Tensor] = None, stream=None):
    """out [m, n] (fp32 or bf16) = A W^T; w the pair of an MXFP4 [n, k], a a bf16 matrix [m, k] or the pair of an MXFP4 [m, k]."""
    m, n, ldc, c_type = _rows_of(out, "out")
    dev = out.device
    to = _begin(dev, stream)
    mw, k = _mx_of(w, "w", n, device=dev)
    if isinstance(a, torch.Tensor):
        rows, cols, lda, a_type = _rows_of(a, "a")
        if a_type != FOCUS_BF16 or a.device != dev:
            _bad("a must be bf16 and on %s", dev)
        a_ptr, a_scales = a.data_ptr(), None
    else:
        ma, cols = _mx_of(a, "a", m, device=dev)
        rows, lda, a_type, a_ptr, a_scales = m, cols, FOCUS_MX4, ma.codes, ma.scales
    if rows != m or cols != k:
        _bad("a is %d x %d, out %d x %d and w has %d columns", rows, cols, m, n, k)
    ws, ws_bytes, keep = _scratch(workspace, focus_mx_gemm_bytes(m, n, k, a_type) if workspace is None else 0, dev, stream)
    rc = _lib.focus_mx_gemm(to, m, n, k, a_type, a_ptr, a_scales, lda, mw, c_type, out.data_ptr(), ldc, ws, ws_bytes)
    if rc:
        _check(rc)
    return out


def focus_mx_experts_bytes(n_experts: int, hidden: int, ffn: int, n_rows: int, k: int) -> int:
    _int32(n_experts, hidden, ffn, n_rows, k)
    nbytes = C.c_size_t()
    _check(_lib.focus_mx_experts_bytes(n_experts, hidden, ffn, n_rows, k, C.byref(nbytes)))
    return nbytes.value


def focus_mx_experts(gate_up, down, x: torch.Tensor, experts: torch.Tensor, weights: torch.Tensor, out: torch.Tensor, add: bool = False,
                     workspace: Optional[torch.Tensor] = None, stream=None):
    """out [rows, hidden] (+)= the routed SwiGLU experts of x [rows, hidden] bf16; gate_up, down the pairs of an MXFP4 [E, 2 ffn, hidden] and
    [E, hidden, ffn]; experts [rows, k] int32, weights [rows, k] fp32."""
    rows, hidden, ldx, x_type = _rows_of(x, "x")
    out_rows, out_cols, ldo, out_type = _rows_of(out, "out")
    dev = out.device
    to = _begin(dev, stream)
    if x_type != FOCUS_BF16 or x.device != dev:
        _bad("x must be bf16 and on %s", dev)
    if gate_up[0].dim() != 3 or experts.dim() != 2:
        _bad("gate_up has three dimensions, experts two")
    (E, two_ffn, _), k = gate_up[0].shape, experts.shape[1]
    _int32(E, k)
    mg, hidden_g = _mx_of(gate_up, "gate_up", E, two_ffn, device=dev)
    md, ffn = _mx_of(down, "down", E, hidden, device=dev)
    if hidden_g != hidden or two_ffn != 2 * ffn or out_rows != rows or out_cols != hidden:
        _bad("x, out, gate_up and down do not fit together")
    _plain(experts, "experts", (rows, k), torch.int32, dev)
    _plain(weights, "weights", (rows, k), torch.float32, dev)
    ws, ws_bytes, keep = _scratch(workspace, focus_mx_experts_bytes(E, hidden, ffn, rows, k) if workspace is None else 0, dev, stream)
    rc = _lib.focus_mx_experts(to, E, hidden, ffn, mg, md, rows, k, x.data_ptr(), ldx, experts.data_ptr(), weights.data_ptr(), out_type, out.data_ptr(), ldo,
                               int(add), ws, ws_bytes)
    if rc:
        _check(rc)
    return out


# -- generation that branches over the paged cache (no context) ---------------------------------------
# A pool is a contiguous tensor [n_layers, n_pages, 2, H_kv, page_size, D], fp32 or bf16 (the values, its second half, are kept transposed: [H_kv, D, page_size]).
# Page tables [rows, stride], lengths, reference counts and lists are contiguous int32 tensors.

def _kv_of(pool: torch.Tensor) -> focus_kv:
    shape = pool.shape
    code = _DTYPES.get(pool.dtype)
    if len(shape) != 6 or shape[2] != 2 or shape[5] == 0 or code is None or not pool.is_contiguous():
        _bad("a pool is a contiguous fp32 or bf16 tensor [n_layers, n_pages, 2, H_kv, page_size, D]")
    _int32(*shape)
    return focus_kv(pool.data_ptr(), code, shape[0], shape[1], shape[4], shape[3], shape[5])


def _table_of(table: torch.Tensor, name: str, device):
    """(rows, stride) of a page table."""
    if table.dim() != 2 or table.dtype != torch.int32 or not table.is_contiguous() or table.device != device:
        _bad("%s must be a contiguous int32 matrix on %s", name, device)
    _int32(*table.shape)
    return table.shape


def _cu_of(cu: torch.Tensor, name: str, n: int, device):
    _plain(cu, name, (n + 1,), torch.int32, device)
    return cu.data_ptr()


def focus_kv_append(pool: torch.Tensor, layer: int, k: torch.Tensor, v: torch.Tensor, cu_rows: torch.Tensor, lens: torch.Tensor, page_table: torch.Tensor, stream=None):
    """Rows of k and v [rows, H_kv * D] become the next tokens of their sequences: row r of sequence b (cu_rows[b] <= r < cu_rows[b + 1]) token
    lens[b] + r - cu_rows[b] of a layer of the pool."""
    kv, dev = _kv_of(pool), pool.device
    to = _begin(dev, stream)
    n, stride = _table_of(page_table, "page_table", dev)
    rows, cols, ldk, k_type = _rows_of(k, "k")
    v_rows, v_cols, ldv, v_type = _rows_of(v, "v")
    if k.device != dev or v.device != dev or k_type != kv.dtype or v_type != kv.dtype or v_rows != rows or cols != kv.n_kv_heads * kv.head_dim or v_cols != cols:
        _bad("k and v must be matrices [rows, %d] of the pool's type on %s", kv.n_kv_heads * kv.head_dim, dev)
    _plain(lens, "lens", (n,), torch.int32, dev)
    _int32(layer)
    rc = _lib.focus_kv_append(kv, to, layer, n, rows, _cu_of(cu_rows, "cu_rows", n, dev), lens.data_ptr(), page_table.data_ptr(), stride, k.data_ptr(), ldk, v.data_ptr(), ldv)
    if rc:
        _check(rc)


def focus_tree_attention(pool: torch.Tensor, layer: int, q: torch.Tensor, cu_rows: torch.Tensor, lens: torch.Tensor, page_table: torch.Tensor,
                         seen: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None, scale: Optional[float] = None, max_rows: int = 0, max_len: int = 0,
                         workspace: Optional[torch.Tensor] = None, stream=None):
    """Attention of the query rows q [rows, H_q * D] over the cached tokens of their sequences and over the drafted ones behind them that the bits of seen
    ([rows] or [rows, words] int64, contiguous; None: a chain) show.  max_rows, max_len: the most rows of a sequence, and the longest lens[b] + rows, as far as
    the caller knows.  scale: 1 / sqrt(D)."""
    kv, dev = _kv_of(pool), pool.device
    to = _begin(dev, stream)
    n, stride = _table_of(page_table, "page_table", dev)
    rows, cols, ldq, q_type = _rows_of(q, "q")
    if q.device != dev or q_type != kv.dtype or cols % kv.head_dim or cols == 0:
        _bad("q must be a matrix of heads of %d, of the pool's type, on %s", kv.head_dim, dev)
    if out is None:
        out = _new((rows, cols), q.dtype, dev, stream)
        ldo = cols
    else:
        out_rows, out_cols, ldo, out_type = _rows_of(out, "out")
        if out_rows != rows or out_cols != cols or out_type != q_type or out.device != dev:
            _bad("out must be like q")
    words = 0
    if seen is not None:
        words = seen.shape[1] if seen.dim() == 2 else 1
        _int32(words)
        _plain(seen, "seen", (rows, words) if seen.dim() == 2 else (rows,), torch.int64, dev)
    _plain(lens, "lens", (n,), torch.int32, dev)
    _int32(layer, max_rows, max_len)
    heads = cols // kv.head_dim
    if workspace is None:
        nbytes = C.c_size_t()
        rc = _lib.focus_tree_attention_bytes(kv, n, rows, max_rows, max_len, stride, heads, nbytes)
        if rc:
            _check(rc)
        ws, ws_bytes, keep = _scratch(None, nbytes.value, dev, stream)
    else:
        ws, ws_bytes, keep = _scratch(workspace, 0, dev, stream)
    rc = _lib.focus_tree_attention(kv, to, layer, n, rows, max_rows, max_len, _cu_of(cu_rows, "cu_rows", n, dev), lens.data_ptr(), page_table.data_ptr(), stride,
                                   None if seen is None else seen.data_ptr(), words, heads, kv.head_dim ** -0.5 if scale is None else scale, q.data_ptr(), ldq,
                                   out.data_ptr(), ldo, ws, ws_bytes)
    if rc:
        _check(rc)
    return out


def focus_kv_compact(pool: torch.Tensor, start: torch.Tensor, cu_keep: torch.Tensor, keep: torch.Tensor, page_table: torch.Tensor, to_table: Optional[torch.Tensor] = None,
                     stream=None):
    """Token start[b] + keep[cu_keep[b] + i] of row b's pages in page_table becomes token start[b] + i of its pages in to_table (None: page_table, in place), in
    every layer.  keep ascends within a sequence."""
    kv, dev = _kv_of(pool), pool.device
    to = _begin(dev, stream)
    n, stride = _table_of(page_table, "page_table", dev)
    if to_table is None:
        to_table = page_table
    to_rows, to_stride = _table_of(to_table, "to_table", dev)
    if to_rows != n:
        _bad("to_table must have a row for each of page_table")
    _plain(start, "start", (n,), torch.int32, dev)
    if keep.dim() != 1:
        _bad("keep must be a list")
    _int32(keep.shape[0])
    _plain(keep, "keep", keep.shape, torch.int32, dev)
    rc = _lib.focus_kv_compact(kv, to, n, keep.shape[0], start.data_ptr(), _cu_of(cu_keep, "cu_keep", n, dev), keep.data_ptr(), page_table.data_ptr(), stride, to_table.data_ptr(),
                               to_stride)
    if rc:
        _check(rc)


def _int32_out(t: Optional[torch.Tensor], name: str, shape, device, stream):
    if t is None:
        return _new(shape, torch.int32, device, stream)
    _plain(t, name, shape, torch.int32, device)
    return t


def focus_kv_fork(pool: torch.Tensor, parents: torch.Tensor, lens: torch.Tensor, page_table: torch.Tensor, refs: torch.Tensor, new_lens: Optional[torch.Tensor] = None,
                  new_table: Optional[torch.Tensor] = None, lacking: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None):
    """(new_lens, new_table, lacking) of rows that continue the rows parents of page_table; refs [n_pages], how many entries hold a page, follows.  No parents: all
    rows give their pages back."""
    kv, dev = _kv_of(pool), pool.device
    to = _begin(dev, stream)
    n_old, stride = _table_of(page_table, "page_table", dev)
    if parents.dim() != 1:
        _bad("parents must be a list")
    n_new = parents.shape[0]
    _int32(n_new)
    _plain(parents, "parents", (n_new,), torch.int32, dev)
    _plain(lens, "lens", (n_old,), torch.int32, dev)
    _plain(refs, "refs", (kv.n_pages,), torch.int32, dev)
    new_lens = _int32_out(new_lens, "new_lens", (n_new,), dev, stream)
    new_table = _int32_out(new_table, "new_table", (n_new, stride), dev, stream)
    lacking = _int32_out(lacking, "lacking", (n_new,), dev, stream)
    if workspace is None:
        nbytes = C.c_size_t()
        rc = _lib.focus_kv_fork_bytes(n_new, nbytes)
        if rc:
            _check(rc)
        ws, ws_bytes, keep = _scratch(None, nbytes.value, dev, stream)
    else:
        ws, ws_bytes, keep = _scratch(workspace, 0, dev, stream)
    rc = _lib.focus_kv_fork(kv, to, n_old, n_new, parents.data_ptr(), lens.data_ptr(), page_table.data_ptr(), stride, new_lens.data_ptr(), new_table.data_ptr(),
                            refs.data_ptr(), lacking.data_ptr(), ws, ws_bytes)
    if rc:
        _check(rc)
    return new_lens, new_table, lacking


def focus_kv_reserve(lens: torch.Tensor, room: int, page_table: torch.Tensor, refs: torch.Tensor, page_size: int, lacking: Optional[torch.Tensor] = None,
                     workspace: Optional[torch.Tensor] = None, stream=None):
    """Gives the rows of page_table the pages that lens + room tokens need; returns how many pages each still lacks."""
    dev = page_table.device
    to = _begin(dev, stream)
    n, stride = _table_of(page_table, "page_table", dev)
    if refs.dim() != 1:
        _bad("refs must be a list")
    _int32(refs.shape[0], room, page_size)
    _plain(refs, "refs", refs.shape, torch.int32, dev)
    _plain(lens, "lens", (n,), torch.int32, dev)
    lacking = _int32_out(lacking, "lacking", (n,), dev, stream)
    if workspace is None:
        nbytes = C.c_size_t()
        rc = _lib.focus_kv_reserve_bytes(n, nbytes)
        if rc:
            _check(rc)
        ws, ws_bytes, keep = _scratch(None, nbytes.value, dev, stream)
    else:
        ws, ws_bytes, keep = _scratch(workspace, 0, dev, stream)
    rc = _lib.focus_kv_reserve(to, n, page_size, refs.shape[0], lens.data_ptr(), room, page_table.data_ptr(), stride, refs.data_ptr(), lacking.data_ptr(), ws, ws_bytes)
    if rc:
        _check(rc)
    return lacking


def focus_beam_select(logits: torch.Tensor, scores: torch.Tensor, k: int, done: Optional[torch.Tensor] = None, end_token: int = 0, rows: Optional[torch.Tensor] = None,
                      tokens: Optional[torch.Tensor] = None, new_scores: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None):
    """(rows, tokens, new_scores), each [n, k]: the k best of every request's candidates; logits [n * n_beams, vocab] fp32 or bf16, scores [n, n_beams] fp32, done
    [n, n_beams] bool or uint8.  rows are rows of logits, -1 where no candidate was left."""
    n_rows, vocab, ld, dtype = _rows_of(logits, "logits")
    dev = logits.device
    to = _begin(dev, stream)
    if scores.dim() != 2 or scores.shape[0] * scores.shape[1] != n_rows:
        _bad("scores must be a matrix with a value for each of the %d rows of logits", n_rows)
    n, beams = scores.shape
    _int32(n, beams, k, end_token)
    _plain(scores, "scores", (n, beams), torch.float32, dev)
    if done is not None:
        _plain(done, "done", (n, beams), torch.bool if done.dtype == torch.bool else torch.uint8, dev)
    nbytes = C.c_size_t()
    rc = _lib.focus_beam_select_bytes(n, beams, vocab, k, nbytes)
    if rc:
        _check(rc)
    rows = _int32_out(rows, "rows", (n, k), dev, stream)
    tokens = _int32_out(tokens, "tokens", (n, k), dev, stream)
    if new_scores is None:
        new_scores = _new((n, k), torch.float32, dev, stream)
    else:
        _plain(new_scores, "new_scores", (n, k), torch.float32, dev)
    ws, ws_bytes, keep = _scratch(workspace, nbytes.value, dev, stream)
    rc = _lib.focus_beam_select(to, n, beams, vocab, k, dtype, logits.data_ptr(), ld, scores.data_ptr(), None if done is None else done.data_ptr(), end_token,
                                rows.data_ptr(), tokens.data_ptr(), new_scores.data_ptr(), ws, ws_bytes)
    if rc:
        _check(rc)
    return rows, tokens, new_scores


def make_step_out(**tensors) -> focus_step_out:
    o = focus_step_out()
    for k, t in tensors.items():
        if k not in _OUT_FIELDS:
            raise KeyError(k)
        setattr(o, k, None if t is None else t.data_ptr())
    return o


class Focus:
    """A context: marshals tensors to the C ABI and keeps the borrowed buffers alive."""

    def __init__(self, cfg: focus_config, embed: torch.Tensor, lm_head: torch.Tensor, final_norm: torch.Tensor,
                 layers: List[Dict[str, torch.Tensor]], kv_pool: torch.Tensor, workspace: Optional[torch.Tensor] = None):
        self.cfg = cfg
        self.keep = [embed, lm_head, final_norm, layers, kv_pool]
        need = focus_workspace_bytes(cfg)
        if workspace is None:
            workspace = torch.empty(need, dtype=torch.uint8, device=kv_pool.device)
        self.workspace = workspace
        w = focus_weights()
        w.embed, w.lm_head, w.final_norm = embed.data_ptr(), lm_head.data_ptr(), final_norm.data_ptr()
        self._arrays = {}
        names = ["attn_norm", "w_qkv", "w_o", "mlp_norm", "w_gate_up", "w_down"]
        if cfg.n_experts > 0:
            names += ["w_router", "w_expert_gate_up", "w_expert_down"] + (["w_shared_gate_up", "w_shared_down"] if cfg.shared_ffn else [])
        for name in names:
            arr = (C.c_void_p * cfg.n_layers)(*[l[name].data_ptr() if name in l else None for l in layers])
            self._arrays[name] = arr
            setattr(w, name, arr)
        self._ctx = C.c_void_p()
        _check(_lib.focus_init(C.byref(cfg), C.byref(w), _ptr(kv_pool), kv_pool.numel() * kv_pool.element_size(),
                               _ptr(workspace), workspace.numel(), C.byref(self._ctx)))

    # -- entry points, same names as the header -------------------------------------------------
    def focus_prefill_kv(self, prefix_len: Sequence[int], page_table: Sequence[Sequence[int]],
                         prompt_tokens: Optional[Sequence[Sequence[int]]] = None,
                         seq_slot: Optional[Sequence[int]] = None, keep_stats: bool = False, stream=None):
        n = len(prefix_len)
        stride = max([len(t) for t in page_table] + [1])
        flat = [-1] * (n * stride)
        for b, t in enumerate(page_table):
            flat[b * stride:b * stride + len(t)] = list(t)
        prompts = None if prompt_tokens is None else [t for row in prompt_tokens for t in row]
        _check(_lib.focus_prefill_kv(self._ctx, self._stream(stream), n, _i32(seq_slot), _i32(list(prefix_len)),
                                     _i32(flat), stride, _i32(prompts), int(keep_stats)), self._ctx)

    def focus_step(self, n_seq: int, seq_slot: Optional[torch.Tensor] = None, k_override: Optional[torch.Tensor] = None,
                   keep_override: Optional[torch.Tensor] = None, out: Optional[focus_step_out] = None, stream=None):
        _check(_lib.focus_step(self._ctx, self._stream(stream), n_seq, _ptr(seq_slot), _ptr(k_override),
                               _ptr(keep_override), None if out is None else C.byref(out)), self._ctx)

    def focus_select_compact(self, n_seq: int, delta_I: torch.Tensor, out: focus_step_out,
                             seq_slot: Optional[torch.Tensor] = None, k_override: Optional[torch.Tensor] = None, stream=None):
        _check(_lib.focus_select_compact(self._ctx, self._stream(stream), n_seq, _ptr(seq_slot), _ptr(delta_I),
                                         _ptr(k_override), C.byref(out)), self._ctx)

    def focus_commit(self, n_seq: int, keep_bits: torch.Tensor, cu_seqlens: torch.Tensor, conf: torch.Tensor,
                     argmax: torch.Tensor, out: Optional[focus_step_out] = None, seq_slot: Optional[torch.Tensor] = None,
                     stream=None):
        _check(_lib.focus_commit(self._ctx, self._stream(stream), n_seq, _ptr(seq_slot), _ptr(keep_bits), _ptr(cu_seqlens),
                                 _ptr(conf), _ptr(argmax), None if out is None else C.byref(out)), self._ctx)

    def focus_run_layers(self, n_seq: int, keep_bits: torch.Tensor, vis_bits: torch.Tensor, layer_begin: int,
                         layer_end: int, hidden: torch.Tensor, seq_slot: Optional[torch.Tensor] = None, stream=None):
        _check(_lib.focus_run_layers(self._ctx, self._stream(stream), n_seq, _ptr(seq_slot), _ptr(keep_bits), _ptr(vis_bits),
                                     layer_begin, layer_end, _ptr(hidden)), self._ctx)

    def focus_finalize_blocks(self, n_seq: int, finalized: Optional[torch.Tensor] = None, seq_slot: Optional[torch.Tensor] = None,
                              stream=None):
        _check(_lib.focus_finalize_blocks(self._ctx, self._stream(stream), n_seq, _ptr(seq_slot), _ptr(finalized)), self._ctx)

    def focus_run_steps(self, n_seq: int, n_steps: int, finalize: bool = True, decoded: Optional[torch.Tensor] = None,
                        out: Optional[focus_step_out] = None, seq_slot: Optional[torch.Tensor] = None, stream=None):
        _check(_lib.focus_run_steps(self._ctx, self._stream(stream), n_seq, _ptr(seq_slot), n_steps, int(finalize), _ptr(decoded),
                                    None if out is None else C.byref(out)), self._ctx)

    def focus_set_route_override(self, experts: Optional[torch.Tensor]):
        self._route_override = experts       # borrowed by the library
        _check(_lib.focus_set_route_override(self._ctx, _ptr(experts)), self._ctx)

    def focus_set_row_hint(self, packed_rows: int, rows_per_seq: int = 0):
        _check(_lib.focus_set_row_hint(self._ctx, packed_rows, rows_per_seq), self._ctx)

    def focus_set_router(self, router: Optional[focus_router], bias: Optional[Sequence[Optional[torch.Tensor]]] = None):
        """bias: one fp32 tensor [E], or None, per layer."""
        E, bias = self.cfg.n_experts, None if bias is None else list(bias)
        for b in bias or ():
            if b is not None:
                _plain(b, "bias", (E,), torch.float32, self.workspace.device)
        if bias is not None and len(bias) != self.cfg.n_layers:
            _bad("one bias per layer")
        arr = None if bias is None else (C.c_void_p * len(bias))(*[None if b is None else b.data_ptr() for b in bias])
        _check(_lib.focus_set_router(self._ctx, None if router is None else C.byref(router), arr), self._ctx)
        self._router_bias = None if router is None else bias             # borrowed by the library

    def focus_set_mx_weights(self, layers: Optional[Sequence[Dict[str, tuple]]]):
        """layers: per layer a dict of matrix name (w_gate_up, w_expert_down, ...) -> pair (codes, scales); {} leaves a layer on the matrices
        the context was made with."""
        if layers is None:
            _check(_lib.focus_set_mx_weights(self._ctx, None), self._ctx)
            self._mx_layers = None
            return
        g = self.cfg
        if len(layers) != g.n_layers:
            _bad("one entry per layer")
        shapes = {"w_gate_up": (2 * g.ffn, g.hidden), "w_down": (g.hidden, g.ffn),
                  "w_expert_gate_up": (g.n_experts, 2 * g.expert_ffn, g.hidden), "w_expert_down": (g.n_experts, g.hidden, g.expert_ffn),
                  "w_shared_gate_up": (2 * g.shared_ffn, g.hidden), "w_shared_down": (g.hidden, g.shared_ffn)}
        layers = [{name: tuple(pair) for name, pair in l.items()} for l in layers]
        for name in {name for l in layers for name in l}.difference(shapes):
            _bad("%s is no matrix of a feed-forward", name)
        w, arrays = focus_mx_weights(), []
        for name in _MX_FIELDS:
            if any(name in l for l in layers):
                pairs = [_mx_of(l[name], name, *shapes[name][:-1], device=self.workspace.device) if name in l else (focus_mx(), shapes[name][-1]) for l in layers]
                if any(k != shapes[name][-1] for _, k in pairs):
                    _bad("%s has another width", name)
                arrays.append((focus_mx * len(layers))(*[m for m, _ in pairs]))
                setattr(w, name, arrays[-1])
        _check(_lib.focus_set_mx_weights(self._ctx, C.byref(w)), self._ctx)
        self._mx_layers = layers             # borrowed by the library

    def focus_get_state(self, slot: int) -> focus_seq_state:
        st = focus_seq_state()
        _check(_lib.focus_get_state(self._ctx, slot, C.byref(st)), self._ctx)
        return st

    def focus_set_state(self, slot: int, st: focus_seq_state):
        _check(_lib.focus_set_state(self._ctx, slot, C.byref(st)), self._ctx)

    def focus_set_timing(self, enable: bool):
        _check(_lib.focus_set_timing(self._ctx, int(enable)), self._ctx)

    def focus_get_kernel_time(self, kernel_class: int):
        ms, n = C.c_float(), C.c_int32()
        _check(_lib.focus_get_kernel_time(self._ctx, kernel_class, C.byref(ms), C.byref(n)), self._ctx)
        return ms.value, n.value

    def focus_free(self):
        if self._ctx:
            _lib.focus_free(self._ctx)
            self._ctx = C.c_void_p()

    def __del__(self):
        try:
            self.focus_free()
        except Exception:
            pass

    @staticmethod
    def _stream(stream):
        if stream is None:
            stream = torch.cuda.current_stream()
        return C.c_void_p(stream.cuda_stream)
