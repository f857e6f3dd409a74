"""Thin ctypes binding of libmuxq.so (the C ABI declared in include/muxq.h).

Argument marshalling only: torch tensors supply device memory and the current
HIP stream; every step of the computation runs inside the library's kernels.
There is no CPU fallback: if the shared library is missing, loading raises.
"""
import ctypes as C
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmuxq.so")

PER_TENSOR, PER_CHANNEL = 0, 1
_GRAN = {"tensor": PER_TENSOR, "channel": PER_CHANNEL, PER_TENSOR: PER_TENSOR,
         PER_CHANNEL: PER_CHANNEL}

EXPORTS = ["muxq_version", "muxq_status_string", "muxq_k_pad", "muxq_wq_bytes",
           "muxq_packed_bytes", "muxq_packed_index", "muxq_detect_scratch_bytes",
           "muxq_workspace_layout", "muxq_workspace_bytes", "muxq_quantize_weight", "muxq_quantize_weight_bits", "muxq_linear_opts",
           "muxq_detect_outliers", "muxq_build_aux", "muxq_linear",
           "muxq_linear_naive_int8", "muxq_gemm_i8", "muxq_init", "muxq_linear_timed",
           "muxq_noalloc_max_bytes", "muxq_linear_noalloc", "muxq_linear_gelu", "muxq_linear_gelu_slabs",
           "muxq_mlp", "muxq_mlp_workspace_bytes",
           "muxq_quantize_weight_smooth", "muxq_smooth_absmax",
           "muxq_probe_mfma_rate", "muxq_gemm_kernel", "muxq_code_kernel", "muxq_static_bytes", "muxq_static_layout_of",
           "muxq_prepare_static", "muxq_linear_static", "muxq_gelu_absmax",
           "muxq_kv_append", "muxq_kv_gather", "muxq_paged_attention", "muxq_paged_attention_workspace_bytes",
           "muxq_lora", "muxq_lora_workspace_bytes", "muxq_norm", "muxq_norm_slabs", "muxq_norm_scratch_bytes",
           "muxq_window_attention", "muxq_window_attention_workspace_bytes", "muxq_tree_attention",
           "muxq_tree_attention_workspace_bytes", "muxq_verify_tree", "muxq_kv_copy", "muxq_kv_compact"]


class MuxqError(RuntimeError):
    pass


class WsLayout(C.Structure):
    _fields_ = [(n, C.c_size_t) for n in
                ("col_absmax", "col_scale", "col_slot", "col_mask", "outlier_idx", "n_outliers",
                 "x_scale", "absmax_partial", "body_q", "aux_q", "w_aux", "cn", "total")] + [("k_pad", C.c_int32)]


class StaticLayout(C.Structure):
    _fields_ = [(n, C.c_size_t) for n in ("col_mask", "outlier_idx", "n_outliers", "w_aux", "total")] + \
               [("k_pad", C.c_int32)]


class ActOpts(C.Structure):
    _fields_ = [("x_gran", C.c_int32), ("ia_bits", C.c_int32), ("absmax_ready", C.c_int32),
                ("aux_own_scale", C.c_int32), ("absmax_slabs", C.c_int32)]


class KvCache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p)] + \
               [(n, C.c_int32) for n in ("type", "n_blocks", "block_size", "n_kv_heads", "head_dim", "reserved")] + \
               [(n, C.c_int64) for n in ("ld_block", "ld_head", "ld_token")]


X_PER_TENSOR, X_PER_TOKEN = 0, 1
_XGRAN = {"tensor": X_PER_TENSOR, "token": X_PER_TOKEN, X_PER_TENSOR: X_PER_TENSOR,
          X_PER_TOKEN: X_PER_TOKEN}

_lib = None


def lib():
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise MuxqError(f"{LIB_PATH} is missing: build it with "
                            "`python -m paper_2604_04701_amd.build` (there is no fallback path)")
        L = C.CDLL(LIB_PATH)
        vp, i, f, sz = C.c_void_p, C.c_int, C.c_float, C.c_size_t
        L.muxq_version.restype = i
        L.muxq_status_string.restype = C.c_char_p
        L.muxq_status_string.argtypes = [i]
        L.muxq_k_pad.restype = i
        L.muxq_k_pad.argtypes = [i]
        L.muxq_wq_bytes.restype = sz
        L.muxq_wq_bytes.argtypes = [i, i]
        L.muxq_packed_bytes.restype = sz
        L.muxq_packed_bytes.argtypes = [i, i]
        L.muxq_packed_index.restype = sz
        L.muxq_packed_index.argtypes = [i, i, i]
        L.muxq_workspace_layout.restype = i
        L.muxq_workspace_layout.argtypes = [i, i, i, i, C.POINTER(WsLayout)]
        L.muxq_workspace_bytes.restype = sz
        L.muxq_workspace_bytes.argtypes = [i, i, i, i]
        L.muxq_quantize_weight.restype = i
        L.muxq_quantize_weight.argtypes = [vp, i, i, i, i, vp, vp, vp]
        L.muxq_detect_outliers.restype = i
        L.muxq_detect_outliers.argtypes = [vp, i, i, i, f, i, vp, vp, vp, vp, vp]
        L.muxq_detect_scratch_bytes.restype = sz
        L.muxq_detect_scratch_bytes.argtypes = [i]
        L.muxq_build_aux.restype = i
        L.muxq_build_aux.argtypes = [vp, i, i, i, vp, vp, vp, i, i, vp, vp, vp, vp, vp]
        L.muxq_linear.restype = i
        L.muxq_linear.argtypes = [vp, i, i, i, vp, vp, i, i, vp, f, i, i, vp, i, vp, sz, vp, vp]
        L.muxq_quantize_weight_bits.restype = i
        L.muxq_quantize_weight_bits.argtypes = [vp, i, i, i, i, i, vp, vp, vp]
        L.muxq_linear_opts.restype = i
        L.muxq_linear_opts.argtypes = [vp, i, i, i, vp, vp, i, i, vp, f, i, i, vp, i, vp, sz, vp,
                                       C.POINTER(ActOpts), vp]
        L.muxq_linear_naive_int8.restype = i
        L.muxq_linear_naive_int8.argtypes = [vp, i, i, i, vp, vp, i, i, vp, vp, i, vp, sz, vp, vp]
        L.muxq_gemm_i8.restype = i
        L.muxq_gemm_i8.argtypes = [vp, i, i, vp, i, vp, vp, vp, i, i, vp, vp, i, vp, vp, i, vp, vp]
        L.muxq_probe_mfma_rate.restype = i
        L.muxq_probe_mfma_rate.argtypes = [vp, vp, sz, i, i, vp, vp]
        L.muxq_init.restype = i
        L.muxq_init.argtypes = []
        L.muxq_mlp_workspace_bytes.restype = sz
        L.muxq_mlp_workspace_bytes.argtypes = [i, i, i, i, i]
        L.muxq_mlp.restype = i
        L.muxq_mlp.argtypes = [vp, i, i, i, vp, vp, i, i, vp, vp, vp, i, i, vp, f, i, i, vp, i, vp, i, vp, sz,
                               C.POINTER(ActOpts), vp]
        L.muxq_noalloc_max_bytes.restype = sz
        L.muxq_noalloc_max_bytes.argtypes = []
        L.muxq_linear_noalloc.restype = i
        L.muxq_linear_noalloc.argtypes = [vp, i, i, i, vp, vp, i, i, vp, f, i, i, vp, i, vp]
        L.muxq_linear_timed.restype = i
        L.muxq_linear_timed.argtypes = [vp, i, i, i, vp, vp, i, i, vp, f, i, i, vp, i, vp, sz,
                                        C.POINTER(ActOpts), vp, vp, vp, vp]
        L.muxq_static_bytes.restype = sz
        L.muxq_static_bytes.argtypes = [i, i, i]
        L.muxq_static_layout_of.restype = i
        L.muxq_static_layout_of.argtypes = [i, i, i, C.POINTER(StaticLayout)]
        L.muxq_prepare_static.restype = i
        L.muxq_prepare_static.argtypes = [vp, i, i, vp, i, i, vp, sz, vp]
        L.muxq_linear_static.restype = i
        L.muxq_linear_static.argtypes = [vp, i, i, i, vp, vp, i, i, vp, i, i, vp, vp, i, vp, sz, vp,
                                         C.POINTER(ActOpts), vp]
        L.muxq_gelu_absmax.restype = i
        L.muxq_gelu_absmax.argtypes = [vp, i, i, i, vp, i, vp, vp]
        L.muxq_quantize_weight_smooth.restype = i
        L.muxq_quantize_weight_smooth.argtypes = [vp, i, i, i, i, i, vp, vp, vp, vp]
        L.muxq_smooth_absmax.restype = i
        L.muxq_smooth_absmax.argtypes = [vp, i, i, i, vp, vp, i, vp, vp]
        L.muxq_gemm_kernel.restype = C.c_char_p
        L.muxq_gemm_kernel.argtypes = [i, i, i]
        L.muxq_code_kernel.restype = C.c_char_p
        L.muxq_code_kernel.argtypes = [i, i, i, i, C.POINTER(ActOpts), i]
        L.muxq_linear_gelu_slabs.restype = i
        L.muxq_linear_gelu_slabs.argtypes = [i, i, i]
        L.muxq_linear_gelu.restype = i
        L.muxq_linear_gelu.argtypes = [vp, i, i, i, vp, vp, i, i, vp, f, i, i, vp, i, vp, sz, vp,
                                       C.POINTER(ActOpts), vp]
        kv = C.POINTER(KvCache)
        L.muxq_kv_append.restype = i
        L.muxq_kv_append.argtypes = [vp, vp, i, i, i, vp, i, i, vp, i, vp, vp, vp, i, i, i, kv, vp]
        L.muxq_kv_gather.restype = i
        L.muxq_kv_gather.argtypes = [vp, i, kv, vp, i, vp, i, vp]
        L.muxq_paged_attention_workspace_bytes.restype = sz
        L.muxq_paged_attention_workspace_bytes.argtypes = [i, i, i, i, i]
        L.muxq_paged_attention.restype = i
        L.muxq_paged_attention.argtypes = [vp, i, i, i, kv, vp, i, vp, i, f, vp, i, vp, sz, vp]
        L.muxq_lora.restype = i
        L.muxq_lora.argtypes = [vp, i, i, i, vp, vp, vp, i, i, vp, vp, i, vp, i, i, vp, i, vp, sz, vp]
        L.muxq_lora_workspace_bytes.restype = sz
        L.muxq_lora_workspace_bytes.argtypes = [i, i, i, i, i]
        L.muxq_norm_slabs.restype = i
        L.muxq_norm_slabs.argtypes = [i, i]
        L.muxq_norm_scratch_bytes.restype = sz
        L.muxq_norm_scratch_bytes.argtypes = [i, i]
        L.muxq_norm.restype = i
        L.muxq_norm.argtypes = [vp, i, i, i, vp, i, f, vp, vp, vp, i, vp, vp, i, f, vp, i, vp, i, vp, vp, sz, vp]
        L.muxq_window_attention_workspace_bytes.restype = sz
        L.muxq_window_attention_workspace_bytes.argtypes = [i, i, i, i, i, i, i, i]
        L.muxq_window_attention.restype = i
        L.muxq_window_attention.argtypes = [vp, i, i, i, kv, vp, i, vp, vp, i, i, i, i, i, f, vp, i, vp, sz, vp]
        L.muxq_tree_attention_workspace_bytes.restype = sz
        L.muxq_tree_attention_workspace_bytes.argtypes = [i, i, i, i, i, i]
        L.muxq_tree_attention.restype = i
        L.muxq_tree_attention.argtypes = [vp, i, i, i, kv, vp, i, vp, vp, vp, i, i, i, f, vp, i, vp, sz, vp]
        L.muxq_verify_tree.restype = i
        L.muxq_verify_tree.argtypes = [vp, i, vp, i, i, i, vp, vp, vp, vp, i, i, vp, vp, vp, vp]
        L.muxq_kv_copy.restype = i
        L.muxq_kv_copy.argtypes = [vp, vp, i, kv, vp]
        L.muxq_kv_compact.restype = i
        L.muxq_kv_compact.argtypes = [vp, vp, vp, vp, vp, i, i, i, i, kv, vp]
        _lib = L
    return _lib


def _check(status: int, what: str):
    if status != 0:
        raise MuxqError(f"{what}: status {status} ({lib().muxq_status_string(status).decode()})")


def _p(t):
    return None if t is None else t.data_ptr()


# The raw handle of the current stream of the current device.  (current_stream() builds a Stream object
# on the way, 2.9 us of the 9 us a call of one token takes on the host.)
if hasattr(torch._C, "_cuda_getCurrentRawStream") and hasattr(torch._C, "_cuda_getDevice"):
    def _stream():
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
else:
    def _stream():
        return torch.cuda.current_stream().cuda_stream


def k_pad(K: int) -> int:
    return lib().muxq_k_pad(K)


def packed_bytes(rows: int, cols: int) -> int:
    return lib().muxq_packed_bytes(rows, cols)


def unpack(buf, rows: int, cols: int):
    """Packed layout (16 x 64 blocks, see include/muxq.h) -> row-major [rows, cols] tensor.
    Pure re-indexing for tests and inspection; works on any device."""
    if cols == 0:
        return buf.new_empty((rows, 0))
    r16 = (rows + 15) // 16
    v = buf.reshape(-1)[:r16 * 16 * cols].view(r16, cols // 64, 16, 64)
    return v.permute(0, 2, 1, 3).reshape(r16 * 16, cols)[:rows]


def pack(mat):
    """Row-major [rows, cols] int8 tensor (cols % 64 == 0) -> packed flat buffer."""
    rows, cols = mat.shape
    r16 = (rows + 15) // 16
    full = mat.new_zeros((r16 * 16, cols))
    full[:rows] = mat
    return full.view(r16, 16, cols // 64, 64).permute(0, 2, 1, 3).contiguous().reshape(-1)


def workspace_layout(M, K, N, r_cap) -> WsLayout:
    L = WsLayout()
    _check(lib().muxq_workspace_layout(M, K, N, r_cap, C.byref(L)), "muxq_workspace_layout")
    return L


def workspace_bytes(M, K, N, r_cap) -> int:
    return lib().muxq_workspace_bytes(M, K, N, r_cap)


def alloc_workspace(M, K, N, r_cap, device="cuda"):
    return torch.empty(workspace_bytes(M, K, N, r_cap), dtype=torch.uint8, device=device)


def muxq_quantize_weight(W, gran="tensor", bits=8, factors=None):
    """W: [K, N] fp16 device tensor (row stride W.stride(0)).  Returns (w_q: packed
    N x k_pad int8 codes as a flat buffer, w_scale [1] or [N] fp32).  factors: optional fp32 [K]
    device tensor, the weight side of a per-channel difficulty migration (W' = fp16(W f[k]))."""
    K, N = W.shape
    g = _GRAN[gran]
    w_q = torch.empty(lib().muxq_wq_bytes(K, N), dtype=torch.int8, device=W.device)
    w_scale = torch.empty(N if g == PER_CHANNEL else 1, dtype=torch.float32, device=W.device)
    if factors is not None:
        _check(lib().muxq_quantize_weight_smooth(_p(W), K, N, W.stride(0), g, bits, _p(factors), _p(w_q),
                                                 _p(w_scale), _stream()), "muxq_quantize_weight_smooth")
    elif bits == 8:
        _check(lib().muxq_quantize_weight(_p(W), K, N, W.stride(0), g, _p(w_q), _p(w_scale),
                                          _stream()), "muxq_quantize_weight")
    else:
        _check(lib().muxq_quantize_weight_bits(_p(W), K, N, W.stride(0), g, bits, _p(w_q),
                                               _p(w_scale), _stream()), "muxq_quantize_weight_bits")
    return w_q, w_scale


def muxq_detect_outliers(X, threshold=6.0, r_cap=64):
    """Returns (col_absmax [K] fp32, outlier_idx [max(r_cap,1)] int32, n_outliers [2] int32)."""
    M, K = X.shape
    col_absmax = torch.empty(K, dtype=torch.float32, device=X.device)
    idx = torch.empty(max(r_cap, 1), dtype=torch.int32, device=X.device)
    n_out = torch.empty(2, dtype=torch.int32, device=X.device)
    scratch = torch.empty(lib().muxq_detect_scratch_bytes(K), dtype=torch.uint8, device=X.device)
    _check(lib().muxq_detect_outliers(_p(X), M, K, X.stride(0), threshold, r_cap, _p(col_absmax),
                                      _p(idx), _p(n_out), _p(scratch), _stream()),
           "muxq_detect_outliers")
    return col_absmax, idx, n_out


def muxq_build_aux(X, col_absmax, outlier_idx, n_outliers, r_cap=64, exp=2):
    """Returns (body_q packed M x k_pad, aux_q packed M x r_cap, x_scale [2] fp32)."""
    M, K = X.shape
    kp = k_pad(K)
    body_q = torch.empty(packed_bytes(M, kp), dtype=torch.int8, device=X.device)
    aux_q = torch.empty(packed_bytes(M, r_cap), dtype=torch.int8, device=X.device)
    x_scale = torch.empty(2, dtype=torch.float32, device=X.device)
    scratch = torch.empty(2 * kp, dtype=torch.int32, device=X.device)
    _check(lib().muxq_build_aux(_p(X), M, K, X.stride(0), _p(col_absmax), _p(outlier_idx),
                                _p(n_outliers), r_cap, exp, _p(body_q),
                                _p(aux_q) if r_cap else None, _p(x_scale), _p(scratch), _stream()),
           "muxq_build_aux")
    return body_q, aux_q, x_scale


def muxq_smooth_absmax(X, factors, workspace=None, layout=None, out=None):
    """X' = fp16(X / factors[k]) (in place when out is X); with workspace / layout also the slab
    maxima of X' for a following call with absmax_ready=True.  Returns X'."""
    M, K = X.shape
    if out is None:
        out = torch.empty_like(X)
    slabs = None if workspace is None else workspace[layout.absmax_partial:]
    _check(lib().muxq_smooth_absmax(_p(X), M, K, X.stride(0), _p(factors), _p(out), out.stride(0),
                                    _p(slabs), _stream()), "muxq_smooth_absmax")
    return out


def muxq_gelu_absmax(Y, workspace, layout: "WsLayout", out=None):
    """X = gelu(Y) (tanh form; in place when out is Y) and the slab maxima of X, left in the
    absmax_partial region of `workspace` (a muxq_linear workspace for the same M, K; `layout`
    its workspace_layout) for a following call with absmax_ready=True.  Returns X."""
    M, K = Y.shape
    if out is None:
        out = torch.empty_like(Y)
    slabs = workspace[layout.absmax_partial:]
    _check(lib().muxq_gelu_absmax(_p(Y), M, K, Y.stride(0), _p(out), out.stride(0), _p(slabs), _stream()),
           "muxq_gelu_absmax")
    return out


def muxq_linear(X, w_q, w_scale, N, w_gran="tensor", bias=None, threshold=6.0, exp=2, r_cap=64,
                out=None, workspace=None, dbg_acc=None, x_gran="tensor", ia_bits=8, absmax_ready=False,
                aux_scale="shared", absmax_slabs=0):
    """Y = MUXQ(X) . W.  X [M, K] fp16; w_q / w_scale from muxq_quantize_weight of a
    K x N weight.  Returns Y [M, N] fp16 (and leaves every intermediate in `workspace`).
    x_gran "token" / ia_bits != 8 / absmax_ready (slab maxima left in `workspace` by
    muxq_gelu_absmax) go through muxq_linear_opts."""
    M, K = X.shape
    if out is None:
        out = torch.empty((M, N), dtype=torch.float16, device=X.device)
    if workspace is None:
        workspace = alloc_workspace(M, K, N, r_cap, X.device)
    own = {"shared": 0, "own": 1}[aux_scale]
    if _XGRAN[x_gran] == X_PER_TENSOR and ia_bits == 8 and not absmax_ready and not own and not absmax_slabs:
        _check(lib().muxq_linear(_p(X), M, K, X.stride(0), _p(w_q), _p(w_scale), _GRAN[w_gran], N,
                                 _p(bias), threshold, exp, r_cap, _p(out), out.stride(0),
                                 _p(workspace), workspace.numel(), _p(dbg_acc), _stream()),
               "muxq_linear")
    else:
        opts = ActOpts(_XGRAN[x_gran], ia_bits, int(bool(absmax_ready)), own, absmax_slabs)
        _check(lib().muxq_linear_opts(_p(X), M, K, X.stride(0), _p(w_q), _p(w_scale), _GRAN[w_gran],
                                      N, _p(bias), threshold, exp, r_cap, _p(out), out.stride(0),
                                      _p(workspace), workspace.numel(), _p(dbg_acc), C.byref(opts),
                                      _stream()), "muxq_linear_opts")
    return out


def muxq_linear_noalloc(X, w_q, w_scale, N, w_gran="tensor", bias=None, threshold=6.0, exp=2, r_cap=64,
                        out=None):
    """muxq_linear with its intermediates in the library's static device array (no workspace,
    no allocation inside the call; `out` is the caller's, allocated here only when not given)."""
    M, K = X.shape
    if out is None:
        out = torch.empty((M, N), dtype=torch.float16, device=X.device)
    _check(lib().muxq_linear_noalloc(_p(X), M, K, X.stride(0), _p(w_q), _p(w_scale), _GRAN[w_gran], N,
                                     _p(bias), threshold, exp, r_cap, _p(out), out.stride(0), _stream()),
           "muxq_linear_noalloc")
    return out


def muxq_linear_gelu(X, w_q, w_scale, N, w_gran="tensor", bias=None, threshold=6.0, exp=2, r_cap=64,
                     out=None, workspace=None, next_workspace=None, next_layout=None, x_gran="tensor",
                     ia_bits=8):
    """H = gelu(MUXQ(X) . W + b) with the GELU fused into the GEMM.  next_workspace / next_layout:
    the workspace (and its workspace_layout) of the layer that consumes H; it receives H's slab
    maxima.  Returns (H, number of slabs written -- pass it on as absmax_slabs with
    absmax_ready=True)."""
    M, K = X.shape
    if out is None:
        out = torch.empty((M, N), dtype=torch.float16, device=X.device)
    if workspace is None:
        workspace = alloc_workspace(M, K, N, r_cap, X.device)
    slabs = None if next_workspace is None else next_workspace[next_layout.absmax_partial:]
    opts = ActOpts(_XGRAN[x_gran], ia_bits, 0, 0, 0)
    _check(lib().muxq_linear_gelu(_p(X), M, K, X.stride(0), _p(w_q), _p(w_scale), _GRAN[w_gran], N,
                                  _p(bias), threshold, exp, r_cap, _p(out), out.stride(0), _p(workspace),
                                  workspace.numel(), _p(slabs), C.byref(opts), _stream()),
           "muxq_linear_gelu")
    return out, lib().muxq_linear_gelu_slabs(M, K, N)


def muxq_mlp(X, w1_q, w1_scale, N1, w2_q, w2_scale, N2, w_gran="tensor", bias1=None, bias2=None,
             threshold=6.0, exp=2, r_cap=64, x_gran="tensor", ia_bits=8, workspace=None, out_h=None, out=None):
    """c_fc, GELU, c_proj as one call: returns (H, Y, workspace).  The workspace holds the first
    layer's workspace at offset 0 and the second layer's behind it (see muxq.h)."""
    M, K = X.shape
    if out_h is None:
        out_h = torch.empty((M, N1), dtype=torch.float16, device=X.device)
    if out is None:
        out = torch.empty((M, N2), dtype=torch.float16, device=X.device)
    if workspace is None:
        n = lib().muxq_mlp_workspace_bytes(M, K, N1, N2, r_cap)
        if n == 0:
            raise MuxqError("muxq_mlp_workspace_bytes: bad shapes")
        workspace = torch.empty(n, dtype=torch.uint8, device=X.device)
    opts = ActOpts(_XGRAN[x_gran], ia_bits, 0, 0, 0)
    _check(lib().muxq_mlp(_p(X), M, K, X.stride(0), _p(w1_q), _p(w1_scale), _GRAN[w_gran], N1, _p(bias1),
                          _p(w2_q), _p(w2_scale), _GRAN[w_gran], N2, _p(bias2), threshold, exp, r_cap,
                          _p(out_h), out_h.stride(0), _p(out), out.stride(0), _p(workspace),
                          workspace.numel(), C.byref(opts), _stream()), "muxq_mlp")
    return out_h, out, workspace


def static_layout(K, N, r_cap) -> StaticLayout:
    lay = StaticLayout()
    _check(lib().muxq_static_layout_of(K, N, r_cap, C.byref(lay)), "muxq_static_layout_of")
    return lay


def muxq_prepare_static(channel_list, K, w_q, N, r_cap=64):
    """channel_list: int32 tensor on the GPU (ascending channel indices found offline), may be
    empty.  Returns the static block (uint8 tensor) muxq_linear_static consumes."""
    lay = static_layout(K, N, r_cap)
    block = torch.empty(lay.total, dtype=torch.uint8, device=w_q.device)
    n = int(channel_list.numel())
    _check(lib().muxq_prepare_static(_p(channel_list) if n else None, n, K, _p(w_q), N, r_cap,
                                     _p(block), block.numel(), _stream()), "muxq_prepare_static")
    return block


def muxq_linear_static(X, w_q, w_scale, N, static_block, w_gran="tensor", bias=None, exp=2, r_cap=64,
                       out=None, workspace=None, dbg_acc=None, x_gran="tensor", ia_bits=8,
                       absmax_ready=False, aux_scale="shared", absmax_slabs=0):
    """muxq_linear with the channel list of a prepared static block instead of the run-time
    detection (per-token activations then need one pass over X)."""
    M, K = X.shape
    if out is None:
        out = torch.empty((M, N), dtype=torch.float16, device=X.device)
    if workspace is None:
        workspace = alloc_workspace(M, K, N, r_cap, X.device)
    opts = ActOpts(_XGRAN[x_gran], ia_bits, int(bool(absmax_ready)), {"shared": 0, "own": 1}[aux_scale],
                   absmax_slabs)
    _check(lib().muxq_linear_static(_p(X), M, K, X.stride(0), _p(w_q), _p(w_scale), _GRAN[w_gran], N,
                                    _p(bias), exp, r_cap, _p(static_block), _p(out), out.stride(0),
                                    _p(workspace), workspace.numel(), _p(dbg_acc), C.byref(opts),
                                    _stream()), "muxq_linear_static")
    return out


def muxq_linear_naive_int8(X, w_q, w_scale, N, w_gran="tensor", bias=None, out=None,
                           workspace=None, dbg_acc=None):
    M, K = X.shape
    if out is None:
        out = torch.empty((M, N), dtype=torch.float16, device=X.device)
    if workspace is None:
        workspace = alloc_workspace(M, K, N, 0, X.device)
    _check(lib().muxq_linear_naive_int8(_p(X), M, K, X.stride(0), _p(w_q), _p(w_scale),
                                        _GRAN[w_gran], N, _p(bias), _p(out), out.stride(0),
                                        _p(workspace), workspace.numel(), _p(dbg_acc), _stream()),
           "muxq_linear_naive_int8")
    return out


def muxq_gemm_i8(a_q, M, K, w_q, N, x_scale, w_scale, w_gran="tensor", aux_q=None, w_aux=None,
                 n_outliers=None, r_cap=0, exp=2, bias=None, out=None, dbg_acc=None):
    """a_q / w_q / aux_q / w_aux: packed buffers (see pack / unpack)."""
    if out is None:
        out = torch.empty((M, N), dtype=torch.float16, device=a_q.device)
    _check(lib().muxq_gemm_i8(_p(a_q), M, K, _p(w_q), N, _p(aux_q), _p(w_aux),
                              _p(n_outliers), r_cap, exp, _p(x_scale), _p(w_scale), _GRAN[w_gran],
                              _p(bias), _p(out), out.stride(0), _p(dbg_acc), _stream()),
           "muxq_gemm_i8")
    return out


def muxq_init():
    """Per-device set-up for the current device (optional; needed before a first call that is
    made under graph capture)."""
    _check(lib().muxq_init(), "muxq_init")


def muxq_linear_timed(X, w_q, w_scale, N, gemm_start, gemm_stop, w_gran="tensor", bias=None,
                      threshold=6.0, exp=2, r_cap=64, out=None, workspace=None, x_gran="tensor",
                      ia_bits=8, absmax_ready=False, wg_ticks=None):
    """muxq_linear that records the raw hipEvent_t handles gemm_start / gemm_stop (ints) around
    its GEMM kernel (measurement aid, include/muxq_measure.h).  wg_ticks: None or an int64
    device tensor of 2048 entries (start / end tick of each workgroup of a persistent GEMM)."""
    M, K = X.shape
    if out is None:
        out = torch.empty((M, N), dtype=torch.float16, device=X.device)
    if workspace is None:
        workspace = alloc_workspace(M, K, N, r_cap, X.device)
    opts = ActOpts(_XGRAN[x_gran], ia_bits, int(bool(absmax_ready)), 0)
    _check(lib().muxq_linear_timed(_p(X), M, K, X.stride(0), _p(w_q), _p(w_scale), _GRAN[w_gran], N,
                                   _p(bias), threshold, exp, r_cap, _p(out), out.stride(0),
                                   _p(workspace), workspace.numel(), C.byref(opts), gemm_start,
                                   gemm_stop, _p(wg_ticks), _stream()), "muxq_linear_timed")
    return out


def gemm_kernel(M: int, K: int, N: int) -> str:
    """Name of the kernel that runs the GEMM of an M x K -> N layer (include/muxq_measure.h)."""
    return lib().muxq_gemm_kernel(M, K, N).decode()


def code_kernel(M: int, K: int, N: int, r_cap=64, x_gran="tensor", absmax_ready=False, aux_scale="shared",
                hands_maxima=False) -> str:
    """Name of the kernel that forms the codes of X in an M x K -> N layer (include/muxq_measure.h)."""
    opts = ActOpts(_XGRAN[x_gran], 8, int(absmax_ready), {"shared": 0, "own": 1}[aux_scale], 0)
    return lib().muxq_code_kernel(M, K, N, r_cap, C.byref(opts), int(hands_maxima)).decode()


def wq_row_sums(w_q, K: int, N: int):
    """The int32 per-output-channel code sums stored behind the packed codes of a weight."""
    off = (packed_bytes(N, k_pad(K)) + 255) // 256 * 256
    return w_q[off:off + 4 * N].view(torch.int32)


def ws_packed(workspace, layout: WsLayout, name: str, M: int, N: int, r_cap: int):
    """The raw packed buffer of body_q / aux_q / w_aux inside a muxq_linear workspace."""
    rows, cols = {"body_q": (M, layout.k_pad), "aux_q": (M, r_cap), "w_aux": (N, r_cap)}[name]
    off = getattr(layout, name)
    return workspace[off:off + packed_bytes(rows, cols)].view(torch.int8)


def ws_view(workspace, layout: WsLayout, name: str, M: int, N: int, r_cap: int):
    """Typed view of one intermediate inside a muxq_linear workspace (the three INT8
    matrices are returned unpacked to row-major)."""
    kp = layout.k_pad
    spec = {
        "col_absmax": (torch.float32, (kp,)),
        "col_scale": (torch.float32, (kp,)),
        "col_slot": (torch.int32, (kp,)),
        "outlier_idx": (torch.int32, (max(r_cap, 1),)),
        "n_outliers": (torch.int32, (2,)),
        "zero_point": (torch.int32, (1,)),
        "zero_point_token": (torch.int32, (M,)),
        "cn": (torch.int32, (N,)),
        "x_scale": (torch.float32, (2,)),
        "aux_scale": (torch.float32, (2,)),
        "x_scale_token": (torch.float32, (2, M)),
        "aux_scale_token": (torch.float32, (2, M)),      # s_aux[M], rho[M] (Aux on its own scale)
        "body_q": (torch.int8, (M, kp)),
        "aux_q": (torch.int8, (M, r_cap)),
        "w_aux": (torch.int8, (N, r_cap)),
    }[name]
    dtype, shape = spec
    if name in ("body_q", "aux_q", "w_aux"):
        off = getattr(layout, name)
        return unpack(workspace[off:off + packed_bytes(*shape)].view(torch.int8), *shape)
    n = 1
    for d in shape:
        n *= d
    if name == "zero_point":
        off = layout.n_outliers + 8
    elif name == "aux_scale":
        off = layout.x_scale + 8
    elif name == "aux_scale_token":
        off = layout.x_scale + 12 * M
    elif name == "zero_point_token":
        off = layout.x_scale + 8 * M
    else:
        off = getattr(layout, "x_scale" if name == "x_scale_token" else name)
    nbytes = n * torch.empty(0, dtype=dtype).element_size()
    return workspace[off:off + nbytes].view(dtype).view(shape)


def muxq_probe_mfma_rate(a_codes, b_codes, iters=4000, n_workgroups=512):
    """Register-only MFMA issue-rate probe on the given operand codes (int8 device tensors).
    Returns (TOP/s, shader GHz)."""
    n = min(a_codes.numel(), b_codes.numel()) // 16 * 16
    clocks = torch.zeros(3, dtype=torch.int64, device=a_codes.device)
    start, stop = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)

    def launch(rounds):
        _check(lib().muxq_probe_mfma_rate(_p(a_codes), _p(b_codes), n, rounds, n_workgroups, _p(clocks),
                                          _stream()), "muxq_probe_mfma_rate")

    launch(1)                           # the first launch on a device loads the kernel, a millisecond that is not timed
    start.record()
    launch(iters)
    stop.record()
    torch.cuda.synchronize()
    ops = n_workgroups * 4 * iters * 8 * 65536.0
    c = clocks.cpu().tolist()
    return ops / (start.elapsed_time(stop) * 1e-3) / 1e12, (c[0] / (c[1] * 10.0) if c[1] else 0.0)


# ---- what stands between the projections of a block (include/muxq_block.h) --------------------

NORM_LAYER, NORM_RMS = 0, 1
_NORM = {"layer": NORM_LAYER, "rms": NORM_RMS, NORM_LAYER: NORM_LAYER, NORM_RMS: NORM_RMS}


_F16, _F32, _I8, _I32 = torch.float16, torch.float32, torch.int8, torch.int32


# (A call of a few microseconds has dozens of checks: each entry point makes them in one expression, and goes through its
# tensors one by one, with _rows and _flat, only to say which of them it refuses.)
def _refuse(what):
    raise MuxqError(what)


def _rows(t, name):
    """t: [rows, heads, d] or [rows, width] of fp16 whose rows are contiguous; returns its row stride."""
    st = t.stride()
    if t.dtype is not _F16 or not t.is_cuda or st[-1] != 1 or (len(st) == 3 and st[1] != t.shape[2] and t.shape[1] != 1):
        _refuse(f"{name}: a GPU tensor of fp16 with contiguous rows is expected")
    return st[0]


def _flat(t, n, dtype, name):
    """t: n contiguous entries of a type (at least, for indices); returns its address, None for None."""
    if t is None:
        return None
    if t.dtype is not dtype or not t.is_cuda or not t.is_contiguous() or (t.numel() != n and (dtype is not _I32 or t.numel() < n)):
        _refuse(f"{name}: a contiguous GPU tensor of {n} {dtype} is expected")
    return t.data_ptr()


def _call(entry, args, workspace, stream, alloc, what):
    """entry(*args, workspace, its bytes, stream).  Without a workspace the call goes out with none: it is refused for a NULL
    pointer, with nothing enqueued, where one is needed, and only then is one allocated."""
    if workspace is not None:
        if not workspace.is_cuda or not workspace.is_contiguous():
            _refuse(f"{what}: the workspace is a contiguous GPU tensor")
        status = entry(*args, workspace.data_ptr(), workspace.nbytes, stream)
    else:
        status = entry(*args, None, 0, stream)
        if status == 1:
            workspace = alloc()
            status = entry(*args, workspace.data_ptr(), workspace.numel(), stream)
    if status != 0:
        _check(status, what)


def _kv(k_cache, v_cache, k_scale, v_scale):
    """The descriptor of a cache given as tensors [pages, heads, tokens of a page, d]: views of any
    strides with contiguous d (transpose a [pages, tokens, heads, d] tensor), fp16 or int8, the latter with scales
    [pages, heads, tokens of a page]."""
    shape, strides, dtype = k_cache.shape, k_cache.stride(), k_cache.dtype
    if v_cache.shape != shape or v_cache.stride() != strides or v_cache.dtype is not dtype or not k_cache.is_cuda or not v_cache.is_cuda:
        _refuse("cache: keys and values are GPU tensors of one shape, type and order")
    n, heads, block, d = shape
    lb, lh, lt, one = strides
    if one != 1:
        _refuse("cache: head dimensions are contiguous")
    # a dimension of one element may carry any stride
    if heads == 1:
        lh = (lt * block + 15) // 16 * 16
    if n == 1:
        lb = max(lb, (block - 1) * lt + (heads - 1) * lh + d + 15) // 16 * 16
    if dtype is _I8:
        if k_scale is None or v_scale is None:
            _refuse("cache: 8-bit codes come with k_scale and v_scale")
        scales = n * heads * block
        return KvCache(k_cache.data_ptr(), v_cache.data_ptr(), _flat(k_scale, scales, _F32, "k_scale"),
                       _flat(v_scale, scales, _F32, "v_scale"), 1, n, block, heads, d, 0, lb, lh, lt)
    if dtype is not _F16 or k_scale is not None or v_scale is not None:
        _refuse("cache: fp16 without scales, or int8 with them")
    return KvCache(k_cache.data_ptr(), v_cache.data_ptr(), None, None, 0, n, block, heads, d, 0, lb, lh, lt)


def alloc_kv_cache(n_blocks, block_size, n_kv_heads, head_dim, dtype=torch.float16, device="cuda"):
    """(k_cache, v_cache, k_scale, v_scale): empty pages, heads before tokens; scales are None for fp16."""
    k, v = (torch.empty((n_blocks, n_kv_heads, block_size, head_dim), dtype=dtype, device=device) for _ in "kv")
    if dtype != torch.int8:
        return k, v, None, None
    ks, vs = (torch.empty((n_blocks, n_kv_heads, block_size), dtype=torch.float32, device=device) for _ in "kv")
    return k, v, ks, vs


def muxq_kv_append(k, v, slots, k_cache, v_cache, k_scale=None, v_scale=None, q=None, q_out=None, positions=None,
                   cos_sin=None, interleaved=False):
    """Keys and values [M, n_kv_heads, d] of new tokens to their slots (int32 [M], page * block_size + place,
    -1: nowhere) of the cache; with cos_sin (float [positions, rot_dim]: cosines, then sines) and positions
    (int32 [M]) rotated on the way, and the queries q [M, n_heads, d] with them.  q, k, v may be column
    ranges of one tensor.  Returns q_out (made when not given; None without q)."""
    M, heads, d = k.shape
    c = _kv(k_cache, v_cache, k_scale, v_scale)
    ks, vs = k.stride(), v.stride()
    if not (k.dtype is v.dtype is _F16 and slots.dtype is _I32 and k.is_cuda and v.is_cuda and slots.is_cuda and v.shape == k.shape and
            heads == c.n_kv_heads and d == c.head_dim and ks[2] == vs[2] == 1 and (heads == 1 or ks[1] == vs[1] == d) and
            slots.is_contiguous() and slots.numel() == M):
        _rows(k, "k"), _rows(v, "v"), _flat(slots, M, _I32, "slots")
        _refuse("muxq_kv_append: k, v, slots and the cache differ in tokens or heads")
    n_heads = ldq = ldqo = 0
    q_at = q_out_at = None
    if q is not None:
        if q_out is None:
            q_out = torch.empty(q.shape, dtype=_F16, device=q.device)
        n_heads = q.shape[1]
        qs, os = q.stride(), q_out.stride()
        if not (q.dtype is q_out.dtype is _F16 and q.is_cuda and q_out.is_cuda and q.shape == q_out.shape == (M, n_heads, d) and
                qs[2] == os[2] == 1 and (n_heads == 1 or qs[1] == os[1] == d)):
            _rows(q, "q"), _rows(q_out, "q_out")
            _refuse("muxq_kv_append: q, q_out and k differ in tokens or head size")
        ldq, ldqo, q_at, q_out_at = qs[0], os[0], q.data_ptr(), q_out.data_ptr()
    n_pos = rot = 0
    cos_at = pos_at = None
    if cos_sin is not None:
        n_pos, rot = cos_sin.shape
        if positions is None:
            _refuse("muxq_kv_append: cos_sin comes with positions")
        cos_at, pos_at = _flat(cos_sin, n_pos * rot, _F32, "cos_sin"), _flat(positions, M, _I32, "positions")
    status = lib().muxq_kv_append(k.data_ptr(), v.data_ptr(), M, ks[0], vs[0], q_at, n_heads, ldq, q_out_at, ldqo, slots.data_ptr(),
                                  pos_at, cos_at, n_pos, rot, int(interleaved), C.byref(c), _stream())
    if status != 0:
        _check(status, "muxq_kv_append")
    return q_out


def muxq_kv_gather(slots, k_cache, v_cache, k_scale=None, v_scale=None, k_out=None, v_out=None):
    """Keys and values of the cache's slots (int32 [M]) as fp16 [M, n_kv_heads, d]; zeros for slots outside."""
    c = _kv(k_cache, v_cache, k_scale, v_scale)
    shape = (slots.numel(), c.n_kv_heads, c.head_dim)
    if k_out is None:
        k_out = torch.empty(shape, dtype=torch.float16, device=k_cache.device)
    if v_out is None:
        v_out = torch.empty(shape, dtype=torch.float16, device=k_cache.device)
    if k_out.shape != shape or v_out.shape != shape:
        _refuse(f"muxq_kv_gather: outputs of shape {shape} are expected")
    status = lib().muxq_kv_gather(_flat(slots, shape[0], _I32, "slots"), shape[0], C.byref(c), k_out.data_ptr(), _rows(k_out, "k_out"),
                                  v_out.data_ptr(), _rows(v_out, "v_out"), _stream())
    if status != 0:
        _check(status, "muxq_kv_gather")
    return k_out, v_out


def attention_workspace_bytes(S, n_heads, n_kv_heads, head_dim, max_length) -> int:
    return lib().muxq_paged_attention_workspace_bytes(S, n_heads, n_kv_heads, head_dim, max_length)


def alloc_attention_workspace(S, n_heads, n_kv_heads, head_dim, max_length, device="cuda"):
    """Workspace of muxq_paged_attention, also good for a smaller S or max_length (empty where none is needed)."""
    return torch.empty(attention_workspace_bytes(S, n_heads, n_kv_heads, head_dim, max_length), dtype=torch.uint8, device=device)


def muxq_paged_attention(q, k_cache, v_cache, block_table, lengths, max_length, scale=None, k_scale=None, v_scale=None,
                         out=None, workspace=None):
    """Attention of one new token of each sequence, q [S, n_heads, d], over the cache's pages that
    block_table (int32 [S, pages]) lists, the first lengths[s] tokens (int32 [S]) of each sequence;
    max_length: a bound on lengths known on the host.  scale: 1 / sqrt(d) when not given."""
    S, n_heads, d = q.shape
    c = _kv(k_cache, v_cache, k_scale, v_scale)
    if out is None:
        out = torch.empty((S, n_heads, d), dtype=torch.float16, device=q.device)
    qs, os, ts = q.stride(), out.stride(), block_table.stride()
    if not (q.dtype is out.dtype is _F16 and block_table.dtype is lengths.dtype is _I32 and q.is_cuda and out.is_cuda and
            block_table.is_cuda and lengths.is_cuda and d == c.head_dim and out.shape == q.shape and qs[2] == os[2] == 1 and
            (n_heads == 1 or qs[1] == os[1] == d) and block_table.shape[0] == S and ts[1] == 1 and lengths.is_contiguous() and
            lengths.numel() == S and max_length <= block_table.shape[1] * c.block_size):
        _rows(q, "q"), _rows(out, "out"), _flat(lengths, S, _I32, "lengths")
        _refuse("muxq_paged_attention: q, out and the cache differ in head size, or block_table is no int32 GPU tensor [S, pages] "
                "with contiguous rows of max_length tokens")
    args = (q.data_ptr(), S, n_heads, qs[0], C.byref(c), block_table.data_ptr(), ts[0] if S > 1 else block_table.shape[1],
            lengths.data_ptr(), max_length, d ** -0.5 if scale is None else scale, out.data_ptr(), os[0])
    _call(lib().muxq_paged_attention, args, workspace, _stream(),
          lambda: alloc_attention_workspace(S, n_heads, c.n_kv_heads, d, max_length, q.device), "muxq_paged_attention")
    return out


def alloc_lora_workspace(M, K, N, r, n_requests, device="cuda"):
    """Workspace of muxq_lora, also good for a smaller M, K, r or number of requests (empty where none is needed)."""
    return torch.empty(lib().muxq_lora_workspace_bytes(M, K, N, r, n_requests), dtype=torch.uint8, device=device)


def muxq_lora(X, A, B, scales, starts, adapters, Y, out=None, workspace=None):
    """out = Y + scales[i] (X A_i^T) B_i^T for rows starts[q]..starts[q + 1] of request q with adapter i =
    adapters[q] (-1: none).  X [M, K], Y [M, N] fp16; A [n, r, K], B [n, N, r] fp16; scales float [n]; starts int32
    [requests + 1], adapters int32 [requests].  out may be Y."""
    M, K = X.shape
    n, r, k = A.shape
    N = Y.shape[1]
    requests = adapters.numel()
    if out is None:
        out = torch.empty((M, N), dtype=torch.float16, device=X.device)
    xs, ys, os = X.stride(), Y.stride(), out.stride()
    if not (X.dtype is A.dtype is B.dtype is Y.dtype is out.dtype is _F16 and scales.dtype is _F32 and starts.dtype is adapters.dtype is _I32 and
            X.is_cuda and A.is_cuda and B.is_cuda and scales.is_cuda and starts.is_cuda and adapters.is_cuda and Y.is_cuda and out.is_cuda and
            k == K and B.shape == (n, N, r) and Y.shape == out.shape == (M, N) and xs[1] == ys[1] == os[1] == 1 and A.is_contiguous() and
            B.is_contiguous() and scales.is_contiguous() and starts.is_contiguous() and adapters.is_contiguous() and
            scales.numel() == n and starts.numel() == requests + 1):
        _rows(X, "X"), _rows(Y, "Y"), _rows(out, "out"), _flat(A, n * r * K, _F16, "A"), _flat(B, n * N * r, _F16, "B")
        _flat(scales, n, _F32, "scales"), _flat(starts, requests + 1, _I32, "starts"), _flat(adapters, requests, _I32, "adapters")
        _refuse("muxq_lora: shapes of X, A, B, starts, adapters, Y and out do not fit")
    args = (X.data_ptr(), M, K, xs[0], A.data_ptr(), B.data_ptr(), scales.data_ptr(), n, r, starts.data_ptr(), adapters.data_ptr(),
            requests, Y.data_ptr(), ys[0], N, out.data_ptr(), os[0])
    _call(lib().muxq_lora, args, workspace, _stream(), lambda: alloc_lora_workspace(M, K, N, r, requests, X.device), "muxq_lora")
    return out


def norm_slabs(M: int, K: int) -> int:
    """Rows of column maxima that muxq_norm leaves for M tokens (absmax_slabs of the next layer)."""
    return lib().muxq_norm_slabs(M, K)


def alloc_norm_scratch(M, K, device="cuda"):
    """Scratch of a muxq_norm call that hands maxima over (empty where none is needed)."""
    return torch.empty(lib().muxq_norm_scratch_bytes(M, K), dtype=torch.uint8, device=device)


def muxq_norm(x, weight, bias=None, residual=None, residual_scale=1.0, post_weight=None, post_bias=None, gate=None,
              kind="layer", eps=1e-5, out=None, residual_out=None, slabs=None, scratch=None):
    """r = residual_scale * residual + gate * post-norm(x) (each part optional), y = norm(r) with kind "layer" or "rms".
    gate: [K], or [M, K] for one per token.  slabs: the absmax_partial region of the next layer's workspace
    (workspace[layout.absmax_partial:]), which then runs with absmax_ready=True, absmax_slabs=norm_slabs(M, K).
    Returns (y, r); r is made when there is something to add or scale, else None."""
    M, K = x.shape
    if out is None:
        out = torch.empty((M, K), dtype=torch.float16, device=x.device)
    if residual_out is None and (residual is not None or gate is not None or post_weight is not None):
        residual_out = torch.empty((M, K), dtype=torch.float16, device=x.device)
    if slabs is not None and not (slabs.is_cuda and slabs.is_contiguous() and
                                  slabs.numel() * slabs.element_size() >= (M if M <= 64 else 1) * ((K + 63) // 64 * 128)):
        _refuse("muxq_norm: slabs are too small")
    shape, xs, os = x.shape, x.stride(), out.stride()
    if not (x.dtype is out.dtype is weight.dtype is _F16 and x.is_cuda and out.is_cuda and weight.is_cuda and out.shape == shape and
            xs[1] == os[1] == 1 and weight.is_contiguous() and weight.numel() == K):
        _rows(x, "x"), _rows(out, "out"), _flat(weight, K, _F16, "weight")
        _refuse("muxq_norm: out and x differ in shape")
    ldr = ldro = ldg = 0
    r_at = r_out_at = gate_at = None
    if residual is not None:
        r_at, ldr = residual.data_ptr(), _rows(residual, "residual")
        if residual.shape != shape:
            _refuse("muxq_norm: residual and x differ in shape")
    if residual_out is not None:
        r_out_at, ldro = residual_out.data_ptr(), _rows(residual_out, "residual_out")
        if residual_out.shape != shape:
            _refuse("muxq_norm: residual_out and x differ in shape")
    if gate is not None:
        gate_at = gate.data_ptr()
        if gate.dim() == 1:
            _flat(gate, K, _F16, "gate")
        elif gate.shape == shape:
            ldg = _rows(gate, "gate")
            if M == 1:                  # (the stride of a single row says nothing)
                ldg = K
        else:
            _refuse("muxq_norm: gate is [K] or [M, K]")
    args = (x.data_ptr(), M, K, xs[0], r_at, ldr, residual_scale,
            None if post_weight is None else _flat(post_weight, K, _F16, "post_weight"),
            None if post_bias is None else _flat(post_bias, K, _F16, "post_bias"), gate_at, ldg, weight.data_ptr(),
            None if bias is None else _flat(bias, K, _F16, "bias"), _NORM[kind], eps, r_out_at, ldro, out.data_ptr(), os[0], _p(slabs))
    _call(lib().muxq_norm, args, scratch, _stream(), lambda: alloc_norm_scratch(M, K, x.device), "muxq_norm")
    return out, residual_out


# ---- several new tokens of a sequence ----------------------------------------------------------

# (get_device() is -1 for host memory: one comparison says that a tensor is on a GPU, and on the current one, whose stream the call
# goes to.)
_device = torch._C._cuda_getDevice if hasattr(torch._C, "_cuda_getDevice") else torch.cuda.current_device


# (ctypes cuts a number to the 32 bits of a C int without a word.)
_INT = (1 << 31) - 1


def _together(what, *tensors):
    """Says of tensors on GPUs why they are not all on the current one."""
    at = {t.get_device() for t in tensors if t is not None}
    if at != {_device()}:
        _refuse(f"{what}: the tensors are on devices {sorted(at)}, the current one is {_device()}")


def alloc_window_attention_workspace(S, n_heads, n_kv_heads, head_dim, max_new, max_length, window=0, sinks=0, device="cuda"):
    """Workspace of muxq_window_attention, also good for fewer sequences and tokens and smaller windows (empty where none is needed)."""
    n = lib().muxq_window_attention_workspace_bytes(S, n_heads, n_kv_heads, head_dim, max_new, max_length, window, sinks)
    return torch.empty(n, dtype=torch.uint8, device=device)


def alloc_tree_attention_workspace(S, n_heads, n_kv_heads, head_dim, max_nodes, max_length, device="cuda"):
    """Workspace of muxq_tree_attention, also good for fewer sequences, nodes and tokens (empty where none is needed)."""
    n = lib().muxq_tree_attention_workspace_bytes(S, n_heads, n_kv_heads, head_dim, max_nodes, max_length)
    return torch.empty(n, dtype=torch.uint8, device=device)


def _rows_args(what, q, k_cache, v_cache, block_table, starts, lengths, max_new, max_length, k_scale, v_scale, out, workspace, parents=None):
    """The checks that both attentions of several new tokens share: (descriptor of the cache, out, arguments up to lengths)."""
    M, n_heads, d = q.shape
    c = _kv(k_cache, v_cache, k_scale, v_scale)
    S = lengths.numel()
    if out is None:
        out = torch.empty((M, n_heads, d), dtype=torch.float16, device=q.device)
    qs, os, ts = q.stride(), out.stride(), block_table.stride()
    if not (q.dtype is out.dtype is _F16 and block_table.dtype is lengths.dtype is starts.dtype is _I32 and
            _device() == q.get_device() == out.get_device() == k_cache.get_device() == v_cache.get_device() == block_table.get_device() ==
            lengths.get_device() == starts.get_device() and (k_scale is None or k_scale.get_device() == v_scale.get_device() == q.get_device()) and
            (parents is None or (parents.dtype is _I32 and parents.get_device() == q.get_device() and parents.is_contiguous() and
                                 parents.numel() == M)) and d == c.head_dim and out.shape == q.shape and
            qs[2] == os[2] == 1 and (n_heads == 1 or qs[1] == os[1] == d) and block_table.dim() == 2 and block_table.shape[0] == S and
            (ts[1] == 1 or block_table.shape[1] == 1) and lengths.is_contiguous() and starts.is_contiguous() and starts.numel() == S + 1 and
            max_length <= block_table.shape[1] * c.block_size and 0 <= qs[0] | os[0] | ts[0] | max_new | max_length <= _INT):
        _rows(q, "q"), _rows(out, "out"), _flat(lengths, S, _I32, "lengths"), _flat(starts, S + 1, _I32, "starts"), _flat(parents, M, _I32, "parents")
        if block_table.is_cuda:
            _together(what, q, out, k_cache, v_cache, k_scale, v_scale, block_table, starts, lengths, parents)
        _refuse(f"{what}: q, out and the cache differ in head size, starts has not one entry more than lengths, or block_table is no "
                "int32 GPU tensor [S, pages] with contiguous rows of max_length tokens, or a row stride or a bound takes more than 31 bits")
    if workspace is not None and workspace.get_device() != _device():
        _refuse(f"{what}: the workspace is no tensor of the current device")
    # (a dimension of one element may carry any stride)
    ldq, ldo = (qs[0], os[0]) if M > 1 else (n_heads * d, n_heads * d)
    return c, out, ldo, S, (q.data_ptr(), M, n_heads, ldq, C.byref(c), block_table.data_ptr(), ts[0] if S > 1 else block_table.shape[1],
                            starts.data_ptr(), lengths.data_ptr())


def muxq_window_attention(q, k_cache, v_cache, block_table, starts, lengths, max_new, max_length, window=0, sinks=0, scale=None,
                          k_scale=None, v_scale=None, out=None, workspace=None):
    """Causal attention of the new tokens of each sequence, q [M, n_heads, d], over the cache, where they stand already: rows
    starts[s]..starts[s + 1] (int32 [S + 1]) are the last of lengths[s] tokens (int32 [S]).  window: how many tokens a row sees, its own the
    last of them (0: all), with the first `sinks` of the sequence beside them.  max_new, max_length: bounds on the rows and tokens of a
    sequence known on the host.  scale: 1 / sqrt(d) when not given."""
    if not 0 <= window | sinks <= _INT:
        _refuse("muxq_window_attention: window and sinks are numbers of tokens, 31 bits at most")
    c, out, ldo, S, args = _rows_args("muxq_window_attention", q, k_cache, v_cache, block_table, starts, lengths, max_new, max_length, k_scale,
                                      v_scale, out, workspace)
    args += (S, max_new, max_length, window, sinks, c.head_dim ** -0.5 if scale is None else scale, out.data_ptr(), ldo)
    _call(lib().muxq_window_attention, args, workspace, _stream(),
          lambda: alloc_window_attention_workspace(S, q.shape[1], c.n_kv_heads, c.head_dim, max_new, max_length, window, sinks, q.device),
          "muxq_window_attention")
    return out


def muxq_tree_attention(q, k_cache, v_cache, block_table, starts, lengths, parents, max_nodes, max_length, scale=None, k_scale=None,
                        v_scale=None, out=None, workspace=None):
    """Attention of the nodes of a drafted tree of each sequence, as muxq_window_attention without a window, but a node sees of the
    new tokens only itself and the nodes above it; parents (int32 [M]): the number of each node's parent within its
    sequence, -1 for a root.  max_nodes: a bound on the nodes of a tree, at most 64.  There is no window for trees."""
    c, out, ldo, S, args = _rows_args("muxq_tree_attention", q, k_cache, v_cache, block_table, starts, lengths, max_nodes, max_length, k_scale,
                                      v_scale, out, workspace, parents)
    args += (parents.data_ptr(), S, max_nodes, max_length, c.head_dim ** -0.5 if scale is None else scale,
             out.data_ptr(), ldo)
    _call(lib().muxq_tree_attention, args, workspace, _stream(),
          lambda: alloc_tree_attention_workspace(S, q.shape[1], c.n_kv_heads, c.head_dim, max_nodes, max_length, q.device),
          "muxq_tree_attention")
    return out


def muxq_verify_tree(target, tokens, starts, parents, max_nodes, draft=None, uniforms=None, path=None, counts=None, next_token=None):
    """Drafted trees against the target's probabilities, target [M, V] float, row m what comes after node m: (path int32 [M], counts
    int32 [S], next_token int32 [S]).  tokens, parents: int32 [M]; starts: int32 [S + 1]; draft [M, V] float: what each
    node's children were drawn from (None: chosen without drawing); uniforms float [M] in [0, 1), None: greedy."""
    M, V = target.shape
    S = starts.numel() - 1
    device = target.device
    path = torch.empty(M, dtype=torch.int32, device=device) if path is None else path
    counts = torch.empty(S, dtype=torch.int32, device=device) if counts is None else counts
    next_token = torch.empty(S, dtype=torch.int32, device=device) if next_token is None else next_token
    if not (target.dtype is _F32 and tokens.dtype is parents.dtype is starts.dtype is path.dtype is counts.dtype is next_token.dtype is _I32 and
            _device() == target.get_device() == tokens.get_device() == parents.get_device() == starts.get_device() == path.get_device() ==
            counts.get_device() == next_token.get_device() and
            (target.stride(1) == 1 or V == 1) and 0 <= target.stride(0) | max_nodes <= _INT and tokens.is_contiguous() and parents.is_contiguous() and starts.is_contiguous() and
            path.is_contiguous() and counts.is_contiguous() and next_token.is_contiguous() and tokens.numel() == parents.numel() == path.numel() == M and
            counts.numel() == next_token.numel() == S and
            (draft is None or (draft.dtype is _F32 and draft.get_device() == target.get_device() and draft.shape == (M, V) and (draft.stride(1) == 1 or V == 1) and
                               draft.stride(0) <= _INT)) and
            (uniforms is None or (uniforms.dtype is _F32 and uniforms.get_device() == target.get_device() and uniforms.is_contiguous() and uniforms.numel() == M))):
        _flat(tokens, M, _I32, "tokens"), _flat(parents, M, _I32, "parents"), _flat(starts, S + 1, _I32, "starts"), _flat(uniforms, M, _F32, "uniforms")
        _flat(path, M, _I32, "path"), _flat(counts, S, _I32, "counts"), _flat(next_token, S, _I32, "next_token")
        if target.is_cuda and (draft is None or draft.is_cuda):
            _together("muxq_verify_tree", target, tokens, starts, parents, draft, uniforms, path, counts, next_token)
        _refuse(f"muxq_verify_tree: target and draft are GPU tensors of float [{M}, {V}] with contiguous rows; tokens, parents and path have a number "
                "for each row, counts and next_token for each sequence; row strides and max_nodes take 31 bits at most")
    # (a dimension of one element may carry any stride)
    ldt = target.stride(0) if M > 1 else V
    ldd = 0 if draft is None else draft.stride(0) if M > 1 else V
    status = lib().muxq_verify_tree(target.data_ptr(), ldt, _p(draft), ldd, M, V, tokens.data_ptr(), parents.data_ptr(), _p(uniforms),
                                    starts.data_ptr(), S, max_nodes, path.data_ptr(), counts.data_ptr(), next_token.data_ptr(), _stream())
    if status != 0:
        _check(status, "muxq_verify_tree")
    return path, counts, next_token


def muxq_kv_copy(src, dst, k_cache, v_cache, k_scale=None, v_scale=None):
    """Pages dst[i] of the cache become copies of pages src[i] (int32 [n]; pairs with a page outside it are left out)."""
    c = _kv(k_cache, v_cache, k_scale, v_scale)
    n = src.numel()
    if not (src.dtype is dst.dtype is _I32 and _device() == src.get_device() == dst.get_device() == k_cache.get_device() == v_cache.get_device() and
            (k_scale is None or k_scale.get_device() == v_scale.get_device() == src.get_device()) and
            src.is_contiguous() and dst.is_contiguous() and dst.numel() == n):
        _flat(src, n, _I32, "src"), _flat(dst, n, _I32, "dst")
        if dst.numel() == n:
            _together("muxq_kv_copy", k_cache, v_cache, k_scale, v_scale, src, dst)
        _refuse("muxq_kv_copy: src and dst differ in length")
    status = lib().muxq_kv_copy(src.data_ptr(), dst.data_ptr(), n, C.byref(c), _stream())
    if status != 0:
        _check(status, "muxq_kv_copy")


def muxq_kv_compact(path, counts, starts, lengths, block_table, k_cache, v_cache, max_nodes, k_scale=None, v_scale=None):
    """The accepted nodes of each tree (path, counts as muxq_verify_tree gives them) become the first of its new tokens in the
    cache; starts, lengths (the nodes among them) and block_table as muxq_tree_attention takes them."""
    c = _kv(k_cache, v_cache, k_scale, v_scale)
    S, M = counts.numel(), path.numel()
    if not (path.dtype is counts.dtype is starts.dtype is lengths.dtype is block_table.dtype is _I32 and
            _device() == path.get_device() == counts.get_device() == starts.get_device() == lengths.get_device() == block_table.get_device() ==
            k_cache.get_device() == v_cache.get_device() and (k_scale is None or k_scale.get_device() == v_scale.get_device() == path.get_device()) and
            path.is_contiguous() and counts.is_contiguous() and
            starts.is_contiguous() and lengths.is_contiguous() and starts.numel() == S + 1 and lengths.numel() == S and block_table.dim() == 2 and
            block_table.shape[0] == S and (block_table.stride(1) == 1 or block_table.shape[1] == 1) and 0 <= block_table.stride(0) | max_nodes <= _INT):
        _flat(path, M, _I32, "path"), _flat(counts, S, _I32, "counts"), _flat(starts, S + 1, _I32, "starts"), _flat(lengths, S, _I32, "lengths")
        if block_table.is_cuda:
            _together("muxq_kv_compact", k_cache, v_cache, k_scale, v_scale, path, counts, starts, lengths, block_table)
        _refuse("muxq_kv_compact: starts has one entry more than counts, lengths as many, and block_table is an int32 GPU tensor [S, pages] with "
                "contiguous rows; its row stride and max_nodes take 31 bits at most")
    status = lib().muxq_kv_compact(path.data_ptr(), counts.data_ptr(), starts.data_ptr(), lengths.data_ptr(), block_table.data_ptr(),
                                   block_table.stride(0) if S > 1 else block_table.shape[1], M, S, max_nodes, C.byref(c), _stream())
    if status != 0:
        _check(status, "muxq_kv_compact")
