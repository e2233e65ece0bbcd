"""Thin ctypes binding of libsla.so: argument marshalling only.

Every function has the name and the semantics of the C entry point declared in
include/sla.h; tensors are torch CUDA tensors used purely as device memory (their
data_ptr() is passed through), the stream is torch's current stream.  There is no CPU
fallback: if the HIP library has not been built, importing the symbols raises.
"""
from __future__ import annotations

import ctypes as C
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsla.so")

SLA_OK, SLA_ERR_INVALID_ARG, SLA_ERR_UNSUPPORTED, SLA_ERR_WORKSPACE, SLA_ERR_HIP = 0, -1, -2, -3, -4
SLA_BF16, SLA_FP8_E4M3 = 0, 1
STATE_ROWS = 65          # rows of one block state: 64 rows of h^T and one row of z
EXPORTS = ["sla_resolve_counts", "sla_workspace_bytes", "sla_forward", "sla_pool_classify", "sla_linear_states",
           "sla_marginal_aggregate", "sla_sparse_combine", "sla_forward_profiled", "sla_wproj_grad", "sla_quantise_e4m3",
           "sla_forward_with_labels", "sla_fp8_linear_workspace_bytes", "sla_fp8_linear", "sla_forward_static", "sla_sparse_combine_f32", "sla_fp8_linear_qkv",
           "sla_fp8_checkpoint_bytes", "sla_fp8_checkpoint_restore", "sla_fp8_linear_grad_workspace_bytes", "sla_fp8_linear_save", "sla_fp8_linear_grad",
           "sla_quantise_mxfp4", "sla_dequantise_mxfp4", "sla_mxfp4_linear_workspace_bytes", "sla_mxfp4_linear",
           "sla_qk_norm_rope", "sla_qk_norm_rope_e4m3", "sla_qk_norm_rope_grad_workspace_bytes", "sla_qk_norm_rope_grad",
           "sla_strerror", "sla_last_error", "sla_stage_name"]
STATIC_WORKSPACE_BYTES = 96 * 1024 * 1024
NUM_STAGES = 6


class SlaParams(C.Structure):
    _fields_ = [("B", C.c_int32), ("H", C.c_int32), ("N", C.c_int32), ("D", C.c_int32),
                ("bq", C.c_int32), ("bk", C.c_int32),
                ("crit_frac", C.c_double), ("neg_frac", C.c_double),
                ("k_crit", C.c_int32), ("k_neg", C.c_int32),
                ("dtype", C.c_int32), ("phi", C.c_int32), ("proj_per_head", C.c_int32),
                ("sm_scale", C.c_float), ("layout", C.c_int32)]


class SlaError(RuntimeError):
    def __init__(self, status: int, where: str, detail: str):
        super().__init__(f"{where}: status {status}: {detail}")
        self.status = status


_lib = None


def lib() -> C.CDLL:
    """Loads the HIP library; raises if it has not been built (no fallback path exists)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: run `python -m paper_2605_11354_amd.build` "
                              "(the SLA forward has no CPU or PyTorch fallback)")
        _lib = C.CDLL(LIB_PATH)
        for name in EXPORTS:
            getattr(_lib, name)                      # raises AttributeError on a missing export
        _lib.sla_strerror.restype = C.c_char_p
        _lib.sla_last_error.restype = C.c_char_p
        _lib.sla_stage_name.restype = C.c_char_p
        for name in EXPORTS[:-3]:                    # all but the three that return text
            getattr(_lib, name).restype = C.c_int
    return _lib


def make_params(B, H, N, bq, bk, crit_frac=0.0, neg_frac=0.0, k_crit=-1, k_neg=-1, dtype="bf16",
                proj_per_head=False, sm_scale=0.0, D=64, phi="softmax", layout="bhnd") -> SlaParams:
    """layout: "bhnd" = Q, K, V, O are [B,H,N,D]; "bnhd" = [B,N,H,D] (rows of a head H*D elements apart)."""
    return SlaParams(B, H, N, D, bq, bk, crit_frac, neg_frac, k_crit, k_neg,
                     SLA_BF16 if dtype == "bf16" else SLA_FP8_E4M3, {"softmax": 0, "elu1": 1}[phi],
                     1 if proj_per_head else 0, sm_scale, {"bhnd": 0, "bnhd": 1}[layout])


def _check(status: int, where: str):
    if status != SLA_OK:
        raise SlaError(status, where, lib().sla_last_error().decode())


def _ptr(t):
    if t is None:
        return C.c_void_p(0)
    assert t.is_cuda and t.is_contiguous(), "device tensors must be contiguous CUDA tensors"
    return C.c_void_p(t.data_ptr())


def _stream():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def sla_resolve_counts(p: SlaParams):
    kc, kn = C.c_int32(), C.c_int32()
    _check(lib().sla_resolve_counts(C.byref(p), C.byref(kc), C.byref(kn)), "sla_resolve_counts")
    return kc.value, kn.value


def sla_workspace_bytes(p: SlaParams) -> int:
    n = C.c_size_t()
    _check(lib().sla_workspace_bytes(C.byref(p), C.byref(n)), "sla_workspace_bytes")
    return n.value


def alloc_workspace(p: SlaParams, device="cuda:0") -> torch.Tensor:
    return torch.empty(max(256, sla_workspace_bytes(p)), dtype=torch.uint8, device=device)


def sla_forward(p, Q, K, V, W_proj, O, labels=None, sQ=None, sK=None, sV=None, workspace=None):
    ws = workspace if workspace is not None else alloc_workspace(p, Q.device)
    _check(lib().sla_forward(C.byref(p), _ptr(Q), _ptr(K), _ptr(V), _ptr(sQ), _ptr(sK), _ptr(sV), _ptr(W_proj),
                             _ptr(O), _ptr(labels), _ptr(ws), C.c_size_t(ws.numel()), _stream()), "sla_forward")
    return O


def sla_forward_static(p, Q, K, V, W_proj, O, labels=None, sQ=None, sK=None, sV=None):
    """sla_forward on the library's own workspace (no allocation; shapes up to STATIC_WORKSPACE_BYTES of workspace)."""
    _check(lib().sla_forward_static(C.byref(p), _ptr(Q), _ptr(K), _ptr(V), _ptr(sQ), _ptr(sK), _ptr(sV), _ptr(W_proj),
                                    _ptr(O), _ptr(labels), _stream()), "sla_forward_static")
    return O


def sla_forward_profiled(p, Q, K, V, W_proj, O, labels=None, sQ=None, sK=None, sV=None, workspace=None):
    """Returns {stage name: milliseconds} for one forward (synchronises the stream)."""
    ws = workspace if workspace is not None else alloc_workspace(p, Q.device)
    ms = (C.c_float * NUM_STAGES)()
    _check(lib().sla_forward_profiled(C.byref(p), _ptr(Q), _ptr(K), _ptr(V), _ptr(sQ), _ptr(sK), _ptr(sV), _ptr(W_proj),
                                      _ptr(O), _ptr(labels), _ptr(ws), C.c_size_t(ws.numel()), _stream(), ms),
           "sla_forward_profiled")
    return {lib().sla_stage_name(i).decode(): float(ms[i]) for i in range(NUM_STAGES)}


def sla_pool_classify(p, Q, K, labels, crit_idx=None, Pc=None, qbar=None, kbar=None, scores=None,
                      sQ=None, sK=None, workspace=None):
    ws = workspace if workspace is not None else alloc_workspace(p, Q.device)
    _check(lib().sla_pool_classify(C.byref(p), _ptr(Q), _ptr(K), _ptr(sQ), _ptr(sK), _ptr(labels), _ptr(crit_idx),
                                   _ptr(Pc), _ptr(qbar), _ptr(kbar), _ptr(scores), _ptr(ws), C.c_size_t(ws.numel()),
                                   _stream()), "sla_pool_classify")
    return labels


def sla_linear_states(p, K, V, hT, sK=None, sV=None):
    _check(lib().sla_linear_states(C.byref(p), _ptr(K), _ptr(V), _ptr(sK), _ptr(sV), _ptr(hT), _stream()),
           "sla_linear_states")
    return hT


def sla_marginal_aggregate(p, labels, hT, Hq, workspace=None):
    ws = workspace if workspace is not None else alloc_workspace(p, hT.device)
    _check(lib().sla_marginal_aggregate(C.byref(p), _ptr(labels), _ptr(hT), _ptr(Hq), _ptr(ws), C.c_size_t(ws.numel()),
                                        _stream()), "sla_marginal_aggregate")
    return Hq


def sla_forward_with_labels(p, Q, K, V, W_proj, labels, O, sQ=None, sK=None, sV=None, workspace=None):
    ws = workspace if workspace is not None else alloc_workspace(p, Q.device)
    _check(lib().sla_forward_with_labels(C.byref(p), _ptr(Q), _ptr(K), _ptr(V), _ptr(sQ), _ptr(sK), _ptr(sV), _ptr(W_proj),
                                         _ptr(labels), _ptr(O), _ptr(ws), C.c_size_t(ws.numel()), _stream()),
           "sla_forward_with_labels")
    return O


def sla_fp8_linear(x, W, bias, y, workspace=None):
    """y bf16 [N,d_out] <- FP8 fake-quantised linear layer of x bf16 [N,d_in] with W bf16 [d_out,d_in] and bias (or None)."""
    import torch
    N, d_in = x.shape
    d_out = W.shape[0]
    n = C.c_size_t(0)
    _check(lib().sla_fp8_linear_workspace_bytes(C.c_int32(N), C.c_int32(d_in), C.c_int32(d_out), C.byref(n)), "sla_fp8_linear_workspace_bytes")
    ws = workspace if workspace is not None else torch.empty(max(n.value, 256), dtype=torch.uint8, device=x.device)
    _check(lib().sla_fp8_linear(_ptr(x), _ptr(W), _ptr(bias), C.c_int32(N), C.c_int32(d_in), C.c_int32(d_out), _ptr(y), _ptr(ws),
                                C.c_size_t(ws.numel()), _stream()), "sla_fp8_linear")
    return y


def sla_quantise_e4m3(X, blk, codes, scales, layout="bhnd"):
    """X bf16 [B,H,N,64] ([B,N,H,64] with layout "bnhd") -> codes uint8 of the same layout, scales fp32 [B,H,ceil(N/blk)]."""
    if layout == "bhnd":
        Bn, H, N, D = X.shape
    else:
        Bn, N, H, D = X.shape
    assert D == 64
    _check(lib().sla_quantise_e4m3(_ptr(X), C.c_int32(Bn), C.c_int32(H), C.c_int32(N), C.c_int32(blk),
                                   C.c_int32({"bhnd": 0, "bnhd": 1}[layout]), _ptr(codes), _ptr(scales), _stream()),
           "sla_quantise_e4m3")
    return codes, scales


def sla_wproj_grad(p, Q, dO, dW, workspace, sQ=None):
    """dW (fp32 [nW,64,64]) <- gradient of sum(O * dO) w.r.t. W_proj; `workspace` is the one sla_forward just used."""
    _check(lib().sla_wproj_grad(C.byref(p), _ptr(Q), _ptr(sQ), _ptr(dO), _ptr(dW), _ptr(workspace),
                                C.c_size_t(workspace.numel()), _stream()), "sla_wproj_grad")
    return dW


def sla_sparse_combine(p, Q, K, V, W_proj, labels, Hq, O, sQ=None, sK=None, sV=None, workspace=None):
    ws = workspace if workspace is not None else alloc_workspace(p, Q.device)
    _check(lib().sla_sparse_combine(C.byref(p), _ptr(Q), _ptr(K), _ptr(V), _ptr(sQ), _ptr(sK), _ptr(sV), _ptr(W_proj),
                                    _ptr(labels), _ptr(Hq), _ptr(O), _ptr(ws), C.c_size_t(ws.numel()), _stream()),
           "sla_sparse_combine")
    return O


def sla_sparse_combine_f32(p, Q, K, V, W_proj, labels, Hq, O32, sQ=None, sK=None, sV=None, workspace=None):
    """sla_sparse_combine with the result in fp32 (O32: float32 tensor of the shape of O)."""
    ws = workspace if workspace is not None else alloc_workspace(p, Q.device)
    _check(lib().sla_sparse_combine_f32(C.byref(p), _ptr(Q), _ptr(K), _ptr(V), _ptr(sQ), _ptr(sK), _ptr(sV), _ptr(W_proj),
                                        _ptr(labels), _ptr(Hq), _ptr(O32), _ptr(ws), C.c_size_t(ws.numel()), _stream()),
           "sla_sparse_combine_f32")
    return O32


def sla_fp8_linear_qkv(x, W, bias, B_, N, H, bq, Q8, K8, V8, sQ, sK, sV, workspace=None):
    """qkv projection with the per-block E4M3 quantiser in the GEMM's epilogue: x [B*N, d_in], W [3*H*64, d_in]."""
    import torch
    d_in = x.shape[1]
    if workspace is None:
        n = C.c_size_t()
        _check(lib().sla_fp8_linear_workspace_bytes(C.c_int32(B_ * N), C.c_int32(d_in), C.c_int32(3 * H * 64), C.byref(n)),
               "sla_fp8_linear_workspace_bytes")
        workspace = torch.empty(max(256, n.value), dtype=torch.uint8, device=x.device)
    _check(lib().sla_fp8_linear_qkv(_ptr(x), _ptr(W), _ptr(bias), C.c_int32(B_), C.c_int32(N), C.c_int32(H), C.c_int32(d_in),
                                    C.c_int32(bq), _ptr(Q8), _ptr(K8), _ptr(V8), _ptr(sQ), _ptr(sK), _ptr(sV),
                                    _ptr(workspace), C.c_size_t(workspace.numel()), _stream()), "sla_fp8_linear_qkv")


# ---- norm and rotation of heads
class SlaHeadsParams(C.Structure):
    _fields_ = [("B", C.c_int32), ("H", C.c_int32), ("N", C.c_int32), ("D", C.c_int32),
                ("norm", C.c_int32), ("norm_per_head", C.c_int32), ("axes", C.c_int32), ("pairing", C.c_int32),
                ("pos_per_item", C.c_int32), ("layout", C.c_int32), ("eps", C.c_float), ("base", C.c_double),
                ("batch_stride", C.c_int64), ("token_stride", C.c_int64), ("head_stride", C.c_int64)]


def make_heads_params(q, norm="layer", norm_per_head=False, eps=1e-5, axes=2, pairing="halves", base=100.0, pos_per_item=False,
                      layout="bhnd") -> SlaHeadsParams:
    """q: a [B,N,H,64] tensor or view with the sizes and strides that q, k, v (and dq, dk, dv) have, e.g. qkv[:, :, 0] of a fused
    projection qkv [B,N,3,H,64].  layout: of the outputs, "bhnd" or "bnhd"."""
    Bn, N, H, D = q.shape
    if q.stride(3) != 1 and D > 1 and q.numel():
        raise ValueError("the 64 channels of a row must be contiguous")
    return SlaHeadsParams(Bn, H, N, D, {"none": 0, "rms": 1, "layer": 2}[norm], int(norm_per_head), axes,
                          {"halves": 0, "adjacent": 1}[pairing], int(pos_per_item), {"bhnd": 0, "bnhd": 1}[layout], eps, base,
                          q.stride(0), q.stride(1), q.stride(2))


def _tensor(t, what, dtype, shape):
    """Pointer of a dense device tensor of this type and shape (None: NULL)."""
    if t is None:
        return None
    if t.dtype != dtype or tuple(t.shape) != shape:
        raise ValueError(f"{what}: {dtype} {list(shape)} expected, got {t.dtype} {list(t.shape)}")
    if not t.is_cuda or t.device.index != torch.cuda.current_device() or not t.is_contiguous():
        raise ValueError(f"{what}: a contiguous tensor on the current device expected")
    return t.data_ptr()


def _rows(p, t, what):
    """Pointer of a [B,N,H,64] tensor with the strides in p."""
    if t is None:
        return None
    shape, strides = (p.B, p.N, p.H, p.D), (p.batch_stride, p.token_stride, p.head_stride, 1)
    if t.dtype != torch.bfloat16 or tuple(t.shape) != shape or any(n > 1 and a != b for n, a, b in zip(shape, t.stride(), strides)):
        raise ValueError(f"{what}: bfloat16 {list(shape)} with strides {list(strides)} expected, got {t.dtype} {list(t.shape)} {list(t.stride())}")
    if not t.is_cuda or t.device.index != torch.cuda.current_device():
        raise ValueError(f"{what}: a tensor on the current device expected")
    return t.data_ptr()


def _heads_parameters(p, pos, *params):
    shape = (p.H, 64) if p.norm_per_head else (64,)
    names = ("q_weight", "q_bias", "k_weight", "k_bias")
    ptrs = [_tensor(t, n, torch.float32, shape) for t, n in zip(params, names)]
    full = (p.B if p.pos_per_item else 1, p.N, p.axes)
    return ptrs, _tensor(pos, "pos", torch.int32, full[1:] if pos is not None and pos.dim() == 2 and full[0] == 1 else full)


def _heads_shape(p):
    return (p.B, p.N, p.H, 64) if p.layout else (p.B, p.H, p.N, 64)


def _ptrs(ptrs):
    return [C.c_void_p(x) for x in ptrs]


def sla_qk_norm_rope(p, q, k, v, Q, K, V, pos=None, q_weight=None, q_bias=None, k_weight=None, k_bias=None):
    """q, k, v bf16 [B,N,H,64] in the strides of p -> Q, K, V bf16 in p's layout; pos int32 [N,axes], [1,N,axes] or [B,N,axes]."""
    w, at = _heads_parameters(p, pos, q_weight, q_bias, k_weight, k_bias)
    shape = _heads_shape(p)
    args = [_rows(p, q, "q"), _rows(p, k, "k"), _rows(p, v, "v"), *w, at, *(_tensor(t, n, torch.bfloat16, shape) for t, n in zip((Q, K, V), "QKV"))]
    _check(lib().sla_qk_norm_rope(C.byref(p), *_ptrs(args), _stream()), "sla_qk_norm_rope")
    return Q, K, V


def sla_qk_norm_rope_e4m3(p, q, k, v, bq, Q8, K8, V8, sQ, sK, sV, pos=None, q_weight=None, q_bias=None, k_weight=None, k_bias=None):
    """The same into E4M3 codes (uint8, p's layout) with block scales fp32 [B,H,ceil(N/bq)], [B,H,ceil(N/64)] twice."""
    w, at = _heads_parameters(p, pos, q_weight, q_bias, k_weight, k_bias)
    shape, blocks = _heads_shape(p), [(p.B, p.H, -(-p.N // max(b, 1))) for b in (bq, 64, 64)]
    args = [_rows(p, q, "q"), _rows(p, k, "k"), _rows(p, v, "v"), *w, at]
    out = [_tensor(t, n, torch.uint8, shape) for t, n in zip((Q8, K8, V8), ("Q8", "K8", "V8"))]
    out += [_tensor(t, n, torch.float32, s) for t, n, s in zip((sQ, sK, sV), ("sQ", "sK", "sV"), blocks)]
    _check(lib().sla_qk_norm_rope_e4m3(C.byref(p), *_ptrs(args), C.c_int32(bq), *_ptrs(out), _stream()), "sla_qk_norm_rope_e4m3")
    return Q8, K8, V8, sQ, sK, sV


def sla_qk_norm_rope_grad_workspace_bytes(p) -> int:
    n = C.c_size_t()
    _check(lib().sla_qk_norm_rope_grad_workspace_bytes(C.byref(p), C.byref(n)), "sla_qk_norm_rope_grad_workspace_bytes")
    return n.value


def sla_qk_norm_rope_grad(p, q, k, dQ, dK, dV, dq, dk, dv, pos=None, q_weight=None, k_weight=None, dq_weight=None, dq_bias=None,
                          dk_weight=None, dk_bias=None, workspace=None):
    """dQ, dK, dV (bf16, p's layout) -> dq, dk, dv (bf16, the strides of q, k, v) and fp32 gradients of the norm's parameters."""
    w, at = _heads_parameters(p, pos, q_weight, None, k_weight, None)
    dw, _ = _heads_parameters(p, None, dq_weight, dq_bias, dk_weight, dk_bias)
    shape = _heads_shape(p)
    if workspace is None:
        workspace = torch.empty(max(256, sla_qk_norm_rope_grad_workspace_bytes(p)), dtype=torch.uint8, device=q.device)
    args = [_rows(p, q, "q"), _rows(p, k, "k"), w[0], w[2], at, *(_tensor(t, n, torch.bfloat16, shape) for t, n in zip((dQ, dK, dV), ("dQ", "dK", "dV"))),
            _rows(p, dq, "dq"), _rows(p, dk, "dk"), _rows(p, dv, "dv"), *dw]
    _check(lib().sla_qk_norm_rope_grad(C.byref(p), *_ptrs(args), _ptr(workspace), C.c_size_t(workspace.numel()), _stream()),
           "sla_qk_norm_rope_grad")
    return dq, dk, dv


# ---- training of the FP8 layer from an 8-bit copy of its input
def _bytes(name, *sizes) -> int:
    n = C.c_size_t()
    _check(getattr(lib(), name)(*[C.c_int32(x) for x in sizes], C.byref(n)), name)
    return n.value


def sla_fp8_checkpoint_bytes(N, d_in) -> int:
    return _bytes("sla_fp8_checkpoint_bytes", N, d_in)


def sla_fp8_linear_grad_workspace_bytes(N, d_in, d_out) -> int:
    return _bytes("sla_fp8_linear_grad_workspace_bytes", N, d_in, d_out)


def _buffer(t, what):
    """(pointer, bytes) of a checkpoint or workspace."""
    p = _tensor(t, what, torch.uint8, (t.numel(),))
    return C.c_void_p(p), C.c_size_t(t.numel())


def _linear_workspace(workspace, N, d_in, d_out, device):
    if workspace is None:
        workspace = torch.empty(max(256, sla_fp8_linear_grad_workspace_bytes(N, d_in, d_out)), dtype=torch.uint8, device=device)
    return _buffer(workspace, "workspace")


def sla_fp8_linear_save(x, W, bias, y, checkpoint, workspace=None):
    """sla_fp8_linear that leaves x in 8 bits in `checkpoint` (uint8, sla_fp8_checkpoint_bytes(N, d_in) long)."""
    (N, d_in), d_out, bf = x.shape, W.shape[0], torch.bfloat16
    args = _ptrs([_tensor(x, "x", bf, (N, d_in)), _tensor(W, "W", bf, (d_out, d_in)), _tensor(bias, "bias", bf, (d_out,))])
    _check(lib().sla_fp8_linear_save(*args, C.c_int32(N), C.c_int32(d_in), C.c_int32(d_out), C.c_void_p(_tensor(y, "y", bf, (N, d_out))),
                                     *_buffer(checkpoint, "checkpoint"), *_linear_workspace(workspace, N, d_in, d_out, x.device), _stream()),
           "sla_fp8_linear_save")
    return y


def sla_fp8_linear_grad(dy, checkpoint, W, dx=None, dW=None, db=None, workspace=None):
    """Gradients of sla_fp8_linear_save's x, W and bias (each may be None; db only with dW) from that of its y."""
    (N, d_out), d_in, bf = dy.shape, W.shape[1], torch.bfloat16
    out = _ptrs([_tensor(dx, "dx", bf, (N, d_in)), _tensor(dW, "dW", bf, (d_out, d_in)), _tensor(db, "db", bf, (d_out,))])
    _check(lib().sla_fp8_linear_grad(C.c_void_p(_tensor(dy, "dy", bf, (N, d_out))), *_buffer(checkpoint, "checkpoint"),
                                     C.c_void_p(_tensor(W, "W", bf, (d_out, d_in))), C.c_int32(N), C.c_int32(d_in), C.c_int32(d_out), *out,
                                     *_linear_workspace(workspace, N, d_in, d_out, dy.device), _stream()), "sla_fp8_linear_grad")
    return dx, dW, db


def sla_fp8_checkpoint_restore(checkpoint, x):
    """x bf16 [N,d_in] <- the layer's input as its forward multiplied it."""
    N, d_in = x.shape
    _check(lib().sla_fp8_checkpoint_restore(*_buffer(checkpoint, "checkpoint"), C.c_int32(N), C.c_int32(d_in),
                                            C.c_void_p(_tensor(x, "x", torch.bfloat16, (N, d_in))), _stream()), "sla_fp8_checkpoint_restore")
    return x


# ---- microscaled 4-bit numbers
def sla_quantise_mxfp4(X, codes, scales):
    """X bf16 [rows, cols] -> codes uint8 [rows, cols/2], scales uint8 [rows, cols/32]."""
    rows, cols = X.shape
    args = _ptrs([_tensor(codes, "codes", torch.uint8, (rows, cols // 2)), _tensor(scales, "scales", torch.uint8, (rows, cols // 32))])
    _check(lib().sla_quantise_mxfp4(C.c_void_p(_tensor(X, "X", torch.bfloat16, (rows, cols))), C.c_int64(rows), C.c_int32(cols), *args, _stream()),
           "sla_quantise_mxfp4")
    return codes, scales


def sla_dequantise_mxfp4(codes, scales, Y):
    """Y bf16 [rows, cols] <- the numbers that codes and scales stand for."""
    rows, cols = Y.shape
    args = _ptrs([_tensor(codes, "codes", torch.uint8, (rows, cols // 2)), _tensor(scales, "scales", torch.uint8, (rows, cols // 32))])
    _check(lib().sla_dequantise_mxfp4(*args, C.c_int64(rows), C.c_int32(cols), C.c_void_p(_tensor(Y, "Y", torch.bfloat16, (rows, cols))), _stream()),
           "sla_dequantise_mxfp4")
    return Y


def sla_mxfp4_linear_workspace_bytes(N, d_in, d_out) -> int:
    return _bytes("sla_mxfp4_linear_workspace_bytes", N, d_in, d_out)


def sla_mxfp4_linear(x, W_codes, W_scales, bias, y, workspace=None):
    """y bf16 [N,d_out] <- linear layer of x bf16 [N,d_in], both factors in microscaled 4-bit numbers."""
    (N, d_in), d_out, bf = x.shape, W_codes.shape[0], torch.bfloat16
    args = _ptrs([_tensor(x, "x", bf, (N, d_in)), _tensor(W_codes, "W_codes", torch.uint8, (d_out, d_in // 2)),
                  _tensor(W_scales, "W_scales", torch.uint8, (d_out, d_in // 32)), _tensor(bias, "bias", bf, (d_out,))])
    if workspace is None:
        workspace = torch.empty(max(256, sla_mxfp4_linear_workspace_bytes(N, d_in, d_out)), dtype=torch.uint8, device=x.device)
    _check(lib().sla_mxfp4_linear(*args, C.c_int32(N), C.c_int32(d_in), C.c_int32(d_out), C.c_void_p(_tensor(y, "y", bf, (N, d_out))),
                                  *_buffer(workspace, "workspace"), _stream()), "sla_mxfp4_linear")
    return y
