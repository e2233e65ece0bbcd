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
# argument kinds of the calls that a decoding step or a short layer makes often: pointer, int32, int64, size_t
_KINDS = {"p": C.c_void_p, "i": C.c_int32, "l": C.c_int64, "z": C.c_size_t}
_ARGUMENTS = {"sla_qk_norm_rope": "p" * 13, "sla_qk_norm_rope_e4m3": "p" * 9 + "i" + "p" * 7, "sla_qk_norm_rope_grad": "p" * 17 + "zp",
              "sla_qk_norm_rope_grad_workspace_bytes": "pp",
              "sla_fp8_checkpoint_bytes": "iip", "sla_fp8_checkpoint_restore": "pziipp", "sla_fp8_linear_grad_workspace_bytes": "iiip",
              "sla_fp8_linear_save": "pppiiippzpzp", "sla_fp8_linear_grad": "ppzpiiippppzp",
              "sla_quantise_mxfp4": "plippp", "sla_dequantise_mxfp4": "pplipp", "sla_mxfp4_linear_workspace_bytes": "iiip",
              "sla_mxfp4_linear": "ppppiiippzp"}
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
        for name, kinds in _ARGUMENTS.items():       # with these, plain integers and None pass for pointers and sizes
            getattr(_lib, name).argtypes = [_KINDS[k] for k in kinds]
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


# ---- what the calls below share: checks of tensors against the sizes that go with the pointers
def _device() -> int:
    """The current device; before any is in use there are no device tensors, and every tensor is refused."""
    return torch.cuda.current_device() if torch.cuda.is_initialized() else -2


def _raw_stream(dev):
    return torch._C._cuda_getCurrentRawStream(dev)       # torch.cuda.current_stream().cuda_stream without the object around it


def _refuse(t, what, dtype, shape, dev):
    if t.dtype != dtype or tuple(t.shape) != shape:
        raise ValueError(f"{what}: {dtype} {list(shape)} expected, got {t.dtype} {list(t.shape)}")
    raise ValueError(f"{what}: a contiguous tensor on the current device expected, got one on {t.device} with strides {list(t.stride())}")


def _tensor(t, what, dtype, shape, dev):
    """Pointer of a dense device tensor of this type and shape (None: NULL)."""
    if t is None:
        return None
    if t.dtype is not dtype or t.shape != shape or t.get_device() != dev or not t.is_contiguous():
        _refuse(t, what, dtype, shape, dev)
    return t.data_ptr()


def _buffer(t, what, dev):
    """(pointer, bytes) of a checkpoint or workspace."""
    n = t.numel()
    return _tensor(t, what, torch.uint8, (n,), dev), n


def _bytes(name, *sizes) -> int:
    n = C.c_size_t()
    _check(getattr(lib(), name)(*sizes, C.byref(n)), name)
    return n.value


def _scratch(need, device):
    return torch.empty(max(256, need), dtype=torch.uint8, device=device)


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


class _Heads:
    """The sizes in p as the tensors of a call have to have them."""

    def __init__(self, p):
        self.p, self.dev = p, _device()
        self.shape = (p.B, p.N, p.H, p.D)
        self.strides = (p.batch_stride, p.token_stride, p.head_stride, 1)
        self.out = self.shape if p.layout else (p.B, p.H, p.N, p.D)

    def rows(self, t, what):
        """Pointer of a [B,N,H,64] tensor with the strides in p."""
        if t is None:
            return None
        if t.dtype is not torch.bfloat16 or t.shape != self.shape or t.get_device() != self.dev or \
                (t.stride() != self.strides and any(n > 1 and a != b for n, a, b in zip(self.shape, t.stride(), self.strides))):
            raise ValueError(f"{what}: bfloat16 {list(self.shape)} with strides {list(self.strides)} on the current device "
                             f"expected, got {t.dtype} {list(t.shape)} {list(t.stride())} on {t.device}")
        return t.data_ptr()

    def dense(self, t, what, dtype=torch.bfloat16):
        return _tensor(t, what, dtype, self.out, self.dev)

    def weight(self, t, what):
        return _tensor(t, what, torch.float32, (self.p.H, 64) if self.p.norm_per_head else (64,), self.dev) if t is not None else None

    def positions(self, pos):
        if pos is None:
            return None
        full = (self.p.B if self.p.pos_per_item else 1, self.p.N, self.p.axes)
        return _tensor(pos, "pos", torch.int32, full[1:] if pos.dim() == 2 and full[0] == 1 else full, self.dev)


def sla_qk_norm_rope(p, q, k, v, Q, K, V, pos=None, q_weight=None, q_bias=None, k_weight=None, k_bias=None):
    """q, k, v bf16 [B,N,H,64] in the strides of p -> Q, K, V bf16 in p's layout; pos int32 [N,axes], [1,N,axes] or [B,N,axes]."""
    h = _Heads(p)
    _check(lib().sla_qk_norm_rope(C.byref(p), h.rows(q, "q"), h.rows(k, "k"), h.rows(v, "v"), h.weight(q_weight, "q_weight"), h.weight(q_bias, "q_bias"),
                                  h.weight(k_weight, "k_weight"), h.weight(k_bias, "k_bias"), h.positions(pos),
                                  h.dense(Q, "Q"), h.dense(K, "K"), h.dense(V, "V"), _raw_stream(h.dev)), "sla_qk_norm_rope")
    return Q, K, V


def sla_qk_norm_rope_e4m3(p, q, k, v, bq, Q8, K8, V8, sQ, sK, sV, pos=None, q_weight=None, q_bias=None, k_weight=None, k_bias=None):
    """The same into E4M3 codes (uint8, p's layout) with block scales fp32 [B,H,ceil(N/bq)], [B,H,ceil(N/64)] twice."""
    h, u8 = _Heads(p), torch.uint8
    scales = lambda t, what, blk: _tensor(t, what, torch.float32, (p.B, p.H, -(-p.N // max(blk, 1))), h.dev)
    _check(lib().sla_qk_norm_rope_e4m3(C.byref(p), h.rows(q, "q"), h.rows(k, "k"), h.rows(v, "v"), h.weight(q_weight, "q_weight"), h.weight(q_bias, "q_bias"),
                                       h.weight(k_weight, "k_weight"), h.weight(k_bias, "k_bias"), h.positions(pos), bq,
                                       h.dense(Q8, "Q8", u8), h.dense(K8, "K8", u8), h.dense(V8, "V8", u8),
                                       scales(sQ, "sQ", bq), scales(sK, "sK", 64), scales(sV, "sV", 64), _raw_stream(h.dev)), "sla_qk_norm_rope_e4m3")
    return Q8, K8, V8, sQ, sK, sV


def sla_qk_norm_rope_grad_workspace_bytes(p) -> int:
    return _bytes("sla_qk_norm_rope_grad_workspace_bytes", C.byref(p))


def sla_qk_norm_rope_grad(p, q, k, dQ, dK, dV, dq, dk, dv, pos=None, q_weight=None, k_weight=None, dq_weight=None, dq_bias=None,
                          dk_weight=None, dk_bias=None, workspace=None):
    """dQ, dK, dV (bf16, p's layout) -> dq, dk, dv (bf16, the strides of q, k, v) and fp32 gradients of the norm's parameters."""
    h = _Heads(p)
    if workspace is None:
        workspace = _scratch(sla_qk_norm_rope_grad_workspace_bytes(p), q.device)
    _check(lib().sla_qk_norm_rope_grad(C.byref(p), h.rows(q, "q"), h.rows(k, "k"), h.weight(q_weight, "q_weight"), h.weight(k_weight, "k_weight"),
                                       h.positions(pos), h.dense(dQ, "dQ"), h.dense(dK, "dK"), h.dense(dV, "dV"),
                                       h.rows(dq, "dq"), h.rows(dk, "dk"), h.rows(dv, "dv"), h.weight(dq_weight, "dq_weight"), h.weight(dq_bias, "dq_bias"),
                                       h.weight(dk_weight, "dk_weight"), h.weight(dk_bias, "dk_bias"), *_buffer(workspace, "workspace", h.dev),
                                       _raw_stream(h.dev)), "sla_qk_norm_rope_grad")
    return dq, dk, dv


# ---- training of the FP8 layer from an 8-bit copy of its input
def sla_fp8_checkpoint_bytes(N, d_in) -> int:
    return _bytes("sla_fp8_checkpoint_bytes", N, d_in)


def sla_fp8_linear_grad_workspace_bytes(N, d_in, d_out) -> int:
    return _bytes("sla_fp8_linear_grad_workspace_bytes", N, d_in, d_out)


def sla_fp8_linear_save(x, W, bias, y, checkpoint, workspace=None):
    """The FP8 layer's training form: y, and x in 8 bits in `checkpoint` (uint8, sla_fp8_checkpoint_bytes(N, d_in) long)."""
    (N, d_in), d_out, bf, dev = x.shape, W.shape[0], torch.bfloat16, _device()
    if workspace is None:
        workspace = _scratch(sla_fp8_linear_grad_workspace_bytes(N, d_in, d_out), x.device)
    _check(lib().sla_fp8_linear_save(_tensor(x, "x", bf, (N, d_in), dev), _tensor(W, "W", bf, (d_out, d_in), dev), _tensor(bias, "bias", bf, (d_out,), dev),
                                     N, d_in, d_out, _tensor(y, "y", bf, (N, d_out), dev), *_buffer(checkpoint, "checkpoint", dev),
                                     *_buffer(workspace, "workspace", dev), _raw_stream(dev)), "sla_fp8_linear_save")
    return y


def sla_fp8_linear_grad(dy, checkpoint, W, dx=None, dW=None, db=None, workspace=None):
    """Gradients of sla_fp8_linear_save's x, W and bias (each may be None; db only with dW) from that of its y."""
    (N, d_out), d_in, bf, dev = dy.shape, W.shape[1], torch.bfloat16, _device()
    if workspace is None:
        workspace = _scratch(sla_fp8_linear_grad_workspace_bytes(N, d_in, d_out), dy.device)
    _check(lib().sla_fp8_linear_grad(_tensor(dy, "dy", bf, (N, d_out), dev), *_buffer(checkpoint, "checkpoint", dev), _tensor(W, "W", bf, (d_out, d_in), dev),
                                     N, d_in, d_out, _tensor(dx, "dx", bf, (N, d_in), dev), _tensor(dW, "dW", bf, (d_out, d_in), dev),
                                     _tensor(db, "db", bf, (d_out,), dev), *_buffer(workspace, "workspace", dev), _raw_stream(dev)), "sla_fp8_linear_grad")
    return dx, dW, db


def sla_fp8_checkpoint_restore(checkpoint, x):
    """x bf16 [N,d_in] <- the layer's input as its forward multiplied it."""
    (N, d_in), dev = x.shape, _device()
    _check(lib().sla_fp8_checkpoint_restore(*_buffer(checkpoint, "checkpoint", dev), N, d_in, _tensor(x, "x", torch.bfloat16, (N, d_in), dev),
                                            _raw_stream(dev)), "sla_fp8_checkpoint_restore")
    return x


# ---- microscaled 4-bit numbers
def sla_quantise_mxfp4(X, codes, scales):
    """X bf16 [rows, cols] -> codes uint8 [rows, cols/2], scales uint8 [rows, cols/32]."""
    (rows, cols), u8, dev = X.shape, torch.uint8, _device()
    _check(lib().sla_quantise_mxfp4(_tensor(X, "X", torch.bfloat16, (rows, cols), dev), rows, cols, _tensor(codes, "codes", u8, (rows, cols // 2), dev),
                                    _tensor(scales, "scales", u8, (rows, cols // 32), dev), _raw_stream(dev)), "sla_quantise_mxfp4")
    return codes, scales


def sla_dequantise_mxfp4(codes, scales, Y):
    """Y bf16 [rows, cols] <- the numbers that codes and scales stand for."""
    (rows, cols), u8, dev = Y.shape, torch.uint8, _device()
    _check(lib().sla_dequantise_mxfp4(_tensor(codes, "codes", u8, (rows, cols // 2), dev), _tensor(scales, "scales", u8, (rows, cols // 32), dev),
                                      rows, cols, _tensor(Y, "Y", torch.bfloat16, (rows, cols), dev), _raw_stream(dev)), "sla_dequantise_mxfp4")
    return Y


def sla_mxfp4_linear_workspace_bytes(N, d_in, d_out) -> int:
    return _bytes("sla_mxfp4_linear_workspace_bytes", N, d_in, d_out)


def sla_mxfp4_linear(x, W_codes, W_scales, bias, y, workspace=None):
    """y bf16 [N,d_out] <- linear layer of x bf16 [N,d_in], both factors in microscaled 4-bit numbers."""
    (N, d_in), d_out, bf, u8, dev = x.shape, W_codes.shape[0], torch.bfloat16, torch.uint8, _device()
    if workspace is None:
        workspace = _scratch(sla_mxfp4_linear_workspace_bytes(N, d_in, d_out), x.device)
    _check(lib().sla_mxfp4_linear(_tensor(x, "x", bf, (N, d_in), dev), _tensor(W_codes, "W_codes", u8, (d_out, d_in // 2), dev),
                                  _tensor(W_scales, "W_scales", u8, (d_out, d_in // 32), dev), _tensor(bias, "bias", bf, (d_out,), dev),
                                  N, d_in, d_out, _tensor(y, "y", bf, (N, d_out), dev), *_buffer(workspace, "workspace", dev), _raw_stream(dev)),
           "sla_mxfp4_linear")
    return y
