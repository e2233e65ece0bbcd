"""Refusals of the norm and rotation of heads: on the host, before any launch."""
import ctypes as C

import pytest
import torch

from paper_2605_11354_amd import binding as B

PTR, NULL = C.c_void_p(4096), C.c_void_p(0)


@pytest.fixture(scope="module")
def lib():
    return B.lib()


def params(**kw):
    p = B.make_heads_params(torch.empty((2, 5, 3, 3, 64), dtype=torch.bfloat16)[:, :, 0])
    for name, value in kw.items():
        setattr(p, name, value)
    return p


def forward(lib, p, q=PTR, k=PTR, v=PTR, qw=NULL, qb=NULL, kw=NULL, kb=NULL, pos=PTR, Q=PTR, K=PTR, V=PTR):
    return lib.sla_qk_norm_rope(C.byref(p), q, k, v, qw, qb, kw, kb, pos, Q, K, V, NULL)


def e4m3(lib, p, bq=64, v=PTR, V=PTR, sQ=PTR, sV=PTR):
    return lib.sla_qk_norm_rope_e4m3(C.byref(p), PTR, PTR, v, NULL, NULL, NULL, NULL, PTR, C.c_int32(bq), PTR, PTR, V, sQ, PTR, sV, NULL)


def grad(lib, p, dV=PTR, dv=PTR, dqw=PTR, ws=PTR, size=1 << 20, dq=PTR):
    return lib.sla_qk_norm_rope_grad(C.byref(p), PTR, PTR, NULL, NULL, PTR, PTR, PTR, dV, dq, PTR, dv, dqw, NULL, NULL, NULL, ws, C.c_size_t(size), NULL)


@pytest.mark.parametrize("kw,status", [
    (dict(D=32), B.SLA_ERR_UNSUPPORTED), (dict(B=-1), B.SLA_ERR_INVALID_ARG), (dict(B=70000), B.SLA_ERR_UNSUPPORTED),
    (dict(N=1 << 30, B=2), B.SLA_ERR_UNSUPPORTED), (dict(norm=3), B.SLA_ERR_INVALID_ARG), (dict(norm=-1), B.SLA_ERR_INVALID_ARG),
    (dict(norm_per_head=2), B.SLA_ERR_INVALID_ARG), (dict(axes=3), B.SLA_ERR_INVALID_ARG), (dict(axes=-1), B.SLA_ERR_INVALID_ARG),
    (dict(pairing=2), B.SLA_ERR_INVALID_ARG), (dict(pos_per_item=2), B.SLA_ERR_INVALID_ARG), (dict(layout=2), B.SLA_ERR_INVALID_ARG),
    (dict(eps=0.0), B.SLA_ERR_INVALID_ARG), (dict(eps=float("nan")), B.SLA_ERR_INVALID_ARG), (dict(eps=float("inf")), B.SLA_ERR_INVALID_ARG),
    (dict(base=0.5), B.SLA_ERR_INVALID_ARG), (dict(base=float("inf")), B.SLA_ERR_INVALID_ARG), (dict(base=float("nan")), B.SLA_ERR_INVALID_ARG),
    (dict(token_stride=2 * 64), B.SLA_ERR_INVALID_ARG),         # rows of neighbouring tokens overlap
    (dict(token_stride=-576), B.SLA_ERR_INVALID_ARG), (dict(token_stride=0), B.SLA_ERR_INVALID_ARG),
    (dict(token_stride=1 << 60), B.SLA_ERR_INVALID_ARG),
    (dict(head_stride=60), B.SLA_ERR_INVALID_ARG), (dict(head_stride=68), B.SLA_ERR_INVALID_ARG),
    (dict(H=70000, B=0), B.SLA_ERR_UNSUPPORTED), (dict(H=1 << 30, N=0, B=0, norm_per_head=1), B.SLA_ERR_UNSUPPORTED),
    (dict(batch_stride=576), B.SLA_ERR_INVALID_ARG), (dict(batch_stride=640), B.SLA_ERR_INVALID_ARG), (dict(batch_stride=128), B.SLA_ERR_INVALID_ARG), (dict(batch_stride=0), B.SLA_ERR_INVALID_ARG),
])
def test_parameters(lib, kw, status):
    p = params(**kw)
    assert forward(lib, p) == status and len(lib.sla_last_error()) > 0
    assert e4m3(lib, p) == status and grad(lib, p) == status
    n = C.c_size_t()
    assert lib.sla_qk_norm_rope_grad_workspace_bytes(C.byref(p), C.byref(n)) == status


def test_pointers(lib):
    p, odd = params(), C.c_void_p(4104)
    for name in ("q", "k", "Q", "K"):
        assert forward(lib, p, **{name: NULL}) == B.SLA_ERR_INVALID_ARG
        assert forward(lib, p, **{name: odd}) == B.SLA_ERR_INVALID_ARG and b"aligned" in lib.sla_last_error()
    for name in ("v", "V", "qw", "qb", "kw", "kb"):
        assert forward(lib, p, **{name: odd}) == B.SLA_ERR_INVALID_ARG
    assert forward(lib, p, v=NULL) == B.SLA_ERR_INVALID_ARG and forward(lib, p, V=NULL) == B.SLA_ERR_INVALID_ARG
    assert forward(lib, p, pos=NULL) == B.SLA_ERR_INVALID_ARG and forward(lib, p, pos=C.c_void_p(4097)) == B.SLA_ERR_INVALID_ARG
    assert forward(lib, params(norm=0), qw=PTR) == B.SLA_ERR_INVALID_ARG and forward(lib, params(norm=0), kb=PTR) == B.SLA_ERR_INVALID_ARG
    assert e4m3(lib, p, bq=96) == B.SLA_ERR_UNSUPPORTED and e4m3(lib, p, sQ=NULL) == B.SLA_ERR_INVALID_ARG
    assert e4m3(lib, p, sV=NULL) == B.SLA_ERR_INVALID_ARG and e4m3(lib, p, v=NULL) == B.SLA_ERR_INVALID_ARG
    assert grad(lib, p, dV=NULL) == B.SLA_ERR_INVALID_ARG and grad(lib, p, dv=NULL) == B.SLA_ERR_INVALID_ARG
    assert grad(lib, p, dq=NULL) == B.SLA_ERR_INVALID_ARG and grad(lib, p, dqw=odd) == B.SLA_ERR_INVALID_ARG
    assert grad(lib, params(norm=0)) == B.SLA_ERR_INVALID_ARG
    assert grad(lib, p, ws=NULL) == B.SLA_ERR_WORKSPACE and grad(lib, p, ws=C.c_void_p(4112)) == B.SLA_ERR_WORKSPACE
    assert grad(lib, p, size=B.sla_qk_norm_rope_grad_workspace_bytes(p) - 1) == B.SLA_ERR_WORKSPACE
    assert lib.sla_qk_norm_rope(None, *[PTR] * 11, NULL) == B.SLA_ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [dict(B=0), dict(H=0), dict(N=0)])
def test_nothing_to_do(lib, kw):
    p = params(**kw)
    assert lib.sla_qk_norm_rope(C.byref(p), *[NULL] * 12) == B.SLA_OK
    assert lib.sla_qk_norm_rope_e4m3(C.byref(p), *[NULL] * 8, C.c_int32(64), *[NULL] * 7) == B.SLA_OK
    assert lib.sla_qk_norm_rope_grad(C.byref(p), *[NULL] * 16, C.c_size_t(0), NULL) == B.SLA_OK
    assert B.sla_qk_norm_rope_grad_workspace_bytes(p) == 0


def test_orders_of_dimensions_and_strides_of_single_elements_do_not_matter(lib):
    n = C.c_size_t()
    for kw in (dict(token_stride=1152, batch_stride=576), dict(token_stride=64, head_stride=320, batch_stride=960),       # other orders of the dimensions
               dict(B=1, batch_stride=-7), dict(N=1, token_stride=0), dict(H=1, head_stride=3)):
        assert lib.sla_qk_norm_rope_grad_workspace_bytes(C.byref(params(**kw)), C.byref(n)) == B.SLA_OK


def test_tensors_of_another_shape_or_type():
    p = params()
    q = torch.empty((2, 5, 3, 3, 64), dtype=torch.bfloat16)[:, :, 0]
    out = [torch.empty((2, 3, 5, 64), dtype=torch.bfloat16) for _ in range(3)]
    with pytest.raises(ValueError, match="current device"):                                  # tensors of the host
        B.sla_qk_norm_rope(p, q, q, q, *out, pos=None)
    with pytest.raises(ValueError, match="strides"):
        B.sla_qk_norm_rope(p, q.contiguous(), q, q, *out)
