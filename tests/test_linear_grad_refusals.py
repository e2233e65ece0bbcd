"""Refusals of the FP8 layer's training calls: on the host, before any launch."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2605_11354_amd import binding as B

PTR, NULL = C.c_void_p(4096), C.c_void_p(0)
BIG = C.c_size_t(1 << 40)


@pytest.fixture(scope="module")
def lib():
    return B.lib()


def save(lib, N=5, d_in=128, d_out=8, x=PTR, W=PTR, b=NULL, y=PTR, ck=PTR, ck_size=BIG, ws=PTR, ws_size=BIG):
    return lib.sla_fp8_linear_save(x, W, b, C.c_int32(N), C.c_int32(d_in), C.c_int32(d_out), y, ck, ck_size, ws, ws_size, NULL)


def grad(lib, N=5, d_in=128, d_out=8, dy=PTR, W=PTR, dx=PTR, dW=PTR, db=PTR, ck=PTR, ck_size=BIG, ws=PTR, ws_size=BIG):
    return lib.sla_fp8_linear_grad(dy, ck, ck_size, W, C.c_int32(N), C.c_int32(d_in), C.c_int32(d_out), dx, dW, db, ws, ws_size, NULL)


@pytest.mark.parametrize("sizes,status", [((5, 64, 8), B.SLA_ERR_UNSUPPORTED), ((5, 128, 12), B.SLA_ERR_UNSUPPORTED), ((-1, 128, 8), B.SLA_ERR_INVALID_ARG),
                                          ((5, 0, 8), B.SLA_ERR_INVALID_ARG), ((5, 128, 0), B.SLA_ERR_INVALID_ARG),
                                          ((1 << 30, 128, 8), B.SLA_ERR_UNSUPPORTED), ((1 << 20, 128, 4096), B.SLA_ERR_UNSUPPORTED)])
def test_sizes(lib, sizes, status):
    n = C.c_size_t()
    assert save(lib, *sizes) == status and grad(lib, *sizes) == status
    assert lib.sla_fp8_linear_grad_workspace_bytes(*map(C.c_int32, sizes), C.byref(n)) == status


def test_pointers_and_buffers(lib):
    odd = C.c_void_p(4104)
    for name in ("x", "W", "y"):
        assert save(lib, **{name: NULL}) == B.SLA_ERR_INVALID_ARG and save(lib, **{name: odd}) == B.SLA_ERR_INVALID_ARG
    assert save(lib, b=odd) == B.SLA_ERR_INVALID_ARG
    for name in ("dy", "W"):
        assert grad(lib, **{name: NULL}) == B.SLA_ERR_INVALID_ARG and grad(lib, **{name: odd}) == B.SLA_ERR_INVALID_ARG
    for name in ("dx", "dW", "db"):
        assert grad(lib, **{name: odd}) == B.SLA_ERR_INVALID_ARG
    assert grad(lib, dW=NULL) == B.SLA_ERR_UNSUPPORTED
    small = B.sla_fp8_checkpoint_bytes(5, 128) - 1, B.sla_fp8_linear_grad_workspace_bytes(5, 128, 8) - 1
    for call in (save, grad):
        for bad in (dict(ck=NULL), dict(ck=C.c_void_p(4112)), dict(ck_size=C.c_size_t(small[0])), dict(ws=NULL), dict(ws=C.c_void_p(4112)), dict(ws_size=C.c_size_t(small[1]))):
            assert call(lib, **bad) == B.SLA_ERR_WORKSPACE, bad
    n = C.c_int32(5)
    assert lib.sla_fp8_checkpoint_restore(PTR, C.c_size_t(small[0]), n, C.c_int32(128), PTR, NULL) == B.SLA_ERR_WORKSPACE
    assert lib.sla_fp8_checkpoint_restore(PTR, BIG, n, C.c_int32(128), NULL, NULL) == B.SLA_ERR_INVALID_ARG
    assert lib.sla_fp8_checkpoint_bytes(n, C.c_int32(128), None) == B.SLA_ERR_INVALID_ARG


def test_nothing_to_do(lib):
    assert save(lib, N=0, x=NULL, W=NULL, y=NULL, ck=NULL, ws=NULL) == B.SLA_OK
    assert grad(lib, dx=NULL, dW=NULL, db=NULL, dy=NULL, W=NULL, ck=NULL, ws=NULL) == B.SLA_OK
    assert grad(lib, N=0, dW=NULL, db=NULL, dy=NULL, W=NULL, ck=NULL, ws=NULL) == B.SLA_OK
    assert lib.sla_fp8_checkpoint_restore(NULL, C.c_size_t(0), C.c_int32(0), C.c_int32(128), NULL, NULL) == B.SLA_OK


def test_the_checkpoint_is_half_of_the_input():
    for N, d in ((1, 128), (197, 384), (43968, 1024)):
        assert N * (d + 4) <= B.sla_fp8_checkpoint_bytes(N, d) < N * (d + 4) + 512


def test_tensors_of_another_shape_type_or_place():
    bf = torch.bfloat16
    x, W, y, ck = torch.empty((5, 128), dtype=bf), torch.empty((8, 128), dtype=bf), torch.empty((5, 8), dtype=bf), torch.empty(4096, dtype=torch.uint8)
    with pytest.raises(ValueError, match="x: a contiguous tensor on the current device"):
        B.sla_fp8_linear_save(x, W, None, y, ck)
    with pytest.raises(ValueError, match="x: "):
        B.sla_fp8_linear_save(x.float(), W, None, y, ck)


def test_the_training_scale_is_no_significand_of_ones():
    """The division step needs that of its divisor: all 128 significands of a bf16 maximum (the scale's exponent plays no part), and 1e-8."""
    for top in list(np.arange(128, 256, dtype=np.float32)) + [np.float32(1e-8)]:
        scale = np.float32(top * (np.float32(1) / np.float32(448)))
        assert scale.view(np.uint32) & 0x7FFFFF != 0x7FFFFF
