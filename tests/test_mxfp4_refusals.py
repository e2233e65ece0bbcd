"""Refusals of the microscaled 4-bit calls: on the host, before any launch."""
import ctypes as C

import pytest
import torch

from paper_2605_11354_amd import binding as B

PTR, NULL, ODD = C.c_void_p(4096), C.c_void_p(0), C.c_void_p(4104)


@pytest.fixture(scope="module")
def lib():
    return B.lib()


def linear(lib, N=40, d_in=128, d_out=8, x=PTR, W=PTR, Ws=PTR, b=NULL, y=PTR, ws=PTR, size=1 << 40):
    return lib.sla_mxfp4_linear(x, W, Ws, b, C.c_int32(N), C.c_int32(d_in), C.c_int32(d_out), y, ws, C.c_size_t(size), NULL)


@pytest.mark.parametrize("sizes,status", [((40, 64, 8), B.SLA_ERR_UNSUPPORTED), ((40, 128, 4), B.SLA_ERR_UNSUPPORTED), ((-1, 128, 8), B.SLA_ERR_INVALID_ARG),
                                          ((40, 0, 8), B.SLA_ERR_INVALID_ARG), ((40, 128, -8), B.SLA_ERR_INVALID_ARG),
                                          ((1 << 30, 128, 8), B.SLA_ERR_UNSUPPORTED), ((1 << 20, 128, 4096), B.SLA_ERR_UNSUPPORTED)])
def test_sizes(lib, sizes, status):
    n = C.c_size_t()
    assert linear(lib, *sizes) == status and lib.sla_mxfp4_linear_workspace_bytes(*map(C.c_int32, sizes), C.byref(n)) == status


@pytest.mark.parametrize("N", [1, 40])
def test_pointers_and_workspace(lib, N):
    for name in ("x", "W", "Ws", "y"):
        assert linear(lib, N, **{name: NULL}) == B.SLA_ERR_INVALID_ARG and linear(lib, N, **{name: ODD}) == B.SLA_ERR_INVALID_ARG
    assert linear(lib, N, b=ODD) == B.SLA_ERR_INVALID_ARG


def test_workspace(lib):
    need = B.sla_mxfp4_linear_workspace_bytes(40, 128, 8)
    assert need >= 40 * 128 * 17 // 32 and B.sla_mxfp4_linear_workspace_bytes(1, 4096, 4096) == 0
    for bad in (dict(ws=NULL), dict(ws=C.c_void_p(4112)), dict(size=need - 1)):
        assert linear(lib, **bad) == B.SLA_ERR_WORKSPACE
    assert lib.sla_mxfp4_linear_workspace_bytes(C.c_int32(40), C.c_int32(128), C.c_int32(8), None) == B.SLA_ERR_INVALID_ARG


def test_matrices(lib):
    for call in (lib.sla_quantise_mxfp4, lib.sla_dequantise_mxfp4):
        def run(rows, cols, a=PTR, b=PTR, c=PTR):
            ptrs = (a, C.c_int64(rows), C.c_int32(cols), b, c) if call is lib.sla_quantise_mxfp4 else (a, b, C.c_int64(rows), C.c_int32(cols), c)
            return call(*ptrs, NULL)
        assert run(-1, 32) == B.SLA_ERR_INVALID_ARG and run(4, 0) == B.SLA_ERR_INVALID_ARG and run(4, 48) == B.SLA_ERR_UNSUPPORTED
        assert run(1 << 40, 32) == B.SLA_ERR_UNSUPPORTED and run(0, 32, NULL, NULL, NULL) == B.SLA_OK
        for k in range(3):
            for bad in (NULL, ODD):
                ptrs = [PTR, PTR, PTR]
                ptrs[k] = bad
                assert run(4, 32, *ptrs) == B.SLA_ERR_INVALID_ARG


def test_nothing_to_do(lib):
    assert linear(lib, 0, x=NULL, W=NULL, Ws=NULL, y=NULL, ws=NULL, size=0) == B.SLA_OK


def test_tensors_of_another_shape_type_or_place():
    bf, u8 = torch.bfloat16, torch.uint8
    x, c, s = torch.empty((4, 128), dtype=bf), torch.empty((8, 64), dtype=u8), torch.empty((8, 4), dtype=u8)
    with pytest.raises(ValueError, match="current device"):
        B.sla_quantise_mxfp4(x, c[:4], s[:4])
    with pytest.raises(ValueError, match="x: "):
        B.sla_mxfp4_linear(x.float(), c, s, None, torch.empty((4, 8), dtype=bf))
