// C ABI of the microscaled 4-bit format (k_mxfp4.hip): parameter checks and launches.
#include "api_util.hpp"
#include "sla_kernels.hpp"

using sla::aligned;
using sla::align_up;
using sla::at;
using sla::fail;

namespace {

sla_status_t check_matrix(int64_t rows, int32_t cols)
{
    if (rows < 0 || cols <= 0) return fail(SLA_ERR_INVALID_ARG, "bad sizes (rows=%ld cols=%d)", (long)rows, cols);
    if (cols % 32 != 0) return fail(SLA_ERR_UNSUPPORTED, "cols = %d; blocks are 32 elements of a row: only multiples of 32 are implemented", cols);
    if (rows > (1L << 42) / cols) return fail(SLA_ERR_UNSUPPORTED, "matrix of 2^42 elements or more");
    return SLA_OK;
}

struct MxPlan { size_t off_scales, off_w, off_ws, total; };      // codes and scales of x, those of W where they are turned
sla_status_t make_mx_plan(int32_t N, int32_t d_in, int32_t d_out, MxPlan &mp)
{
    if (N < 0 || d_in <= 0 || d_out <= 0) return fail(SLA_ERR_INVALID_ARG, "bad sizes (N=%d d_in=%d d_out=%d)", N, d_in, d_out);
    if (d_in % 128 != 0) return fail(SLA_ERR_UNSUPPORTED, "d_in = %d; only multiples of 128 are implemented", d_in);
    if (d_out % 8 != 0) return fail(SLA_ERR_UNSUPPORTED, "d_out = %d; only multiples of 8 are implemented", d_out);
    if ((double)N * d_in >= 4.0e9 || (double)d_out * d_in >= 4.0e9 || (double)N * d_out >= 4.0e9) return fail(SLA_ERR_UNSUPPORTED, "matrix of 4e9 elements or more");
    if (d_in > 1 << 24) return fail(SLA_ERR_UNSUPPORTED, "d_in = %d; at most 2^24 are implemented", d_in);       // 256 rows of codes within 2 GB
    const bool turned = sla::mxfp4_turns_weights(N, d_out);
    mp.off_scales = align_up((size_t)N, 16) * d_in / 2;
    mp.off_w = mp.off_scales + align_up((size_t)N * d_in / 32, 256);
    mp.off_ws = mp.off_w + (turned ? align_up((size_t)d_out, 16) * d_in / 2 : 0);
    mp.total = sla::mxfp4_few(N, d_out, d_in) ? 0 : mp.off_ws + (turned ? align_up((size_t)d_out * d_in / 32, 256) : 0);
    return SLA_OK;
}

}  // namespace

extern "C" {

sla_status_t sla_quantise_mxfp4(const void *X, int64_t rows, int32_t cols, void *codes, void *scales, void *stream)
{
    const sla_status_t s = check_matrix(rows, cols);
    if (s != SLA_OK || rows == 0) return s;
    SLA_REQ_PTR(X); SLA_REQ_PTR(codes); SLA_REQ_PTR(scales);
    SLA_HIP(sla::launch_quantise_mxfp4(X, rows, cols, codes, scales, (hipStream_t)stream));
    return SLA_OK;
}

sla_status_t sla_dequantise_mxfp4(const void *codes, const void *scales, int64_t rows, int32_t cols, void *Y, void *stream)
{
    const sla_status_t s = check_matrix(rows, cols);
    if (s != SLA_OK || rows == 0) return s;
    SLA_REQ_PTR(codes); SLA_REQ_PTR(scales); SLA_REQ_PTR(Y);
    SLA_HIP(sla::launch_dequantise_mxfp4(codes, scales, rows, cols, Y, (hipStream_t)stream));
    return SLA_OK;
}

sla_status_t sla_mxfp4_linear_workspace_bytes(int32_t N, int32_t d_in, int32_t d_out, size_t *bytes)
{
    MxPlan mp;
    const sla_status_t s = make_mx_plan(N, d_in, d_out, mp);
    if (s != SLA_OK) return s;
    if (!bytes) return fail(SLA_ERR_INVALID_ARG, "bytes is NULL");
    *bytes = mp.total;
    return SLA_OK;
}

sla_status_t sla_mxfp4_linear(const void *x, const void *W_codes, const void *W_scales, const void *bias, int32_t N, int32_t d_in,
                              int32_t d_out, void *y, void *workspace, size_t workspace_bytes, void *stream)
{
    MxPlan mp;
    const sla_status_t s = make_mx_plan(N, d_in, d_out, mp);
    if (s != SLA_OK || N == 0) return s;
    SLA_REQ_PTR(x); SLA_REQ_PTR(W_codes); SLA_REQ_PTR(W_scales); SLA_REQ_PTR(y);
    SLA_OPT_PTR(bias);
    hipStream_t st = (hipStream_t)stream;
    if (sla::mxfp4_few(N, d_out, d_in)) {
        SLA_HIP(sla::launch_mxfp4_few(x, W_codes, W_scales, bias, N, d_out, d_in, y, st));
        return SLA_OK;
    }
    if (!workspace) return fail(SLA_ERR_WORKSPACE, "workspace is NULL (%zu bytes needed)", mp.total);
    if (!aligned(workspace, 256)) return fail(SLA_ERR_WORKSPACE, "workspace must be 256-byte aligned");
    if (workspace_bytes < mp.total) return fail(SLA_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", workspace_bytes, mp.total);
    const bool turned = sla::mxfp4_turns_weights(N, d_out);
    void *const codes = workspace, *const scales = at<void>(workspace, mp.off_scales);
    void *const W = turned ? at<void>(workspace, mp.off_w) : nullptr, *const Ws = at<void>(workspace, mp.off_ws);
    SLA_HIP(sla::launch_mxfp4_operands(x, N, d_in, codes, scales, W_codes, W_scales, d_out, W, Ws, st));
    SLA_HIP(sla::launch_mxfp4_gemm(codes, scales, turned ? W : W_codes, turned ? Ws : W_scales, turned, bias, N, d_out, d_in, y, st));
    return SLA_OK;
}

}  // extern "C"
