// Gradients of the FP8 fake-quantised linear layer y = x_fp8 W_fp8^T + b (Alg. 2 of the paper, straight through the
// quantisers) from the E4M3 codes that its forward multiplied:
//     dx = dy W_fp8          [N, d_in]         summed over the d_out channels
//     dW = dy^T x_fp8        [d_out, d_in]     summed over the N tokens
//     db = sum over tokens of dy
// x is kept for the backward pass as those codes and one fp32 scale per token: N (d_in + 4) bytes instead of 2 N d_in.
//
// Both products have one form: C[m][n] = sum_k A(m,k) B(k,n), with B the code matrix (rows k = channels of W or tokens of x, in the
// fragment order of k_linear.hip) times the scale of the row, rounded to bf16, and A = dy, read as it lies (dx) or transposed (dW).
// The scale belongs to the summation index, so it cannot wait for the epilogue.  Rounding code x scale to bf16 is off by at
// most 2^-8 of it, as the rounding of x to bf16 was in the first place; products are exact in the fp32 accumulators.
#include "sla_common.hpp"
#include "sla_kernels.hpp"

#include <type_traits>

namespace sla {

namespace {
constexpr int kStepK = 32;                           // summation indices of a step: one group of rows of the code matrix
typedef __attribute__((ext_vector_type(4))) short s16x4;

// Tiles that lie [k][column] in LDS: a row is 2 columns bytes, its 16-byte piece c at position c ^ swizzle(k).  Four
// consecutive k then put the same 64 bytes of columns into four different quarters of the banks (the transposing read takes 64 bytes of
// four rows at a time), and writes of one piece by consecutive k go to sixteen different places.
__device__ __forceinline__ int swizzle(int k) { return 4 * (k & 3) | ((k >> 2) & 3); }

// MFMA operand of 32 columns n0 .. n0 + 31 and the 16 indices of step t from a tile that lies [k][column]: lane l gets column
// l % 32, k = 16 t + 8 (l / 32) .. + 7.  Each ds_read_b64_tr_b16 turns, in every 16 lanes, 4 rows x 16 columns around.
template <int COLS> __device__ __forceinline__ bf16x8 read_turned(const uint8_t *tile, int n0, int t, int lane)
{
    const int i = lane & 15, g = lane >> 5, chunk = n0 / 8 + 2 * ((lane >> 4) & 1) + ((i & 3) >> 1);
    s16x4 r[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int k = 16 * t + 8 * g + 4 * j + (i >> 2);
        const uint8_t *const at = tile + k * (2 * COLS) + (chunk ^ (4 * (i >> 2) | ((2 * g + j) & 3))) * 16 + (i & 1) * 8;
        r[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)at);
    }
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(r[0], r[1], 0, 1, 2, 3, 4, 5, 6, 7));
}

// sixteen E4M3 codes times a scale, rounded to bf16
__device__ __forceinline__ void restore16(uint4 c, float s, uint4 (&out)[2])
{
    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
    uint32_t o[8];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[q], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[q], true);
        o[2 * q] = pack_bf16(lo[0] * s, lo[1] * s);
        o[2 * q + 1] = pack_bf16(hi[0] * s, hi[1] * s);
    }
    out[0] = make_uint4(o[0], o[1], o[2], o[3]);
    out[1] = make_uint4(o[4], o[5], o[6], o[7]);
}
}  // namespace

// TURN: A(m,k) = A[k][m] (dW), else A[m][k] (dx); A is bf16 with `lda` elements to a row.  Workgroup tile 64 TM x 64 TN, four waves as
// 2 x 2.  Split `s` of the summation covers k from s k_split on; with part != nullptr the tile goes there in fp32, [split][M][cols],
// and, from the first tile of columns, the sums of A over k to part_db [split][M].
template <int TM, int TN, bool TURN>
__global__ __launch_bounds__(256) void linear_grad_kernel(const uint16_t *__restrict__ A, int lda, const uint8_t *__restrict__ codes,
                                                          const float *__restrict__ scales, int M, int cols, int K, int k_split, int n_nt,
                                                          int tiles, int total, uint16_t *__restrict__ C, float *__restrict__ part,
                                                          float *__restrict__ part_db)
{
    constexpr int BM = 64 * TM, BN = 64 * TN, kA = BM * kStepK * 2, kB = BN * kStepK * 2, kStage = kA + kB;
    __shared__ __attribute__((aligned(1024))) uint8_t smem[2 * kStage];
    const int item = (int)xcd_remap(blockIdx.x, total);
    if (item >= total) return;
    const int split = item / tiles, tile = item - split * tiles, mt = tile / n_nt, nt = tile - mt * n_nt;
    const int m0 = mt * BM, n0 = nt * BN, k0 = split * k_split, k1 = min(K, k0 + k_split);
    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, g = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = (wave & 1) * 32 * TM, wn = (wave >> 1) * 32 * TN;

    constexpr int kPb = TN / 2;                      // pieces of B a thread brings in a step
    uint4 ra[TM], rb[kPb];
    float rs[kPb];
    auto load = [&](int k) {
#pragma unroll
        for (int x = 0; x < TM; ++x) {
            const int id = x * 256 + tid;
            ra[x] = make_uint4(0, 0, 0, 0);
            if constexpr (TURN) {
                const int kk = k + id / (BM / 8), m = m0 + id % (BM / 8) * 8;
                if (kk < k1 && m < M) ra[x] = *(const uint4 *)(A + (size_t)kk * lda + m);
            } else {
                const int m = m0 + id / 4, kk = k + id % 4 * 8;
                if (kk < k1 && m < M) ra[x] = *(const uint4 *)(A + (size_t)m * lda + kk);
            }
        }
        const int R = min(32, K - k);                // rows of the group of code rows that starts at k
#pragma unroll
        for (int x = 0; x < kPb; ++x) {
            const int slice = x * 2 + (tid >> 7), run = (tid >> 5) & 3, r = tid & 31;
            rb[x] = make_uint4(0, 0, 0, 0);
            rs[x] = 0.f;
            if (r < R && n0 + 64 * slice < cols) {
                rb[x] = *(const uint4 *)(codes + (size_t)k * cols + (size_t)(n0 / 64 + slice) * R * 64 + (run * R + r) * 16);
                rs[x] = scales[k + r];
            }
        }
    };
    auto store = [&](uint8_t *st) {
#pragma unroll
        for (int x = 0; x < TM; ++x) {
            const int id = x * 256 + tid;
            if constexpr (TURN) {
                const int kk = id / (BM / 8), c = id % (BM / 8);
                *(uint4 *)(st + kk * (2 * BM) + (c ^ swizzle(kk)) * 16) = ra[x];
            } else {
                const int m = id / 4, c = id % 4;
                *(uint4 *)(st + m * 64 + (c ^ ((m >> 2) & 3)) * 16) = ra[x];
            }
        }
#pragma unroll
        for (int x = 0; x < kPb; ++x) {
            const int slice = x * 2 + (tid >> 7), run = (tid >> 5) & 3, r = tid & 31;
            const int c = 8 * slice + 2 * (2 * (run & 1) + (run >> 1));        // run h * 2 + g holds the pieces of channels 32 g + 16 h
            uint4 v[2];
            restore16(rb[x], rs[x], v);
            uint8_t *const row = st + kA + r * (2 * BN);
            *(uint4 *)(row + (c ^ swizzle(r)) * 16) = v[0];
            *(uint4 *)(row + ((c + 1) ^ swizzle(r)) * 16) = v[1];
        }
    };

    f32x16 acc[TN][TM];
#pragma unroll
    for (int b = 0; b < TN; ++b)
#pragma unroll
        for (int a = 0; a < TM; ++a)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[b][a][e] = 0.f;
    float sums[TM];
#pragma unroll
    for (int a = 0; a < TM; ++a) sums[a] = 0.f;
    const bool summing = TURN && part_db && nt == 0 && wn == 0;

    const int steps = (k1 - k0 + kStepK - 1) / kStepK;
    load(k0);
    store(smem);
    __syncthreads();
    for (int s = 0; s < steps; ++s) {
        const uint8_t *const st = smem + (s & 1) * kStage;
        if (s + 1 < steps) load(k0 + (s + 1) * kStepK);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            bf16x8 af[TM], bf[TN];
#pragma unroll
            for (int a = 0; a < TM; ++a) {
                if constexpr (TURN) af[a] = read_turned<BM>(st, wm + 32 * a, t, lane);
                else {
                    const int m = wm + 32 * a + l32;
                    af[a] = *(const bf16x8 *)(st + m * 64 + ((2 * t + g) ^ ((m >> 2) & 3)) * 16);
                }
            }
#pragma unroll
            for (int b = 0; b < TN; ++b) bf[b] = read_turned<BN>(st + kA, wn + 32 * b, t, lane);
#pragma unroll
            for (int b = 0; b < TN; ++b)
#pragma unroll
                for (int a = 0; a < TM; ++a) acc[b][a] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bf[b], af[a], acc[b][a], 0, 0, 0);
            if (summing) {
#pragma unroll
                for (int a = 0; a < TM; ++a) {
                    const uint4 u = __builtin_bit_cast(uint4, af[a]);
                    sums[a] = dot2_bf16(u.x, 0x3F803F80u, dot2_bf16(u.y, 0x3F803F80u, dot2_bf16(u.z, 0x3F803F80u, dot2_bf16(u.w, 0x3F803F80u, sums[a]))));
                }
            }
        }
        if (s + 1 < steps) store(smem + ((s + 1) & 1) * kStage);
        __syncthreads();
    }

    // register 4q + r of acc[b][a], lane (l32, g): n = 32 b + 8 q + 4 g + r, m = 32 a + l32
#pragma unroll
    for (int a = 0; a < TM; ++a) {
        const int m = m0 + wm + 32 * a + l32;
        if (summing) {
            const float v = sums[a] + xchg32(sums[a]);
            if (g == 0 && m < M) part_db[(size_t)split * M + m] = v;
        }
#pragma unroll
        for (int b = 0; b < TN; ++b)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int n = n0 + wn + 32 * b + 8 * q + 4 * g;
                if (m >= M || n >= cols) continue;
                const float v[4] = {acc[b][a][4 * q], acc[b][a][4 * q + 1], acc[b][a][4 * q + 2], acc[b][a][4 * q + 3]};
                if (part) *(float4 *)(part + ((size_t)split * M + m) * cols + n) = make_float4(v[0], v[1], v[2], v[3]);
                else *(uint2 *)(C + (size_t)m * cols + n) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
            }
    }
}

// out[i] = bf16(sum of the splits' partials, in order); count values (a multiple of 8)
__global__ __launch_bounds__(256) void linear_grad_reduce_kernel(const float *__restrict__ part, int splits, long count, uint16_t *__restrict__ out)
{
    const long i = ((long)blockIdx.x * 256 + threadIdx.x) * 4;
    if (i >= count) return;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int s = 0; s < splits; ++s) {
        const float4 u = *(const float4 *)(part + s * count + i);
        v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;
    }
    *(uint2 *)(out + i) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
}

// bf16 rows [rows, cols] of codes in fragment order and their scales: sixteen channels a thread
__global__ __launch_bounds__(256) void restore_rows_kernel(const uint8_t *__restrict__ codes, const float *__restrict__ scales, long rows, int cols,
                                                           uint16_t *__restrict__ X)
{
    const long at = (long)blockIdx.x * 256 + threadIdx.x, pieces = cols / 16;      // a piece is sixteen codes; threads walk them as they lie
    if (at >= rows * pieces) return;
    const long grp = at / (32 * pieces);
    const int R = (int)min(32L, rows - 32 * grp), in = (int)(at - grp * 32 * pieces);
    const int slice = in / (4 * R), rest = in - slice * 4 * R, run = rest / R, r = rest - run * R;
    uint4 v[2];
    restore16(*(const uint4 *)(codes + at * 16), scales[32 * grp + r], v);
    uint16_t *const x = X + (32 * grp + r) * cols + 64 * slice + 16 * (2 * (run & 1) + (run >> 1));
    *(uint4 *)x = v[0];
    *(uint4 *)(x + 8) = v[1];
}

namespace {
constexpr int kGradTile = 128;                       // rows and columns of a workgroup's tile

template <bool TURN>
hipError_t launch_grad(const void *A, int lda, const void *codes, const float *scales, int M, int cols, int K, int splits, void *C, float *part,
                       float *part_db, hipStream_t st)
{
    const int n_mt = (M + kGradTile - 1) / kGradTile, n_nt = (cols + kGradTile - 1) / kGradTile;
    const long tiles = (long)n_mt * n_nt, total = tiles * splits;
    if (total > 0x7FFFFFF0L) return hipErrorInvalidValue;
    const int steps = (K + kStepK - 1) / kStepK, k_split = (steps + splits - 1) / splits * kStepK;
    linear_grad_kernel<2, 2, TURN><<<(unsigned)xcd_grid(total), 256, 0, st>>>((const uint16_t *)A, lda, (const uint8_t *)codes, scales, M, cols, K, k_split,
                                                                              n_nt, (int)tiles, (int)total, (uint16_t *)C, part, part_db);
    return hipGetLastError();
}
}  // namespace

// Splits of the sum over the tokens: enough workgroups for the chip where dW has few tiles, each with at least eight steps.
int linear_grad_splits(int N, int d_in, int d_out)
{
    const long tiles = (long)((d_out + kGradTile - 1) / kGradTile) * ((d_in + kGradTile - 1) / kGradTile);
    const int steps = (N + kStepK - 1) / kStepK;
    long s = 768 / tiles;
    s = s > steps / 8 ? steps / 8 : s;
    s = s < 1 ? 1 : s;
    return steps ? (int)((steps + (steps + s - 1) / s - 1) / ((steps + s - 1) / s)) : 0;     // no split without steps
}

hipError_t launch_linear_dx(const void *dy, const void *w8, const float *sw, int N, int d_in, int d_out, void *dx, hipStream_t st)
{
    return launch_grad<false>(dy, d_out, w8, sw, N, d_in, d_out, 1, dx, nullptr, nullptr, st);
}

hipError_t launch_linear_dw(const void *dy, const void *x8, const float *sx, int N, int d_in, int d_out, void *dW, void *db, float *part, hipStream_t st)
{
    const int splits = linear_grad_splits(N, d_in, d_out);
    const long count = (long)d_out * d_in;
    float *const part_db = part + (size_t)splits * count;
    if (splits) {
        const hipError_t e = launch_grad<true>(dy, d_out, x8, sx, d_out, d_in, N, splits, nullptr, part, db ? part_db : nullptr, st);
        if (e != hipSuccess) return e;
    }
    linear_grad_reduce_kernel<<<(unsigned)((count / 4 + 255) / 256), 256, 0, st>>>(part, splits, count, (uint16_t *)dW);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !db) return e;
    linear_grad_reduce_kernel<<<(unsigned)((d_out / 4 + 255) / 256), 256, 0, st>>>(part_db, splits, d_out, (uint16_t *)db);
    return hipGetLastError();
}

hipError_t launch_restore_rows(const void *codes, const float *scales, long rows, int cols, void *X, hipStream_t st)
{
    restore_rows_kernel<<<(unsigned)((rows * (cols / 16) + 255) / 256), 256, 0, st>>>((const uint8_t *)codes, scales, rows, cols, (uint16_t *)X);
    return hipGetLastError();
}

}  // namespace sla
