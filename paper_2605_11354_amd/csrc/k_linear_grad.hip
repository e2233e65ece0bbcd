// Gradients of the FP8 fake-quantised linear layer y = x_fp8 W_fp8^T + b (Alg. 2 of the paper, straight through the
// quantisers) from the E4M3 codes that its forward multiplied:
//     dx = dy W_fp8          [N, d_in]         summed over the d_out channels
//     dW = dy^T x_fp8        [d_out, d_in]     summed over the N tokens
//     db = sum over tokens of dy
// x is kept for the backward pass as those codes and one fp32 scale per token: N (d_in + 4) bytes instead of 2 N d_in.
//
// Both products have one form: C[m][n] = sum_k A(m,k) B(k,n), with B the code matrix (rows k = channels of W or tokens of x) times the
// scale of the row, rounded to bf16, and A = dy, read as it lies (dx) or transposed (dW).  The scale belongs to the summation
// index, so it cannot wait for the epilogue.  Rounding code x scale to bf16 is off by at most 2^-8 of it, as the rounding of x to bf16
// was in the first place; products are exact in the fp32 accumulators.
//
// B is restored once, by restore_turned_kernel, into the order in which the matrix unit's operands are read: column groups of 32, of
// a group 16 k after 16 k, 1 KB each, lane l's 16 bytes (column l % 32, k = 8 (l / 32) ..) one after the other; k past the end are
// zeros up to a multiple of 32.  (Converted on the way to LDS instead, every tile of rows converts it again: four vector instructions
// for each matrix instruction, 540 us instead of 30 for the restoring and what the products then take.)
#include "sla_common.hpp"
#include "sla_kernels.hpp"

#include <type_traits>

namespace sla {

namespace {
constexpr int kStepK = 32;                           // summation indices of a step
typedef __attribute__((ext_vector_type(4))) short s16x4;

// Tiles that lie [k][column] in LDS: a row is 2 columns bytes, its 16-byte piece c at position c ^ swizzle(k).  Four
// consecutive k then put the same 64 bytes of columns into four different quarters of the banks (the transposing read takes 64 bytes of
// four rows at a time), and writes of one piece by consecutive k go to sixteen different places.
__device__ __forceinline__ int swizzle(int k) { return 4 * (k & 3) | ((k >> 2) & 3); }

// MFMA operand of 32 columns n0 .. n0 + 31 and the 16 indices of part t from a tile that lies [k][column]: lane l gets column
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
__device__ __forceinline__ void restore16(i32x4 c, float s, i32x4 (&out)[2])
{
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(c[q], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(c[q], true);
        out[q >> 1][2 * (q & 1)] = (int)pack_bf16(lo[0] * s, lo[1] * s);
        out[q >> 1][2 * (q & 1) + 1] = (int)pack_bf16(hi[0] * s, hi[1] * s);
    }
}
}  // namespace

// rows x cols codes (fragment order of k_linear.hip) and the scales of the rows -> B as described above.  A wave takes 32 rows and
// 128 columns; the turn is ds_read_b64_tr_b16's.
__global__ __launch_bounds__(256) void restore_turned_kernel(const uint8_t *__restrict__ codes, const float *__restrict__ scales, int rows, int cols, uint8_t *__restrict__ B)
{
    __shared__ __attribute__((aligned(1024))) uint8_t smem[4 * 8192];
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63;
    const int spans = cols / 128, groups = (rows + 31) / 32;
    const long at = (long)blockIdx.x * 4 + wave;
    if (at >= (long)groups * spans) return;          // the whole wave leaves; nothing below synchronises across waves
    const int grp = (int)(at / spans), span = (int)(at - (long)grp * spans), R = min(32, rows - 32 * grp), r = lane & 31;
    uint8_t *const tile = smem + wave * 8192;
    const uint8_t *const from = codes + (size_t)grp * 32 * cols + (size_t)span * 128 * R;
    const float scale = r < R ? scales[32 * grp + r] : 0.f;
    i32x4 c[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) {                    // piece (slice, run): 16 columns of row r
        const int slice = x >> 1, run = (x & 1) * 2 + (lane >> 5);
        c[x] = r < R ? *(const i32x4 *)(from + slice * R * 64 + (run * R + r) * 16) : i32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        const int run = (x & 1) * 2 + (lane >> 5), col = 8 * (x >> 1) + 2 * (2 * (run & 1) + (run >> 1));      // run h * 2 + g holds the pieces of channels 32 g + 16 h
        i32x4 v[2];
        restore16(c[x], scale, v);
        *(i32x4 *)(tile + r * 256 + (col ^ swizzle(r)) * 16) = v[0];
        *(i32x4 *)(tile + r * 256 + ((col + 1) ^ swizzle(r)) * 16) = v[1];
    }
    wave_lds_sync();
#pragma unroll
    for (int x = 0; x < 4; ++x)                      // column groups; two slices of 16 k, 2 KB in a row
#pragma unroll
        for (int t = 0; t < 2; ++t)
            *(bf16x8 *)(B + (((size_t)(span * 4 + x) * groups + grp) * 2 + t) * 1024 + lane * 16) = read_turned<128>(tile, 32 * x, t, lane);
}

// TURN: A(m,k) = A[k][m] (dW), else A[m][k] (dx); A is bf16 with `lda` elements to a row.  Workgroup tile 64 TM x 64 TN, four waves as
// 2 x 2.  Split `s` of the summation covers k from s k_split on; with part != nullptr the tile goes there in fp32, [split][M][cols],
// and, from the first tile of columns, the sums of A over k to part_db [split][M].
//
// Steps of 32 k, four stages in LDS, filled by copies three steps ahead.  A step has two parts of 16 k; the operands of a
// part are read while the products of the one before run (two sets of registers).  The one barrier of a step stands before the products of its
// second part, whose operands are in registers by then: everybody has read the stage, the next one is whole (its copies were asked for three
// steps ago), and its first operands are read under those products.
// With TM = TN = 4 a wave holds 256 accumulators and a CU one workgroup: a part takes 8 operands per 16 matrix instructions from
// LDS, half of what its bandwidth allows (128 x 64 per wave: three quarters, with the writes all of it).
template <int TM, int TN, bool TURN>
__global__ __launch_bounds__(256, TM == 4 ? 1 : 2) void linear_grad_kernel(const uint16_t *__restrict__ A, int lda, const uint8_t *__restrict__ B, int M, int cols,
                                                          int K, int k_split, int n_nt, int tiles, int total, uint16_t *__restrict__ C,
                                                          float *__restrict__ part, float *__restrict__ part_db)
{
    constexpr int BM = 64 * TM, BN = 64 * TN, kA = BM * kStepK * 2, kB = BN * kStepK * 2, kStage = kA + kB, kStages = 4;
    constexpr int kCopies = kStage / 4096, kCopiesA = kA / 4096;               // copies of 1 KB a wave makes in a step
    __shared__ __attribute__((aligned(1024))) uint8_t smem[kStages * kStage];
    const int item = (int)xcd_remap(blockIdx.x, total);
    if (item >= total) return;
    const int split = item / tiles, tile = item - split * tiles, mt = tile / n_nt, nt = tile - mt * n_nt;
    const int m0 = mt * BM, n0 = nt * BN, k0 = split * k_split, k1 = min(K, k0 + k_split);
    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, g = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = (wave & 1) * 32 * TM, wn = (wave >> 1) * 32 * TN;
    const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)smem;

    // ---- copies: copy x of wave w brings bytes 1024 (w kCopiesA + x) .. of the stage's A, or of its B.  Rows and pieces past the end
    // repeat the last ones: results of rows past M and columns past `cols` are not stored, and what of A lies past K is cleared (clear_tail).
    uint32_t va[kCopiesA];
    auto place = [&](int left) {                     // left: summation indices that are there, from the step's first on
#pragma unroll
        for (int x = 0; x < kCopiesA; ++x) {
            const int at = (wave * kCopiesA + x) * 1024 + lane * 16;
            if constexpr (TURN) {
                const int k = at / (2 * BM), c = (at % (2 * BM) / 16) ^ swizzle(k);
                va[x] = (uint32_t)min(k, left - 1) * (uint32_t)lda * 2u + (uint32_t)min(m0 + 8 * c, M - 8) * 2u;
            } else {
                const int m = at / 64, c = (at / 16 % 4) ^ (m >> 2 & 3);
                va[x] = (uint32_t)min(m, M - 1 - m0) * (uint32_t)lda * 2u + (uint32_t)min(c, left / 8 - 1) * 16u;
            }
        }
    };
    const int groups = (K + 31) / 32;
    const uint8_t *pb[kCopies - kCopiesA];           // two copies are a column group's step
#pragma unroll
    for (int x = 0; x < kCopies - kCopiesA; ++x) {
        const int id = wave * (kCopies - kCopiesA) + x;
        pb[x] = B + ((size_t)min(n0 / 32 + (id >> 1), cols / 32 - 1) * groups * 2 + (id & 1)) * 1024;
    }
    const uint8_t *base;                             // of the step that is copied next
    uint32_t to;
    auto aim = [&](int k, int stage) {
        if (K - k < kStepK) place(K - k);            // the last step of all
        base = (const uint8_t *)A + (TURN ? (size_t)k * lda * 2 : (size_t)m0 * lda * 2 + (size_t)k * 2);
        to = lds_base + stage * kStage;
    };
    auto copy_one = [&](int k, int x) {
        if (x < kCopiesA) copy_1k_to_lds(base, va[x], to + (wave * kCopiesA + x) * 1024);
        else copy_1k_to_lds(pb[x - kCopiesA] + (size_t)k * 64, lane * 16, to + kA + (wave * (kCopies - kCopiesA) + x - kCopiesA) * 1024);
    };
    auto clear_tail = [&](int left, int stage) {     // whole pieces (dx: K is a multiple of 8) or rows (dW)
        for (int at = tid * 16; at < kA; at += 4096) {
            const int k = TURN ? at / (2 * BM) : 8 * ((at / 16 % 4) ^ (at / 256 & 3));
            if (k >= left) *(i32x4 *)(smem + stage * kStage + at) = i32x4{0, 0, 0, 0};
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
    const int steps = (k1 - k0 + kStepK - 1) / kStepK;                           // at least one

    bf16x8 af[2][TM], bf[2][TN];
    auto read_one = [&](int set, int stage, int t, int x) {                      // operand x: TN of B, then TM of A
        const uint8_t *const st = smem + stage * kStage;
        if (x < TN) bf[set][x] = *(const bf16x8 *)(st + kA + ((wn / 32 + x) * 2 + t) * 1024 + lane * 16);
        else if constexpr (TURN) af[set][x - TN] = read_turned<BM>(st, wm + 32 * (x - TN), t, lane);
        else {
            const int m = wm + 32 * (x - TN) + l32;
            af[set][x - TN] = *(const bf16x8 *)(st + m * 64 + ((2 * t + g) ^ (m >> 2 & 3)) * 16);
        }
    };
    // the products of a part; what `between` does goes behind each of them, since a wave is alone on its SIMD: everything that is not
    // issued in the 28 cycles that a matrix instruction goes on by itself leaves the matrix unit idle
    auto multiply = [&](int set, auto between) {
#pragma unroll
        for (int i = 0; i < TM * TN; ++i) {
            const int b = i / TM, a = i % TM;
            acc[b][a] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bf[set][b], af[set][a], acc[b][a], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
            between(i);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (summing) {
#pragma unroll
            for (int a = 0; a < TM; ++a) {
                const uint4 u = __builtin_bit_cast(uint4, af[set][a]);
                sums[a] = dot2_bf16(u.x, 0x3F803F80u, dot2_bf16(u.y, 0x3F803F80u, dot2_bf16(u.z, 0x3F803F80u, dot2_bf16(u.w, 0x3F803F80u, sums[a]))));
            }
        }
    };
    // the next stage is whole and everybody is done with the one before it; AHEAD: later steps whose copies may still be under way
    auto change = [&](auto ahead) {
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(decltype(ahead)::value * kCopies) : "memory");
        lds_barrier();
    };
    auto change_to_last = [&](int stage) {           // and what of it lies past K is cleared
        const int left = K - (k0 + (steps - 1) * kStepK);
        if (left < kStepK) {
            clear_tail(left, stage);
            lds_barrier();
        }
    };
    constexpr int kOperands = TM + TN, kEvery = TM * TN / kCopies > 0 ? TM * TN / kCopies : 1;
    auto step = [&](int s, auto copies, auto ahead, auto last) {
        constexpr bool kCopy = decltype(copies)::value, kLast = decltype(last)::value;
        const int k3 = k0 + (s + 3) * kStepK;
        if constexpr (kCopy) aim(k3, (s + 3) & 3);
        multiply(0, [&](int i) {
            if (i < kOperands) read_one(1, s & 3, 1, i);
            if constexpr (kCopy)
                if (i % kEvery == 0 && i / kEvery < kCopies) copy_one(k3, i / kEvery);
        });
        if constexpr (!kLast) {
            change(ahead);
            if constexpr (decltype(ahead)::value == 0) change_to_last((s + 1) & 3);
        }
        multiply(1, [&](int i) {
            if constexpr (!kLast)
                if (i < kOperands) read_one(0, (s + 1) & 3, 0, i);
        });
    };
    static_assert(kOperands <= TM * TN && kCopies * kEvery <= TM * TN, "a part has room for its reads and copies");
    using Ahead0 = std::integral_constant<int, 0>;
    using Ahead1 = std::integral_constant<int, 1>;
    using Ahead2 = std::integral_constant<int, 2>;
    using Yes = std::true_type;
    using No = std::false_type;

    place(kStepK);
    for (int s = 0; s < min(steps, 3); ++s) {
        aim(k0 + s * kStepK, s);
#pragma unroll
        for (int x = 0; x < kCopies; ++x) copy_one(k0 + s * kStepK, x);
    }
    if (steps > 2) change(Ahead2{});
    else if (steps == 2) change(Ahead1{});
    else change(Ahead0{});
    if (steps == 1) change_to_last(0);
#pragma unroll
    for (int x = 0; x < kOperands; ++x) read_one(0, 0, 0, x);
    int s = 0;
    for (; s + 3 < steps; ++s) step(s, Yes{}, Ahead2{}, No{});
    if (s + 2 < steps) step(s++, No{}, Ahead1{}, No{});
    if (s + 1 < steps) step(s++, No{}, Ahead0{}, No{});
    step(s, No{}, Ahead0{}, Yes{});

    // register 4q + r of acc[b][a], lane (l32, g): n = 32 b + 8 q + 4 g + r, m = 32 a + l32
    auto swap32 = [](uint32_t &lo, uint32_t &hi) {                               // upper lanes of lo <-> lower lanes of hi
        const auto r = __builtin_amdgcn_permlane32_swap(lo, hi, false, false);
        lo = r[0];
        hi = r[1];
    };
#pragma unroll
    for (int a = 0; a < TM; ++a) {
        const int m = m0 + wm + 32 * a + l32;
        if (summing) {
            const float v = sums[a] + xchg32(sums[a]);
            if (g == 0 && m < M) part_db[(size_t)split * M + m] = v;
        }
#pragma unroll
        for (int b = 0; b < TN; ++b) {
            const f32x16 &v = acc[b][a];
            if (part) {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int n = n0 + wn + 32 * b + 8 * q + 4 * g;
                    if (m < M && n < cols) *(float4 *)(part + ((size_t)split * M + m) * cols + n) = make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
                }
            } else {
#pragma unroll
                for (int q = 0; q < 4; q += 2) {
                    uint32_t x0 = pack_bf16(v[4 * q], v[4 * q + 1]), y0 = pack_bf16(v[4 * q + 2], v[4 * q + 3]);
                    uint32_t x1 = pack_bf16(v[4 * q + 4], v[4 * q + 5]), y1 = pack_bf16(v[4 * q + 6], v[4 * q + 7]);
                    swap32(x0, x1);
                    swap32(y0, y1);
                    const int n = n0 + wn + 32 * b + 8 * q + 8 * g;
                    if (m < M && n < cols) *(uint4 *)(C + (size_t)m * cols + n) = make_uint4(x0, y0, x1, y1);
                }
            }
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
    i32x4 v[2];
    restore16(*(const i32x4 *)(codes + at * 16), scales[32 * grp + r], v);
    uint16_t *const x = X + (32 * grp + r) * cols + 64 * slice + 16 * (2 * (run & 1) + (run >> 1));
    *(i32x4 *)x = v[0];
    *(i32x4 *)(x + 8) = v[1];
}

namespace {
template <int T, bool TURN>
hipError_t launch_grad(const void *A, int lda, const void *B, int M, int cols, int K, int splits, void *C, float *part, float *part_db, hipStream_t st)
{
    const int n_mt = (M + 64 * T - 1) / (64 * T), n_nt = (cols + 64 * T - 1) / (64 * T);
    const long tiles = (long)n_mt * n_nt, total = tiles * splits;
    if (total > 0x7FFFFFF0L) return hipErrorInvalidValue;
    const int steps = (K + kStepK - 1) / kStepK, k_split = (steps + splits - 1) / splits * kStepK;
    linear_grad_kernel<T, T, TURN><<<(unsigned)xcd_grid(total), 256, 0, st>>>((const uint16_t *)A, lda, (const uint8_t *)B, M, cols, K, k_split,
                                                                              n_nt, (int)tiles, (int)total, (uint16_t *)C, part, part_db);
    return hipGetLastError();
}
hipError_t launch_restore_turned(const void *codes, const float *scales, int rows, int cols, void *B, hipStream_t st)
{
    const long waves = (long)((rows + 31) / 32) * (cols / 128);
    restore_turned_kernel<<<(unsigned)((waves + 3) / 4), 256, 0, st>>>((const uint8_t *)codes, scales, rows, cols, (uint8_t *)B);
    return hipGetLastError();
}
long tiles_of(int M, int cols, int size) { return (long)((M + size - 1) / size) * ((cols + size - 1) / size); }

// Tiles and splits of dW: enough workgroups for the chip, each split with at least eight steps, none without steps.
struct GradPlan { int wide, splits; };
GradPlan dw_plan(int N, int d_in, int d_out)
{
    const int steps = (N + kStepK - 1) / kStepK;
    GradPlan p;
    p.wide = tiles_of(d_out, d_in, 256) * (steps / 8) >= 256;
    long s = p.wide ? 256 / tiles_of(d_out, d_in, 256) : 512 / tiles_of(d_out, d_in, 128);
    s = s > steps / 8 ? steps / 8 : s;
    s = s < 1 ? 1 : s;
    p.splits = steps ? (int)((steps + (steps + s - 1) / s - 1) / ((steps + s - 1) / s)) : 0;
    return p;
}
}  // namespace

int linear_grad_splits(int N, int d_in, int d_out) { return dw_plan(N, d_in, d_out).splits; }

size_t linear_grad_turned_bytes(int rows, int cols) { return (size_t)((rows + 31) / 32) * 32 * cols * 2; }

hipError_t launch_linear_dx(const void *dy, const void *w8, const float *sw, int N, int d_in, int d_out, void *dx, void *turned, hipStream_t st)
{
    const hipError_t e = launch_restore_turned(w8, sw, d_out, d_in, turned, st);
    if (e != hipSuccess) return e;
    if (tiles_of(N, d_in, 256) >= 160) return launch_grad<4, false>(dy, d_out, turned, N, d_in, d_out, 1, dx, nullptr, nullptr, st);
    return launch_grad<2, false>(dy, d_out, turned, N, d_in, d_out, 1, dx, nullptr, nullptr, st);
}

hipError_t launch_linear_dw(const void *dy, const void *x8, const float *sx, int N, int d_in, int d_out, void *dW, void *db, void *turned, float *part, hipStream_t st)
{
    const GradPlan p = dw_plan(N, d_in, d_out);
    const int splits = p.splits;
    const long count = (long)d_out * d_in;
    float *const part_db = part + (size_t)splits * count;
    if (splits) {
        hipError_t e = launch_restore_turned(x8, sx, N, d_in, turned, st);
        if (e != hipSuccess) return e;
        e = p.wide ? launch_grad<4, true>(dy, d_out, turned, d_out, d_in, N, splits, nullptr, part, db ? part_db : nullptr, st)
                   : launch_grad<2, true>(dy, d_out, turned, d_out, d_in, N, splits, nullptr, part, db ? part_db : nullptr, st);
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
