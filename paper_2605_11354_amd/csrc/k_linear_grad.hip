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
// was in the first place; products are exact in the fp32 accumulators.  dx and dW come out 1.8e-3 to 2.5e-3 from 64 bits in the 2-norm, of which their
// store is 1.66e-3; operands of more bits would take the matrix unit twice as long.
//
// B is restored once, by grad_operands_kernel, into the order in which the matrix unit's operands are read: column groups of 32, of
// a group 16 k after 16 k, 1 KB each, lane l's 16 bytes (column l % 32, k = 8 (l / 32) ..) one after the other; k past the end are
// zeros up to a multiple of 32.  (Converted on the way to LDS instead, every tile of rows converts it again: four vector instructions
// for each matrix instruction, 540 us instead of 30 for the restoring and what the products then take.)
#include "gemm_common.hpp"
#include "sla_kernels.hpp"

#include <algorithm>
#include <type_traits>

namespace sla {

namespace {
constexpr int kStepK = 32, kStages = 4;              // summation indices of a step; steps in LDS
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

// Codes of a 32 x 128 tile, lane l's four pieces (columns 16 (x / 2 * 4 + 2 (run % 2) + run / 2) .. of row l % 32, run = x % 2 * 2 + l / 32:
// the order of k_linear.hip), times the scale of the lane's row -> B as described above: column groups 4 span .. + 3, row group grp.
// `tile`: 8 KB of the wave's own LDS; the turn is ds_read_b64_tr_b16's.
__device__ __forceinline__ void turn_tile(const i32x4 (&c)[4], float scale, uint8_t *tile, int lane, int span, int grp, int groups, uint8_t *B)
{
    const int r = lane & 31;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        const int run = (x & 1) * 2 + (lane >> 5), col = 8 * (x >> 1) + 2 * (2 * (run & 1) + (run >> 1));
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

// Both products' B in one launch.  The first w_blocks workgroups quantise W (bf16 [d_out, cols]) as the layer's forward does and turn
// the numbers at once: `parts` workgroups share 32 rows, 128 columns at a time for each of their waves, and each needs the maxima of the whole
// rows.  The others turn the kept codes of x: 32 rows and 128 columns a wave.  HBM bound: 43968 tokens, 1024 -> 4096 28 us (45 MB of codes in, 90 MB out, and W: 5.2 TB/s).
__global__ __launch_bounds__(256) void grad_operands_kernel(const uint16_t *__restrict__ W, int d_out, uint8_t *__restrict__ Bw, unsigned w_blocks, unsigned parts,
                                                            const uint8_t *__restrict__ codes, const float *__restrict__ scales, int rows,
                                                            uint8_t *__restrict__ Bx, int cols)
{
    __shared__ __attribute__((aligned(1024))) uint8_t smem[4 * 8192];
    __shared__ float red[4][32];
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63, r = lane & 31;
    const int spans = cols / 128;
    i32x4 c[4];
    if (blockIdx.x < w_blocks) {
        const int grp = (int)(blockIdx.x / parts), part = (int)(blockIdx.x - grp * parts);
        const int R = min(32, d_out - 32 * grp);
        const uint16_t *const from = W + (size_t)32 * grp * cols;
        float top[4] = {0.f, 0.f, 0.f, 0.f};         // of rows lane / 8 + 8 i, over 64 columns at a time
        const int n = cols / 64, turn = (int)(blockIdx.x % (unsigned)n);          // workgroups begin at columns, and so channels of the L2, of their own
#pragma unroll 4
        for (int s0 = wave; s0 < n; s0 += 4) {
            const int s = s0 + turn < n ? s0 + turn : s0 + turn - n;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint4 u = *(const uint4 *)(from + (size_t)min((lane >> 3) + 8 * i, R - 1) * cols + 64 * s + 8 * (lane & 7));
                const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                for (int q = 0; q < 4; ++q) top[i] = fmaxf(top[i], fmaxf(fabsf(bf16_lo(w[q])), fabsf(bf16_hi(w[q]))));
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            // over eight lanes
            top[i] = fmaxf(top[i], __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(top[i]), 0xB1, 0xf, 0xf, true)));
            top[i] = fmaxf(top[i], __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(top[i]), 0x4E, 0xf, 0xf, true)));
            top[i] = fmaxf(top[i], __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(top[i]), 0x141, 0xf, 0xf, true)));
            if ((lane & 7) == 0) red[wave][(lane >> 3) + 8 * i] = top[i];
        }
        __syncthreads();
        const float scale = training_scale(fmaxf(fmaxf(red[0][r], red[1][r]), fmaxf(red[2][r], red[3][r])));
        const BlockDivisor divide(scale);
        for (int span = part * 4 + wave; span < spans; span += 4 * (int)parts) {
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int run = (x & 1) * 2 + (lane >> 5), col = 16 * (4 * (x >> 1) + 2 * (run & 1) + (run >> 1));
                const uint16_t *const at = from + (size_t)min(r, R - 1) * cols + 128 * span + col;
                const uint4 u = *(const uint4 *)at, v = *(const uint4 *)(at + 8);
                const uint32_t w[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
                c[x] = __builtin_bit_cast(i32x4, quantise16(w, divide));
            }
            // rows that are not there: zeros, of finite scale
            if (r >= R) for (int x = 0; x < 4; ++x) c[x] = i32x4{0, 0, 0, 0};
            turn_tile(c, r < R ? scale : 0.f, smem + wave * 8192, lane, span, grp, (d_out + 31) / 32, Bw);
            wave_lds_sync();                         // the tile has been read
        }
    } else {
        const int groups = (rows + 31) / 32;
        const long at = (long)(blockIdx.x - w_blocks) * 4 + wave;
        if (at >= (long)groups * spans) return;
        const int grp = (int)(at / spans), span = (int)(at - (long)grp * spans), R = min(32, rows - 32 * grp);
        const uint8_t *const from = codes + (size_t)grp * 32 * cols + (size_t)span * 128 * R;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const int run = (x & 1) * 2 + (lane >> 5);
            c[x] = r < R ? *(const i32x4 *)(from + (x >> 1) * R * 64 + (run * R + r) * 16) : i32x4{0, 0, 0, 0};
        }
        turn_tile(c, r < R ? scales[32 * grp + r] : 0.f, smem + wave * 8192, lane, span, grp, groups, Bx);
    }
}

// One of the two products: C [M, cols] = A B, A bf16 with `lda` elements to a row, B as described above.  Split s of the summation covers k
// from s k_split on.  With part != nullptr a tile goes there in fp32, [split][M][cols], else to C; db (dW only, may be NULL): the sums of A
// over k, from the first tile of columns, to db or, split, to part_db [split][M].
struct GradProduct {
    const uint16_t *A;
    const uint8_t *B;
    int lda, M, cols, K, k_split, n_nt, tiles, total;
    uint16_t *C, *db;
    float *part, *part_db;
};

// TURN: A(m,k) = A[k][m] (dW), else A[m][k] (dx).  Workgroup tile 64 TM x 64 TN, four waves as 2 x 2.
//
// Steps of 32 k, four stages in LDS, filled by copies three steps ahead.  A step has two parts of 16 k; the operands of a
// part are read while the products of the one before run (two sets of registers).  The one barrier of a step stands before the products of its
// second part, whose operands are in registers by then: everybody has read the stage, the next one is whole (its copies were asked for three
// steps ago), and its first operands are read under those products.
// With TM = TN = 4 a wave holds 256 accumulators and a CU one workgroup: a part takes 8 operands per 16 matrix instructions from
// LDS, half of what its bandwidth allows (128 x 64 per wave: three quarters, with the writes all of it).
// Measured: both products of 43968 tokens, 1024 -> 4096 604 us in a stream of passes, 629 from rest (1.2 PFLOP/s: the clock that the chip grants); as library
// products on that machine 361 and 459.
// The matrix unit is busy 78 % of the cycles in which a CU has work; with all copies from the L2 a tenth less time, with a fifth stage the same.
template <int TM, int TN, bool TURN>
__device__ __forceinline__ void grad_tile(const GradProduct &p, int item, uint8_t *smem)
{
    constexpr int BM = 64 * TM, BN = 64 * TN, kA = BM * kStepK * 2, kB = BN * kStepK * 2, kStage = kA + kB;
    constexpr int kCopies = kStage / 4096, kCopiesA = kA / 4096;               // copies of 1 KB a wave makes in a step
    const uint16_t *const A = p.A;
    const uint8_t *const B = p.B;
    const int lda = p.lda, M = p.M, cols = p.cols, K = p.K, tiles = p.tiles, n_nt = p.n_nt, k_split = p.k_split;
    float *const part = p.part;
    const int split = item / tiles, tile = item - split * tiles;
    const auto [mt, nt] = tile_at(tile, (M + BM - 1) / BM, n_nt);
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
    const bool summing = TURN && p.db && nt == 0 && wn == 0;
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
    // the next stage is whole and everybody is done with the one before it; AHEAD: copies of later steps, which may still be under way
    auto change = [&](auto ahead) {
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(decltype(ahead)::value) : "memory");
        lds_barrier();
    };
    auto change_to_last = [&](int stage) {           // and what of it lies past K is cleared
        const int left = K - (k0 + (steps - 1) * kStepK);
        if (left < kStepK) {
            clear_tail(left, stage);
            lds_barrier();
        }
    };
    // 256 x 256: half of the copies behind the last products of either part, every second one: the first have the reads behind them, and the six
    // instructions of a copy fill a gap (all in the first part: 43968 tokens, 1024 -> 4096 646 us, so 634).  128 x 128, where another workgroup
    // fills the gaps: all behind the first part's, the sooner the better (10992 tokens, 1024 -> 1024, the whole step 107.7 us, halves 109.8)
    constexpr int kOperands = TM + TN, kSecond = TM == 4 ? kCopies / 2 : 0, kGap = TM == 4 ? 2 : 1, kFirst = TM * TN - (kCopies - kSecond) * kGap;
    auto copy_behind = [&](int i, int k, int done, int count) {
        if (i >= kFirst && (i - kFirst) % kGap == 0 && (i - kFirst) / kGap < count) copy_one(k, done + (i - kFirst) / kGap);
    };
    auto step = [&](int s, auto copies, auto ahead, auto last) {
        constexpr bool kCopy = decltype(copies)::value, kLast = decltype(last)::value;
        const int k3 = k0 + (s + 3) * kStepK;
        if constexpr (kCopy) aim(k3, (s + 3) & 3);
        multiply(0, [&](int i) {
            if (i < kOperands) read_one(1, s & 3, 1, i);
            if constexpr (kCopy) copy_behind(i, k3, 0, kCopies - kSecond);
        });
        if constexpr (!kLast) {
            change(ahead);
            if constexpr (decltype(ahead)::value == 0) change_to_last((s + 1) & 3);
        }
        multiply(1, [&](int i) {
            if constexpr (!kLast)
                if (i < kOperands) read_one(0, (s + 1) & 3, 0, i);
            if constexpr (kCopy) copy_behind(i, k3, kCopies - kSecond, kSecond);
        });
    };
    static_assert(kOperands <= TM * TN && kCopies % 2 == 0 && kFirst >= 0, "a part has room for its reads and copies");
    using Ahead0 = std::integral_constant<int, 0>;
    using Ahead1 = std::integral_constant<int, kCopies>;
    using Ahead2 = std::integral_constant<int, 2 * kCopies>;
    using InLoop = std::integral_constant<int, 2 * kCopies - kSecond>;           // those of step s + 3's are asked for behind the barrier
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
    for (; s + 3 < steps; ++s) step(s, Yes{}, InLoop{}, No{});
    if (s + 2 < steps) step(s++, No{}, Ahead1{}, No{});
    if (s + 1 < steps) step(s++, No{}, Ahead0{}, No{});
    step(s, No{}, Ahead0{}, Yes{});

    // register 4q + r of acc[b][a], lane (l32, g): n = 32 b + 8 q + 4 g + r, m = 32 a + l32
#pragma unroll
    for (int a = 0; a < TM; ++a) {
        const int m = m0 + wm + 32 * a + l32;
        if (summing) {
            const float v = sums[a] + xchg32(sums[a]);
            if (g == 0 && m < M) {
                if (part) p.part_db[(size_t)split * M + m] = v;
                else p.db[m] = (uint16_t)pack_bf16(v, v);
            }
        }
        if (part) {
#pragma unroll
            for (int b = 0; b < TN; ++b)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const f32x16 &v = acc[b][a];
                    const int n = n0 + wn + 32 * b + 8 * q + 4 * g;
                    if (m < M && n < cols) *(float4 *)(part + ((size_t)split * M + m) * cols + n) = make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
                }
        }
    }
    if (!part) {
        lds_barrier();                               // everybody has read the last stage
        store_tile<TM, TN>(smem + wave * kStoreBytes<TN>, [&](int b, int a, int q, float (&v)[4]) {
#pragma unroll
            for (int r = 0; r < 4; ++r) v[r] = acc[b][a][4 * q + r];
        }, lane, M - m0 - wm, cols - n0 - wn, p.C + (size_t)(m0 + wm) * cols + n0 + wn, (size_t)cols);
    }
}

// The first grid_w workgroups (a multiple of 8) take the tiles of dW, the others those of dx: one launch, and the longer sums first.
template <int T>
__global__ __launch_bounds__(256, T == 4 ? 1 : 2) void linear_grad_kernel(GradProduct w, GradProduct x, unsigned grid_w)
{
    __shared__ __attribute__((aligned(1024))) uint8_t smem[kStages * 64 * (T + T) * kStepK * 2];
    if (blockIdx.x < grid_w) {
        const int item = (int)xcd_remap(blockIdx.x, w.total);
        if (item < w.total) grad_tile<T, T, true>(w, item, smem);
    } else {
        const int item = (int)xcd_remap(blockIdx.x - grid_w, x.total);
        if (item < x.total) grad_tile<T, T, false>(x, item, smem);
    }
}

// HBM bound: four splits of 1024 x 1024 4 to 5 us, two of 4096 x 1024 8 us (42 MB, 5 TB/s).  out[i] = bf16(sum of the splits' partials, in order), for up to three outputs; counts are multiples of 8
struct GradSums {
    const float *part[3];
    uint16_t *out[3];
    long count[3];
    int splits[3];
    unsigned first[4];                               // first workgroup of each, and their number
};
__global__ __launch_bounds__(256) void linear_grad_reduce_kernel(GradSums g)
{
    const int which = blockIdx.x >= g.first[2] ? 2 : blockIdx.x >= g.first[1] ? 1 : 0;
    const long i = ((long)(blockIdx.x - g.first[which]) * 256 + threadIdx.x) * 4, count = g.count[which];
    if (i >= count) return;
    const float *const part = g.part[which];
    const int splits = g.splits[which];
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int s = 0; s < splits; ++s) {
        const float4 u = *(const float4 *)(part + s * count + i);
        v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;
    }
    *(uint2 *)(g.out[which] + i) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
}

// bf16 rows [rows, cols] of codes in fragment order and their scales: sixteen channels a thread; HBM bound: 43968 x 1024 32 us (4.2 TB/s)
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
long tiles_of(int M, int cols, int size) { return (long)((M + size - 1) / size) * ((cols + size - 1) / size); }

// splits of `steps` steps into at most `most`, none without steps
int even_splits(int steps, long most)
{
    if (most < 1) most = 1;
    const int per = (int)((steps + most - 1) / most);
    return steps ? (steps + per - 1) / per : 0;
}
size_t up256(size_t x) { return (x + 255) / 256 * 256; }

// Tiles and splits.  256 x 256 tiles reach 1.2 PFLOP/s, 128 x 128 tiles 0.85, where either fills the chip; what speaks for the small ones is that
// half a round of them is less, and that a sum split less often leaves fewer partials (fp32, written and read again).  Both products
// take the same, so that one launch has them: where one ends the other fills its CUs (10992 tokens, 1024 -> 1024: 78 us in launches of 256 for
// dx and of 128 for dW, 70 in one of 128).  256 from 128 such tiles of dx and 100 steps of both products for each CU on:
//     us, 128 and 256:   43968 tokens, 1024 -> 1024 (172 steps) 224, 212;  10992, 1024 -> 4096 (172) 210, 199;  10992, 4096 -> 1024 (172) 226, 212;
//     2048, 4096 -> 4096 (128) 184, 187;  21984, 1024 -> 1024 (86) 116, 130;  5496, 4096 -> 1024 (86) 120, 139;  43968, 384 -> 1152 (72) 100, 134;
//     4096, 1024 -> 4096 (64) 85, 136
//   dW  split into parts of at least twenty steps: beside dx, which has as much work, for half of the places (128 or, small, 256 workgroups),
//       alone for all of them.  us, all and half: 1374, 1024 -> 4096 54 and 43;  10992, 1024 -> 1024 72 and 67;  10992, 384 -> 1152 44 and 38;
//       43968, 1024 -> 1024 227 and 212;  43968, 1024 -> 4096 672 and 657;  10992, 1024 -> 4096 193 and 199.  Parts of eight and of twenty:
//       700, 1024 -> 1024 23.5 and 19.4;  1374, 384 -> 1152 22.7 and 20.5
//   dx  128 wide, fewer than 256 tiles: split into parts as long as those of dW beside it and at least eight steps, where what that saves (0.27 us a step) is
//       more than the launch and the partials of the sum cost; alone as beside dW, so that its bits do not depend on what else is asked for.  us, split and whole: 197, 1024 -> 4096 24 and 43;  197, 384 -> 1152 13.2 and 15.4;
//       197, 128 -> 512 11.8 and 10.3;  394, 1024 -> 1024 19.9 and 17.8;  1374, 384 -> 1152 26.2 and 22.7;  197, 4096 -> 1024 36 and 30
struct Plan {
    bool wide;
    int splits_x, splits_w;
    size_t off_bx, off_part_x, off_part_w, off_part_db, total;                   // the operand of dx comes first
};
Plan make_plan(int N, int d_in, int d_out, bool both)
{
    Plan p;
    const long w256 = tiles_of(d_out, d_in, 256), x128 = tiles_of(N, d_in, 128), w128 = tiles_of(d_out, d_in, 128);
    const int x_steps = (d_out + kStepK - 1) / kStepK, w_steps = (N + kStepK - 1) / kStepK;
    p.wide = tiles_of(N, d_in, 256) >= 128 && 2 * (long)N * d_in / 65536 * d_out / kStepK >= 100 * 256;
    const long places = p.wide ? 128 : 256, w_tiles = p.wide ? w256 : w128;
    const int beside = even_splits(w_steps, std::min(places / w_tiles, (long)w_steps / 20));         // of dW beside dx
    p.splits_w = both ? beside : even_splits(w_steps, std::min(2 * places / w_tiles, (long)w_steps / 20));
    p.splits_x = 1;
    if (!p.wide && N && x128 < 256) {
        const int part = std::max(8, (w_steps + beside - 1) / beside), splits = even_splits(x_steps, std::min(256 / x128, (long)x_steps / part));
        if (0.27 * (x_steps - x_steps / splits) > 2.5 + 0.028 * x128 * splits) p.splits_x = splits;
    }
    p.off_bx = (size_t)((d_out + 31) / 32) * 64 * d_in;
    p.off_part_x = p.off_bx + (size_t)((N + 31) / 32) * 64 * d_in;
    p.off_part_w = p.off_part_x + (p.splits_x > 1 ? up256((size_t)p.splits_x * N * d_in * 4) : 0);
    p.off_part_db = p.off_part_w + (p.splits_w > 1 ? up256((size_t)p.splits_w * d_out * d_in * 4) : 0);
    p.total = p.off_part_db + (p.splits_w > 1 ? up256((size_t)p.splits_w * d_out * 4) : 0);
    return p;
}

bool set_product(GradProduct &g, bool wide, int splits)
{
    const int size = wide ? 256 : 128, steps = (g.K + kStepK - 1) / kStepK;
    const long tiles = tiles_of(g.M, g.cols, size), total = tiles * splits;
    g.n_nt = (g.cols + size - 1) / size;
    g.tiles = (int)tiles;
    g.total = (int)total;
    g.k_split = (steps + splits - 1) / splits * kStepK;
    return total <= 0x3FFFFFF0L;
}
hipError_t launch_products(bool wide, const GradProduct &w, const GradProduct &x, hipStream_t st)
{
    const unsigned grid_w = w.total ? (unsigned)xcd_grid(w.total) : 0, grid = grid_w + (x.total ? (unsigned)xcd_grid(x.total) : 0);
    if (wide) linear_grad_kernel<4><<<grid, 256, 0, st>>>(w, x, grid_w);
    else      linear_grad_kernel<2><<<grid, 256, 0, st>>>(w, x, grid_w);
    return hipGetLastError();
}
}  // namespace

size_t linear_grad_workspace(int N, int d_in, int d_out) { return std::max(make_plan(N, d_in, d_out, true).total, make_plan(N, d_in, d_out, false).total); }

hipError_t launch_linear_grad(const void *dy, const void *x8, const float *sx, const void *W, int N, int d_in, int d_out, void *dx, void *dW, void *db,
                              void *workspace, hipStream_t st)
{
    const Plan p = make_plan(N, d_in, d_out, dx && dW);
    char *const ws = (char *)workspace;
    GradSums sums = {};
    auto add = [&](int i, const float *part, void *out, long count, int splits) {
        sums.part[i] = part; sums.out[i] = (uint16_t *)out; sums.count[i] = count; sums.splits[i] = splits;
    };
    if (N > 0) {
        uint8_t *const bw = (uint8_t *)ws, *const bx = (uint8_t *)ws + p.off_bx;
        const int spans = d_in / 128;
        // parts: workgroups for the whole chip, no more, since each reads all of its rows (4096 x 4096: two for each 32 rows 24 us, eight 54)
        const int w_groups = (d_out + 31) / 32, parts = std::max(1, std::min(256 / w_groups, (spans + 3) / 4));
        const long w_blocks = dx ? (long)w_groups * parts : 0, x_blocks = dW ? ((long)((N + 31) / 32) * spans + 3) / 4 : 0;
        if (w_blocks + x_blocks > 0x7FFFFFFFL) return hipErrorInvalidValue;
        grad_operands_kernel<<<(unsigned)(w_blocks + x_blocks), 256, 0, st>>>((const uint16_t *)W, d_out, bw, (unsigned)w_blocks, (unsigned)parts, (const uint8_t *)x8, sx, N, bx, d_in);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        GradProduct x = {}, w = {};
        if (dx) {
            x.A = (const uint16_t *)dy; x.B = bw; x.lda = d_out; x.M = N; x.cols = d_in; x.K = d_out; x.C = (uint16_t *)dx;
            x.part = p.splits_x > 1 ? (float *)(ws + p.off_part_x) : nullptr;
            if (!set_product(x, p.wide, p.splits_x)) return hipErrorInvalidValue;
            if (x.part) add(0, x.part, dx, (long)N * d_in, p.splits_x);
        }
        if (dW) {
            w.A = (const uint16_t *)dy; w.B = bx; w.lda = d_out; w.M = d_out; w.cols = d_in; w.K = N; w.C = (uint16_t *)dW; w.db = (uint16_t *)db;
            w.part = p.splits_w > 1 ? (float *)(ws + p.off_part_w) : nullptr;
            w.part_db = (float *)(ws + p.off_part_db);
            if (!set_product(w, p.wide, p.splits_w)) return hipErrorInvalidValue;
            if (w.part) add(1, w.part, dW, (long)d_out * d_in, p.splits_w);
            if (w.part && db) add(2, w.part_db, db, d_out, p.splits_w);
        }
        e = launch_products(p.wide, w, x, st);
        if (e != hipSuccess) return e;
    } else {                                         // no tokens: sums of nothing
        if (dW) add(1, nullptr, dW, (long)d_out * d_in, 0);
        if (db) add(2, nullptr, db, d_out, 0);
    }
    for (int i = 0; i < 3; ++i) sums.first[i + 1] = sums.first[i] + (unsigned)((sums.count[i] / 4 + 255) / 256);
    if (!sums.first[3]) return hipSuccess;
    linear_grad_reduce_kernel<<<sums.first[3], 256, 0, st>>>(sums);
    return hipGetLastError();
}

hipError_t launch_restore_rows(const void *codes, const float *scales, long rows, int cols, void *X, hipStream_t st)
{
    restore_rows_kernel<<<(unsigned)((rows * (cols / 16) + 255) / 256), 256, 0, st>>>((const uint8_t *)codes, scales, rows, cols, (uint16_t *)X);
    return hipGetLastError();
}

}  // namespace sla
