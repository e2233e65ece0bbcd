// Microscaled 4-bit floating point: 32 consecutive elements of a row share a power of two 2^(s - 127), s one byte, and are
// E2M1 numbers c (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives), two to a byte, the even element in the low half.
//     s = max(exponent field of the block's largest magnitude - 2, 0),   c = E2M1(x 2^(127 - s)), to nearest even, at most 6
// A block with an infinity or NaN gets s = 255 (NaN) and codes 0.  The linear layer
//     y[i][o] = sum over blocks of 2^(sx + sw - 254) sum of c_x c_w + bias[o]
// runs on the scaled matrix instructions, which take both scales beside the codes: products are exact, sums are fp32.
#include "gemm_common.hpp"
#include "sla_kernels.hpp"

#include <type_traits>

namespace sla {

namespace {
constexpr int kFp4 = 4;                              // operand format of the scaled matrix instructions

// largest magnitude of eight bf16 (bits without the sign; infinities and NaN order above all numbers)
__device__ __forceinline__ uint32_t top_bits(uint4 u)
{
    typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
    auto mag = [](uint32_t w) { return __builtin_bit_cast(u16x2, w & 0x7FFF7FFFu); };
    const u16x2 m = __builtin_elementwise_max(__builtin_elementwise_max(mag(u.x), mag(u.y)), __builtin_elementwise_max(mag(u.z), mag(u.w)));
    return m[0] > m[1] ? m[0] : m[1];
}
// of a block, eight elements in each of four neighbouring lanes
__device__ __forceinline__ uint32_t block_top(uint4 u)
{
    uint32_t top = top_bits(u);
    top = max(top, (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0xB1, 0xf, 0xf, true));
    return max(top, (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0x4E, 0xf, 0xf, true));
}
// scale byte of a block with that largest magnitude
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) { return top >= 0x7F80u ? 255u : (top >> 7) < 2 ? 0u : (top >> 7) - 2; }

// eight codes of eight bf16; scale = 2^(s - 127) as fp32 bits (subnormal for s = 0).  Blocks with s = 255 are the caller's.
__device__ __forceinline__ uint32_t codes8(uint4 u, float scale)
{
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, u.x), scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, u.y), scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, u.z), scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, u.w), scale, 3);
}
__device__ __forceinline__ float scale_value(uint32_t s) { return __uint_as_float(s ? s << 23 : 0x00400000u); }
}  // namespace

// Four lanes to a block, 16 bytes of it each: 2 bytes in, 17/32 out per element, bound by HBM: 43968 x 1024 25 us (4.6 TB/s), x 4096 84 us (5.4 TB/s).
// BY_STEPS: both as the product below takes them, in steps of 128 elements, so that what a copy to LDS brings lies side by side:
//     codes   of sixteen rows and a step 1 KB, row after row, steps after one another:  ((r / 16) steps + s) 1024 + (r % 16) 64
//     scales  the dword of row r and step s at s rows + r                               (rows x steps dwords)
// and the workgroups from first_w on bring the weights (O rows) into the same order.  As they lie by rows, K / 2 bytes apart, often a power
// of two, the rows of a step come from one or two of the sixteen channels of the L2, and every dword of scales is a request of its own.
struct WeightsIn {
    const i32x4 *codes;
    const uint32_t *scales;
    i32x4 *codes_out;
    uint32_t *scales_out;
    int O;
    unsigned first_w;
};
template <bool BY_STEPS>
__global__ __launch_bounds__(256) void quantise_mxfp4_kernel(const uint4 *__restrict__ X, long pieces, uint32_t *__restrict__ codes, uint8_t *__restrict__ scales,
                                                             int rows, int steps, WeightsIn w)
{
    const long at = (long)blockIdx.x * 256 + threadIdx.x;      // pieces is a multiple of four: a block's lanes all work or all leave
    if constexpr (BY_STEPS)
        if (blockIdx.x >= w.first_w) {                         // four codes' pieces and a dword of scales to (row, step): 16 bytes a thread
            const unsigned i = (blockIdx.x - w.first_w) * 256 + threadIdx.x, row = i / (4u * steps), q = i - row * 4u * steps, s = q >> 2;
            if (row >= (unsigned)w.O) return;
            w.codes_out[((size_t)(row >> 4) * steps + s) * 64 + (row & 15) * 4 + (q & 3)] = w.codes[i];
            if ((q & 3) == 0) w.scales_out[(size_t)s * w.O + row] = w.scales[(size_t)row * steps + s];
            return;
        }
    if (at >= pieces) return;
    const uint4 u = X[at];
    const uint32_t s = scale_byte(block_top(u)), code = s == 255 ? 0u : codes8(u, scale_value(s));
    if constexpr (BY_STEPS) {
        const unsigned row = (unsigned)at / (16u * steps), q = (unsigned)at - row * 16u * steps, st = q >> 4;
        codes[((size_t)(row >> 4) * steps + st) * 256 + (row & 15) * 16 + (q & 15)] = code;
        if ((q & 3) == 0) scales[((size_t)st * rows + row) * 4 + (q >> 2 & 3)] = (uint8_t)s;
    } else {
        codes[at] = code;
        if ((at & 3) == 0) scales[at >> 2] = (uint8_t)s;
    }
}

// Eight elements a thread; HBM bound: 43968 x 1024 18 us.
__global__ __launch_bounds__(256) void dequantise_mxfp4_kernel(const uint32_t *__restrict__ codes, const uint8_t *__restrict__ scales, long pieces, uint4 *__restrict__ Y)
{
    const long at = (long)blockIdx.x * 256 + threadIdx.x;
    if (at >= pieces) return;
    const uint32_t c = codes[at], s = scales[at >> 2];
    const float scale = s == 255 ? __builtin_nanf("") : scale_value(s);
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t m = (c >> (4 * e)) & 7;       // 2 |c|: 0 1 2 3 4 6 8 12, sixteen to a dword pair
        const float mag = 0.5f * (float)((0xC8643210u >> (4 * m)) & 15u);
        v[e] = ((c >> (4 * e)) & 8 ? -mag : mag) * scale;
    }
    Y[at] = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
}

// Large products.  A [M, K] tokens, by steps (see above); W [O, K] channels, by steps (by_steps) or as they lie: a few tiles of tokens
// do not pay for the turn.
// Workgroup tile 64 TM tokens x 64 TN channels, four waves as 2 x 2.  Steps of 128 elements: 64 bytes and one dword of scales of
// every row, copied straight to LDS, four stages, copies three steps ahead.  In LDS the 16-byte piece c of row r is at position
// c ^ (r / 4 % 4): sixteen rows' reads of one piece meet all banks once.  A step has two parts of 64 elements (one matrix instruction
// deep); the operands of a part are read while the products of the one before run, and reads and copies stand between the products,
// because a wave of the largest tile is alone on its SIMD.  The one barrier of a step stands before the products of its second part,
// whose operands are in registers by then.
// Measured: 43968 tokens, 4096 -> 1024 107 us in a stream of passes (3.5 PFLOP/s), 114 to 130 from rest.
// D[channel][token] (W is the first operand): a lane's four consecutive registers are consecutive channels.
template <int TM, int TN>
__global__ __launch_bounds__(256, TM == 4 ? 1 : 2) void mxfp4_gemm_kernel(const uint8_t *__restrict__ A, const uint8_t *__restrict__ As, const uint8_t *__restrict__ W,
                                                            const uint8_t *__restrict__ Ws, int by_steps, const uint16_t *__restrict__ bias, int M, int O,
                                                            int K, int n_ot, int total, uint16_t *__restrict__ Y)
{
    constexpr int BM = 64 * TM, BN = 64 * TN, kRows = BM + BN, kStage = kRows * 68, kStages = 4;      // codes of all rows, tokens first, then their scales
    constexpr int kScales = (kRows / 64 + 3) / 4, kCopies = TM + TN + kScales;   // copies a wave makes in a step: of 1 KB (A, W), of 256 bytes
    constexpr int kOpsA = (TM + 1) / 2, kOpsW = TN / 2, kCopyOps = kOpsA + kOpsW + kScales;       // in pairs
    __shared__ __attribute__((aligned(1024))) uint8_t smem[kStages * kStage];
    const int item = (int)xcd_remap(blockIdx.x, total);
    if (item >= total) return;
    const auto [it, ot] = tile_at(item, (M + BM - 1) / BM, n_ot);
    const int i0 = it * BM, o0 = ot * BN;
    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, g = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wi = (wave & 1) * 32 * TM, wo = (wave >> 1) * 32 * TN;
    const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)smem;

    // copies of wave w: sixteen rows' pieces each of tokens from row 16 TM w of the tile on and of channels from row 16 TN w on, the scales
    // of 64 rows from row 64 kScales w of both on; rows past the end repeat the last one: their results are not stored
    const int steps = K / 128;
    const int w_row = by_steps ? 64 : K / 2, ws_row = by_steps ? 4 : K / 32;
    const size_t w_step = by_steps ? 1024 : 64, ws_step = by_steps ? 4 * (size_t)O : 4;
    uint32_t va[TM], vw[TN], vs[kScales];
    auto place = [&](int r, int last, int row_bytes) {                           // of the lane's piece; sixteen rows are 1024 steps bytes in either order
        const int at = min(r, last);
        return (uint32_t)(at >> 4) * 1024u * (uint32_t)steps + (uint32_t)(at & 15) * (uint32_t)row_bytes + (((lane & 3) ^ (r >> 2)) & 3) * 16;
    };
#pragma unroll
    for (int x = 0; x < TM; ++x) va[x] = place((wave * TM + x) * 16 + (lane >> 2), M - 1 - i0, 64);
#pragma unroll
    for (int x = 0; x < TN; ++x) vw[x] = place((wave * TN + x) * 16 + (lane >> 2), O - 1 - o0, w_row);
    int ks = item % steps;                           // step that the next copies bring: tiles that share rows start at steps of their own
    const uint8_t *ba, *bw, *bs[kScales];            // where that step begins
    const uint8_t *const a0 = A + (size_t)i0 * (K / 2), *const w0 = W + (size_t)o0 * (K / 2), *s0[kScales];
    size_t s_step[kScales];
    int sr[kScales];                                 // first row of a copy of scales (64 x 128 tiles: two waves make the same)
#pragma unroll
    for (int x = 0; x < kScales; ++x) {
        sr[x] = min(wave * kScales + x, kRows / 64 - 1) * 64;
        const bool tokens = sr[x] < BM;
        s0[x] = tokens ? As + (size_t)i0 * 4 : Ws + (size_t)o0 * ws_row;
        s_step[x] = tokens ? 4 * (size_t)M : ws_step;
        vs[x] = (uint32_t)min((tokens ? sr[x] : sr[x] - BM) + lane, (tokens ? M - i0 : O - o0) - 1) * (uint32_t)(tokens ? 4 : ws_row);
    }
    auto aim = [&] {
        ba = a0 + (size_t)ks * 1024;
        bw = w0 + ks * w_step;
#pragma unroll
        for (int x = 0; x < kScales; ++x) bs[x] = s0[x] + ks * s_step[x];
        ks = ks + 1 == steps ? 0 : ks + 1;
    };
    auto copy_one = [&](int s, int x) {
        const uint32_t to = lds_base + (s & (kStages - 1)) * kStage;
        if (x < kOpsA) {
            if constexpr (TM == 1) copy_1k_to_lds(ba, va[0], to + wave * 1024);
            else copy_2k_to_lds(ba, va[2 * x], va[2 * x + 1], to + (wave * TM + 2 * x) * 1024);
        } else if (x < kOpsA + kOpsW) {
            const int p = x - kOpsA;
            copy_2k_to_lds(bw, vw[2 * p], vw[2 * p + 1], to + BM * 64 + (wave * TN + 2 * p) * 1024);
        } else {
            const int p = x - kOpsA - kOpsW;
            copy_256_to_lds(bs[p], vs[p], to + kRows * 64 + sr[p] * 4);
        }
    };

    f32x16 acc[TN][TM];
#pragma unroll
    for (int a = 0; a < TN; ++a)
#pragma unroll
        for (int b = 0; b < TM; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[a][b][e] = 0.f;
    constexpr int kOps = TM + TN;                                                // operands of a part: TN of W, then TM of x
    i32x4 op[2][kOps];
    int sc[kOps], next_sc[kOps];
    // LDS bytes of the lane's piece of operand 0 of W and of x in part 0 and 1, and of their scales; other operands are 32 rows on
    const uint32_t row_w = BM + wo + l32, row_x = wi + l32, piece0 = ((g ^ (l32 >> 2)) & 3) * 16, piece1 = (((2 + g) ^ (l32 >> 2)) & 3) * 16;
    const uint32_t at_w[2] = {row_w * 64 + piece0, row_w * 64 + piece1}, at_x[2] = {row_x * 64 + piece0, row_x * 64 + piece1};
    const uint32_t at_sw = kRows * 64 + row_w * 4, at_sx = kRows * 64 + row_x * 4;
    auto read_op = [&](int set, uint32_t stage, int t, int x) {
        op[set][x] = *(const i32x4 *)(x < TN ? smem + (stage + at_w[t]) + x * 2048 : smem + (stage + at_x[t]) + (x - TN) * 2048);
    };
    auto read_scale = [&](uint32_t stage, int x) { return *(const int *)(x < TN ? smem + (stage + at_sw) + x * 128 : smem + (stage + at_sx) + (x - TN) * 128); };
    auto mine = [&](int dword) { return (int)((uint32_t)dword >> (8 * g)); };    // this half's two blocks of the step: bytes 0 and 2
    auto wide = [](i32x4 u) { return i32x8{u[0], u[1], u[2], u[3], 0, 0, 0, 0}; };
    // the products of a part; what `between` does is spread over the gaps behind them
    auto multiply = [&](auto part, auto between) {
        constexpr int t = decltype(part)::value;
#pragma unroll
        for (int i = 0; i < TM * TN; ++i) {
            const int a = i / TM, b = i % TM;
            acc[a][b] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wide(op[t][a]), wide(op[t][TN + b]), acc[a][b], kFp4, kFp4, 2 * t, sc[a], 2 * t, sc[TN + b]);
            __builtin_amdgcn_sched_barrier(0);
            between(i);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto spread = [](int i, int count, auto f) {     // the share of `count` things that goes behind product i
#pragma unroll
        for (int x = 0; x < count; ++x)
            if (x * (TM * TN) / count == i) f(x);
    };
    using Part0 = std::integral_constant<int, 0>;
    using Part1 = std::integral_constant<int, 1>;
    using Two = std::integral_constant<int, 2>;
    using Yes = std::true_type;
    using No = std::false_type;
    // AHEAD: later steps than the next one whose copies may still be under way
    auto step = [&](int s, auto copies, auto ahead, auto last) {
        constexpr bool kCopy = decltype(copies)::value, kLast = decltype(last)::value;
        const uint32_t stage = (s & (kStages - 1)) * kStage, next = ((s + 1) & (kStages - 1)) * kStage;
        if constexpr (kCopy) aim();
        multiply(Part0{}, [&](int i) {
            spread(i, kOps, [&](int x) { read_op(1, stage, 1, x); });
            if constexpr (kCopy) spread(i, kCopyOps, [&](int x) { copy_one(s + 3, x); });
        });
        if constexpr (!kLast) {
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(decltype(ahead)::value * kCopies) : "memory");
            lds_barrier();
        }
        multiply(Part1{}, [&](int i) {
            if constexpr (!kLast) {
                spread(i, kOps, [&](int x) { read_op(0, next, 0, x); });
                spread(i, kOps, [&](int x) { next_sc[x] = read_scale(next, x); });
            }
        });
        if constexpr (!kLast) {
#pragma unroll
            for (int x = 0; x < kOps; ++x) sc[x] = mine(next_sc[x]);
        }
    };

    for (int s = 0; s < min(steps, 3); ++s) {
        aim();
#pragma unroll
        for (int x = 0; x < kCopyOps; ++x) copy_one(s, x);
    }
    if (steps > 2)       asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * kCopies) : "memory");
    else if (steps == 2) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kCopies) : "memory");
    else                 asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    lds_barrier();
#pragma unroll
    for (int x = 0; x < kOps; ++x) {
        read_op(0, 0, 0, x);
        sc[x] = mine(read_scale(0, x));
    }
    int s = 0;
    for (; s + 3 < steps; ++s) step(s, Yes{}, Two{}, No{});
    if (s + 2 < steps) step(s++, No{}, Part1{}, No{});
    if (s + 1 < steps) step(s++, No{}, Part0{}, No{});
    step(s, No{}, Part0{}, Yes{});

    // register 4q + r of acc[a][b], lane (l32, g): channel 32 a + 8 q + 4 g + r, token 32 b + l32
    lds_barrier();                                   // everybody has read the last stage
    const int ch0 = o0 + wo, tok0 = i0 + wi;
    float bi[TN][4][4];
#pragma unroll
    for (int a = 0; a < TN; ++a)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int o = min(ch0 + 32 * a + 8 * q + 4 * g, O - 4);
            const uint2 u = bias ? *(const uint2 *)(bias + o) : make_uint2(0, 0);
            bi[a][q][0] = bf16_lo(u.x); bi[a][q][1] = bf16_hi(u.x); bi[a][q][2] = bf16_lo(u.y); bi[a][q][3] = bf16_hi(u.y);
        }
    store_tile<TM, TN>(smem + wave * kStoreBytes<TN>, [&](int a, int b, int q, float (&v)[4]) {
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = acc[a][b][4 * q + r] + bi[a][q][r];
    }, lane, M - tok0, O - ch0, Y + (size_t)tok0 * O + ch0, (size_t)O);
}

// Few tokens (at most 4 Q): one launch, bound by the weights' bytes and by latency.  A wave takes 16 channels and a part of K
// in steps of 128: of W lane l holds the 32 elements 32 (l / 16) .. of row l % 16, one whole block, as it lies.  x is quantised on the way:
// sixteen lanes read the 256 bytes of a token's step, four to a block, and the codes and scales go through the wave's own LDS to the lanes
// that multiply them.  The next step's bytes are asked for before this one's are used (two or four steps ahead take registers from other
// workgroups: 4 tokens, 1152 -> 8208 3.8 us and 4.7).  Without a condition on the number of tokens inside, the four tokens' forty instructions each
// go into one another: 16 tokens through 4096 x 4096 6.8 us and 5.8.  One token: 4.6 us for 8.9 MB of weights, four steps of latency and a launch.
// `parts` waves (a power of two) share 16 channels, 8 / parts groups of channels share a workgroup; their sums are added in order.
template <int Q>
__global__ __launch_bounds__(512) void mxfp4_few_kernel(const uint16_t *__restrict__ X, const uint8_t *__restrict__ W, const uint8_t *__restrict__ Ws,
                                                        const uint16_t *__restrict__ bias, int M, int O, int K, int parts, uint16_t *__restrict__ Y)
{
    constexpr int T = (Q + 3) / 4;                   // sixteens of tokens
    __shared__ float sums[8][T][16][17];             // [wave][16 tokens][token][channel]
    __shared__ __attribute__((aligned(16))) uint32_t x_codes[8][T][256];         // [wave][16 tokens][token][block][dword]
    __shared__ uint8_t x_scales[8][T][64];                                       // [wave][16 tokens][token][block]
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63, r16 = lane & 15, c = lane >> 4;
    const int part = wave & (parts - 1), group = wave / parts, o0 = ((int)blockIdx.x * (8 / parts) + group) * 16;
    const int steps = K / 128, mine = (steps - part + parts - 1) / parts;        // steps part, part + parts, ...: at least one
    const int o = min(o0 + r16, O - 1);              // rows past the end repeat the last one
    f32x4 acc[T];
#pragma unroll
    for (int t = 0; t < T; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    const uint8_t *const w = W + (size_t)o * (K / 2) + c * 16, *const ws = Ws + (size_t)o * (K / 32) + c;
    const uint16_t *x[Q];                            // instruction j reads tokens 4 j + l / 16; those past the end repeat the last one
#pragma unroll
    for (int j = 0; j < Q; ++j) x[j] = X + (size_t)min(4 * j + c, M - 1) * K + 8 * r16;
    uint4 wn, xn[Q];
    uint32_t sn;
    auto load = [&](int k) {                         // the wave's step k
        const int s = part + parts * k;
        wn = *(const uint4 *)(w + s * 64);
        sn = ws[s * 4];
#pragma unroll
        for (int j = 0; j < Q; ++j) xn[j] = *(const uint4 *)(x[j] + s * 128);
    };
    load(0);
    if (Q < 4) {                                     // tokens that are not there: zeros
        *(uint4 *)(x_codes[wave][0] + 4 * lane) = make_uint4(0, 0, 0, 0);
        x_scales[wave][0][lane] = 0;
        wave_lds_sync();
    }
    for (int k = 0; k < mine; ++k) {
        const i32x8 wf = {(int)wn.x, (int)wn.y, (int)wn.z, (int)wn.w, 0, 0, 0, 0};
        const int sw = (int)sn;
#pragma unroll
        for (int j = 0; j < Q; ++j) {
            const uint32_t sx = scale_byte(block_top(xn[j]));
            x_codes[wave][j / 4][64 * (j % 4) + lane] = codes8(xn[j], scale_value(sx)) & (sx == 255 ? 0u : ~0u);
            x_scales[wave][j / 4][16 * (j % 4) + (lane >> 2)] = (uint8_t)sx;
        }
        if (k + 1 < mine) load(k + 1);
        wave_lds_sync();
#pragma unroll
        for (int t = 0; t < T; ++t) {
            const uint4 u = *(const uint4 *)(x_codes[wave][t] + 16 * r16 + 4 * c);
            const i32x8 xf = {(int)u.x, (int)u.y, (int)u.z, (int)u.w, 0, 0, 0, 0};
            acc[t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wf, xf, acc[t], kFp4, kFp4, 0, sw, 0, (int)x_scales[wave][t][4 * r16 + c]);
        }
        wave_lds_sync();
    }
    // register r of acc[t]: channel 4 c + r, token 16 t + r16
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) sums[wave][t][r16][4 * c + r] = acc[t][r];
    __syncthreads();
    const int groups = 8 / parts, out = groups * T * 256;
    for (int at = threadIdx.x; at < out; at += 512) {
        const int ch = at & 15, tok = (at >> 4) & 15, t = (at >> 8) % T, gr = (at >> 8) / T;
        const int oo = ((int)blockIdx.x * groups + gr) * 16 + ch, i = 16 * t + tok;
        float v = 0.f;
        for (int p = 0; p < parts; ++p) v += sums[gr * parts + p][t][tok][ch];
        if (i < M && oo < O) {
            bf16x2 b;
            b[0] = (__bf16)(v + (bias ? bf16_bits_to_f32(bias[oo]) : 0.f));
            Y[(size_t)i * O + oo] = __builtin_bit_cast(uint16_t, b[0]);
        }
    }
}

hipError_t launch_quantise_mxfp4(const void *X, long rows, int cols, void *codes, void *scales, hipStream_t st)
{
    const long pieces = rows * (cols / 8), grid = (pieces + 255) / 256;
    if (grid > 0x7FFFFFFFL) return hipErrorInvalidValue;
    quantise_mxfp4_kernel<false><<<(unsigned)grid, 256, 0, st>>>((const uint4 *)X, pieces, (uint32_t *)codes, (uint8_t *)scales, 0, 0, WeightsIn{});
    return hipGetLastError();
}

hipError_t launch_mxfp4_operands(const void *X, int M, int K, void *codes, void *scales, const void *W, const void *Ws, int O, void *W_out, void *Ws_out, hipStream_t st)
{
    const long pieces = (long)M * (K / 8), first_w = (pieces + 255) / 256, grid = first_w + (W_out ? ((long)O * (K / 32) + 255) / 256 : 0);
    if (grid > 0x7FFFFFFFL) return hipErrorInvalidValue;
    const WeightsIn w = {(const i32x4 *)W, (const uint32_t *)Ws, (i32x4 *)W_out, (uint32_t *)Ws_out, O, (unsigned)first_w};
    quantise_mxfp4_kernel<true><<<(unsigned)grid, 256, 0, st>>>((const uint4 *)X, pieces, (uint32_t *)codes, (uint8_t *)scales, M, K / 128, w);
    return hipGetLastError();
}

hipError_t launch_dequantise_mxfp4(const void *codes, const void *scales, long rows, int cols, void *Y, hipStream_t st)
{
    const long pieces = rows * (cols / 8), grid = (pieces + 255) / 256;
    if (grid > 0x7FFFFFFFL) return hipErrorInvalidValue;
    dequantise_mxfp4_kernel<<<(unsigned)grid, 256, 0, st>>>((const uint32_t *)codes, (const uint8_t *)scales, pieces, (uint4 *)Y);
    return hipGetLastError();
}

// One launch while quantising x in every workgroup costs less than a launch of its own: 32 tokens through 4096 x 4096 8.9 us (13.0 with two launches),
// 1024 x 1024 4.1 (6.9), 4096 -> 8192 12.9 (12.8); up to 64 where four or eight waves share K, none has much of it, and each workgroup has a CU of its own: 48 tokens
// through 1024 x 1024 4.9 (7.0), 64 tokens 5.7 (7.0), 2048 x 2048 8.1 (8.7), but 4096 x 4096 14.6 (13.3), 128 -> 1024 7.6 (5.4),
// 2048 -> 8192 16.6 (8.9).
bool mxfp4_few(int M, int O, int K) { return M <= 32 || (M <= 64 && K >= 512 && O <= 4096 && (M + 15) / 16 * ((K + 1023) / 1024) <= 12); }

namespace {
template <int Q> hipError_t launch_few(const void *X, const void *W, const void *Ws, const void *bias, int M, int O, int K, void *Y, hipStream_t st)
{
    int parts = 1;                                   // waves that share a channel group's K, each with a step at least
    while (parts < 8 && 2 * parts <= K / 128) parts *= 2;
    const int channels = 16 * (8 / parts);
    mxfp4_few_kernel<Q><<<(unsigned)((O + channels - 1) / channels), 512, 0, st>>>((const uint16_t *)X, (const uint8_t *)W, (const uint8_t *)Ws,
                                                                                  (const uint16_t *)bias, M, O, K, parts, (uint16_t *)Y);
    return hipGetLastError();
}
template <int TM, int TN>
hipError_t launch_gemm(const void *A, const void *As, const void *W, const void *Ws, bool by_steps, const void *bias, int M, int O, int K, void *Y, hipStream_t st)
{
    const int n_it = (M + 64 * TM - 1) / (64 * TM), n_ot = (O + 64 * TN - 1) / (64 * TN);
    const long total = (long)n_it * n_ot;
    if (total > 0x7FFFFFF0L) return hipErrorInvalidValue;
    mxfp4_gemm_kernel<TM, TN><<<(unsigned)xcd_grid(total), 256, 0, st>>>((const uint8_t *)A, (const uint8_t *)As, (const uint8_t *)W, (const uint8_t *)Ws, by_steps,
                                                                         (const uint16_t *)bias, M, O, K, n_ot, (int)total, (uint16_t *)Y);
    return hipGetLastError();
}
}  // namespace

hipError_t launch_mxfp4_few(const void *X, const void *W, const void *Ws, const void *bias, int M, int O, int K, void *Y, hipStream_t st)
{
    if (M <= 4) return launch_few<1>(X, W, Ws, bias, M, O, K, Y, st);
    if (M <= 8) return launch_few<2>(X, W, Ws, bias, M, O, K, Y, st);
    if (M <= 16) return launch_few<4>(X, W, Ws, bias, M, O, K, Y, st);
    if (M <= 32) return launch_few<8>(X, W, Ws, bias, M, O, K, Y, st);
    if (M <= 48) return launch_few<12>(X, W, Ws, bias, M, O, K, Y, st);
    return launch_few<16>(X, W, Ws, bias, M, O, K, Y, st);
}

// W by steps costs its quantiser launch (17/32 O K bytes read and written): where both products take as long as that, with M = O
// (4096 tokens x 4096 -> 4096: 53.2 us as it lies, 51.6 turned; 4096 x 1024 -> 4096: 21.3 both), it is not worth the workspace; with M = 2 O it is
// (8192 x 4096 -> 4096: 100 and 95; 8192 x 1024 -> 4096: 36.2 and 34.6).
bool mxfp4_turns_weights(int M, int O) { return M >= 2L * O; }

// Tiles.  64 x 128 while each has a CU of its own (256 of them, 2048 x 1024 -> 1024: 6.1 us, 6.7 with 128 x 128; 352, 700 x 1024 -> 4096: 7.5 and
// 7.0, from 4096 channels 23.3 and 17.0).  A 256 x 256 tile reads half as much from LDS and L2 for a product as four of 128 x 128, but has a CU to
// itself, with nothing under its start and end: from 192 on, whatever K is, which loses on short rows there (us, 256 x 256 and 128 x 128: 172,
// 10992 x 1024 -> 1024: 15.2 and 12.9; 192, 3000 x 1024 -> 4096: 16.0 and 14.0, x 4096: 34.8 and 41.0; 2752, 43968 x 1024 -> 4096: 150 and 154; 688, 43968 x 4096 -> 1024: 102 and 108).
hipError_t launch_mxfp4_gemm(const void *A, const void *As, const void *W, const void *Ws, bool by_steps, const void *bias, int M, int O, int K, void *Y, hipStream_t st)
{
    const long wide = (long)((M + 255) / 256) * ((O + 255) / 256), narrow = (long)((M + 63) / 64) * ((O + 127) / 128);
    if (wide >= 192) return launch_gemm<4, 4>(A, As, W, Ws, by_steps, bias, M, O, K, Y, st);
    if (narrow > 256) return launch_gemm<2, 2>(A, As, W, Ws, by_steps, bias, M, O, K, Y, st);
    return launch_gemm<1, 2>(A, As, W, Ws, by_steps, bias, M, O, K, Y, st);
}

}  // namespace sla
