// What lies between a qkv projection and the attention, in one pass over the data: the norm of every head's query and key
// rows over their 64 channels, the position rotation, and the layout (for the E4M3 path also the data type and the block
// scales) in which the attention takes Q, K and V; and the gradients of all of it.
//     u = (x - m) r,  n = u w + b             m = mean(x) (layer norm; 0 for the RMS norm),  r = 1 / sqrt(mean((x - m)^2) + eps)
//     y_i = n_i cos a - n_p sin a,  y_p = n_p cos a + n_i sin a      (i, p) a pair of channels, a = position base^(-2 i / S)
// backward, with d the gradient of n (that of y rotated back) and g = d w:
//     dx = r (g - mean(g) - u mean(g u))      (no mean(g) term for the RMS norm),   dw = sum d u,   db = sum d
//
// Unit of work: 64 tokens of one head of one tensor, a wave's.  Lane l holds eight channels of tokens l / 8 + 8 k: a row is one
// 128-byte line, its sums are three cross-lane steps inside groups of eight lanes, the partner of a rotated channel is in the
// same lane or one cross-lane operand away, and the unit is a scale block of the E4M3 path.  The workgroup's four waves take
// neighbouring heads of the same tokens, so the lines of a token that lie side by side are read side by side, and the cosines and
// sines of those tokens are computed once, into LDS, for all heads and both tensors.
// HBM bound: 2 bytes in, 2 (E4M3: 1) out per element; backward 4 in, 2 out.  At the copy rate a CU has twenty vector instructions
// for an element, so each is counted: the root is v_rsq_f32 (one unit in the last place), rotation is a product and a
// multiply-add with a cross-lane operand (the table holds the sines with both signs), the E4M3 codes come from the three steps of BlockDivisor.
// Measured, layer norm and two axes, in a stream of calls: 43968 tokens of 16 heads, q, k and v: bf16 110 to 118 us (540 MB, 4.6 to 4.9 TB/s), E4M3 96 us with
// 64-row query blocks (405 MB, 4.2 TB/s) and 110 to 115 with 128-row ones; 10992 tokens bf16 28 to 30 us (4.5 to 4.8 TB/s); gradients of 13814 tokens of 12 heads
// with weights of each head 45 us (170 MB, 3.8 TB/s) and 4 to 5 for the sums; 32 tokens of 16 heads 4.6 us, a launch and three trips to memory.
#include "sla_common.hpp"
#include "sla_kernels.hpp"

#include <type_traits>

namespace sla {

namespace {
// floats per token of the table: 32 cosines, 32 sines, 32 negated sines, one 16-byte step of padding
constexpr int kCsPitch = 100;

// The group of eight channels that lane c of a row's eight holds: 0 1 2 3 7 6 5 4, so that the partner of a pair (i, i + 32) is the
// lane mirrored within eight, and that of (i, i + 16) within a half of 32 the lane two on or back: one DPP operand either way.
__device__ __forceinline__ int channel_group(int c) { return c < 4 ? c : 11 - c; }
template <int ROT> __device__ __forceinline__ float partner(float v)
{
    return __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), ROT == 1 ? 0x141 : 0x4E, 0xf, 0xf, true));
}

// sum over the eight lanes of a row, in all of them
__device__ __forceinline__ float row_sum(float v)
{
    auto step = [](float a, auto ctrl) { return a + __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(a), decltype(ctrl)::value, 0xf, 0xf, true)); };
    v = step(v, std::integral_constant<int, 0xB1>{});
    v = step(v, std::integral_constant<int, 0x4E>{});
    return step(v, std::integral_constant<int, 0x141>{});
}

// sum over the eight lanes l % 8 of a wave, in all of them
__device__ __forceinline__ float group_sum(float v)
{
    v += __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), 0x128, 0xf, 0xf, true));      // eight lanes on, within sixteen
    const uint32_t u = __float_as_uint(v);
    const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    return pair_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

__device__ __forceinline__ void unpack8(uint4 u, float (&x)[8])
{
    x[0] = bf16_lo(u.x); x[1] = bf16_hi(u.x); x[2] = bf16_lo(u.y); x[3] = bf16_hi(u.y);
    x[4] = bf16_lo(u.z); x[5] = bf16_hi(u.z); x[6] = bf16_lo(u.w); x[7] = bf16_hi(u.w);
}
__device__ __forceinline__ uint4 packed8(const float (&x)[8])
{
    return make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
}

// n rotated by the angles of its token (back = 0) or back (1); o = the lane's group of eight channels, cs = the token's
// row of the table.  ROT: 1 = channels (i, i + 32) are a pair, 2 = (i, i + 16) within each half of 32, 3 = (2 i, 2 i + 1)
template <int ROT> __device__ __forceinline__ void rotate(float (&n)[8], const float *cs, int o, int back)
{
    if constexpr (ROT == 1 || ROT == 2) {
        const int at = ROT == 1 ? 8 * (o & 3) : 16 * (o >> 2) + 8 * (o & 1);
        const bool adds = ((o & (ROT == 1 ? 4 : 2)) != 0) != (back != 0);       // the second of a pair adds, the first subtracts
        const int sines = adds ? 32 : 64;
        float c[8], s[8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            *(float4 *)(c + 4 * h) = *(const float4 *)(cs + at + 4 * h);
            *(float4 *)(s + 4 * h) = *(const float4 *)(cs + sines + at + 4 * h);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float p = partner<ROT>(n[e]);
            n[e] = fmaf(p, s[e], n[e] * c[e]);
        }
    } else if constexpr (ROT == 3) {
        const float4 c4 = *(const float4 *)(cs + 4 * o), s4 = *(const float4 *)(cs + (back ? 64 : 32) + 4 * o);
        const float c[4] = {c4.x, c4.y, c4.z, c4.w}, s[4] = {s4.x, s4.y, s4.z, s4.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float a = n[2 * i], b = n[2 * i + 1];
            n[2 * i] = fmaf(-b, s[i], a * c[i]);
            n[2 * i + 1] = fmaf(a, s[i], b * c[i]);
        }
    }
}

// x -> u (see above) of one row, and r
__device__ __forceinline__ float normalise(float (&x)[8], int norm, float eps)
{
    if (norm == 0) return 1.f;
    if (norm == 2) {
        const float m = row_sum(((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]))) * (1.0f / 64.0f);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] -= m;
    }
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fmaf(x[e], x[e], s);
    const float r = __builtin_amdgcn_rsqf(fmaf(row_sum(s), 1.0f / 64.0f, eps));
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= r;
    return r;
}

// cos and sin of `quarters` quarter turns, reduced in 64 bits: a position of 2^31 still leaves 2^-22 of a turn.  Taylor series on half a
// quarter to either side: the first terms left out are below 3e-8.
__device__ __forceinline__ float2 cos_sin(double quarters)
{
    const double whole = rint(quarters);
    const float t = (float)(quarters - whole) * 1.57079632679f, z = t * t;
    const float s = t * fmaf(z, fmaf(z, fmaf(z, fmaf(z, 1.0f / 362880.0f, -1.0f / 5040.0f), 1.0f / 120.0f), -1.0f / 6.0f), 1.0f);
    const float c = fmaf(z, fmaf(z, fmaf(z, fmaf(z, 1.0f / 40320.0f, -1.0f / 720.0f), 1.0f / 24.0f), -0.5f), 1.0f);
    const int q = (int)whole;
    const float a = q & 1 ? s : c, b = q & 1 ? c : s;
    return make_float2((q + 1) & 2 ? -a : a, q & 2 ? -b : b);
}

// Where the rows of the workgroup's tokens lie.  TOK tokens; those past `valid` repeat the last one.  SEQ: the tokens are one
// sequence's (b, first ..), else they run through all sequences.
template <int TOK, bool SEQ>
__device__ __forceinline__ void lay_out_tokens(const HeadsArgs &a, int b, long first, int valid, long *in_off, long *out_off, int *pos_row)
{
    const int tid = threadIdx.x;
    if (tid < TOK) {
        const long f = first + min(tid, valid - 1);
        const int item = SEQ ? b : (int)((unsigned)f / (unsigned)a.N), t = SEQ ? (int)f : (int)f - item * a.N;
        in_off[tid] = item * a.bs + t * a.ts;
        out_off[tid] = item * a.obs + t * a.ots;
        if constexpr (!SEQ) pos_row[tid] = a.pos_per_item ? item * a.N + t : t;
    }
    __syncthreads();
}
// Their angles
template <class Row>
__device__ __forceinline__ void make_table(const HeadsArgs &a, int valid, Row pos_row, float *table)
{
    const int tid = threadIdx.x, j = tid & 31, per = 32 / a.axes, axis = j / per;
    const double turn = a.turn[j];
    const int rows = (valid + 7) & ~7;               // whole groups of eight: the rows behind the last one repeat it, here too
    for (int r = tid >> 5; r < rows; r += 8) {
        const float2 cs = cos_sin((double)a.pos[(size_t)pos_row(r) * a.axes + axis] * turn);
        float *const row = table + r * kCsPitch;
        row[j] = cs.x;
        row[32 + j] = cs.y;
        row[64 + j] = -cs.y;
    }
    lds_barrier();
}

// `otherwise` where there are none: 1 and -0, which keep the sign of a zero
__device__ __forceinline__ void load_weights(const float *p, int head, int per_head, int o, float otherwise, float (&w)[8])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = otherwise;
    if (p) {
        p += (per_head ? (size_t)head * 64 : 0) + 8 * o;
        *(float4 *)w = *(const float4 *)p;
        *(float4 *)(w + 4) = *(const float4 *)(p + 4);
    }
}
}  // namespace

namespace {
// what an item (tensor, head) of a workgroup's list is
struct Item { int tensor, head; };
__device__ __forceinline__ Item item_of(const HeadsArgs &a, int item)
{
    const int tensor = item / a.H;
    return Item{tensor, item - tensor * a.H};
}
template <class T> __device__ __forceinline__ T pick(T const (&p)[3], int tensor) { return tensor == 0 ? p[0] : tensor == 1 ? p[1] : p[2]; }
}  // namespace

// bf16 outputs.  A unit is TOK tokens of 8 ROWS / TOK neighbouring items, ROWS rows a lane: where tokens are few, a workgroup takes few of them and all the
// heads rather than many tokens of few heads, for which it would compute as many angles.  The rows of the next unit are asked
// for before this one's are stored: a load behind a store would wait for it.
template <int ROT, int TOK, int ROWS>
__global__ __launch_bounds__(256, 4) void heads_kernel(HeadsArgs a)
{
    constexpr int kOct = TOK / 8, kItems = ROWS / kOct;
    __shared__ long in_off[TOK], out_off[TOK];
    __shared__ int pos_row[TOK];
    __shared__ __attribute__((aligned(16))) float table[ROT ? TOK * kCsPitch : 4];
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63, o = channel_group(lane & 7), r0 = lane >> 3;
    const unsigned blk = blockIdx.x / (unsigned)a.splits, part = blockIdx.x - blk * (unsigned)a.splits;
    const long first = (long)blk * TOK;
    const int valid = (int)min((long)TOK, (long)a.B * a.N - first);
    lay_out_tokens<TOK, false>(a, 0, first, valid, in_off, out_off, pos_row);
    const int i0 = (int)part * a.chunk, i1 = min(i0 + a.chunk, a.tensors * a.H);
    uint4 rows[ROWS], nxt[ROWS];
    auto load = [&](int unit) {
#pragma unroll
        for (int k = 0; k < ROWS; ++k)
            if (8 * (k % kOct) < valid && unit + k / kOct < i1) {
                const Item it = item_of(a, unit + k / kOct);
                nxt[k] = *(const uint4 *)(pick(a.x, it.tensor) + it.head * a.hs + 8 * o + in_off[r0 + 8 * (k % kOct)]);
            }
    };
    load(i0 + wave * kItems);
    if constexpr (ROT != 0) make_table(a, valid, [&](int r) { return (long)pos_row[r]; }, table);
    float w[8], bias[8];
    int have = -1;                                   // tensor whose weights these are
    for (int unit = i0 + wave * kItems; unit < i1; unit += 4 * kItems) {
#pragma unroll
        for (int k = 0; k < ROWS; ++k) rows[k] = nxt[k];
        load(unit + 4 * kItems);
        Item it;
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
            if (unit + k / kOct >= i1) break;
            const int r = r0 + 8 * (k % kOct);
            if (k % kOct == 0) {
                it = item_of(a, unit + k / kOct);
                if (it.tensor < 2 && (a.per_head || it.tensor != have)) {
                    load_weights(a.w[it.tensor], it.head, a.per_head, o, 1.f, w);
                    load_weights(a.b[it.tensor], it.head, a.per_head, o, -0.f, bias);
                    have = it.tensor;
                }
            }
            if (8 * (k % kOct) >= valid) continue;
            if (it.tensor < 2) {
                float x[8];
                unpack8(rows[k], x);
                (void)normalise(x, a.norm, a.eps);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = fmaf(x[e], w[e], bias[e]);
                if constexpr (ROT != 0) rotate<ROT>(x, table + r * kCsPitch, o, 0);
                rows[k] = packed8(x);
            }
            if (r < valid) *(uint4 *)((uint16_t *)pick(a.y, it.tensor) + out_off[r] + it.head * a.ohs + 8 * o) = rows[k];
        }
    }
}

// E4M3 outputs with query blocks of 64 SUB tokens; a workgroup takes 64 SUB tokens of one sequence, a unit is 64 tokens of one
// item.  With SUB = 2 two waves share an item, each with its half of the query block, and exchange the block's maximum through LDS.
// On 43968 tokens of 16 heads norm, rotation and their angles take 18 of 112 us that do not hide behind the copies, in the 64-row form, without the
// exchange, 5 of 96 (called without norm and rotation: 93 and 90).
// The codes are those of the fp32 quotient y / scale, as with the stand-alone quantiser: rounded once, to E4M3.  The scale of q and k can have any significand;
// for all 2^23 of them the three-step quotient is the division's wherever it lies within six units of a border between two codes (gone
// through on the host; tests/test_division_step_any_scale.py has a selection), and elsewhere a unit in its last place does not matter.
template <int ROT, int SUB>
__global__ __launch_bounds__(256, 3) void heads_e4m3_kernel(HeadsArgs a)
{
    constexpr int kTok = 64 * SUB, kAtOnce = 4 / SUB;
    __shared__ long in_off[kTok], out_off[kTok];
    __shared__ float red[2][4];
    __shared__ __attribute__((aligned(16))) float table[ROT ? kTok * kCsPitch : 4];
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63, o = channel_group(lane & 7), r0 = lane >> 3;
    const unsigned blk = blockIdx.x / (unsigned)a.splits, part = blockIdx.x - blk * (unsigned)a.splits;
    const unsigned per = (unsigned)(a.N + kTok - 1) / kTok;
    const int b = (int)(blk / per);
    const long first = (long)(blk - (unsigned)b * per) * kTok;
    const int valid = (int)min((long)kTok, a.N - first);
    lay_out_tokens<kTok, true>(a, b, first, valid, in_off, out_off, nullptr);

    const int sub = SUB == 2 ? wave & 1 : 0, row0 = 64 * sub + r0, mine = min(64, valid - 64 * sub);      // this wave's tokens
    const int i0 = (int)part * a.chunk, i1 = min(i0 + a.chunk, a.tensors * a.H);
    const int steps = (i1 - i0 + kAtOnce - 1) / kAtOnce, at0 = i0 + (SUB == 2 ? wave >> 1 : wave);
    uint4 rows[8];
    auto load = [&](int item) {
        if (item >= i1) return;
        const Item it = item_of(a, item);
        const uint16_t *const x = pick(a.x, it.tensor) + it.head * a.hs + 8 * o;
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (8 * k < mine) rows[k] = *(const uint4 *)(x + in_off[row0 + 8 * k]);
    };
    load(at0);
    if constexpr (ROT != 0) make_table(a, valid, [&](int r) { return (a.pos_per_item ? (long)b * a.N : 0) + first + min(r, valid - 1); }, table);
    for (int s = 0; s < steps; ++s) {
        const int item = at0 + s * kAtOnce;
        const bool active = item < i1 && mine > 0;
        const Item it = item_of(a, item);
        float y[8][8], amax = 0.f;
        if (active) {
            float w[8], bias[8];
            if (it.tensor < 2) {
                load_weights(a.w[it.tensor], it.head, a.per_head, o, 1.f, w);
                load_weights(a.b[it.tensor], it.head, a.per_head, o, -0.f, bias);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if (8 * k >= mine) continue;
                unpack8(rows[k], y[k]);
                if (it.tensor < 2) {
                    (void)normalise(y[k], a.norm, a.eps);
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[k][e] = fmaf(y[k][e], w[e], bias[e]);
                    if constexpr (ROT != 0) rotate<ROT>(y[k], table + (row0 + 8 * k) * kCsPitch, o, 0);
                }
#pragma unroll
                for (int e = 0; e < 8; e += 2) amax = fmaxf(amax, fmaxf(fabsf(y[k][e]), fabsf(y[k][e + 1])));
            }
            load(item + kAtOnce);                    // before this item's stores: a load behind a store would wait for it
        }
        amax = wave_max_dpp(amax);
        if constexpr (SUB == 2) {
            if (i0 + s * kAtOnce < a.H) {            // a step of queries, for all waves alike
                if (lane == 0) red[s & 1][wave] = active ? amax : 0.f;
                lds_barrier();
            }
            if (it.tensor == 0) amax = fmaxf(red[s & 1][wave], red[s & 1][wave ^ 1]);
        }
        if (!active) continue;
        const int span = it.tensor == 0 ? kTok : 64, nblk = (a.N + span - 1) / span;
        const float scale = fmaxf(amax, 1e-8f) / 448.0f;
        const int at = (int)(first / span) + (it.tensor == 0 ? 0 : sub);
        if (lane == 0 && (it.tensor != 0 || sub == 0)) pick(a.scales, it.tensor)[((size_t)b * a.H + it.head) * nblk + at] = scale;
        const BlockDivisor divide(scale);
        uint8_t *const out = (uint8_t *)pick(a.y, it.tensor) + it.head * a.ohs + 8 * o;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if (8 * k >= mine) continue;
#pragma unroll
            for (int e = 0; e < 8; ++e) y[k][e] = __builtin_amdgcn_fmed3f(divide(y[k][e]), -448.0f, 448.0f);       // NaN gives -448, as with the stand-alone quantiser
            if (r0 + 8 * k < mine)
                *(uint2 *)(out + out_off[row0 + 8 * k]) = make_uint2(pack_e4m3(y[k][0], y[k][1], y[k][2], y[k][3]), pack_e4m3(y[k][4], y[k][5], y[k][6], y[k][7]));
        }
    }
}

// Gradients.  a.x: the inputs; g: the gradients of the outputs, in their layout; dx: those of the inputs, in the inputs' strides.
// Sums over tokens for dw and db: in registers over a wave's units, over its eight tokens at a time at the end, over the four
// waves through LDS (weights shared by the heads) or not at all (weights of each head: a unit is one head's), then over the
// partials part[tensor][head or 0][slot][dw | db][64] in heads_grad_reduce_kernel: all in fp32 and in a fixed order.
// TOK as in heads_kernel; with weights of each head TOK is 64.
template <int ROT, int TOK>
__global__ __launch_bounds__(256, 3) void heads_grad_kernel(HeadsArgs a, HeadsGrads d)
{
    constexpr int kOct = TOK / 8, kItems = 64 / TOK;
    __shared__ long in_off[TOK], out_off[TOK];
    __shared__ int pos_row[TOK];
    __shared__ __attribute__((aligned(16))) float table[ROT ? TOK * kCsPitch : 4];
    __shared__ __attribute__((aligned(16))) float sums[4][2][128];
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63, o = channel_group(lane & 7), r0 = lane >> 3;
    const unsigned blk = blockIdx.x / (unsigned)a.splits, split = blockIdx.x - blk * (unsigned)a.splits;
    const long first = (long)blk * TOK;
    const int valid = (int)min((long)TOK, (long)a.B * a.N - first);
    lay_out_tokens<TOK, false>(a, 0, first, valid, in_off, out_off, pos_row);
    const int i0 = (int)split * a.chunk, i1 = min(i0 + a.chunk, a.tensors * a.H);
    const bool weights = d.part != nullptr;
    float dw[8], db[8];
    auto clear = [&] {
#pragma unroll
        for (int e = 0; e < 8; ++e) dw[e] = db[e] = 0.f;
    };
    auto flush = [&](float *to) {                    // the lanes of a channel group add up; the first eight write
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            dw[e] = group_sum(dw[e]);
            db[e] = group_sum(db[e]);
        }
        if (lane < 8) {
#pragma unroll
            for (int e = 0; e < 8; e += 4) {
                *(float4 *)(to + 8 * o + e) = make_float4(dw[e], dw[e + 1], dw[e + 2], dw[e + 3]);
                *(float4 *)(to + 64 + 8 * o + e) = make_float4(db[e], db[e + 1], db[e + 2], db[e + 3]);
            }
        }
        clear();
    };
    clear();
    int flushed = 0;                                 // tensors whose sums (shared weights) are in LDS
    // half units of four rows a lane: their eight loads are asked for before the half unit in front of them is stored
    uint4 xs[4], gs[4], nx[4], ng[4];
    auto load = [&](int unit, int half) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int k = 4 * half + j;
            if (8 * (k % kOct) < valid && unit + k / kOct < i1) {
                const Item it = item_of(a, unit + k / kOct);
                const int r = r0 + 8 * (k % kOct);
                ng[j] = *(const uint4 *)(pick(d.g, it.tensor) + it.head * a.ohs + 8 * o + out_off[r]);
                if (it.tensor < 2) nx[j] = *(const uint4 *)(a.x[it.tensor] + it.head * a.hs + 8 * o + in_off[r]);
            }
        }
    };
    load(i0 + wave * kItems, 0);
    if constexpr (ROT != 0) make_table(a, valid, [&](int r) { return (long)pos_row[r]; }, table);
    float w[8];
    int have = -1;                                   // tensor whose weights these are
    for (int unit = i0 + wave * kItems; unit < i1; unit += 4 * kItems) {
        Item it = item_of(a, unit);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
#pragma unroll
            for (int j = 0; j < 4; ++j) { xs[j] = nx[j]; gs[j] = ng[j]; }
            load(half ? unit + 4 * kItems : unit, half ^ 1);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int k = 4 * half + j, r = r0 + 8 * (k % kOct);
                if (unit + k / kOct >= i1) break;
                if (k % kOct == 0) {
                    it = item_of(a, unit + k / kOct);
                    if (weights && !a.per_head)
                        for (; flushed < min(it.tensor, 2); ++flushed) flush(sums[wave][flushed]);
                    if (it.tensor < 2 && (a.per_head || it.tensor != have)) {
                        load_weights(a.w[it.tensor], it.head, a.per_head, o, 1.f, w);
                        have = it.tensor;
                    }
                }
                if (8 * (k % kOct) >= valid) continue;
                uint4 res = gs[j];
                if (it.tensor < 2) {
                    float u[8], n[8];
                    unpack8(xs[j], u);
                    unpack8(gs[j], n);
                    const float rs = normalise(u, a.norm, a.eps);
                    if constexpr (ROT != 0) rotate<ROT>(n, table + r * kCsPitch, o, 1);
                    if (r < valid) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) { dw[e] = fmaf(n[e], u[e], dw[e]); db[e] += n[e]; }
                    }
                    if (a.norm != 0) {
                        float m = 0.f, c = 0.f;
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            n[e] *= w[e];
                            m += n[e];
                            c = fmaf(n[e], u[e], c);
                        }
                        m = a.norm == 2 ? row_sum(m) * (1.0f / 64.0f) : 0.f;
                        c = row_sum(c) * (1.0f / 64.0f);
#pragma unroll
                        for (int e = 0; e < 8; ++e) n[e] = rs * (fmaf(-u[e], c, n[e]) - m);
                    }
                    res = packed8(n);
                }
                if (r < valid) *(uint4 *)(pick(d.dx, it.tensor) + it.head * a.hs + 8 * o + in_off[r]) = res;
            }
        }
        if (TOK == 64 && weights && a.per_head && it.tensor < 2) flush(d.part + (((size_t)it.tensor * a.H + it.head) * d.slots + blk) * 128);
    }
    if (weights && !a.per_head) {
        for (; flushed < 2; ++flushed) flush(sums[wave][flushed]);
        __syncthreads();
        const int t = threadIdx.x >> 7, c = threadIdx.x & 127;
        d.part[((size_t)t * d.slots + blockIdx.x) * 128 + c] = (sums[0][t][c] + sums[1][t][c]) + (sums[2][t][c] + sums[3][t][c]);
    }
}

// dw, db of (tensor, head) = sum of its partials: slice s of a workgroup adds slots s, s + 64, ..., then the slices in order.
// A workgroup owns 16 of a partial's 128 columns, so that one pair of shared weights still gives 16 workgroups of 64 slices.
__global__ __launch_bounds__(1024) void heads_grad_reduce_kernel(const float *__restrict__ part, int slots, int heads, HeadsGrads d)
{
    __shared__ float sums[64][16];
    const int c = threadIdx.x & 15, s = threadIdx.x >> 4, col = (blockIdx.x & 7) * 16 + c;
    const int pair = blockIdx.x >> 3, tensor = pair / heads, head = pair - tensor * heads;
    const float *const p = part + (size_t)pair * slots * 128 + col;
    float v = 0.f;
#pragma unroll 4
    for (int k = s; k < slots; k += 64) v += p[(size_t)k * 128];
    sums[s][c] = v;
    __syncthreads();
    if (threadIdx.x < 16) {
        float t = 0.f;
        for (int k = 0; k < 64; ++k) t += sums[k][c];
        float *const out = col < 64 ? d.dw[tensor] : d.db[tensor];
        if (out) out[(size_t)head * 64 + (col & 63)] = t;
    }
}

namespace {
// Workgroups: the items of a block of tokens are split over several; each computes the block's angles anew.
// bf16 and gradients: into 4096 workgroups or what the items give.  us, by workgroups of a block of tokens, the rule's in brackets: bf16, 43968 tokens
// of 16 heads 1: 118, 2: 127, 4: 118, [6]: 110, 12: 113;  8 x 1374 tokens 1: 27, 2: 33, [3]: 28;  gradients with weights of each head, 2 x 6907 tokens of 12 heads
// 1: 59, 2: 53, 3: 41.5, 4: 41.6, 6: 46, [9]: 44;  43968 tokens of 16 heads 1: 159, 2: 178, [6]: 160, 12: 165;  1374 tokens 1: 72, 6: 22, [12]: 16;  with shared
// weights 2 x 6907 tokens 1: 39, 2: 54, [3]: 45;  43968 1: 157, [6]: 164, 12: 182;  1374 1: 25, [3]: 16.  So gradients of middle sizes lose up to 6 % by
// it, with shared weights 14 %; no one number of workgroups suits them all.
// E4M3: a CU holds three workgroups, and the angles of 128 tokens cost as much as four items, so whole rounds of 768 count: the
// number of parts with the shortest rounds.  43968 tokens of 16 heads, 128-row blocks 1: 130, [2]: 110, 3: 117, 4: 112, 6: 106, 12: 110;  64-row blocks [1]: 95,
// 2: 105, 3: 97, 6: 96;  8 x 1374 tokens, 64-row 1: 47, 2: 37, [4]: 29.5, 6: 30.7, 128-row 4: 42, [8]: 32.5, 12: 35;  10992 tokens of 12 heads, 128-row 3: 40,
// [6]: 29.5, 9: 31;  137400 tokens 1: 311, [2]: 305, 3: 281, 4: 295, 6: 281: where there are several rounds either way it gives up 4 to 8 %.
void split_items(HeadsArgs &a, long blocks, int at_once, bool rounds)
{
    const int items = a.tensors * a.H, most = (items + at_once - 1) / at_once;
    long parts = (4096 + blocks - 1) / blocks;
    if (rounds) {
        long best = 0x7FFFFFFFFFFFL;
        for (int s = 1; s <= most && (s == 1 || blocks * s <= 4 * 768); ++s) {
            const long cost = (blocks * s + 767) / 768 * ((most + s - 1) / s * at_once + 4);
            if (cost < best) { best = cost; parts = s; }
        }
    }
    parts = parts < 1 ? 1 : parts > most ? most : parts;
    a.chunk = (int)((items + parts - 1) / parts);
    a.chunk = (a.chunk + at_once - 1) / at_once * at_once;
    a.splits = (items + a.chunk - 1) / a.chunk;
}
int rotation_form(const HeadsArgs &a) { return a.axes == 0 ? 0 : a.adjacent ? 3 : a.axes; }
bool few_tokens(const HeadsArgs &a) { return (long)a.B * a.N < 64 * 512; }
long token_blocks(const HeadsArgs &a, int tok) { return ((long)a.B * a.N + tok - 1) / tok; }

template <int ROT> hipError_t launch_heads_rot(HeadsArgs a, int bq, hipStream_t st)
{
    // units of two rows a lane instead of eight where even those make few workgroups: one after the other in a wave they are latency
    // (32 tokens of 16 heads: 8.3 us and 5.9)
    const bool few = few_tokens(a), least = few && token_blocks(a, 16) * a.tensors * a.H <= 4 * 512;
    const int tok = bq ? bq : few ? 16 : 64;
    const long blocks = bq ? (long)a.B * ((a.N + tok - 1) / tok) : token_blocks(a, tok);
    split_items(a, blocks, bq == 128 ? 2 : bq || !few || least ? 4 : 16, bq != 0);
    const long grid = blocks * a.splits;
    if (grid > 0x7FFFFFFFL) return hipErrorInvalidValue;
    if (bq == 64)       heads_e4m3_kernel<ROT, 1><<<(unsigned)grid, 256, 0, st>>>(a);
    else if (bq == 128) heads_e4m3_kernel<ROT, 2><<<(unsigned)grid, 256, 0, st>>>(a);
    else if (least)     heads_kernel<ROT, 16, 2><<<(unsigned)grid, 256, 0, st>>>(a);
    else if (few)       heads_kernel<ROT, 16, 8><<<(unsigned)grid, 256, 0, st>>>(a);
    else                heads_kernel<ROT, 64, 8><<<(unsigned)grid, 256, 0, st>>>(a);
    return hipGetLastError();
}
// the plan of a gradient's launch: tokens of a workgroup, and the slots of its partial sums
int plan_grad(HeadsArgs &a, int &slots)
{
    const int tok = few_tokens(a) && !a.per_head ? 16 : 64;
    const long blocks = token_blocks(a, tok);
    slots = 0;
    if (!blocks) return tok;
    split_items(a, blocks, tok == 16 ? 16 : 4, false);
    slots = (int)(a.per_head ? blocks : blocks * a.splits);
    return tok;
}
template <int ROT> hipError_t launch_heads_grad_rot(HeadsArgs a, HeadsGrads d, hipStream_t st)
{
    const int tok = plan_grad(a, d.slots);
    if (a.B * (long)a.N) {
        const long grid = token_blocks(a, tok) * a.splits;
        if (grid > 0x7FFFFFFFL) return hipErrorInvalidValue;
        if (tok == 16) heads_grad_kernel<ROT, 16><<<(unsigned)grid, 256, 0, st>>>(a, d);
        else           heads_grad_kernel<ROT, 64><<<(unsigned)grid, 256, 0, st>>>(a, d);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (!d.part && !d.dw[0] && !d.dw[1] && !d.db[0] && !d.db[1]) return hipSuccess;
    const int heads = a.per_head ? a.H : 1;
    heads_grad_reduce_kernel<<<16u * heads, 1024, 0, st>>>(d.part, d.slots, heads, d);
    return hipGetLastError();
}
}  // namespace

size_t heads_grad_part_bytes(int B, int H, int N, int tensors, int per_head)
{
    HeadsArgs a = {};
    a.B = B; a.H = H; a.N = N; a.tensors = tensors; a.per_head = per_head;
    int slots;
    plan_grad(a, slots);
    return (size_t)2 * (per_head ? H : 1) * slots * 128 * sizeof(float);
}

hipError_t launch_heads(const HeadsArgs &a, int bq, hipStream_t st)
{
    switch (rotation_form(a)) {
    case 0: return launch_heads_rot<0>(a, bq, st);
    case 1: return launch_heads_rot<1>(a, bq, st);
    case 2: return launch_heads_rot<2>(a, bq, st);
    default: return launch_heads_rot<3>(a, bq, st);
    }
}
hipError_t launch_heads_grad(const HeadsArgs &a, const HeadsGrads &d, hipStream_t st)
{
    switch (rotation_form(a)) {
    case 0: return launch_heads_grad_rot<0>(a, d, st);
    case 1: return launch_heads_grad_rot<1>(a, d, st);
    case 2: return launch_heads_grad_rot<2>(a, d, st);
    default: return launch_heads_grad_rot<3>(a, d, st);
    }
}

}  // namespace sla
