// What lies between a qkv projection and the attention, in one pass over the data: the norm of every head's query and key
// rows over their 64 channels, the position rotation, and the layout (for the E4M3 path also the data type and the block
// scales) in which the attention takes Q, K and V; and the gradients of all of it.
//     u = (x - m) r,  n = u w + b             m = mean(x) (layer norm; 0 for the RMS norm),  r = 1 / sqrt(mean((x - m)^2) + eps)
//     y_i = n_i cos a - n_p sin a,  y_p = n_p cos a + n_i sin a      (i, p) a pair of channels, a = position base^(-2 i / S)
// backward, with d the gradient of n (that of y rotated back) and g = d w:
//     dx = r (g - mean(g) - u mean(g u))      (no mean(g) term for the RMS norm),   dw = sum d u,   db = sum d
//
// Unit of work: 64 tokens of one head of one tensor, a wave's.  Lane l holds channels 8 (l % 8) .. + 7 of token l / 8 + 8 k:
// a row is one 128-byte line, its sums are three cross-lane steps inside groups of eight lanes, the partner of a rotated
// channel is in the same lane or in one of the same eight, and the unit is a scale block of the E4M3 path.  The workgroup's
// four waves take neighbouring heads of the same tokens, so the lines of a token that lie side by side are read side by side,
// and the cosines and sines of those tokens are computed once, into LDS, for all heads and both tensors.
// All of it is bound by HBM: 2 bytes in, 2 (E4M3: 1) out per element; backward 4 in, 2 out.
#include "sla_common.hpp"
#include "sla_kernels.hpp"

#include <type_traits>

namespace sla {

namespace {
constexpr int kCsPitch = 68;                         // floats per token of the table: 32 cosines, 32 sines, one 16-byte step of padding

// value of lane l ^ X (X = 2 or 4)
template <int X> __device__ __forceinline__ float lane_xor(float v)
{
    int u = (int)__float_as_uint(v);
    if constexpr (X == 2) u = __builtin_amdgcn_mov_dpp(u, 0x4E, 0xf, 0xf, true);               // quad_perm [2,3,0,1]
    else {
        u = __builtin_amdgcn_mov_dpp(u, 0x141, 0xf, 0xf, true);                                // l -> 7 - l within eight
        u = __builtin_amdgcn_mov_dpp(u, 0x1B, 0xf, 0xf, true);                                 // and back within each four
    }
    return __uint_as_float((uint32_t)u);
}

// sum over the eight lanes of a row, in all of them
__device__ __forceinline__ float row_sum(float v)
{
    auto step = [](float a, auto ctrl) { return a + __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(a), decltype(ctrl)::value, 0xf, 0xf, true)); };
    v = step(v, std::integral_constant<int, 0xB1>{});
    v = step(v, std::integral_constant<int, 0x4E>{});
    return step(v, std::integral_constant<int, 0x141>{});
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

// n rotated by the angles of its token (dir = 1) or back (dir = -1); o = the lane's group of eight channels, cs = the token's
// row of the table.  ROT: 1 = channels (i, i + 32) are a pair, 2 = (i, i + 16) within each half of 32, 3 = (2 i, 2 i + 1)
template <int ROT> __device__ __forceinline__ void rotate(float (&n)[8], const float *cs, int o, float dir)
{
    if constexpr (ROT == 1 || ROT == 2) {
        const int at = ROT == 1 ? 8 * (o & 3) : 16 * (o >> 2) + 8 * (o & 1);
        const float sign = (o & (ROT == 1 ? 4 : 2)) ? dir : -dir;
        float c[8], s[8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            *(float4 *)(c + 4 * h) = *(const float4 *)(cs + at + 4 * h);
            *(float4 *)(s + 4 * h) = *(const float4 *)(cs + 32 + at + 4 * h);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float p = lane_xor<ROT == 1 ? 4 : 2>(n[e]);
            n[e] = fmaf(n[e], c[e], p * (s[e] * sign));
        }
    } else if constexpr (ROT == 3) {
        const float4 c4 = *(const float4 *)(cs + 4 * o), s4 = *(const float4 *)(cs + 32 + 4 * o);
        const float c[4] = {c4.x, c4.y, c4.z, c4.w}, s[4] = {s4.x, s4.y, s4.z, s4.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float a = n[2 * i], b = n[2 * i + 1], t = s[i] * dir;
            n[2 * i] = fmaf(a, c[i], -(b * t));
            n[2 * i + 1] = fmaf(b, c[i], a * t);
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
    const float r = 1.0f / sqrtf(fmaf(row_sum(s), 1.0f / 64.0f, eps));
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= r;
    return r;
}

// Where the rows of the workgroup's tokens lie, and their angles.  TOK tokens; those past `valid` repeat the last one.
// SEQ: the tokens are one sequence's (b, first ..), else they run through all sequences.
template <int TOK, bool SEQ, bool TABLE>
__device__ __forceinline__ void lay_out_tokens(const HeadsArgs &a, int b, long first, int valid, long *in_off, long *out_off, int *pos_row, float *table)
{
    const int tid = threadIdx.x;
    if (tid < TOK) {
        const long f = first + min(tid, valid - 1);
        const int item = SEQ ? b : (int)((unsigned)f / (unsigned)a.N), t = SEQ ? (int)f : (int)f - item * a.N;
        in_off[tid] = item * a.bs + t * a.ts;
        out_off[tid] = item * a.obs + t * a.ots;
        pos_row[tid] = a.pos_per_item ? item * a.N + t : t;
    }
    __syncthreads();
    if constexpr (TABLE) {
        // the angle in turns, reduced in 64 bits: a position of 2^31 still leaves 2^-23 of a turn
        const int j = tid & 31, per = 32 / a.axes, axis = j / per;
        const double turn = a.turn[j];
        const int rows = (valid + 7) & ~7;           // whole groups of eight: the rows behind the last one repeat it, here too
        for (int r = tid >> 5; r < rows; r += 8) {
            double u = (double)a.pos[(size_t)pos_row[r] * a.axes + axis] * turn;
            u -= rint(u);
            float s, c;
            sincospif(2.0f * (float)u, &s, &c);
            table[r * kCsPitch + j] = c;
            table[r * kCsPitch + 32 + j] = s;
        }
        __syncthreads();
    }
}

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

// OUT: 0 = bf16; 1, 2 = E4M3 with query blocks of 64 OUT tokens.  An E4M3 workgroup takes 64 OUT tokens of one sequence: with
// OUT = 2 two waves share a head, each with its half of the query block, and exchange the block's maximum through LDS.
// The codes are those of y in fp32: the quotient by the scale is rounded once, to E4M3.
template <int ROT, int OUT>
__global__ __launch_bounds__(256) void heads_kernel(HeadsArgs a)
{
    constexpr int kSub = OUT == 2 ? 2 : 1, kTok = 64 * kSub, kAtOnce = 4 / kSub;
    __shared__ long in_off[kTok], out_off[kTok];
    __shared__ int pos_row[kTok];
    __shared__ float red[2][4];
    __shared__ __attribute__((aligned(16))) float table[ROT ? kTok * kCsPitch : 4];
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63, o = lane & 7, r0 = lane >> 3;
    const unsigned blk = blockIdx.x / (unsigned)a.splits, part = blockIdx.x - blk * (unsigned)a.splits;
    int b = 0, valid;                                // tokens of the workgroup
    long first;
    if constexpr (OUT == 0) {
        first = (long)blk * kTok;
        valid = (int)min((long)kTok, (long)a.B * a.N - first);
    } else {
        const unsigned per = (unsigned)(a.N + kTok - 1) / kTok;
        b = (int)(blk / per);
        first = (long)(blk - (unsigned)b * per) * kTok;
        valid = (int)min((long)kTok, a.N - first);
    }
    lay_out_tokens<kTok, OUT != 0, ROT != 0>(a, b, first, valid, in_off, out_off, pos_row, table);

    const int sub = kSub == 2 ? wave & 1 : 0, row0 = 64 * sub + r0, mine = min(64, valid - 64 * sub);      // this wave's tokens
    const int i0 = (int)part * a.chunk, i1 = min(i0 + a.chunk, a.tensors * a.H);
    const int steps = (i1 - i0 + kAtOnce - 1) / kAtOnce, at0 = i0 + (kSub == 2 ? wave >> 1 : wave);
    uint4 cur[8], nxt[8];
    auto load = [&](int item, uint4 (&into)[8]) {
        if (item >= i1) return;
        const int tensor = item / a.H, head = item - tensor * a.H;
        const uint16_t *const x = (tensor == 0 ? a.x[0] : tensor == 1 ? a.x[1] : a.x[2]) + head * a.hs + 8 * o;
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (8 * k < mine) into[k] = *(const uint4 *)(x + in_off[row0 + 8 * k]);
    };
    load(at0, nxt);
    for (int s = 0; s < steps; ++s) {
        const int item = at0 + s * kAtOnce;
#pragma unroll
        for (int k = 0; k < 8; ++k) cur[k] = nxt[k];
        load(item + kAtOnce, nxt);
        const bool active = item < i1 && mine > 0;
        const int tensor = item / a.H, head = item - tensor * a.H;
        float w[8], bias[8], y[OUT ? 8 : 1][8], amax = 0.f;
        if (active && tensor < 2) {
            load_weights(tensor ? a.w[1] : a.w[0], head, a.per_head, o, 1.f, w);
            load_weights(tensor ? a.b[1] : a.b[0], head, a.per_head, o, 0.f, bias);
        }
        const long out_head = head * a.ohs + 8 * o;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if (!active || 8 * k >= mine) continue;
            float x[8];
            unpack8(cur[k], x);
            if (tensor < 2) {
                (void)normalise(x, a.norm, a.eps);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = fmaf(x[e], w[e], bias[e]);
                if constexpr (ROT != 0) rotate<ROT>(x, table + (row0 + 8 * k) * kCsPitch, o, 1.f);
            }
            if constexpr (OUT == 0) {
                if (r0 + 8 * k < mine) *(uint4 *)((uint16_t *)(tensor == 0 ? a.y[0] : tensor == 1 ? a.y[1] : a.y[2]) + out_off[row0 + 8 * k] + out_head) = tensor < 2 ? packed8(x) : cur[k];
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    y[k][e] = x[e];
                    amax = fmaxf(amax, fabsf(x[e]));
                }
            }
        }
        if constexpr (OUT != 0) {
            amax = wave_max_dpp(amax);
            if constexpr (kSub == 2) {
                if (lane == 0) red[s & 1][wave] = active ? amax : 0.f;
                __syncthreads();
                if (tensor == 0) amax = fmaxf(red[s & 1][wave], red[s & 1][wave ^ 1]);
            }
            if (!active) continue;
            const int span = tensor == 0 ? kTok : 64, nblk = (a.N + span - 1) / span;
            const float scale = fmaxf(amax, 1e-8f) / 448.0f;
            float *const scales = tensor == 0 ? a.scales[0] : tensor == 1 ? a.scales[1] : a.scales[2];
            const int at = (int)(first / span) + (tensor == 0 ? 0 : sub);
            if (lane == 0 && (tensor != 0 || sub == 0)) scales[((size_t)b * a.H + head) * nblk + at] = scale;
            const BlockDivisor divide(scale);
            uint8_t *const out = (uint8_t *)(tensor == 0 ? a.y[0] : tensor == 1 ? a.y[1] : a.y[2]) + out_head;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if (8 * k >= mine) continue;
#pragma unroll
                for (int e = 0; e < 8; ++e) y[k][e] = fminf(fmaxf(divide(y[k][e]), -448.0f), 448.0f);
                if (r0 + 8 * k < mine)
                    *(uint2 *)(out + out_off[row0 + 8 * k]) = make_uint2(pack_e4m3(y[k][0], y[k][1], y[k][2], y[k][3]), pack_e4m3(y[k][4], y[k][5], y[k][6], y[k][7]));
            }
        }
    }
}

// Gradients.  a.x: the inputs; g: the gradients of the outputs, in their layout; dx: those of the inputs, in the inputs' strides.
// Sums over tokens for dw and db: in registers over a wave's units, over its eight tokens at a time at the end, over the four
// waves through LDS (weights shared by the heads) or not at all (weights of each head: a unit is one head's), then over the
// partials part[tensor][head or 0][slot][dw | db][64] in heads_grad_reduce_kernel: all in fp32 and in a fixed order.
template <int ROT>
__global__ __launch_bounds__(256) void heads_grad_kernel(HeadsArgs a, HeadsGrads d)
{
    __shared__ long in_off[64], out_off[64];
    __shared__ int pos_row[64];
    __shared__ __attribute__((aligned(16))) float table[ROT ? 64 * kCsPitch : 4];
    __shared__ __attribute__((aligned(16))) float sums[4][2][128];
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63, o = lane & 7, r0 = lane >> 3;
    const unsigned blk = blockIdx.x / (unsigned)a.splits, split = blockIdx.x - blk * (unsigned)a.splits;
    const long first = (long)blk * 64;
    const int valid = (int)min(64L, (long)a.B * a.N - first);
    lay_out_tokens<64, false, ROT != 0>(a, 0, first, valid, in_off, out_off, pos_row, table);
    const int i0 = (int)split * a.chunk, i1 = min(i0 + a.chunk, a.tensors * a.H);
    const bool weights = d.part != nullptr;
    float dw[8], db[8];
    auto clear = [&] {
#pragma unroll
        for (int e = 0; e < 8; ++e) dw[e] = db[e] = 0.f;
    };
    auto flush = [&](float *to) {                    // the lanes of a channel group add up; lanes 0 .. 7 write
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
            for (int x = 8; x < 64; x <<= 1) {
                dw[e] += __shfl_xor(dw[e], x, 64);
                db[e] += __shfl_xor(db[e], x, 64);
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
    for (int item = i0 + wave; item < i1; item += 4) {
        const int tensor = item / a.H, head = item - tensor * a.H;
        if (weights && !a.per_head)
            for (; flushed < min(tensor, 2); ++flushed) flush(sums[wave][flushed]);
        const uint16_t *const x = (tensor == 0 ? a.x[0] : a.x[1]) + head * a.hs + 8 * o;
        const uint16_t *const g = (tensor == 0 ? d.g[0] : tensor == 1 ? d.g[1] : d.g[2]) + head * a.ohs + 8 * o;
        uint16_t *const dx = (tensor == 0 ? d.dx[0] : tensor == 1 ? d.dx[1] : d.dx[2]) + head * a.hs + 8 * o;
        float w[8];
        if (tensor < 2) load_weights(tensor ? a.w[1] : a.w[0], head, a.per_head, o, 1.f, w);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            if (32 * half >= valid) continue;
            uint4 xs[4], gs[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int r = r0 + 8 * k + 32 * half;
                gs[k] = *(const uint4 *)(g + out_off[r]);
                if (tensor < 2) xs[k] = *(const uint4 *)(x + in_off[r]);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int r = r0 + 8 * k + 32 * half;
                uint4 res = gs[k];
                if (tensor < 2) {
                    float u[8], n[8];
                    unpack8(xs[k], u);
                    unpack8(gs[k], n);
                    const float rs = normalise(u, a.norm, a.eps);
                    if constexpr (ROT != 0) rotate<ROT>(n, table + r * kCsPitch, o, -1.f);
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
                if (r < valid) *(uint4 *)(dx + in_off[r]) = res;
            }
        }
        if (weights && a.per_head && tensor < 2) flush(d.part + (((size_t)tensor * a.H + head) * d.slots + blk) * 128);
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
    const int c = threadIdx.x & 15, s = threadIdx.x >> 4, col = blockIdx.x * 16 + c;
    const int tensor = blockIdx.y / heads, head = blockIdx.y - tensor * heads;
    const float *const p = part + (size_t)blockIdx.y * slots * 128 + col;
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
// Workgroups: the heads of a block of tokens are split over several until there are about four for every CU; each computes
// the block's angles anew (an eighth of the work on one head, nothing beside the traffic of a dozen).
void split_items(HeadsArgs &a, long blocks, int at_once)
{
    const int items = a.tensors * a.H, most = (items + at_once - 1) / at_once;
    long want = (1024 + blocks - 1) / blocks;
    want = want < 1 ? 1 : want > most ? most : want;
    a.chunk = (int)((items + want - 1) / want);
    a.chunk = (a.chunk + at_once - 1) / at_once * at_once;
    a.splits = (items + a.chunk - 1) / a.chunk;
}
int rotation_form(const HeadsArgs &a) { return a.axes == 0 ? 0 : a.adjacent ? 3 : a.axes; }

template <int ROT> hipError_t launch_heads_rot(HeadsArgs a, int bq, hipStream_t st)
{
    const int tok = bq == 128 ? 128 : 64;
    const long blocks = bq == 0 ? ((long)a.B * a.N + 63) / 64 : (long)a.B * ((a.N + tok - 1) / tok);
    split_items(a, blocks, bq == 128 ? 2 : 4);
    const long grid = blocks * a.splits;
    if (grid > 0x7FFFFFFFL) return hipErrorInvalidValue;
    if (bq == 0)       heads_kernel<ROT, 0><<<(unsigned)grid, 256, 0, st>>>(a);
    else if (bq == 64) heads_kernel<ROT, 1><<<(unsigned)grid, 256, 0, st>>>(a);
    else               heads_kernel<ROT, 2><<<(unsigned)grid, 256, 0, st>>>(a);
    return hipGetLastError();
}
template <int ROT> hipError_t launch_heads_grad_rot(HeadsArgs a, HeadsGrads d, hipStream_t st)
{
    const long blocks = ((long)a.B * a.N + 63) / 64;
    if (blocks) {
        split_items(a, blocks, 4);
        if (blocks * a.splits > 0x7FFFFFFFL) return hipErrorInvalidValue;
        d.slots = (int)(a.per_head ? blocks : blocks * a.splits);
        heads_grad_kernel<ROT><<<(unsigned)(blocks * a.splits), 256, 0, st>>>(a, d);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    } else d.slots = 0;
    if (!d.part && !d.dw[0] && !d.dw[1] && !d.db[0] && !d.db[1]) return hipSuccess;
    const int heads = a.per_head ? a.H : 1;
    heads_grad_reduce_kernel<<<dim3(8, 2 * heads), 1024, 0, st>>>(d.part, d.slots, heads, d);
    return hipGetLastError();
}
}  // namespace

size_t heads_grad_part_bytes(int B, int H, int N, int tensors, int per_head)
{
    const long blocks = ((long)B * N + 63) / 64;
    if (!blocks) return 0;
    HeadsArgs a = {};
    a.H = H; a.tensors = tensors;
    split_items(a, blocks, 4);
    return (size_t)2 * (per_head ? (size_t)H * blocks : (size_t)blocks * a.splits) * 128 * sizeof(float);
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
