// What the matrix products share: copies of scales and the store of a wave's tile.
#pragma once
#include "sla_common.hpp"

namespace sla {

// Row and column of a tile among `cols` tiles to a row of `rows`: along the rows, or, where these are longer than eight, eight rows at a time and
// down the columns: workgroups that run side by side on an XCD then share rows and columns.  us, along the rows and by eights: gradients of 1374 x 4096 -> 1152
// 64.8, 53.9, 4096 x 4096 -> 1152 121.5, 106.0, 43968 x 4096 -> 2048 1277, 1255, 4096 x 6144 -> 8192 741, 763, the others within 2 % or faster; 4-bit products of
// 4096 x 1024 -> 8192 41.8, 35.8, 43968 x 512 -> 8192 249, 229, 1374 x 2048 -> 2048 12.3, 13.3, 4096 x 512 -> 4096 16.6, 17.6, 43968 x 8192 -> 2048 532, 532.
struct TileAt { int row, col; };
__device__ __forceinline__ TileAt tile_at(int item, int rows, int cols)
{
    const int row = (int)((unsigned)item / (unsigned)cols);
    if (cols <= 8) return {row, item - row * cols};
    const int first = row & ~7, in = item - first * cols, high = min(8, rows - first), col = (int)((unsigned)in / (unsigned)high);
    return {first + in - col * high, col};
}

// two copies of 1 KB as copy_1k_to_lds makes them, the second 1 KB behind the first in LDS: four scalar instructions less
__device__ __forceinline__ void copy_2k_to_lds(const uint8_t *base, uint32_t voff0, uint32_t voff1, uint32_t lds_addr)
{
    uint32_t saved_m0;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %4\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %3\n\ts_add_u32 m0, m0, 0x400\n\ts_nop 0\n\t"
                 "global_load_lds_dwordx4 %2, %3\n\ts_mov_b32 m0, %0"
                 : "=&s"(saved_m0) : "v"(voff0), "v"(voff1), "s"(base), "s"(lds_addr) : "memory", "scc");
}

// 256 bytes global -> LDS: lane l moves the dword at base + voff(l) to LDS byte lds_addr + 4 l (otherwise as copy_1k_to_lds)
__device__ __forceinline__ void copy_256_to_lds(const uint8_t *base, uint32_t voff, uint32_t lds_addr)
{
    uint32_t saved_m0;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %3\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2\n\ts_mov_b32 m0, %0"
                 : "=&s"(saved_m0) : "v"(voff), "s"(base), "s"(lds_addr) : "memory");
}

// Bytes of LDS of its own that a wave needs for store_tile
template <int TN> constexpr int kStoreBytes = 32 * (64 * TN + 16);

// A wave's tile of 32 TM rows x 32 TN columns to bf16 memory, rows `pitch` elements apart, C at its first element; rows_left and
// cols_left (a multiple of 8) of it are there.  value(a, b, q, v): columns 32 a + 8 q + 4 g .. + 3 of row 32 b + l % 32, g = l / 32, as the
// matrix unit leaves them.  Thirty-two rows at a time go through LDS, so that every store is of whole 64 TN bytes of a row: straight
// from the registers it would be thirty-two bytes of each of 32 rows.  16 bytes of padding a row: 16 rows' pieces in different banks.
template <int TM, int TN, class Value>
__device__ __forceinline__ void store_tile(uint8_t *lds, Value value, int lane, int rows_left, int cols_left, uint16_t *C, size_t pitch)
{
    constexpr int kPitch = 64 * TN + 16, kLanes = 4 * TN, kRows = 64 / kLanes;   // lanes to a row, rows to a store
    const int l32 = lane & 31, g = lane >> 5, c = lane % kLanes, r0 = lane / kLanes;
#pragma unroll
    for (int b = 0; b < TM; ++b) {
#pragma unroll
        for (int a = 0; a < TN; ++a)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float v[4];
                value(a, b, q, v);
                *(i32x2 *)(lds + l32 * kPitch + (32 * a + 8 * q + 4 * g) * 2) = i32x2{(int)pack_bf16(v[0], v[1]), (int)pack_bf16(v[2], v[3])};
            }
        wave_lds_sync();
#pragma unroll
        for (int r = r0; r < 32; r += kRows) {
            const i32x4 u = *(const i32x4 *)(lds + r * kPitch + c * 16);
            if (32 * b + r < rows_left && 8 * c < cols_left) *(i32x4 *)(C + (size_t)(32 * b + r) * pitch + 8 * c) = u;
        }
        wave_lds_sync();
    }
}

}  // namespace sla
