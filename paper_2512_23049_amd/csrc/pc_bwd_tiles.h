// LDS tiles of the gradients' kernels (gfx950): the same tile read by row and by column.
#ifndef PC_BWD_TILES_H_
#define PC_BWD_TILES_H_

#include "pc_pieces.h"

#define MFMA32(a, b, c) __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0)
#define TILE_BYTES 8192

namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef const __attribute__((address_space(3))) bf16x8 *lds_frag;
typedef __attribute__((address_space(3))) s16x4 *lds_tr;

__device__ __forceinline__ float ex2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ bf16x8 frag4(uint32_t a, uint32_t b, uint32_t c, uint32_t d) { return __builtin_bit_cast(bf16x8, make_uint4(a, b, c, d)); }
__device__ __forceinline__ bf16x8 read_tr(unsigned at0, unsigned at1)       // rows 0..3 and 4..7 of the lane's column
{
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_tr)(uintptr_t)at0);
    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_tr)(uintptr_t)at1);
    const uint2 x = __builtin_bit_cast(uint2, a), y = __builtin_bit_cast(uint2, b);
    return frag4(x.x, x.y, y.x, y.y);
}
template <int N> __device__ __forceinline__ void wait_vm() { __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | ((N >> 4) << 14)); }
__device__ __forceinline__ void ring_barrier() { asm volatile("s_barrier" ::: "memory"); }

// Swizzle of a row-major tile [32 rows][16 chunks of 16 bytes]: chunk c of row r sits at position c ^ swz(r).  The
// 16 rows of a fragment read hit different banks, and so do the 4 consecutive rows of a transposing one.
__device__ __forceinline__ int swz(int r) { return ((r & 3) << 2) | ((r >> 2) & 3); }

// Fragment addresses of a row-major tile at LDS offset `tile`:
//   by row:    lane's row `row` (any), dims 16 ks + 8 hh + 0..7
//   by column: lane's dim 32 db + (lane & 31), rows 16 s + 8 hh + 0..7
struct RowMajor {
    unsigned row_at, col_at[2];
    __device__ RowMajor(int row, int lane)
    {
        const int hh = lane >> 5, nh = (lane >> 4) & 1, l = lane & 15;
        row_at = (unsigned)(row * 256 + ((hh ^ swz(row)) << 4));
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int key = 8 * hh + 4 * e + (l >> 2);
            col_at[e] = (unsigned)(key * 256 + (((2 * nh + ((l & 3) >> 1)) ^ swz(key)) << 4) + (l & 1) * 8);
        }
    }
    __device__ bf16x8 by_row(unsigned tile, int ks) const { return *(lds_frag)(uintptr_t)((row_at ^ (ks << 5)) + tile); }
    __device__ bf16x8 by_col(unsigned tile, int s, int db) const
    {
        return read_tr((col_at[0] ^ (db << 6)) + tile + s * 4096, (col_at[1] ^ (db << 6)) + tile + s * 4096);
    }
    // the same with the addresses of a tile made once: `at` the tile's position behind them, a constant
    struct Cols { unsigned base[4][2]; };
    __device__ Cols cols(unsigned tile) const
    {
        Cols c;
#pragma unroll
        for (int db = 0; db < 4; ++db)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                c.base[db][e] = (col_at[e] ^ (db << 6)) + tile;
                asm volatile("" : "+v"(c.base[db][e]));  // (or every read gets an addition of its own)
            }
        return c;
    }
    static __device__ bf16x8 by_col(const Cols &c, unsigned at, int s, int db) { return read_tr(c.base[db][0] + (at + s * 4096), c.base[db][1] + (at + s * 4096)); }
};
// the row of the first product's left operand this lane reads: rows are permuted so that result registers 0..7 / 8..15
// of a lane are rows 8 hh + 0..7 / 16 + 8 hh + 0..7, the order in which the second product takes them
__device__ __forceinline__ int perm_row(int n) { return 16 * (n >> 4) + 8 * ((n >> 2) & 1) + 4 * ((n >> 3) & 1) + (n & 3); }

// Values by key from a tile in the V store's order, [4 groups][128 dims][8 keys], chunk (group, dim) at position
// 128 group + (dim ^ 4 (group & 1)): lane's key, dims 16 ks + 8 hh + 0..7.  PERM: the lane's key is perm_row(lane & 31).
template <bool PERM>
struct ValuesByKey {
    unsigned at[2];
    __device__ ValuesByKey(int lane)
    {
        const int hh = lane >> 5, nh = (lane >> 4) & 1, l = lane & 15, c4 = l & 3;
        const int grp = 2 * nh + (PERM ? (c4 & 1) : (c4 >> 1)), half = PERM ? (c4 >> 1) : (c4 & 1);
#pragma unroll
        for (int e = 0; e < 2; ++e) at[e] = (unsigned)((grp * 128 + 8 * hh + 4 * (e ^ (grp & 1)) + (l >> 2)) * 16 + half * 8);
    }
    __device__ bf16x8 get(unsigned tile, int ks) const { return read_tr(at[0] + tile + ks * 256, at[1] + tile + ks * 256); }
};
__device__ __forceinline__ int v_src_chunk(int pos) { return (pos & ~127) | ((pos & 127) ^ (4 * ((pos >> 7) & 1))); }   // what belongs at a position

}  // namespace

#endif
