// How a PC_MX4 cache holds keys and values, and the launch wrappers of what reads them (internal to the library).
//
// A head's row of 128 values is four blocks of 32.  A block is a power of two 2^e, the least with max|x| < 7 2^e (-60 <= e <= 60),
// and a 4-bit code for each value: sign, and one of {0, 1/2, 1, 3/2, 2, 3, 4, 6} 2^e, the nearest (ties to the even code; 6.5 and
// above would be 8, which there is not: 6).  Tiles of 32 slots follow each other for each KV head, 68 bytes a slot:
//   keys    [32 slots][4 blocks][16 bytes] codes (the first value in the low half of a byte), then [32 slots][4 blocks] exponents e + 127
//   values  [4 groups of 8 slots][16 m][8 db] words, word (m, db): value 16 db + m of the eight slots, the first slot lowest;
//           then [4 groups][4 blocks][8 slots] exponents 60 - e
// so that a lane's part of a key (a block) and of the values (a dimension's eight slots) is what the matrix instructions take from it.
// The values that codes stand for are exact in bf16.  A token whose key or value holds an infinity or a NaN has keys of exponent 255
// (NaN) in that head: rows that see it are NaN there, and others do not notice.
#ifndef PC_MX4_H_
#define PC_MX4_H_

#include "pc_internal.h"

#define PC_MX4_ROW 68                 // bytes of a slot's key or value of one KV head
#define PC_MX4_CODES 2048             // bytes of codes in a tile of keys or of values
#define PC_MX4_TILE (PC_TILE * PC_MX4_ROW)
#define PC_MX4_E_MAX 60
#define PC_MX4_HALF 13                // exponents from -13 to 13: the values are exact, and normal numbers, in fp16
#define PC_MX4_COPIED 24              // exponents of values that a long prefill's walk over a copy takes, at most
#define PC_MX4_NAN 255                // exponent of a block of keys that are NaN

struct PcWin;
// Rows of prompts: what a launch makes in front of their attention.
struct PcMx4Prepare {
    const void   *from;               // the call's lists (n16 pieces of 16 bytes), or null: in the arguments
    void         *ws;                 // where they go
    int32_t       n16;
    int32_t       off_q_pos, off_rot, off_tiles;      // within them: positions (int32), runs' rotations (int64), first slots of the tiles that rows see (int32)
    int32_t       n_rows, n_rot, n_tiles;
    int32_t       n_q_heads, n_kv_heads;
    float         scale_log2;         // rides on the queries
    _Float16     *rot_run;            // [n_rot][2][64]: cosines and sines of their turns back
    const void   *q;
    uint2        *q_abs;              // queries turned by their positions, in their units, fp16 (see mx4_query_at)
    float        *q_unit;             // [n_q_heads][rows, rounded up to 32]: 2^e
    const double *inv_freq;
    int64_t       slots;
    const void   *v_store;
    void         *v_to;               // [n_kv_heads][4 n_tiles][128][8]: the tiles' values as a bf16 cache has them, or so in fp16
    int32_t       list_blocks, query_blocks;          // of the grid
    const uint32_t *mark;             // null, or: nothing is done unless *mark is mark_value
    uint32_t      mark_value;
    const uint32_t *bf16_only;        // not 0: some values of the cache are outside fp16
};
void pc_launch_mx4_prepare(PcMx4Prepare P, const PcArgBlob *blob, hipStream_t st);
// What the attention of rows needs besides PcWin (whose v_store and rot_q are not read).
struct PcMx4Rows {
    const uint2   *q_abs;
    const uint32_t *rot_run;          // (pairs)
    const float   *q_unit;
    const int32_t *places;            // of each run: what is added to a slot for its place among v_tiles' slots
    const void    *v_tiles;
    int64_t        v_slots;
    int32_t        n_rows;
    uint32_t       mark_value;        // as in PcMx4Prepare
    const uint32_t *mark, *bf16_only; // (as there)
};
void pc_launch_win_prefill_mx4(const PcWin &W, const PcMx4Rows &M, int n_items, hipStream_t st);

#ifdef __HIPCC__
// the code of |x| 2^-e (a, not NaN), without its sign
__device__ __forceinline__ uint32_t mx4_code(float a)
{
    a = fminf(a, 8.f);
    const float per = a < 2.f ? 2.f : a < 4.f ? 1.f : 0.5f;          // codes a unit
    const int from = a < 2.f ? 0 : a < 4.f ? 2 : 4;
    return (uint32_t)min((int)__builtin_rintf(a * per) + from, 7);
}
__device__ __forceinline__ uint32_t mx4_code(double a)
{
    a = fmin(a, 8.);
    const double per = a < 2. ? 2. : a < 4. ? 1. : 0.5;
    const int from = a < 2. ? 0 : a < 4. ? 2 : 4;
    return (uint32_t)min((int)__builtin_rint(a * per) + from, 7);
}
// e of a block whose largest magnitude is top: top = m 2^x with m in [1/2, 1) is below 7 2^(x - 3) where m < 7/8
__device__ __forceinline__ int mx4_exponent(float top)
{
    const uint32_t b = __float_as_uint(top);
    const int e = (int)(b >> 23 & 255) - 126 - 3 + ((b >> 21 & 3) == 3);
    return max(-PC_MX4_E_MAX, min(PC_MX4_E_MAX, e));
}
__device__ __forceinline__ int mx4_exponent(double top)
{
    const uint32_t b = (uint32_t)__double2hiint(top);
    const int e = (int)(b >> 20 & 2047) - 1022 - 3 + ((b >> 18 & 3) == 3);
    return max(-PC_MX4_E_MAX, min(PC_MX4_E_MAX, e));
}
__device__ __forceinline__ float mx4_power(float, int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
__device__ __forceinline__ double mx4_power(double, int e) { return __hiloint2double((int)((uint32_t)(e + 1023) << 20), 0); }
// what a code (in the low bits) stands for under 2^e
__device__ __forceinline__ float mx4_value(uint32_t code, int e)
{
    const uint32_t m = code & 7;
    const float a = m < 4 ? 0.5f * (float)m : m < 6 ? (float)m - 2.f : 2.f * (float)m - 8.f;
    return (code & 8 ? -a : a) * mx4_power(0.f, e);
}
// Where a query's dims stand among those that are turned by their positions: four of them (lane half hh, s = 0..3: 16 hh + 4 s, s = 4..7:
// 32 + 16 hh + 4 (s - 4), s + 8: 64 further), rows side by side.  So lanes have what the matrix instruction takes from them as bytes
// (its k of a half hh: 16 hh to 16 hh + 15, and 32 further), and a pair of a turn is in one lane.
__device__ __forceinline__ int64_t mx4_query_at(int64_t groups, int h, int64_t R, int hh, int s) { return ((h * groups + (R >> 5)) * 16 + s) * 64 + hh * 32 + (R & 31); }
// where word (m, db) of a value's dimension d stands in its group
__device__ __forceinline__ int mx4_word(int d) { return (d & 15) * 8 + (d >> 4); }
#endif

#endif
