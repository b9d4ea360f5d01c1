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
#define PC_MX4_NAN 255                // exponent of a block of keys that are NaN

// Tiles whose keys and values are laid out as a bf16 cache has them, for the kernels of many rows.
struct PcMx4Unpack {
    const int32_t *slots;             // [n_tiles] first slot of each
    int32_t        n_tiles;
    int32_t        n_kv_heads;
    int64_t        slots_from;        // capacity of the cache
    const void    *k_store, *v_store;
    void          *k_to, *v_to;       // [n_kv_heads][32 n_tiles][128], [n_kv_heads][4 n_tiles][128][8]
};
void pc_launch_mx4_unpack(const PcMx4Unpack &U, hipStream_t st);

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
// where word (m, db) of a value's dimension d stands in its group
__device__ __forceinline__ int mx4_word(int d) { return (d & 15) * 8 + (d >> 4); }
#endif

#endif
