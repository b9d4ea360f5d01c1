// What the kernels that read a PC_MX4 cache multiply with (gfx950): codes by 8-bit pieces of queries, values by probabilities.
#ifndef PC_MX4_PRODUCTS_H_
#define PC_MX4_PRODUCTS_H_

#include "pc_mx4.h"
#include "pc_mfma_common.h"

#include <type_traits>

#define MFMA16(a, b, c) __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0)

typedef int mx4_i32x8 __attribute__((ext_vector_type(8)));
typedef uint16_t mx4_u16x2 __attribute__((ext_vector_type(2)));
typedef short mx4_s16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float ex2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ int imax3(int a, int b, int c) { return max(max(a, b), c); }
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
// a wave's own LDS accesses happen in the order they are issued: the compiler is to keep it
__device__ __forceinline__ void in_order() { asm volatile("" ::: "memory"); }
// One 16-byte (4-byte) per lane direct load: lane l's bytes land at lds_wave_base + 16 l (4 l); completion is awaited by its count.
__device__ __forceinline__ void mx4_dma16(const void *gbase_uniform, unsigned lane_off, unsigned lds_wave_base)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                 ::"s"(lds_wave_base), "v"(lane_off), "s"(gbase_uniform) : "memory", "m0");
}
__device__ __forceinline__ void mx4_dma4(const void *gbase_uniform, unsigned lane_off, unsigned lds_wave_base)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2"
                 ::"s"(lds_wave_base), "v"(lane_off), "s"(gbase_uniform) : "memory", "m0");
}

// Codes (cbsz 4) by e4m3 (blgp 0), each with the exponent in a byte of its scale.  16 keys of 128 dims: lane (m, a) has block a of key m; of the
// queries lane (n, a) has dims 16 a + 0..15 and 64 + 16 a + 0..15 of column n.  32 keys of 64 dims: lane (m, h) has block h;
// lane (n, h) dims 16 h + 0..15 and 32 + 16 h + 0..15.
__device__ __forceinline__ f32x4 mx4_scores16(uint4 codes, int e_codes, mx4_i32x8 q, int e_q, f32x4 c)
{
    const mx4_i32x8 a = {(int)codes.x, (int)codes.y, (int)codes.z, (int)codes.w, 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, q, c, 4, 0, 0, e_codes, 0, e_q);
}
template <int BYTE> __device__ __forceinline__ f32x16 mx4_scores32(uint4 codes, int e_codes, mx4_i32x8 q, int e_q, f32x16 c)
{
    const mx4_i32x8 a = {(int)codes.x, (int)codes.y, (int)codes.z, (int)codes.w, 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, q, c, 4, 0, BYTE, e_codes, 0, e_q);
}
// the eight slots of a dimension, in bf16 and in units of their powers
__device__ __forceinline__ bf16x8 mx4_of_codes(uint32_t w)
{
    const uint4 u = make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.f, 0)),
                               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.f, 1)),
                               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.f, 2)),
                               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.f, 3)));
    return __builtin_bit_cast(bf16x8, u);
}
// bf16 x 2^(60 - d) for two probabilities: d as bytes 0 and 1 (or 2 and 3) of `d`; what would be below the least normal number is zero
template <int PAIR> __device__ __forceinline__ uint32_t mx4_lowered(uint32_t p, uint32_t d)
{
    const uint32_t e = __builtin_amdgcn_perm(0u, d, PAIR == 0 ? 0x010C000Cu : 0x030C020Cu) >> 1;
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_sub_sat(__builtin_bit_cast(mx4_u16x2, p), __builtin_bit_cast(mx4_u16x2, e)));
}
// Two slots of a dimension in bf16 (pair PAIR of the word's four), by their powers: 60 - exponent as bytes of d (pairs 0 and 1: of slots 0 to 3; 2 and
// 3: of 4 to 7).  (A slot behind a message's last token holds codes of zero, or another owner's: any number will do.)
template <int PAIR> __device__ __forceinline__ uint32_t mx4_values(uint32_t w, uint32_t d, std::integral_constant<int, PAIR>)
{
    const uint32_t x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 0x1p60f, PAIR));
    return mx4_lowered<PAIR & 1>(x & 0x7FFF7FFFu, d) | (x & 0x80008000u);
}

// The same in fp16, which holds probabilities to 2^-11 where bf16 has 2^-8: exponents from -13 to 13 (others give any number).
template <int PAIR> __device__ __forceinline__ uint32_t mx4_halfs(uint32_t w, uint32_t d, std::integral_constant<int, PAIR>)
{
    static_assert(PC_MX4_HALF == 13 && PC_MX4_E_MAX == 60, "");
    const uint32_t x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 0x1p13f, PAIR));
    const mx4_u16x2 e = __builtin_bit_cast(mx4_u16x2, __builtin_amdgcn_perm(0u, d, (PAIR & 1) == 0 ? 0x0C010C00u : 0x0C030C02u));
    const mx4_u16x2 by = __builtin_elementwise_sub_sat(e, (mx4_u16x2){47, 47}) << (mx4_u16x2){10, 10};
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_sub_sat(__builtin_bit_cast(mx4_u16x2, x & 0x7FFF7FFFu), by)) | (x & 0x80008000u);
}
// two probabilities for the products, and the products, in fp16 or bf16
typedef _Float16 mx4_f16x8 __attribute__((ext_vector_type(8)));
template <bool HALF> __device__ __forceinline__ uint32_t mx4_pack(float a, float b)
{
    if constexpr (HALF) {
        typedef float f32x2 __attribute__((ext_vector_type(2)));
        typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){a, b}, f16x2));
    } else return pack_bf16(a, b);
}
template <bool HALF> __device__ __forceinline__ f32x4 mx4_mfma16(bf16x8 a, bf16x8 b, f32x4 c)
{
    if constexpr (HALF) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(mx4_f16x8, a), __builtin_bit_cast(mx4_f16x8, b), c, 0, 0, 0);
    else return MFMA16(a, b, c);
}
template <bool HALF, int PAIR> __device__ __forceinline__ uint32_t mx4_numbers(uint32_t w, uint32_t d, std::integral_constant<int, PAIR> p)
{
    if constexpr (HALF) return mx4_halfs(w, d, p);
    else return mx4_values(w, d, p);
}

// c + the two probabilities, as the products take them: their rounding cancels where a row has few large ones (calls of 8 to 200 rows take 1.2 us
// less than with two additions of what was not rounded yet)
typedef __bf16 mx4_bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 mx4_f16x2 __attribute__((ext_vector_type(2)));
template <bool HALF> __device__ __forceinline__ float mx4_sum(uint32_t p, float c)
{
    if constexpr (HALF) return __builtin_amdgcn_fdot2(__builtin_bit_cast(mx4_f16x2, p), (mx4_f16x2){(_Float16)1.f, (_Float16)1.f}, c, false);
    else return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(mx4_bf16x2, p), __builtin_bit_cast(mx4_bf16x2, 0x3F803F80u), c, false);
}
template <bool HALF> __device__ __forceinline__ f32x16 mx4_mfma32(bf16x8 a, bf16x8 b, f32x16 c)
{
    if constexpr (HALF) return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(mx4_f16x8, a), __builtin_bit_cast(mx4_f16x8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// (cos, sin) of a turn: positions are below 2^30 and theta is at least 1 (pc_cache_create), so that what queries are turned by is below 3 x 2^30
// radians, and its turns are off by 2^-24 of one in fp64.  (As polynomials in fp64: 40 instructions where these are 7.)
__device__ __forceinline__ float2 mx4_rotation(double x)
{
    const float part = (float)__builtin_amdgcn_fract(x * 0.15915494309189533577);        // 1 / (2 pi)
    return make_float2(__builtin_amdgcn_cosf(part), __builtin_amdgcn_sinf(part));
}

// The larger of top and two bf16 numbers' magnitudes; fine: they are numbers.
__device__ __forceinline__ float mx4_top(float top, uint32_t w, bool &fine)
{
    fine &= ((w & 0x7F80u) != 0x7F80u) & ((w & 0x7F800000u) != 0x7F800000u);
    return fmaxf(top, fmaxf(fabsf(bf_lo(w)), fabsf(bf_hi(w))));
}
// The unit of a row's pieces, the same for every turn: a turn keeps a pair's norm, sqrt(2) times the larger value at most, and the row's largest comes
// between 128 and 256 of it (448 is the largest number of the pieces; one above is NaN).
__device__ __forceinline__ float mx4_unit(float top)
{
    const int e = max(-100, min(121, (int)(__float_as_uint(top * 1.4142137f) >> 23 & 255) - 134));
    return __uint_as_float((uint32_t)(127 + e) << 23);
}
__device__ __forceinline__ int mx4_e4m3(const float (&x)[4], float unit)
{
    mx4_s16x2 r;
    asm("" : "=v"(r));                                // (both halves are written: nothing to start from)
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, x[0], x[1], unit, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, x[2], x[3], unit, true);
    return __builtin_bit_cast(int, r);
}
// Four values as e4m3 in that unit, and what is left of them in a sixteenth of it: off by 2^-4 of 2^-4 of a value.
__device__ __forceinline__ void mx4_pieces(const float (&x)[4], float unit, int &hi, int &rest)
{
    hi = mx4_e4m3(x, unit);
    const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(hi, unit, false), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(hi, unit, true);
    const float y[4] = {x[0] - a[0], x[1] - a[1], x[2] - b[0], x[3] - b[1]};
    rest = mx4_e4m3(y, unit * 0.0625f);
}

// The same of a row of queries in fp16, in that unit (128 to 256 at most: off by 2^-11 of a value, an eighth of what pieces are off by), two values
// an instruction: 16 values and their partners in the upper half, from what came, scaled, by 16 rotations (cosines and sines, in fp16).
__device__ __forceinline__ mx4_f16x2 mx4_half(uint32_t x) { return __builtin_bit_cast(mx4_f16x2, x); }
// eight bf16 numbers times `by`
__device__ __forceinline__ uint4 mx4_halves(uint4 x, float by)
{
    return make_uint4(pack_f16(bf_lo(x.x) * by, bf_hi(x.x) * by), pack_f16(bf_lo(x.y) * by, bf_hi(x.y) * by),
                      pack_f16(bf_lo(x.z) * by, bf_hi(x.z) * by), pack_f16(bf_lo(x.w) * by, bf_hi(x.w) * by));
}
__device__ __forceinline__ int mx4_e4m3(mx4_f16x2 x, mx4_f16x2 y, float unit)
{
    mx4_s16x2 r;
    asm("" : "=v"(r));
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(r, x, unit, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(r, y, unit, true);
    return __builtin_bit_cast(int, r);
}
__device__ __forceinline__ void mx4_pieces(mx4_f16x2 x, mx4_f16x2 y, int &hi, int &rest)
{
    hi = mx4_e4m3(x, y, 1.f);
    rest = mx4_e4m3(x - __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, false), y - __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, true), 0.0625f);
}
// four values and their partners
__device__ __forceinline__ void mx4_turned(uint2 low, uint2 high, uint2 c, uint2 s, int &u_hi, int &u_rest, int &v_hi, int &v_rest)
{
    const mx4_f16x2 x0 = mx4_half(low.x), x1 = mx4_half(low.y), y0 = mx4_half(high.x), y1 = mx4_half(high.y);
    const mx4_f16x2 c0 = mx4_half(c.x), c1 = mx4_half(c.y), s0 = mx4_half(s.x), s1 = mx4_half(s.y);
    mx4_pieces(x0 * c0 - y0 * s0, x1 * c1 - y1 * s1, u_hi, u_rest);
    mx4_pieces(x0 * s0 + y0 * c0, x1 * s1 + y1 * c1, v_hi, v_rest);
}
__device__ __forceinline__ uint2 mx4_two(uint4 x, int second) { return second ? make_uint2(x.z, x.w) : make_uint2(x.x, x.y); }

#endif
