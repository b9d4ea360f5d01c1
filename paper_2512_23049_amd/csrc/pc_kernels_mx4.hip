// Attention of single tokens over a PC_MX4 cache, and its tiles unpacked for the kernels of many rows (gfx950).  What a row sees, and how
// the host states it: pc_window.h; how the cache holds keys and values: pc_mx4.h.
#include "pc_window.h"
#include "pc_mx4.h"
#include "pc_mfma_common.h"

#define MFMA16(a, b, c) __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0)

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float ex2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
// a wave's own LDS accesses happen in the order they are issued: the compiler is to keep it
__device__ __forceinline__ void in_order() { asm volatile("" ::: "memory"); }
__device__ __forceinline__ const __attribute__((address_space(4))) char *arguments()
{
    return (const __attribute__((address_space(4))) char *)__builtin_amdgcn_kernarg_segment_ptr();
}
// codes (cbsz 4) by e4m3 (blgp 0), each with the exponent in the low byte of its scale
__device__ __forceinline__ f32x4 scores16(uint4 codes, int e_codes, i32x8 q, int e_q, f32x4 c)
{
    const i32x8 a = {(int)codes.x, (int)codes.y, (int)codes.z, (int)codes.w, 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, q, c, 4, 0, 0, e_codes, 0, e_q);
}
// the eight slots of a dimension, in bf16 and in units of their powers
__device__ __forceinline__ bf16x8 of_codes(uint32_t w)
{
    const uint4 u = make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.f, 0)),
                               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.f, 1)),
                               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.f, 2)),
                               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.f, 3)));
    return __builtin_bit_cast(bf16x8, u);
}
// bf16 x 2^(60 - d): d as bytes 0 and 1 (or 2 and 3) of `d`; what would be below the least normal number is zero
template <int PAIR> __device__ __forceinline__ uint32_t lowered(uint32_t p, uint32_t d)
{
    const uint32_t e = __builtin_amdgcn_perm(0u, d, PAIR == 0 ? 0x010C000Cu : 0x030C020Cu) >> 1;
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_sub_sat(__builtin_bit_cast(u16x2, p), __builtin_bit_cast(u16x2, e)));
}

struct Mx4Tile {
    uint4 k[2];               // lane (m, a): block a of key 8 (m >> 2) + 4 half + (m & 3), its codes
    uint32_t ke[2];           // and the exponents of that key's four blocks
    uint4 v[2];               // dimensions 16 db + m of keys 8 a + 0..7: words of db 0..3, 4..7
    uint4 ve[2];              // 60 - exponent: blocks 0 and 1 (keys 8 a + 0..7 each), 2 and 3
    WinTile d;
};

}  // namespace

// One query row a call.  A workgroup is 4 waves over one item of one KV head, each with a contiguous share of its tiles; the g <= 16
// heads of the KV head are the columns of the products.
//   scores   codes of keys as they are stored, by the turned query as the sum of two e4m3 numbers under one power of two for the row
//            (the second has what the first leaves, at 1/16: off by 2^-8 of a value, like bf16): v_mfma_scale 16x16x128, a key's blocks and
//            exponents where the instruction wants them, nothing is unpacked;
//   values   eight slots of a dimension are a word: four conversions make the operand, in units of the slots' powers.  The powers ride
//            on the probabilities, by block of 32 dimensions: probabilities are held 2^60 times as large, and a saturating
//            subtraction from their exponents takes the powers (-60 to 60) off again.
// Bound: memory, 4352 bytes a tile and KV head.
__device__ __forceinline__ void mx4_decode(const PcWin &W, const PcWinItem *items, const PcWinRun *runs, const int32_t *q_pos)
{
    __shared__ __attribute__((aligned(16))) float s_acc[4][16][PC_D + 4];
    __shared__ float s_m[4][16], s_l[4][16];
    __shared__ __attribute__((aligned(16))) float2 s_rot[4][PC_D / 2];

    const int kh = blockIdx.x % W.n_kv_heads;          // consecutive workgroups (one per XCD) take different KV heads
    const int which = blockIdx.x / W.n_kv_heads;
    PcWinItem item;
    {
        const auto *p = reinterpret_cast<const __attribute__((address_space(4))) win_i32x4 *>(reinterpret_cast<uintptr_t>(items + which));
        const win_i32x4 a = p[0], b = p[1];
        item = PcWinItem{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    }
    const int g = W.n_q_heads / W.n_kv_heads;
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const int n = lane & 15, a = lane >> 4;
    const int pos = *reinterpret_cast<const __attribute__((address_space(4))) int32_t *>(reinterpret_cast<uintptr_t>(q_pos + item.q_off));
    const int lo = win_low(pos, W.window);
    const int share = item.n_tiles / 4, more = item.n_tiles % 4;
    const int n_tiles = share + (wave < more), skip = item.skip + wave * share + min(wave, more);

    float m_run = -INFINITY, l_run = 0.f;
    f32x4 acc[8];
#pragma unroll
    for (int db = 0; db < 8; ++db) acc[db] = (f32x4){0.f, 0.f, 0.f, 0.f};
    if (n_tiles > 0) {
        const unsigned char *kb = (const unsigned char *)W.k_store + (int64_t)kh * (W.slots / PC_TILE) * PC_MX4_TILE;
        const unsigned char *vb = (const unsigned char *)W.v_store + (int64_t)kh * (W.slots / PC_TILE) * PC_MX4_TILE;
        WinWalk walk(runs + item.run0, skip, n_tiles);
        int asked = 0;
        const unsigned k_at = (unsigned)((8 * (n >> 2) + (n & 3)) * 64 + 16 * a), ke_at = (unsigned)(PC_MX4_CODES + (8 * (n >> 2) + (n & 3)) * 4);
        const unsigned v_at = (unsigned)(a * 512 + n * 32), ve_at = (unsigned)(PC_MX4_CODES + a * 32);
        auto fetch = [&](Mx4Tile &T) __attribute__((always_inline)) {
            if (asked > 0 && asked < n_tiles) walk.next();
            ++asked;
            T.d = walk.tile();
            T.d.rot = (int)((walk.run - reinterpret_cast<uintptr_t>(runs)) / sizeof(PcWinRun));       // (the run)
            const unsigned char *kt = kb + (int64_t)(T.d.slot0 / PC_TILE) * PC_MX4_TILE, *vt = vb + (int64_t)(T.d.slot0 / PC_TILE) * PC_MX4_TILE;
#pragma unroll
            for (int tau = 0; tau < 2; ++tau) {
                T.k[tau] = ldg16(kt + k_at + tau * 256);
                T.ke[tau] = *reinterpret_cast<const uint32_t *>(kt + ke_at + tau * 16);
                T.v[tau] = ldg16(vt + v_at + tau * 16);
                T.ve[tau] = ldg16(vt + ve_at + tau * 16);
            }
        };
        // the column's head, as it came (from the cache each time: registers): dims 16 a + 0..15, then 64 up
        const unsigned char *qp = (const unsigned char *)W.q + ((int64_t)item.q_off * W.n_q_heads + kh * g + min(n, g - 1)) * (PC_D * 2) + 32 * a;
        const double freq = W.inv_freq[lane];
        Mx4Tile A, B;
        fetch(A);
        if (n_tiles > 1) fetch(B);
        int cur = -1, e_hi = 127, e_lo = 127;
        int64_t cur_turn = 0;
        i32x8 q_hi, q_lo;
        auto compute = [&](Mx4Tile &T) __attribute__((always_inline)) {
            if (T.d.rot != cur) {                        // another run: another rotation?
                const int64_t turn = pos - T.d.rot_pos;
                const bool fresh = cur < 0 || turn != cur_turn;
                cur = T.d.rot; cur_turn = turn;
                if (fresh) {
                    const float2 cs = rope_angle((double)turn * freq);
                    s_rot[wave][lane] = make_float2(cs.x * W.scale_log2, cs.y * W.scale_log2);
                    in_order();
                    float x[16], y[16], top = 0.f;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        uint4 lq = ldg16(qp + 16 * i), hq = ldg16(qp + 128 + 16 * i);
                        if (n >= g) lq = hq = make_uint4(0, 0, 0, 0);
                        const uint32_t lw[4] = {lq.x, lq.y, lq.z, lq.w}, hw[4] = {hq.x, hq.y, hq.z, hq.w};
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float4 r = *reinterpret_cast<const float4 *>(&s_rot[wave][16 * a + 8 * i + 2 * j]);
                            const float x0 = bf_lo(lw[j]), x1 = bf_hi(lw[j]), y0 = bf_lo(hw[j]), y1 = bf_hi(hw[j]);
                            x[8 * i + 2 * j] = x0 * r.x - y0 * r.y; x[8 * i + 2 * j + 1] = x1 * r.z - y1 * r.w;
                            y[8 * i + 2 * j] = x0 * r.y + y0 * r.x; y[8 * i + 2 * j + 1] = x1 * r.w + y1 * r.z;
                        }
                    }
                    in_order();
#pragma unroll
                    for (int i = 0; i < 16; ++i) top = fmaxf(top, fmaxf(fabsf(x[i]), fabsf(y[i])));
                    top = fmaxf(top, __shfl_xor(top, 16));
                    top = fmaxf(top, __shfl_xor(top, 32));
                    // the row's largest value between 128 and 256 (the largest number there is: 448)
                    const int e = max(-100, min(100, (int)(__float_as_uint(top) >> 23 & 255) - 134));
                    const float unit = __uint_as_float((uint32_t)(127 - e) << 23) * (top < INFINITY ? 1.f : __builtin_nanf(""));
                    e_hi = 127 + e; e_lo = 123 + e;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float *p = i < 4 ? x + 4 * i : y + 4 * (i - 4);
                        const float f0 = p[0] * unit, f1 = p[1] * unit, f2 = p[2] * unit, f3 = p[3] * unit;
                        int hi = __builtin_amdgcn_cvt_pk_fp8_f32(f0, f1, 0, false);
                        hi = __builtin_amdgcn_cvt_pk_fp8_f32(f2, f3, hi, true);
                        const auto b0 = __builtin_amdgcn_cvt_pk_f32_fp8(hi, false), b1 = __builtin_amdgcn_cvt_pk_f32_fp8(hi, true);
                        int rest = __builtin_amdgcn_cvt_pk_fp8_f32((f0 - b0[0]) * 16.f, (f1 - b0[1]) * 16.f, 0, false);
                        rest = __builtin_amdgcn_cvt_pk_fp8_f32((f2 - b1[0]) * 16.f, (f3 - b1[1]) * 16.f, rest, true);
                        q_hi[i] = hi; q_lo[i] = rest;
                    }
                }
            }
            f32x4 s[2];
#pragma unroll
            for (int tau = 0; tau < 2; ++tau) {
                const int e = (int)(T.ke[tau] >> (8 * a));
                s[tau] = scores16(T.k[tau], e, q_lo, e_lo, (f32x4){0.f, 0.f, 0.f, 0.f});
                s[tau] = scores16(T.k[tau], e, q_hi, e_hi, s[tau]);
            }
            float sc[8];                                 // keys 8 a + 0..7 of column n
#pragma unroll
            for (int j = 0; j < 8; ++j) sc[j] = s[j >> 2][j & 3];
            const uint32_t sees = win_sees(T.d.pos0, T.d.valid, T.d.sink, false, lo, 0);        // (the only row sees all of the new message)
            if (sees != ~0u) {                           // (uniform; values need no mask: codes are finite)
                const uint32_t mine = sees >> (8 * a);
#pragma unroll
                for (int j = 0; j < 8; ++j) sc[j] = (mine >> j) & 1 ? sc[j] : -INFINITY;
            }
            float mx = fmaxf(fmaxf(fmaxf(sc[0], sc[1]), fmaxf(sc[2], sc[3])), fmaxf(fmaxf(sc[4], sc[5]), fmaxf(sc[6], sc[7])));
            mx = fmaxf(mx, __shfl_xor(mx, 16));
            mx = fmaxf(mx, __shfl_xor(mx, 32));
            const float m_new = fmaxf(m_run, mx), m_safe = m_new == -INFINITY ? 0.f : m_new, alpha = ex2(m_run - m_safe), m_up = m_safe - PC_MX4_E_MAX;
            uint32_t pk[4];
            float ps = 0.f;                              // (of the probabilities as the products take them: their rounding cancels)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                pk[j] = pack_bf16(ex2(sc[2 * j] - m_up), ex2(sc[2 * j + 1] - m_up));
                ps += bf_lo(pk[j]) + bf_hi(pk[j]);
            }
            l_run = l_run * alpha + ps;
            m_run = m_new;
            if (__builtin_amdgcn_ballot_w64(alpha != 1.f) != 0) {           // rare once the running maxima have settled
#pragma unroll
                for (int db = 0; db < 8; ++db) acc[db] *= alpha;
            }
            const uint32_t vw[8] = {T.v[0].x, T.v[0].y, T.v[0].z, T.v[0].w, T.v[1].x, T.v[1].y, T.v[1].z, T.v[1].w};
            const uint32_t ew[8] = {T.ve[0].x, T.ve[0].y, T.ve[0].z, T.ve[0].w, T.ve[1].x, T.ve[1].y, T.ve[1].z, T.ve[1].w};
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const bf16x8 p = __builtin_bit_cast(bf16x8, make_uint4(lowered<0>(pk[0], ew[2 * b]), lowered<1>(pk[1], ew[2 * b]),
                                                                       lowered<0>(pk[2], ew[2 * b + 1]), lowered<1>(pk[3], ew[2 * b + 1])));
#pragma unroll
                for (int i = 0; i < 2; ++i) acc[2 * b + i] = MFMA16(of_codes(vw[2 * b + i]), p, acc[2 * b + i]);
            }
        };
        for (int t = 0;;) {
            compute(A);
            if (t + 2 < n_tiles) fetch(A);
            if (++t >= n_tiles) break;
            compute(B);
            if (t + 2 < n_tiles) fetch(B);
            if (++t >= n_tiles) break;
        }
    }
    l_run += __shfl_xor(l_run, 16);
    l_run += __shfl_xor(l_run, 32);
    if (a == 0) { s_m[wave][n] = m_run; s_l[wave][n] = l_run * 0x1p-60f; }
#pragma unroll
    for (int db = 0; db < 8; ++db) *reinterpret_cast<f32x4 *>(&s_acc[wave][n][16 * db + 4 * a]) = acc[db];
    __syncthreads();
    for (int idx = threadIdx.x; idx < g * (PC_D / 2); idx += 256) {
        const int col = idx / (PC_D / 2), dim = 2 * (idx % (PC_D / 2)), h = kh * g + col;
        float m = -INFINITY;
#pragma unroll
        for (int w = 0; w < 4; ++w) m = fmaxf(m, s_m[w][col]);
        float o0 = 0.f, o1 = 0.f, l = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            // (a wave whose scores were not numbers has a sum that is none; one that saw nothing has a sum of 0)
            const float f = s_l[w][col] == 0.f ? 0.f : ex2(s_m[w][col] - (m == -INFINITY ? 0.f : m));
            const float2 x = *reinterpret_cast<const float2 *>(&s_acc[w][col][dim]);
            if (s_l[w][col] != 0.f) { o0 += x.x * f; o1 += x.y * f; l += s_l[w][col] * f; }
        }
        if (item.part < 0) {
            const float inv = l == 0.f ? 0.f : 1.f / l;
            *reinterpret_cast<uint32_t *>((uint16_t *)W.out + ((int64_t)item.q_off * W.n_q_heads + h) * PC_D + dim) = pack_bf16(o0 * inv, o1 * inv);
            if (W.lse && dim == 0) W.lse[(int64_t)item.q_off * W.n_q_heads + h] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
        } else {
            *reinterpret_cast<float2 *>(W.part_o + ((int64_t)item.part * W.n_q_heads + h) * PC_D + dim) = make_float2(o0, o1);
            if (dim == 0) *reinterpret_cast<float2 *>(W.part_ml + ((int64_t)item.part * W.n_q_heads + h) * 2) = make_float2(l == 0.f ? -INFINITY : m, l);
        }
    }
}

__global__ __launch_bounds__(256, 2) void pc_mx4_decode_kernel(PcWin W) { mx4_decode(W, W.items, W.runs, W.q_pos); }
__global__ __launch_bounds__(256, 2) void pc_mx4_decode_arg_kernel(PcArgBlob, PcWinDecode O, PcWin W)
{
    const char *lists = (const char *)arguments();       // (the blob comes first)
    if (blockIdx.x == 0 && (int)threadIdx.x < O.n16) reinterpret_cast<uint4 *>(O.ws)[threadIdx.x] = reinterpret_cast<const uint4 *>(lists)[threadIdx.x];
    mx4_decode(W, reinterpret_cast<const PcWinItem *>(lists + O.off_items), reinterpret_cast<const PcWinRun *>(lists + O.off_runs),
               reinterpret_cast<const int32_t *>(lists + O.off_q_pos));
}

void pc_launch_win_decode_mx4(const PcWin &W, int n_items, const PcArgBlob *blob, const PcWinDecode &O, hipStream_t st)
{
    if (n_items <= 0) return;
    const unsigned grid = (unsigned)n_items * W.n_kv_heads;
    if (blob) pc_mx4_decode_arg_kernel<<<grid, 256, 0, st>>>(*blob, O, W);
    else pc_mx4_decode_kernel<<<grid, 256, 0, st>>>(W);
}

// ------------------------------------------------------------------------------------------------------------ unpack
// A tile of one KV head as a bf16 cache has it: what the codes stand for is exact there.  Bound: memory (68 bytes read and 256
// written for each key and value).
__global__ __launch_bounds__(256) void pc_mx4_unpack_kernel(PcMx4Unpack U)
{
    const int kh = blockIdx.y;
    const int64_t from = ((int64_t)kh * U.slots_from + U.slots[blockIdx.x]) / PC_TILE * PC_MX4_TILE;
    const char *kt = (const char *)U.k_store + from, *vt = (const char *)U.v_store + from;
    const int64_t to = ((int64_t)kh * U.n_tiles + blockIdx.x) * (PC_TILE * PC_D * 2);
    {
        const int row = threadIdx.x >> 3, c = threadIdx.x & 7;           // values 16 c to 16 c + 15
        const uint2 w = *reinterpret_cast<const uint2 *>(kt + row * 64 + 8 * c);
        const int e = (uint8_t)kt[PC_MX4_CODES + row * 4 + (c >> 1)];
        const float unit = __uint_as_float((uint32_t)min(e, 254) << 23);
        uint4 x[2];
        uint32_t *o = reinterpret_cast<uint32_t *>(x);
        const uint32_t words[2] = {w.x, w.y};
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            o[4 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(words[i], unit, 0));
            o[4 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(words[i], unit, 1));
            o[4 * i + 2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(words[i], unit, 2));
            o[4 * i + 3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(words[i], unit, 3));
        }
        if (e == PC_MX4_NAN) x[0] = x[1] = make_uint4(0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u);
        uint4 *dst = reinterpret_cast<uint4 *>((char *)U.k_to + to + threadIdx.x * 32);
        dst[0] = x[0];
        dst[1] = x[1];
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int grp = (threadIdx.x >> 7) + 2 * i, d = threadIdx.x & 127;
        const uint32_t w = reinterpret_cast<const uint32_t *>(vt + grp * 512)[mx4_word(d)];
        const uint2 ex = *reinterpret_cast<const uint2 *>(vt + PC_MX4_CODES + grp * 32 + d / 32 * 8);
        const uint4 codes = __builtin_bit_cast(uint4, of_codes(w));
        const uint32_t cw[4] = {codes.x, codes.y, codes.z, codes.w};
        uint32_t o[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t es = (j < 2 ? ex.x : ex.y) >> 16 * (j & 1);
            const float u0 = __uint_as_float((187u - min(es & 255u, 120u)) << 23), u1 = __uint_as_float((187u - min(es >> 8 & 255u, 120u)) << 23);
            o[j] = pack_bf16(bf_lo(cw[j]) * u0, bf_hi(cw[j]) * u1);
        }
        *reinterpret_cast<uint4 *>((char *)U.v_to + to + (grp * 128 + d) * 16) = make_uint4(o[0], o[1], o[2], o[3]);
    }
}

void pc_launch_mx4_unpack(const PcMx4Unpack &U, hipStream_t st)
{
    if (U.n_tiles > 0) pc_mx4_unpack_kernel<<<dim3((unsigned)U.n_tiles, (unsigned)U.n_kv_heads), 256, 0, st>>>(U);
}
