// Rows of a layer's projections on their way into the cache, the gradient of that way, and messages read back (gfx950).
//
//   y = x / sqrt(mean(x^2) + eps) * w             for every head of queries and keys,
//   stored key = y turned to its position          pairs (i, i + D/2) by pos theta^(-2i/D), angles in 64 bits,
// values as they are; in a PC_MX4 cache keys (from 64 bits on) and values in the 4 bits of pc_mx4.h.
#include "pc_project.h"
#include "pc_mx4.h"
#include "pc_mfma_common.h"

#include <algorithm>
#include <type_traits>

namespace {

__device__ __forceinline__ const __attribute__((address_space(4))) char *arguments()
{
    return (const __attribute__((address_space(4))) char *)__builtin_amdgcn_kernarg_segment_ptr();
}

// the item that a block belongs to: the last one whose block0 is not behind it
template <class Item> __device__ __forceinline__ Item item_of(const Item *items, int n, int block)
{
    int a = 0, b = n;
    while (b - a > 1) {
        const int mid = (a + b) / 2;
        if (items[mid].block0 <= block) a = mid; else b = mid;
    }
    return items[a];
}

// E = D / 16 values from the lower half of a head's row and as many from the upper one, in 32 bits
template <typename T, int E> __device__ __forceinline__ void load_run(const T *p, float (&x)[E])
{
    if constexpr (sizeof(T) == 2) {
        static_assert(E == 8, "");
        const uint4 u = ldg16(p);
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) { x[2 * j] = bf_lo(w[j]); x[2 * j + 1] = bf_hi(w[j]); }
    } else {
#pragma unroll
        for (int j = 0; j < E / 4; ++j) {
            const float4 f = reinterpret_cast<const float4 *>(p)[j];
            x[4 * j] = f.x; x[4 * j + 1] = f.y; x[4 * j + 2] = f.z; x[4 * j + 3] = f.w;
        }
    }
}
template <typename T, int E> __device__ __forceinline__ void store_run(T *p, const float (&x)[E])
{
    if constexpr (sizeof(T) == 2) {
        *reinterpret_cast<uint4 *>(p) = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
    } else {
#pragma unroll
        for (int j = 0; j < E / 4; ++j) reinterpret_cast<float4 *>(p)[j] = make_float4(x[4 * j], x[4 * j + 1], x[4 * j + 2], x[4 * j + 3]);
    }
}
template <int E> __device__ __forceinline__ void load_weight(const float *w, int at, float (&x)[E])
{
#pragma unroll
    for (int j = 0; j < E; ++j) x[j] = w ? w[at + j] : 1.f;
}
// over the eight lanes of a head's row
template <typename F> __device__ __forceinline__ F sum8(F x)
{
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) x += __shfl_xor(x, o);
    return x;
}

}  // namespace

// ------------------------------------------------------------------------------------------------------------ append
// A block takes a group of eight slots and eight heads of one kind: part below `kv`: keys and values, else queries.  Parts of a group follow each
// other, so that the work on keys hides behind the queries' traffic (8192 rows into 4 bits: all keys first 74 us, so 68).  A head's
// row is eight lanes, each with E values of the lower half and their partners in the upper half: turns stay in a lane, sums
// take three steps.  Rotations are made once a block (8 tokens x D/2) and shared by its heads.
// Bound: memory, where there are many rows (bf16, 2208 rows of 32 heads over 8, 54 MB: 11.7 us, 4.6 TB/s; 4 bits, 8192 rows of 64 heads over 8, 311 MB: 66 us, 4.7 TB/s,
// keys in 64 bits: a key next to the middle of two codes goes to the one that its exact value is nearer to); latency where there are few
// (four rows 5.2 us, a launch of nothing 3).
template <int STORE, int D>           // STORE: PC_F32, PC_BF16, PC_MX4
__device__ __forceinline__ void rows_block(const PcRows &R, const PcRowsItem *items)
{
    using T = std::conditional_t<STORE == 0, float, uint16_t>;
    using F = std::conditional_t<STORE == 2, double, float>;            // of keys
    constexpr int E = D / 16, HALF = D / 2;
    struct Turn { F c, s; };
    __shared__ __attribute__((aligned(16))) Turn s_turn[PC_ROWS_GROUP][HALF];
    const int kv = (R.n_kv_heads + PC_ROWS_HEADS - 1) / PC_ROWS_HEADS, chunks = kv + (R.q_out ? (R.n_q_heads + PC_ROWS_HEADS - 1) / PC_ROWS_HEADS : 0);
    const int block = R.block0 + (int)blockIdx.x / chunks, part = (int)blockIdx.x % chunks;
    const PcRowsItem it = item_of(items, R.n_items, block);
    const int t0 = 8 * (it.slot0 / 8 + block - it.block0) - it.slot0;          // the group's first token (may lie in front of the item's)
    const int c = threadIdx.x & 7, hd = threadIdx.x >> 3 & 7, tt0 = threadIdx.x >> 6;     // the thread's tokens: t0 + tt0, and four on
    const int lo = E * c, hi = HALF + E * c;

    if (part >= kv) {
        const int h = (part - kv) * PC_ROWS_HEADS + hd;
        if (h >= R.n_q_heads) return;
        float w0[E], w1[E], x0[2][E], x1[2][E];
        load_weight<E>(R.q_weight, lo, w0);
        load_weight<E>(R.q_weight, hi, w1);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int t = min(max(t0 + tt0 + 4 * u, 0), it.n - 1);
            const T *src = (const T *)it.q + (int64_t)t * R.q_stride + h * D;
            load_run<T, E>(src + lo, x0[u]);
            load_run<T, E>(src + hi, x1[u]);
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int t = t0 + tt0 + 4 * u;
            float sq = 0.f;
#pragma unroll
            for (int j = 0; j < E; ++j) sq += x0[u][j] * x0[u][j] + x1[u][j] * x1[u][j];
            const float r = 1.f / sqrtf(sum8(sq) * (1.f / D) + R.eps);
#pragma unroll
            for (int j = 0; j < E; ++j) { x0[u][j] *= r * w0[j]; x1[u][j] *= r * w1[j]; }
            if (t < 0 || t >= it.n) continue;
            T *dst = (T *)R.q_out + ((it.q_row + t) * R.n_q_heads + h) * D;
            store_run<T, E>(dst + lo, x0[u]);
            store_run<T, E>(dst + hi, x1[u]);
        }
        return;
    }

    if (part == 0 && block == it.block0 && threadIdx.x == 0) {
        if (it.fresh) R.table[it.msg] = PcMsgEntry{it.slot0, it.len, 0, 0};
        else R.table[it.msg].len = it.len;
    }
    for (int e = threadIdx.x; e < PC_ROWS_GROUP * HALF; e += 256) {
        const int t = t0 + e / HALF;
        if (t < 0 || t >= it.n) continue;
        if constexpr (STORE == 2) {
            double s, co;
            sincos((double)(it.pos0 + t) * R.inv_freq[e % HALF], &s, &co);
            s_turn[e / HALF][e % HALF] = Turn{co, s};
        } else {
            const float2 cs = rope_turn(it.pos0 + t, R.inv_freq[e % HALF]);
            s_turn[e / HALF][e % HALF] = Turn{cs.x, cs.y};
        }
    }
    const int h0 = part * PC_ROWS_HEADS, h = min(h0 + hd, R.n_kv_heads - 1);
    const bool head_ok = h0 + hd < R.n_kv_heads;
    [[maybe_unused]] bool bad[2] = {false, false};       // (4 bits) the value holds what is no number

    if constexpr (STORE == 2) {                          // values: codes by token, then words of eight slots
        __shared__ __attribute__((aligned(16))) uint8_t s_code[PC_ROWS_HEADS][D][8];
        float x0[2][E], x1[2][E];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const T *src = (const T *)it.v + (int64_t)min(max(t0 + tt0 + 4 * u, 0), it.n - 1) * R.v_stride + h * D;
            load_run<T, E>(src + lo, x0[u]);
            load_run<T, E>(src + hi, x1[u]);
        }
        const int64_t tile = ((int64_t)h * R.slots + (it.slot0 + t0)) / PC_TILE;           // (slots: a multiple of the tile)
        const int grp = (it.slot0 + t0) % PC_TILE / 8;
        char *vt = (char *)R.v_store + tile * PC_MX4_TILE;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int tt = tt0 + 4 * u, t = t0 + tt;
            const bool there = t >= 0 && t < it.n;
            float m0 = 0.f, m1 = 0.f;
#pragma unroll
            for (int j = 0; j < E; ++j) { m0 = fmaxf(m0, fabsf(x0[u][j])); m1 = fmaxf(m1, fabsf(x1[u][j])); }
            bool b = false;
#pragma unroll
            for (int j = 0; j < E; ++j) b |= !(fabsf(x0[u][j]) < INFINITY) | !(fabsf(x1[u][j]) < INFINITY);
#pragma unroll
            for (int o = 1; o < 4; o <<= 1) { m0 = fmaxf(m0, __shfl_xor(m0, o)); m1 = fmaxf(m1, __shfl_xor(m1, o)); }
            int all = b;
#pragma unroll
            for (int o = 1; o < 8; o <<= 1) all |= __shfl_xor(all, o);
            bad[u] = all != 0;
            const int e0 = mx4_exponent(m0), e1 = mx4_exponent(m1);
            const float p0 = mx4_power(0.f, -e0), p1 = mx4_power(0.f, -e1);
            if (there && head_ok && !bad[u] && ((m0 > 0.f && abs(e0) > PC_MX4_HALF) || (m1 > 0.f && abs(e1) > PC_MX4_HALF))) *R.wide = 1;
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const bool none = bad[u] || !there;
                s_code[hd][lo + j][tt] = none ? 0 : (uint8_t)(mx4_code(fabsf(x0[u][j]) * p0) | (__float_as_uint(x0[u][j]) >> 28 & 8));
                s_code[hd][hi + j][tt] = none ? 0 : (uint8_t)(mx4_code(fabsf(x1[u][j]) * p1) | (__float_as_uint(x1[u][j]) >> 28 & 8));
            }
            if (there && head_ok && (c & 3) == 0) {      // blocks c / 4 and 2 + c / 4
                char *ex = vt + PC_MX4_CODES + grp * 32 + tt;
                ex[(c >> 2) * 8] = (char)(PC_MX4_E_MAX - (bad[u] ? 0 : e0));
                ex[(2 + (c >> 2)) * 8] = (char)(PC_MX4_E_MAX - (bad[u] ? 0 : e1));
            }
        }
        __syncthreads();
        // (slots of the group that are not the item's keep what they hold; those of a new message hold nothing)
        const int first = max(0, -t0), last = min(8, it.n - t0);
        const uint32_t mine = (last >= 8 ? ~0u : (1u << 4 * last) - 1u) & ~((1u << 4 * first) - 1u);
        for (int e = threadIdx.x; e < PC_ROWS_HEADS * D; e += 256) {
            const int hh = h0 + e / D, at = e % D, d = (at & 7) * 16 + at / 8;             // (word at: dimension d)
            if (hh >= R.n_kv_heads) break;
            const uint2 b = *reinterpret_cast<const uint2 *>(&s_code[e / D][d][0]);
            auto four = [](uint32_t x) { x = (x | x >> 4) & 0x00FF00FFu; return (x | x >> 8) & 0xFFFFu; };
            uint32_t w = four(b.x) | four(b.y) << 16;
            uint32_t *to = reinterpret_cast<uint32_t *>((char *)R.v_store + ((int64_t)hh * R.slots + (it.slot0 + t0)) / PC_TILE * PC_MX4_TILE + grp * 512) + at;
            if (!it.fresh && mine != ~0u) w = (w & mine) | (*to & ~mine);
            *to = w;
        }
    } else if constexpr (STORE == 1) {
        // a thread: two dims of a head over the eight slots (rows behind a new message's last token get zeros)
        const bool whole = it.fresh || (t0 >= 0 && t0 + 8 <= it.n);
        for (int e = threadIdx.x; e < PC_ROWS_HEADS * HALF; e += 256) {
            const int hh = h0 + e / HALF, d = 2 * (e % HALF);
            if (hh >= R.n_kv_heads) break;
            uint32_t in[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int t = t0 + j;
                in[j] = t >= 0 && t < it.n ? *reinterpret_cast<const uint32_t *>((const uint16_t *)it.v + (int64_t)t * R.v_stride + hh * D + d) : 0u;
            }
            uint16_t *dst = (uint16_t *)R.v_store + (((int64_t)hh * R.slots + it.slot0 + t0) / 8 * D + d) * 8;
            if (whole) {
                uint4 a, b;
                uint32_t *ew = reinterpret_cast<uint32_t *>(&a), *ow = reinterpret_cast<uint32_t *>(&b);
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    ew[w] = (in[2 * w] & 0xFFFFu) | in[2 * w + 1] << 16;
                    ow[w] = in[2 * w] >> 16 | (in[2 * w + 1] & 0xFFFF0000u);
                }
                *reinterpret_cast<uint4 *>(dst) = a;
                *reinterpret_cast<uint4 *>(dst + 8) = b;
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (t0 + j >= 0 && t0 + j < it.n) { dst[j] = (uint16_t)in[j]; dst[8 + j] = (uint16_t)(in[j] >> 16); }
            }
        }
    } else {
        constexpr int P = D / 4;                         // 16-byte pieces of a row
        for (int e = threadIdx.x; e < PC_ROWS_GROUP * PC_ROWS_HEADS * P; e += 256) {
            const int hh = h0 + e / P % PC_ROWS_HEADS, t = t0 + e / (P * PC_ROWS_HEADS);
            if (hh >= R.n_kv_heads || t < 0 || t >= (it.fresh ? it.rows : it.n)) continue;
            const float4 x = t < it.n ? *reinterpret_cast<const float4 *>((const float *)it.v + (int64_t)t * R.v_stride + hh * D + 4 * (e % P)) : make_float4(0.f, 0.f, 0.f, 0.f);
            *reinterpret_cast<float4 *>((float *)R.v_store + ((int64_t)hh * R.slots + it.slot0 + t) * D + 4 * (e % P)) = x;
        }
    }

    // keys
    float w0[E], w1[E], x0[2][E], x1[2][E];
    load_weight<E>(R.k_weight, lo, w0);
    load_weight<E>(R.k_weight, hi, w1);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const T *src = (const T *)it.k + (int64_t)min(max(t0 + tt0 + 4 * u, 0), it.n - 1) * R.k_stride + h * D;
        load_run<T, E>(src + lo, x0[u]);
        load_run<T, E>(src + hi, x1[u]);
    }
    __syncthreads();                                     // (the rotations)
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int tt = tt0 + 4 * u, t = t0 + tt;
        const bool there = t >= 0 && t < it.n;
        F y0[E], y1[E];
#pragma unroll
        for (int j = 0; j < E; ++j) { y0[j] = x0[u][j]; y1[j] = x1[u][j]; }
        if (R.norm) {
            F sq = 0;
#pragma unroll
            for (int j = 0; j < E; ++j) sq += y0[j] * y0[j] + y1[j] * y1[j];
            sq = sum8(sq) * (F)(1. / D) + (F)R.eps;
            const F r = (F)1 / (STORE == 2 ? (F)sqrt((double)sq) : (F)sqrtf((float)sq));
#pragma unroll
            for (int j = 0; j < E; ++j) { y0[j] *= r * w0[j]; y1[j] *= r * w1[j]; }
        }
        if (there) {
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const Turn cs = s_turn[tt][lo + j];
                const F a = y0[j], b = y1[j];
                y0[j] = a * cs.c - b * cs.s;
                y1[j] = a * cs.s + b * cs.c;
            }
        }
        if constexpr (STORE == 2) {
            double m0 = 0, m1 = 0;
            bool b = bad[u];
#pragma unroll
            for (int j = 0; j < E; ++j) { m0 = fmax(m0, fabs(y0[j])); m1 = fmax(m1, fabs(y1[j])); }
#pragma unroll
            for (int j = 0; j < E; ++j) b |= !(fabs(y0[j]) < INFINITY) | !(fabs(y1[j]) < INFINITY);
#pragma unroll
            for (int o = 1; o < 4; o <<= 1) { m0 = fmax(m0, __shfl_xor(m0, o)); m1 = fmax(m1, __shfl_xor(m1, o)); }
            int all = b;
#pragma unroll
            for (int o = 1; o < 8; o <<= 1) all |= __shfl_xor(all, o);
            if (!there || !head_ok) continue;
            const int e0 = mx4_exponent(m0), e1 = mx4_exponent(m1);
            const double p0 = mx4_power(0., -e0), p1 = mx4_power(0., -e1);
            uint32_t k0 = 0, k1 = 0;
#pragma unroll
            for (int j = 0; j < E; ++j) {
                k0 |= (mx4_code(fabs(y0[j]) * p0) | (y0[j] < 0 ? 8u : 0u)) << 4 * j;
                k1 |= (mx4_code(fabs(y1[j]) * p1) | (y1[j] < 0 ? 8u : 0u)) << 4 * j;
            }
            if (all) k0 = k1 = 0;
            char *kt = (char *)R.k_store + ((int64_t)h * R.slots + it.slot0 + t) / PC_TILE * PC_MX4_TILE;
            const int row = (it.slot0 + t) % PC_TILE;
            *reinterpret_cast<uint32_t *>(kt + row * 64 + 4 * c) = k0;           // (lane c: values 8 c to 8 c + 7 of a half)
            *reinterpret_cast<uint32_t *>(kt + row * 64 + 32 + 4 * c) = k1;
            if ((c & 3) == 0) {
                kt[PC_MX4_CODES + row * 4 + (c >> 2)] = (char)(all ? PC_MX4_NAN : e0 + 127);
                kt[PC_MX4_CODES + row * 4 + 2 + (c >> 2)] = (char)(all ? PC_MX4_NAN : e1 + 127);
            }
        } else {
            if (!head_ok || t < 0 || t >= (it.fresh ? it.rows : it.n)) continue;
            if (!there) {
#pragma unroll
                for (int j = 0; j < E; ++j) y0[j] = y1[j] = 0;
            }
            T *dst = (T *)R.k_store + ((int64_t)h * R.slots + it.slot0 + t) * D;
            store_run<T, E>(dst + lo, y0);
            store_run<T, E>(dst + hi, y1);
        }
    }
}

template <int STORE, int D> __global__ __launch_bounds__(256) void pc_rows_kernel(PcRows R) { rows_block<STORE, D>(R, R.items); }
template <int STORE, int D> __global__ __launch_bounds__(256) void pc_rows_arg_kernel(PcArgBlob, PcRows R)
{
    rows_block<STORE, D>(R, (const PcRowsItem *)arguments());           // (the blob comes first)
}

void pc_launch_rows(int dtype, PcRows R, const PcArgBlob *blob, hipStream_t st)
{
    auto chunks = [](int heads) { return (heads + PC_ROWS_HEADS - 1) / PC_ROWS_HEADS; };
    const int parts = chunks(R.n_kv_heads) + (R.q_out ? chunks(R.n_q_heads) : 0), most = std::max(1, (1 << 23) / parts);       // (a launch has fewer than 2^32 threads)
    for (R.block0 = 0; R.block0 < R.n_blocks; R.block0 += most) {
        const unsigned grid = (unsigned)(std::min(most, R.n_blocks - R.block0) * parts);
        auto go = [&](auto store, auto dim) {
            constexpr int S = decltype(store)::value, D = decltype(dim)::value;
            if (blob) pc_rows_arg_kernel<S, D><<<grid, 256, 0, st>>>(*blob, R);
            else pc_rows_kernel<S, D><<<grid, 256, 0, st>>>(R);
        };
        using std::integral_constant;
        if (dtype == 2) go(integral_constant<int, 2>{}, integral_constant<int, 128>{});
        else if (dtype == 1) go(integral_constant<int, 1>{}, integral_constant<int, 128>{});
        else if (R.D == 64) go(integral_constant<int, 0>{}, integral_constant<int, 64>{});
        else go(integral_constant<int, 0>{}, integral_constant<int, 128>{});
    }
}

// ---------------------------------------------------------------------------------------------------------- gradient
// With r = 1 / sqrt(mean(x^2) + eps), u = x r, g = dy w:   dx = r (g - u mean(g u)),   dw = the sum of dy u over rows and heads.
// Of keys dy is the gradient of the keys as stored, turned back.  A block takes block_rows rows and eight heads of one kind
// (blockIdx.y: queries' chunks of heads, then keys', then values'); its sums for the weights leave as one row of partial results, which the
// last block, or a second launch, adds up in order.
// Bound: memory (8192 rows of 64 heads over 8, 654 MB: 129 us, 5.1 TB/s; 939 rows of 32 heads over 8: 11 us; sums behind them 6.5 and 3.7: 64 threads
// a dimension, eight loads each at once).
template <typename T, int D>
__device__ __forceinline__ void rows_backward(const PcRowsBwd &B, const PcRowsBwdItem *items)
{
    constexpr int E = D / 16, HALF = D / 2;
    __shared__ __attribute__((aligned(16))) float2 s_turn[4][HALF];
    __shared__ __attribute__((aligned(16))) float s_sum[4][D];
    const PcRowsBwdItem it = item_of(items, B.n_items, blockIdx.x);
    const int nq = B.q ? (B.n_q_heads + 7) / 8 : 0, nk = (B.n_kv_heads + 7) / 8;
    const int c = threadIdx.x & 7, hd = threadIdx.x >> 3 & 7, wave = threadIdx.x >> 6;
    const int lo = E * c, hi = HALF + E * c;
    const int t0 = ((int)blockIdx.x - it.block0) * B.block_rows, t1 = min(t0 + B.block_rows, it.n);
    const int kind = (int)blockIdx.y < nq ? 0 : (int)blockIdx.y < nq + nk ? 1 : 2;
    const int chunk = (int)blockIdx.y - (kind == 0 ? 0 : kind == 1 ? nq : nq + nk);
    const int heads = kind == 0 ? B.n_q_heads : B.n_kv_heads, h = min(8 * chunk + hd, heads - 1);
    const bool head_ok = 8 * chunk + hd < heads;
    if (kind == 2) {                                     // values: as they are, in the rows' type
        for (int t = t0 + wave; t < t1; t += 4) {
            float y0[E], y1[E];
            const float *src = B.d_v + ((int64_t)(it.slot0 + t) * heads + h) * D;
            load_run<float, E>(src + lo, y0);
            load_run<float, E>(src + hi, y1);
            if (!head_ok) continue;
            T *dst = (T *)B.to_v + (it.row0 + t) * B.to_v_stride + h * D;
            store_run<T, E>(dst + lo, y0);
            store_run<T, E>(dst + hi, y1);
        }
        return;
    }
    float w0[E], w1[E], dw0[E], dw1[E];
    load_weight<E>(kind == 0 ? B.q_weight : B.k_weight, lo, w0);
    load_weight<E>(kind == 0 ? B.q_weight : B.k_weight, hi, w1);
#pragma unroll
    for (int j = 0; j < E; ++j) dw0[j] = dw1[j] = 0.f;
    for (int t = t0 + wave; t < t1; t += 4) {
        const int64_t row = it.row0 + t;
        const T *src = kind == 0 ? (const T *)B.q + row * B.q_stride + h * D : (const T *)B.k + row * B.k_stride + h * D;
        const float *grad = kind == 0 ? B.d_q + (row * heads + h) * D : B.d_k + ((int64_t)(it.slot0 + t) * heads + h) * D;
        float x0[E], x1[E], y0[E], y1[E];
        load_run<T, E>(src + lo, x0);
        load_run<T, E>(src + hi, x1);
        load_run<float, E>(grad + lo, y0);
        load_run<float, E>(grad + hi, y1);
        if (kind == 1) {                                 // (a wave has a row: its own rotations)
            for (int f = threadIdx.x & 63; f < HALF; f += 64) s_turn[wave][f] = rope_turn(it.pos0 + t, B.inv_freq[f]);
            asm volatile("" ::: "memory");               // (a wave's own LDS accesses happen in order)
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const float2 cs = s_turn[wave][lo + j];
                const float a = y0[j], b = y1[j];
                y0[j] = a * cs.x + b * cs.y;
                y1[j] = b * cs.x - a * cs.y;
            }
            asm volatile("" ::: "memory");
        }
        float sq = 0.f, gx = 0.f;
#pragma unroll
        for (int j = 0; j < E; ++j) {
            sq += x0[j] * x0[j] + x1[j] * x1[j];
            gx += y0[j] * w0[j] * x0[j] + y1[j] * w1[j] * x1[j];
        }
        const float r = 1.f / sqrtf(sum8(sq) * (1.f / D) + B.eps), k = sum8(gx) * (1.f / D) * r * r;
        if (!head_ok) continue;
#pragma unroll
        for (int j = 0; j < E; ++j) {
            dw0[j] += y0[j] * x0[j] * r;
            dw1[j] += y1[j] * x1[j] * r;
            x0[j] = r * (y0[j] * w0[j] - x0[j] * k);
            x1[j] = r * (y1[j] * w1[j] - x1[j] * k);
        }
        T *dst = kind == 0 ? (T *)B.to_q + row * B.to_q_stride + h * D : (T *)B.to_k + row * B.to_k_stride + h * D;
        store_run<T, E>(dst + lo, x0);
        store_run<T, E>(dst + hi, x1);
    }
    if (!(kind == 0 ? B.to_q_weight : B.to_k_weight)) return;
#pragma unroll
    for (int j = 0; j < E; ++j)
#pragma unroll
        for (int o = 8; o < 64; o <<= 1) { dw0[j] += __shfl_xor(dw0[j], o); dw1[j] += __shfl_xor(dw1[j], o); }
    if (hd == 0) {
#pragma unroll
        for (int j = 0; j < E; ++j) { s_sum[wave][lo + j] = dw0[j]; s_sum[wave][hi + j] = dw1[j]; }
    }
    __syncthreads();
    float *to = kind == 0 ? B.q_part + ((int64_t)blockIdx.x * nq + chunk) * D : B.k_part + ((int64_t)blockIdx.x * nk + chunk) * D;
    const int d = threadIdx.x;
    const float sum = d < D ? s_sum[0][d] + s_sum[1][d] + s_sum[2][d] + s_sum[3][d] : 0.f;
    if (B.n_done == 0) {
        if (d < D) to[d] = sum;
        return;
    }
    __shared__ bool s_last;
    if (d < D) __hip_atomic_store(to + d, sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __builtin_amdgcn_s_waitcnt(0x0F70);                  // vmcnt(0): this wave's part is out
    __syncthreads();
    if (threadIdx.x == 0) {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "agent");
        s_last = atomicInc(B.done, B.n_done - 1) == B.n_done - 1;        // (wraps to zero with the last block: ready for the next call)
    }
    __syncthreads();
    if (!s_last) return;
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
    // (in shares of parts, and these in order: the same sum whichever block is last)
    constexpr int SHARES = 256 / D;
    const int share = threadIdx.x / D, e = threadIdx.x % D;
    for (int w = 0; w < 2; ++w) {
        float *out = w == 0 ? B.to_q_weight : B.to_k_weight;
        if (!out) continue;
        const float *part = w == 0 ? B.q_part : B.k_part;
        const int n = B.n_blocks * (w == 0 ? nq : nk);
        float x = 0.f;
        for (int i = share; i < n; i += 16 * SHARES) {
            float y[16];
#pragma unroll
            for (int u = 0; u < 16; ++u) y[u] = i + SHARES * u < n ? part[(int64_t)(i + SHARES * u) * D + e] : 0.f;
#pragma unroll
            for (int u = 0; u < 16; ++u) x += y[u];
        }
        __syncthreads();
        s_sum[share][e] = x;
        __syncthreads();
        if (share == 0) {
            x = 0.f;
#pragma unroll
            for (int k = 0; k < SHARES; ++k) x += s_sum[k][e];
            out[e] = x;
        }
    }
}

template <typename T, int D> __global__ __launch_bounds__(256) void pc_rows_bwd_kernel(PcRowsBwd B) { rows_backward<T, D>(B, B.items); }
template <typename T, int D> __global__ __launch_bounds__(256) void pc_rows_bwd_arg_kernel(PcArgBlob, PcRowsBwd B)
{
    rows_backward<T, D>(B, (const PcRowsBwdItem *)arguments());         // (the blob comes first)
}

// The partial sums of the weights' gradients, in order: a block 16 dims of one of them, 64 threads a dim.
__global__ __launch_bounds__(1024) void pc_rows_bwd_sum_kernel(PcRowsBwd B)
{
    __shared__ float s_sum[64][17];
    float *to = blockIdx.y == 0 ? B.to_q_weight : B.to_k_weight;
    if (!to) return;
    const float *part = blockIdx.y == 0 ? B.q_part : B.k_part;
    const int n = B.n_blocks * ((blockIdx.y == 0 ? B.n_q_heads : B.n_kv_heads) + 7 >> 3);
    const int d = blockIdx.x * 16 + (threadIdx.x & 15), share = threadIdx.x >> 4;
    float x = 0.f;
    for (int i = share; i < n; i += 8 * 64) {            // (eight at a time: the loads' latency is what this costs)
        float y[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) y[u] = i + 64 * u < n ? part[(int64_t)(i + 64 * u) * B.D + d] : 0.f;
#pragma unroll
        for (int u = 0; u < 8; ++u) x += y[u];
    }
    s_sum[share][threadIdx.x & 15] = x;
    __syncthreads();
    if (share == 0) {
        x = 0.f;
#pragma unroll
        for (int k = 0; k < 64; ++k) x += s_sum[k][threadIdx.x];
        to[d] = x;
    }
}

void pc_launch_rows_backward(int dtype, const PcRowsBwd &B, const PcArgBlob *blob, hipStream_t st)
{
    if (B.n_blocks <= 0) return;
    const unsigned nq = B.q ? (unsigned)(B.n_q_heads + 7) / 8 : 0u, nk = (unsigned)(B.n_kv_heads + 7) / 8;
    const dim3 grid((unsigned)B.n_blocks, nq + 2 * nk);
    auto go = [&](auto zero, auto dim) {
        using T = decltype(zero);
        constexpr int D = decltype(dim)::value;
        if (blob) pc_rows_bwd_arg_kernel<T, D><<<grid, 256, 0, st>>>(*blob, B);
        else pc_rows_bwd_kernel<T, D><<<grid, 256, 0, st>>>(B);
    };
    using std::integral_constant;
    if (dtype == 1) go((uint16_t)0, integral_constant<int, 128>{});
    else if (B.D == 64) go(0.f, integral_constant<int, 64>{});
    else go(0.f, integral_constant<int, 128>{});
    if (B.n_done == 0 && (B.to_q_weight || B.to_k_weight)) pc_rows_bwd_sum_kernel<<<dim3((unsigned)B.D / 16, 2), 1024, 0, st>>>(B);
}

// -------------------------------------------------------------------------------------------------------------- read
// What extents hold, as rows of tokens: a block eight slots and eight heads.  Keys: a thread 16 dims of two tokens' rows (as the append has
// them).  Values: of 4 bits, and of bf16, a thread has eight tokens of its dims at hand, and writes its part of eight rows.
// Bound: memory (8192 tokens of 8 KV heads in 4 bits: 8.9 MB read, 34 written, 14.6 us).
template <int STORE, int D> __device__ __forceinline__ void read_block(const PcRead &R, const PcReadItem *items)
{
    using T = std::conditional_t<STORE == 0, float, uint16_t>;
    constexpr int E = D / 16, HALF = D / 2;
    const PcReadItem it = item_of(items, R.n_items, blockIdx.x);
    const int t0 = 8 * ((int)blockIdx.x - it.block0);
    {
        const int c = threadIdx.x & 7, h = (int)blockIdx.y * 8 + (threadIdx.x >> 3 & 7);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int t = t0 + (threadIdx.x >> 6) + 4 * u;
            if (t >= it.n || h >= R.n_kv_heads) continue;
            const int64_t at = (int64_t)h * R.slots + it.slot0 + t, to = ((it.row0 + t) * R.n_kv_heads + h) * D;
            const int row = (it.slot0 + t) % PC_TILE;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int d = half * HALF + E * c;
                float k[E];
                if constexpr (STORE == 2) {
                    const char *kt = (const char *)R.k_store + at / PC_TILE * PC_MX4_TILE;
                    const uint32_t codes = *reinterpret_cast<const uint32_t *>(kt + row * 64 + d / 2);
                    const int e = (uint8_t)kt[PC_MX4_CODES + row * 4 + d / 32];
#pragma unroll
                    for (int j = 0; j < E; ++j) k[j] = e == PC_MX4_NAN ? __builtin_nanf("") : mx4_value(codes >> 4 * j, e - 127);
                } else {
                    load_run<T, E>((const T *)R.k_store + at * D + d, k);
                }
                if (R.k) store_run<T, E>((T *)R.k + to + d, k);
                if constexpr (STORE == 0) {
                    load_run<T, E>((const T *)R.v_store + at * D + d, k);
                    if (R.v) store_run<T, E>((T *)R.v + to + d, k);
                }
            }
        }
    }
    if constexpr (STORE != 0) {
        if (!R.v) return;
        const int h = (int)blockIdx.y * 8 + (threadIdx.x >> 4 & 7), d = 8 * (threadIdx.x & 15), half = threadIdx.x >> 7;           // (half: tokens 4 half + 0..3)
        if (h >= R.n_kv_heads) return;
        const int64_t at = (int64_t)h * R.slots + it.slot0 + t0;
        [[maybe_unused]] uint32_t w[8];
        [[maybe_unused]] uint2 x[8];
        [[maybe_unused]] uint32_t ex = 0;
        if constexpr (STORE == 2) {
            const char *vt = (const char *)R.v_store + at / PC_TILE * PC_MX4_TILE;
            const int grp = (it.slot0 + t0) % PC_TILE / 8;
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = reinterpret_cast<const uint32_t *>(vt + grp * 512)[mx4_word(d + j)];
            ex = *reinterpret_cast<const uint32_t *>(vt + PC_MX4_CODES + grp * 32 + d / 32 * 8 + 4 * half);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = *reinterpret_cast<const uint2 *>((const uint16_t *)R.v_store + (at / 8 * D + d + j) * 8 + 4 * half);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = t0 + 4 * half + i;
            if (t >= it.n) break;
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if constexpr (STORE == 2) v[j] = mx4_value(w[j] >> 4 * (4 * half + i), PC_MX4_E_MAX - (int)(ex >> 8 * i & 255u));
                else { const uint32_t p = i < 2 ? x[j].x : x[j].y; v[j] = i & 1 ? bf_hi(p) : bf_lo(p); }
            }
            store_run<uint16_t, 8>((uint16_t *)R.v + ((it.row0 + t) * R.n_kv_heads + h) * D + d, v);
        }
    }
}
template <int STORE, int D> __global__ __launch_bounds__(256) void pc_read_kernel(PcRead R) { read_block<STORE, D>(R, R.items); }
template <int STORE, int D> __global__ __launch_bounds__(256) void pc_read_arg_kernel(PcArgBlob, PcRead R)
{
    read_block<STORE, D>(R, (const PcReadItem *)arguments());           // (the blob comes first)
}

void pc_launch_read(int dtype, const PcRead &R, const PcArgBlob *blob, hipStream_t st)
{
    if (R.n_blocks <= 0) return;
    const dim3 grid((unsigned)R.n_blocks, (unsigned)(R.n_kv_heads + 7) / 8);
    auto go = [&](auto store, auto dim) {
        constexpr int S = decltype(store)::value, D = decltype(dim)::value;
        if (blob) pc_read_arg_kernel<S, D><<<grid, 256, 0, st>>>(*blob, R);
        else pc_read_kernel<S, D><<<grid, 256, 0, st>>>(R);
    };
    using std::integral_constant;
    if (dtype == 2) go(integral_constant<int, 2>{}, integral_constant<int, 128>{});
    else if (dtype == 1) go(integral_constant<int, 1>{}, integral_constant<int, 128>{});
    else if (R.D == 64) go(integral_constant<int, 0>{}, integral_constant<int, 64>{});
    else go(integral_constant<int, 0>{}, integral_constant<int, 128>{});
}
