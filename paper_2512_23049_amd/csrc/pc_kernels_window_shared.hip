// Single tokens of many calls that list the same messages, under a window, bf16 caches (gfx950).
//
// On its own every call reads all that it sees; here a workgroup takes a range of the tiles that any of up to 16 * 16 columns' calls
// see, reads each once, and multiplies it with the queries of those that see it.  A wave holds the columns of one or two groups of 16
// (as many calls as have 16 heads of the KV head together) and their sums for its whole life; what a call sees of a range of
// consecutive tiles (a visit) stands in a list, with the angle its queries are turned by.  What a workgroup has of a row is a split
// of it.  Tiles come by direct loads, in a ring of four pairs.
//
// What bounds it is the memory behind the caches as long as several calls see a tile: 32 calls of 8 heads a KV head over 410 of 512
// messages each, window 16 384: see the launch below.
#include "pc_window.h"
#include "pc_mfma_common.h"

#define TILE_BYTES 8192
#define MFMA16(a, b, c) __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0)

namespace {

typedef const __attribute__((address_space(3))) win_i32x4 *lds16;
__device__ __forceinline__ float ex2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
template <int N> __device__ __forceinline__ void wait_vm() { __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | ((N >> 4) << 14)); }
__device__ __forceinline__ void ring_barrier() { asm volatile("s_barrier" ::: "memory"); }
// One 16-byte per lane direct load: lane l's bytes land at lds_wave_base + 16 l; completion is awaited with wait_vm.
__device__ __forceinline__ void dma16(const void *gbase_uniform, unsigned lane_off, unsigned lds_wave_base)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                 ::"s"(lds_wave_base), "v"(lane_off), "s"(gbase_uniform) : "memory", "m0");
}
// the lane's number, made where it stands: kept from the kernel's start it would wait in memory, and who fetches a register from
// there waits for all loads before it
__device__ __forceinline__ int lane_again()
{
    int x;
    asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(x));
    return x;
}
// list entries, uniform: scalar loads (a vector load's wait would be one for all direct loads)
__device__ __forceinline__ int32_t listed(const int32_t *p) { return *reinterpret_cast<const __attribute__((address_space(4))) int32_t *>(reinterpret_cast<uintptr_t>(p)); }
__device__ __forceinline__ win_i32x4 listed4(const void *p) { return *reinterpret_cast<const __attribute__((address_space(4))) win_i32x4 *>(reinterpret_cast<uintptr_t>(p)); }

}  // namespace

template <int C>
__global__ __launch_bounds__(512, 2) void pc_win_shared_decode_bf16_kernel(PcWin W, PcWinShared S)
{
    constexpr int RING = 4, AHEAD = 3, SLOT = 4 * TILE_BYTES;        // a step: two tiles
    __shared__ __attribute__((aligned(1024))) unsigned char s_kv[RING][SLOT];
    __shared__ __attribute__((aligned(16))) float2 s_rot[8][PC_D / 2];
    __shared__ int4 s_see[8][C][16];                     // what a column's call sees of the wave's visit: pos0, n_tok, sink, lo
    __shared__ double s_freq[PC_D / 2];

    const int kh = blockIdx.x % W.n_kv_heads;
    const win_i32x4 i0 = listed4(S.items + blockIdx.x / W.n_kv_heads), i1 = listed4((const char *)(S.items + blockIdx.x / W.n_kv_heads) + 16);
    const int visit0 = i0.x, n_tiles = i0.y, call0 = i0.z, n_calls = i0.w, lanes_of = i1.x, split0 = i1.y;
    const int g = W.n_q_heads / W.n_kv_heads, per = 16 / g;          // calls a group of columns
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const int n = lane & 15, a = lane >> 4, sub = n / g;
    const int my = wave % lanes_of, rep = wave / lanes_of, reps = 8 / lanes_of;       // its groups of columns; its share of the tiles

    const unsigned char *kb = (const unsigned char *)W.k_store + (int64_t)kh * W.slots * (PC_D * 2);
    const unsigned char *vb = (const unsigned char *)W.v_store + (int64_t)kh * W.slots * (PC_D * 2);
    const unsigned ring = (unsigned)(uintptr_t)&s_kv[0][0];
    // chunk c of key r of K sits at position c ^ turn(r): the 16 keys of a fragment hit different banks
    auto turn_of = [](int r) { return ((r & 3) << 2) | (r >> 3); };

    // the columns' queries, as they came: dims 32 ks + 8 a + 0..7, then 64 up
    uint4 q[C][4];
    if (wave == 0) s_freq[lane] = W.inv_freq[lane];
    bool real[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int call = (my * C + c) * per + sub;
        real[c] = sub < per && call < n_calls;
        const int row = S.calls[call0 + (real[c] ? call : 0)].row;
        const unsigned char *qp = (const unsigned char *)W.q + ((int64_t)row * W.n_q_heads + kh * g + n % g) * (PC_D * 2) + 16 * a;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) q[c][ks] = real[c] ? ldg16(qp + 64 * ks) : make_uint4(0, 0, 0, 0);
    }
    // (they are here before the first direct load is asked for: the compiler's wait for them would be one for all of those)
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) asm volatile("" : "+v"(q[c][ks].x), "+v"(q[c][ks].y), "+v"(q[c][ks].z), "+v"(q[c][ks].w));

    const int n_steps = (n_tiles + 1) / 2;
    int to_visit = visit0, to_tile = 0, to_asked = 0, to_slot = 0, to_has = 0;
    if (n_tiles > 0) { to_slot = listed(&S.visits[visit0].slot0); to_has = listed(&S.visits[visit0].n_tiles); }
    auto request = [&](int place) __attribute__((always_inline)) {
        const int l = lane_again(), k_row = 4 * wave + (l >> 4);
        const unsigned k_src = (unsigned)(k_row * 256 + (((l & 15) ^ turn_of(k_row)) << 4)), v_src = (unsigned)(wave * 1024 + l * 16);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            if (to_asked > 0 && to_asked < n_tiles) {    // (behind the last tile: it again, so that every step is four loads)
                if (++to_tile == to_has) {
                    ++to_visit; to_tile = 0;
                    to_slot = listed(&S.visits[to_visit].slot0); to_has = listed(&S.visits[to_visit].n_tiles);
                }
            }
            ++to_asked;
            const int64_t at = ((int64_t)to_slot + PC_TILE * to_tile) * (PC_D * 2);
            const unsigned to = ring + place * SLOT + half * 2 * TILE_BYTES + wave * 1024;
            dma16(kb + at, k_src, to);
            dma16(vb + at, v_src, to + TILE_BYTES);
        }
    };
    for (int i = 0; i < min(AHEAD, n_steps); ++i) request(i);

    float m_run[C], l_run[C];
    f32x4 acc[C][8];
    bf16x8 qop[C][4];                                    // turned and scaled
    int listers[C];                                      // entries of the group (uniform)
#pragma unroll
    for (int c = 0; c < C; ++c) {
        m_run[c] = -INFINITY; l_run[c] = 0.f; listers[c] = 0;
#pragma unroll
        for (int db = 0; db < 8; ++db) acc[c][db] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) qop[c][ks] = __builtin_bit_cast(bf16x8, make_uint4(0, 0, 0, 0));
    }
    int visit = visit0 - 1, tile = 0, has = 0;           // the walk of what is computed
#pragma unroll 1
    for (int step = 0, place = 0; step < n_steps; ++step, place = (place + 1) & (RING - 1)) {
        if (step + AHEAD <= n_steps) wait_vm<4 * (AHEAD - 1)>();
        else wait_vm<0>();
        ring_barrier();
        if (step + AHEAD < n_steps) request((place + AHEAD) & (RING - 1));
#pragma unroll 1
        for (int half = 0; half < 2; ++half) {
            const int t = 2 * step + half;
            if (t >= n_tiles) break;
            if (++tile >= has) {
                ++visit; tile = 0;
                has = listed(&S.visits[visit].n_tiles);
                const int e0 = listed(&S.visits[visit].e0);
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    const int first = listed(&S.visits[visit].off[my * C + c]), end = listed(&S.visits[visit].off[my * C + c + 1]);
                    listers[c] = end - first;
                    asm volatile("" ::: "memory");       // (a wave's own LDS accesses happen in order)
                    if (a == 0) s_see[wave][c][n] = make_int4(0, 0, 0, 0);
#pragma unroll 1
                    for (int e = first; e < end; ++e) {
#pragma unroll
                        for (int ks = 0; ks < 4; ++ks)   // (its 32 numbers, taken apart once and kept, would not fit the registers)
                            asm volatile("" : "+v"(q[c][ks].x), "+v"(q[c][ks].y), "+v"(q[c][ks].z), "+v"(q[c][ks].w));
                        const win_i32x4 x = listed4(S.sees + e0 + e), y = listed4((const char *)(S.sees + e0 + e) + 16);
                        const bool mine = sub == y.z;
                        if (mine && a == 0) s_see[wave][c][n] = make_int4(x.x, x.y, x.z, x.w);
                        const int64_t turn = (int64_t)(((uint64_t)(uint32_t)y.y << 32) | (uint32_t)y.x);
                        const float2 cs = rope_angle((double)turn * s_freq[lane]);
                        asm volatile("" ::: "memory");
                        s_rot[wave][lane] = make_float2(cs.x * W.scale_log2, cs.y * W.scale_log2);
                        asm volatile("" ::: "memory");
#pragma unroll
                        for (int ks = 0; ks < 2; ++ks) {
                            const uint32_t lw[4] = {q[c][ks].x, q[c][ks].y, q[c][ks].z, q[c][ks].w}, hw[4] = {q[c][ks + 2].x, q[c][ks + 2].y, q[c][ks + 2].z, q[c][ks + 2].w};
                            uint4 was[2] = {__builtin_bit_cast(uint4, qop[c][ks]), __builtin_bit_cast(uint4, qop[c][ks + 2])};
                            uint32_t xo[4] = {was[0].x, was[0].y, was[0].z, was[0].w}, yo[4] = {was[1].x, was[1].y, was[1].z, was[1].w};
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const float4 r = *reinterpret_cast<const float4 *>(&s_rot[wave][32 * ks + 8 * a + 2 * j]);
                                const float x0 = bf_lo(lw[j]), x1 = bf_hi(lw[j]), y0 = bf_lo(hw[j]), y1 = bf_hi(hw[j]);
                                const uint32_t px = pack_bf16(x0 * r.x - y0 * r.y, x1 * r.z - y1 * r.w), py = pack_bf16(x0 * r.y + y0 * r.x, x1 * r.w + y1 * r.z);
                                xo[j] = mine ? px : xo[j]; yo[j] = mine ? py : yo[j];
                            }
                            qop[c][ks] = __builtin_bit_cast(bf16x8, make_uint4(xo[0], xo[1], xo[2], xo[3]));
                            qop[c][ks + 2] = __builtin_bit_cast(bf16x8, make_uint4(yo[0], yo[1], yo[2], yo[3]));
                        }
                    }
                }
            }
            if (t % reps != rep) continue;
            uint32_t sees[C];
            bool some[C], any = false;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                auto first = [](unsigned k) { return k >= 32u ? ~0u : (1u << k) - 1u; };
                if (listers[c] == 0) { sees[c] = 0; some[c] = false; continue; }
                asm volatile("" ::: "memory");
                const int4 w = s_see[wave][c][n];
                const int p = w.x + PC_TILE * tile;
                const unsigned below = w.w <= p ? 0u : (unsigned)w.w - (unsigned)p;
                sees[c] = first((unsigned)max(w.y - PC_TILE * tile, 0)) & (~first(below) | first((unsigned)max(w.z - PC_TILE * tile, 0)));
                some[c] = __builtin_amdgcn_ballot_w64(sees[c] != 0) != 0;
                any |= some[c];
            }
            if (!any) continue;
            const unsigned kt = ring + place * SLOT + half * 2 * TILE_BYTES, vt = kt + TILE_BYTES;
            f32x4 s[C][2];
            {
                win_i32x4 k[2][4];
                // (chunk a + 4 ks of a key stands where (a ^ turn) ^ 4 ks says)
                const int l = lane_again(), r = 8 * ((l & 15) >> 2) + (l & 3);
                const unsigned at = (unsigned)(r * 256 + (((l >> 4) ^ turn_of(r)) << 4));
#pragma unroll
                for (int tau = 0; tau < 2; ++tau) {
#pragma unroll
                    for (int ks = 0; ks < 4; ++ks) k[tau][ks] = *(lds16)(uintptr_t)(kt + (at ^ (ks << 6)) + tau * 1024);
                }
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    if (!some[c]) continue;
#pragma unroll
                    for (int tau = 0; tau < 2; ++tau) {
                        s[c][tau] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int ks = 0; ks < 4; ++ks) s[c][tau] = MFMA16(__builtin_bit_cast(bf16x8, k[tau][ks]), qop[c][ks], s[c][tau]);
                    }
                }
            }
#pragma unroll
            for (int c = 0; c < C; ++c) {
                __builtin_amdgcn_sched_barrier(0);
                if (!some[c]) continue;
                const int l = lane_again();
                const unsigned v_at = (unsigned)(((l >> 4) * PC_D + (l & 15)) * 16);
                win_i32x4 v[8];                          // (read again for the second group: registers)
#pragma unroll
                for (int db = 0; db < 8; ++db) v[db] = *(lds16)(uintptr_t)(vt + v_at + 256 * db);
                const uint32_t mine = sees[c] >> (8 * a);
                float sc[8];                             // keys 8 a + 0..7 of column n
#pragma unroll
                for (int j = 0; j < 8; ++j) sc[j] = (mine >> j) & 1 ? s[c][j >> 2][j & 3] : -INFINITY;
                float mx = fmaxf(fmaxf(fmaxf(sc[0], sc[1]), fmaxf(sc[2], sc[3])), fmaxf(fmaxf(sc[4], sc[5]), fmaxf(sc[6], sc[7])));
                mx = fmaxf(mx, __shfl_xor(mx, 16));
                mx = fmaxf(mx, __shfl_xor(mx, 32));
                const float m_new = fmaxf(m_run[c], mx), m_safe = m_new == -INFINITY ? 0.f : m_new, alpha = m_run[c] == m_new ? 1.f : ex2(m_run[c] - m_safe);
                uint32_t pk[4];
                float ps = 0.f;                          // (of the probabilities as the products take them: their rounding cancels)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    pk[j] = pack_bf16(ex2(sc[2 * j] - m_safe), ex2(sc[2 * j + 1] - m_safe));
                    ps += bf_lo(pk[j]) + bf_hi(pk[j]);
                }
                l_run[c] = l_run[c] * alpha + ps;
                m_run[c] = m_new;
                if (__builtin_amdgcn_ballot_w64(alpha != 1.f) != 0) {       // rare once the running maxima have settled
#pragma unroll
                    for (int db = 0; db < 8; ++db) acc[c][db] *= alpha;
                }
                const bf16x8 p = __builtin_bit_cast(bf16x8, make_uint4(pk[0], pk[1], pk[2], pk[3]));
                const bool whole = sees[c] == ~0u;
                if (__builtin_amdgcn_ballot_w64(real[c] && !whole) == 0) {
#pragma unroll
                    for (int db = 0; db < 8; ++db) acc[c][db] = MFMA16(__builtin_bit_cast(bf16x8, v[db]), p, acc[c][db]);
                } else if (__builtin_amdgcn_ballot_w64(sees[c] != 0 && !whole) == 0) {
                    // columns that see nothing of the tile keep what they have: a value need not be finite, and 0 times it would not be 0
#pragma unroll
                    for (int db = 0; db < 8; ++db) {
                        const f32x4 was = acc[c][db], x = MFMA16(__builtin_bit_cast(bf16x8, v[db]), p, was);
#pragma unroll
                        for (int j = 0; j < 4; ++j) acc[c][db][j] = whole ? x[j] : was[j];
                    }
                } else {
                    // a call at a time, the values of keys that it does not see cleared
#pragma unroll 1
                    for (int i = 0; i < per; ++i) {
                        const uint32_t its = (uint32_t)__builtin_amdgcn_readlane((int)sees[c], i * g);
                        if (its == 0) continue;
                        const uint32_t part = its >> (8 * a);
                        win_i32x4 keep;
#pragma unroll
                        for (int j = 0; j < 4; ++j) keep[j] = (int)( ((part >> (2 * j)) & 1 ? 0xFFFFu : 0u) | ((part >> (2 * j + 1)) & 1 ? 0xFFFF0000u : 0u));
#pragma unroll
                        for (int db = 0; db < 8; ++db) {
                            const f32x4 was = acc[c][db], x = MFMA16(__builtin_bit_cast(bf16x8, v[db] & keep), p, was);
#pragma unroll
                            for (int j = 0; j < 4; ++j) acc[c][db][j] = sub == i ? x[j] : was[j];
                        }
                    }
                }
            }
        }
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
        l_run[c] += __shfl_xor(l_run[c], 16);
        l_run[c] += __shfl_xor(l_run[c], 32);
        if (!real[c]) continue;
        const int64_t at = ((int64_t)S.calls[call0 + (my * C + c) * per + sub].part0 + split0 + rep) * W.n_q_heads + kh * g + n % g;
#pragma unroll
        for (int db = 0; db < 8; ++db) *reinterpret_cast<f32x4 *>(W.part_o + at * PC_D + 16 * db + 4 * a) = acc[c][db];
        if (a == 0) *reinterpret_cast<float2 *>(W.part_ml + at * 2) = make_float2(l_run[c] == 0.f ? -INFINITY : m_run[c], l_run[c]);
    }
}

void pc_launch_win_shared_decode_bf16(const PcWin &W, const PcWinShared &S, hipStream_t st)
{
    if (S.n_items <= 0) return;
    const unsigned grid = (unsigned)S.n_items * W.n_kv_heads;
    if (S.wide) pc_win_shared_decode_bf16_kernel<2><<<grid, 512, 0, st>>>(W, S);
    else pc_win_shared_decode_bf16_kernel<1><<<grid, 512, 0, st>>>(W, S);
}
