// Single tokens of many calls that list the same messages, under a window, bf16 caches (gfx950).
//
// On its own every call reads all that it sees; here a workgroup takes a range of the tiles that any of a set of calls (up to 256 columns)
// see, reads each once, and multiplies it with the queries of those that see it.  A wave holds a group of 16 columns (as many
// calls as have 16 heads of the KV head together) and their sums for its whole life; what a call sees of a range of
// consecutive tiles (a visit) stands in a list, with the angle its queries are turned by.  What a workgroup has of a row is a split
// of it.  Tiles come by direct loads, in a ring of
// three steps.
//
// 32 calls of 8 heads a KV head over 410 of 512 messages each, window 16 384: 197 us for 343 MB (call by call 375 us for 2.1 GB, from
// the caches).  What bounds it is no longer the memory but what lies between two barriers: the longest of 16 waves, of which a third
// has anything to do in a step, and whose chain of a step (limits, scores, exponentials, values) takes 3.5 thousand cycles;
// a visit's turns are 1.5 thousand a call.  Steps of one tile took 240 us, of three 235 (registers: three tiles' values wait in
// memory), 8 waves with two groups each 250.
#include "pc_window.h"
#include "pc_mfma_common.h"

#define TILE_BYTES 8192
#define LAZY_LOG2 64.0f
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

template <int NW>
__global__ __launch_bounds__(64 * NW, NW / 4) void pc_win_shared_decode_bf16_kernel(PcWin W, PcWinShared S)
{
    constexpr int TILES = PC_WIN_STEP_TILES, RING = TILES == 2 ? 4 : 3, AHEAD = RING - 1, SLOT = 2 * TILES * TILE_BYTES, LOADS = 16 / NW * TILES;
    __shared__ __attribute__((aligned(1024))) unsigned char s_kv[RING][SLOT];
    __shared__ __attribute__((aligned(16))) float2 s_rot[NW][PC_D / 2];
    __shared__ int4 s_see[NW][16];                       // what a column's call sees of the wave's visit: pos0, n_tok, sink, lo
    __shared__ double s_freq[PC_D / 2];
    __shared__ int s_odd[RING];                          // of a place in the ring: a value is not finite

    const int kh = blockIdx.x % W.n_kv_heads;
    const win_i32x4 i0 = listed4(S.items + blockIdx.x / W.n_kv_heads), i1 = listed4((const char *)(S.items + blockIdx.x / W.n_kv_heads) + 16);
    const int visit0 = i0.x, n_steps = i0.y, call0 = i0.z, n_calls = i0.w, waves = i1.x, split0 = i1.y;
    const int g = W.n_q_heads / W.n_kv_heads, per = 16 / g;          // calls a group of columns
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const int n = lane & 15, a = lane >> 4, sub = n / g;
    const int my = wave % waves, rep = wave / waves, reps = NW / waves;      // its group of columns; its share of the steps

    const unsigned char *kb = (const unsigned char *)W.k_store + (int64_t)kh * W.slots * (PC_D * 2);
    const unsigned char *vb = (const unsigned char *)W.v_store + (int64_t)kh * W.slots * (PC_D * 2);
    const unsigned ring = (unsigned)(uintptr_t)&s_kv[0][0];
    // chunk c of key r of K sits at position c ^ turn(r): the 16 keys of a fragment hit different banks
    auto turn_of = [](int r) { return ((r & 3) << 2) | (r >> 3); };

    // the columns' queries, as they came: dims 32 ks + 8 a + 0..7, then 64 up
    const int call = my * per + sub;
    const bool real = sub < per && call < n_calls;
    uint4 q[4];
    {
        const int row = S.calls[call0 + (real ? call : 0)].row;
        const unsigned char *qp = (const unsigned char *)W.q + ((int64_t)row * W.n_q_heads + kh * g + n % g) * (PC_D * 2) + 16 * a;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) q[ks] = real ? ldg16(qp + 64 * ks) : make_uint4(0, 0, 0, 0);
    }
    if (wave == 0) s_freq[lane] = W.inv_freq[lane];
    if (wave == 0 && lane < RING) s_odd[lane] = 0;
    // (all of it is here before the first direct load is asked for: the compiler's wait would be one for all of those)
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) asm volatile("" : "+v"(q[ks].x), "+v"(q[ks].y), "+v"(q[ks].z), "+v"(q[ks].w));
    __syncthreads();

    int to_visit = visit0, to_tile = 0, to_asked = 0, to_slot = 0, to_has = 0;
    if (n_steps > 0) { to_slot = listed(&S.visits[visit0].slot0); to_has = listed(&S.visits[visit0].n_tiles); }
    auto request = [&](int place) __attribute__((always_inline)) {
        // (a tile's K and V are eight pieces each)
        const int l = lane_again(), piece = wave % 8, k_row = 4 * piece + (l >> 4);
        const unsigned k_src = (unsigned)(k_row * 256 + (((l & 15) ^ turn_of(k_row)) << 4)), v_src = (unsigned)(piece * 1024 + l * 16);
        if (to_asked > 0) {
            to_tile += TILES;
            if (to_tile >= to_has) {
                ++to_visit; to_tile = 0;
                to_slot = listed(&S.visits[to_visit].slot0); to_has = listed(&S.visits[to_visit].n_tiles);
            }
        }
        ++to_asked;
#pragma unroll
        for (int t = 0; t < TILES; ++t) {                // (behind a visit's last tile: it again, so that every step is as many loads)
            const int64_t at = ((int64_t)to_slot + PC_TILE * min(to_tile + t, to_has - 1)) * (PC_D * 2);
            const unsigned to = ring + place * SLOT + t * 2 * TILE_BYTES + piece * 1024;
            if (NW == 8 || wave < 8) dma16(kb + at, k_src, to);
            if (NW == 8 || wave >= 8) dma16(vb + at, v_src, to + TILE_BYTES);
        }
    };
    // whether a step's values are all finite: who asked for a piece of them looks at it once it is here
    auto look = [&](int place) __attribute__((always_inline)) {
        if (NW == 16 && wave < 8) return;
        const int l = lane_again();
        win_i32x4 odd = {0, 0, 0, 0};
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
            const win_i32x4 w = *(lds16)(uintptr_t)(ring + place * SLOT + t * 2 * TILE_BYTES + TILE_BYTES + (wave & 7) * 1024 + l * 16);
            // a bf16 whose exponent is all ones carries into the bit above it when one is added to the exponent
            odd |= ((w & 0x7F807F80) + 0x00800080) & (int)0x80008000;
        }
        if (__builtin_amdgcn_ballot_w64((odd.x | odd.y | odd.z | odd.w) != 0) != 0 && l == 0) s_odd[place] = 1;
    };
    for (int i = 0; i < min(AHEAD, n_steps); ++i) request(i);

    float m_ref = -INFINITY;
    f32x4 sums = {0.f, 0.f, 0.f, 0.f};                   // of the column's probabilities (four times the same)
    f32x4 acc[8];
    bf16x8 qop[4];                                       // turned and scaled
    int listers = 0;                                     // entries of the group
#pragma unroll
    for (int db = 0; db < 8; ++db) acc[db] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) qop[ks] = __builtin_bit_cast(bf16x8, make_uint4(0, 0, 0, 0));
    int visit = visit0 - 1, tile = 0, has = 0;           // the walk of what is computed
#pragma unroll 1
    for (int step = 0, place = 0; step < n_steps; ++step, place = place == RING - 1 ? 0 : place + 1) {
        if (step + AHEAD <= n_steps) wait_vm<LOADS * (AHEAD - 1)>();
        else wait_vm<0>();
        look(place);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        ring_barrier();
        const int before = place == 0 ? RING - 1 : place - 1;            // (free: the next but one step's)
        if (wave == 0 && lane_again() == 0) s_odd[before] = 0;
        tile += TILES;
        if (tile >= has) {
            ++visit; tile = 0;
            has = listed(&S.visits[visit].n_tiles);
            const int e0 = listed(&S.visits[visit].e0);
            const int first = listed(&S.visits[visit].off[my]), end = listed(&S.visits[visit].off[my + 1]);
            listers = end - first;
            asm volatile("" ::: "memory");               // (a wave's own LDS accesses happen in order)
            if (a == 0) s_see[wave][n] = make_int4(0, 0, 0, 0);
#pragma unroll 1
            for (int e = first; e < end; ++e) {
#pragma unroll
                for (int ks = 0; ks < 4; ++ks)           // (its 32 numbers, taken apart once and kept, would not fit the registers)
                    asm volatile("" : "+v"(q[ks].x), "+v"(q[ks].y), "+v"(q[ks].z), "+v"(q[ks].w));
                const win_i32x4 x = listed4(S.sees + e0 + e), y = listed4((const char *)(S.sees + e0 + e) + 16);
                const bool mine = sub == y.z;
                if (mine && a == 0) s_see[wave][n] = make_int4(x.x, x.y, x.z, x.w);
                const int64_t turn = (int64_t)(((uint64_t)(uint32_t)y.y << 32) | (uint32_t)y.x);
                const float2 cs = rope_angle((double)turn * s_freq[lane]);
                asm volatile("" ::: "memory");
                s_rot[wave][lane] = make_float2(cs.x * W.scale_log2, cs.y * W.scale_log2);
                asm volatile("" ::: "memory");
#pragma unroll
                for (int ks = 0; ks < 2; ++ks) {
                    const uint32_t lw[4] = {q[ks].x, q[ks].y, q[ks].z, q[ks].w}, hw[4] = {q[ks + 2].x, q[ks + 2].y, q[ks + 2].z, q[ks + 2].w};
                    const uint4 was[2] = {__builtin_bit_cast(uint4, qop[ks]), __builtin_bit_cast(uint4, qop[ks + 2])};
                    uint32_t xo[4] = {was[0].x, was[0].y, was[0].z, was[0].w}, yo[4] = {was[1].x, was[1].y, was[1].z, was[1].w};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float4 r = *reinterpret_cast<const float4 *>(&s_rot[wave][32 * ks + 8 * a + 2 * j]);
                        const float x0 = bf_lo(lw[j]), x1 = bf_hi(lw[j]), y0 = bf_lo(hw[j]), y1 = bf_hi(hw[j]);
                        const uint32_t px = pack_bf16(x0 * r.x - y0 * r.y, x1 * r.z - y1 * r.w), py = pack_bf16(x0 * r.y + y0 * r.x, x1 * r.w + y1 * r.z);
                        xo[j] = mine ? px : xo[j]; yo[j] = mine ? py : yo[j];
                    }
                    qop[ks] = __builtin_bit_cast(bf16x8, make_uint4(xo[0], xo[1], xo[2], xo[3]));
                    qop[ks + 2] = __builtin_bit_cast(bf16x8, make_uint4(yo[0], yo[1], yo[2], yo[3]));
                }
            }
        }
        uint32_t sees[TILES], some = 0, all = ~0u;       // bit: key of a tile; of any tile, of all there are
#pragma unroll
        for (int t = 0; t < TILES; ++t) sees[t] = 0;
        if (listers > 0 && (reps == 1 || step % reps == rep)) {
            auto first = [](unsigned k) { return k >= 32u ? ~0u : (1u << k) - 1u; };
            asm volatile("" ::: "memory");
            const int4 w = s_see[wave][n];
#pragma unroll
            for (int t = 0; t < TILES; ++t) {
                const int skip = PC_TILE * (tile + t), p = w.x + skip;
                const unsigned below = w.w <= p ? 0u : (unsigned)w.w - (unsigned)p;
                sees[t] = tile + t >= has ? 0u : first((unsigned)max(w.y - skip, 0)) & (~first(below) | first((unsigned)max(w.z - skip, 0)));
            }
#pragma unroll
            for (int t = 0; t < TILES; ++t) { some |= sees[t]; all &= sees[t]; }
        }
        if (__builtin_amdgcn_ballot_w64(some != 0) != 0) {
            const unsigned kt = ring + place * SLOT;
            float sc[8 * TILES];                         // keys 32 t + 8 a + 0..7 of column n
            {
                // (chunk a + 4 ks of a key stands where (a ^ turn) ^ 4 ks says)
                const int l = lane_again(), r = 8 * ((l & 15) >> 2) + (l & 3);
                const unsigned at = (unsigned)(r * 256 + (((l >> 4) ^ turn_of(r)) << 4));
#pragma unroll
                for (int t = 0; t < TILES; ++t)
#pragma unroll
                    for (int tau = 0; tau < 2; ++tau) {
                        f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int ks = 0; ks < 4; ++ks)
                            s = MFMA16(__builtin_bit_cast(bf16x8, *(lds16)(uintptr_t)(kt + t * 2 * TILE_BYTES + (at ^ (ks << 6)) + tau * 1024)), qop[ks], s);
#pragma unroll
                        for (int j = 0; j < 4; ++j) sc[8 * t + 4 * tau + j] = s[j];
                    }
            }
            __builtin_amdgcn_sched_barrier(0);
            const bool whole = all == ~0u;
            if (__builtin_amdgcn_ballot_w64(some != 0 && !whole) == 0) {     // (all or nothing)
#pragma unroll
                for (int j = 0; j < 8 * TILES; ++j) sc[j] = whole ? sc[j] : -INFINITY;
            } else {
#pragma unroll
                for (int t = 0; t < TILES; ++t) {
                    const uint32_t mine = sees[t] >> (8 * a);
#pragma unroll
                    for (int j = 0; j < 8; ++j) sc[8 * t + j] = (mine >> j) & 1 ? sc[8 * t + j] : -INFINITY;
                }
            }
            float mx = fmaxf(fmaxf(sc[0], sc[1]), fmaxf(sc[2], sc[3]));
#pragma unroll
            for (int j = 4; j < 8 * TILES; j += 4) mx = fmaxf(mx, fmaxf(fmaxf(sc[j], sc[j + 1]), fmaxf(sc[j + 2], sc[j + 3])));
            // The reference of a column's exponents moves only where a score is 2^LAZY above it (a column's first always is):
            // probabilities up to that are as exact, and the lanes of a column need not agree on a maximum step by step.
            if (__builtin_expect(__builtin_amdgcn_ballot_w64(mx > m_ref + LAZY_LOG2) != 0, 0)) {
                mx = fmaxf(mx, __shfl_xor(mx, 16));
                mx = fmaxf(mx, __shfl_xor(mx, 32));
                const float m_new = mx > m_ref + LAZY_LOG2 ? mx : m_ref, f = m_new == m_ref ? 1.f : ex2(m_ref - m_new);
                m_ref = m_new;
                sums *= f;
#pragma unroll
                for (int db = 0; db < 8; ++db) acc[db] *= f;
            }
            const float ref = m_ref == -INFINITY ? 0.f : m_ref;
            bf16x8 p[TILES];
#pragma unroll
            for (int t = 0; t < TILES; ++t) {
                uint32_t pk[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) pk[j] = pack_bf16(ex2(sc[8 * t + 2 * j] - ref), ex2(sc[8 * t + 2 * j + 1] - ref));
                p[t] = __builtin_bit_cast(bf16x8, make_uint4(pk[0], pk[1], pk[2], pk[3]));
            }
            // (the denominator: of the probabilities as the products take them, so that their rounding cancels)
            const bf16x8 ones = __builtin_bit_cast(bf16x8, make_uint4(0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u));
#pragma unroll
            for (int t = 0; t < TILES; ++t) sums = MFMA16(ones, p[t], sums);
            __builtin_amdgcn_sched_barrier(0);           // (values read any earlier would not fit the registers)
            const int lv = lane_again();
            const unsigned vt = kt + TILE_BYTES + (unsigned)(((lv >> 4) * PC_D + (lv & 15)) * 16);
            auto value = [&](int t, int db) __attribute__((always_inline)) { return *(lds16)(uintptr_t)(vt + t * 2 * TILE_BYTES + 256 * db); };
            if (__builtin_expect(uniform(s_odd[place]) == 0, 1)) {
#pragma unroll
                for (int db = 0; db < 8; ++db)
#pragma unroll
                    for (int t = 0; t < TILES; ++t) acc[db] = MFMA16(__builtin_bit_cast(bf16x8, value(t, db)), p[t], acc[db]);
            } else {
                // A value that is not finite: 0 times it would not be 0.  A call at a time, the values of keys that it does not see
                // cleared, and the other columns keep what they have.
#pragma unroll 1
                for (int i = 0; i < per; ++i) {
                    if ((__builtin_amdgcn_readlane((int)some, i * g)) == 0) continue;
                    const bool mine = sub == i;
#pragma unroll
                    for (int t = 0; t < TILES; ++t) {
                        const uint32_t part = (uint32_t)__builtin_amdgcn_readlane((int)sees[t], i * g) >> (8 * a);
                        win_i32x4 keep;
#pragma unroll
                        for (int j = 0; j < 4; ++j) keep[j] = (int)(((part >> (2 * j)) & 1 ? 0xFFFFu : 0u) | ((part >> (2 * j + 1)) & 1 ? 0xFFFF0000u : 0u));
#pragma unroll
                        for (int db = 0; db < 8; ++db) {
                            const f32x4 x = MFMA16(__builtin_bit_cast(bf16x8, value(t, db) & keep), p[t], acc[db]);
#pragma unroll
                            for (int j = 0; j < 4; ++j) acc[db][j] = mine ? x[j] : acc[db][j];
                            __builtin_amdgcn_sched_barrier(0);
                        }
                    }
                }
            }
        }
        // (what is asked for comes behind this step's products: the waves that have none are at it meanwhile)
        if (step + AHEAD < n_steps) request(before);
    }
    if (!real) return;
    const int64_t at = ((int64_t)S.calls[call0 + call].part0 + split0 + rep) * W.n_q_heads + kh * g + n % g;
#pragma unroll
    for (int db = 0; db < 8; ++db) *reinterpret_cast<f32x4 *>(W.part_o + at * PC_D + 16 * db + 4 * a) = acc[db];
    if (a == 0) *reinterpret_cast<float2 *>(W.part_ml + at * 2) = make_float2(sums[0] == 0.f ? -INFINITY : m_ref, sums[0]);
}

void pc_launch_win_shared_decode_bf16(const PcWin &W, const PcWinShared &S, hipStream_t st)
{
    if (S.n_items <= 0) return;
    const unsigned grid = (unsigned)S.n_items * W.n_kv_heads;
    if (S.wide) pc_win_shared_decode_bf16_kernel<16><<<grid, 1024, 0, st>>>(W, S);
    else pc_win_shared_decode_bf16_kernel<8><<<grid, 512, 0, st>>>(W, S);
}
