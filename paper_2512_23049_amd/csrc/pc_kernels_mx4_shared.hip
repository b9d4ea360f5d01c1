// Single tokens of many calls that list the same messages, over a PC_MX4 cache (gfx950): every tile once, as pc_kernels_window_shared.hip has
// it for bf16 (its lists, its walk over visits, its lazy reference), with the products of pc_kernels_mx4.hip.
//
// A workgroup takes a range of the tiles that any of a set of calls (up to 256 columns) see; a wave holds a group of 16 columns and
// their sums for its whole life.  Tiles come as they are stored, 4352 bytes, by direct loads into a ring of four steps of two; the
// workgroup converts a step's values to fp16 (or bf16, where fp16 does not hold them) together, one step ahead, so that no wave has their codes and powers to take apart.  A
// wave's queries are turned for all of a visit's calls at once, each lane by its own call's rotation.
//
// Bound: no unit alone.  32 calls over 410 of 512 messages of 160 tokens each, 64 heads over 8 (2850 distinct tiles): 195 us, of which
// the vector unit is busy in 48 %, shared memory in 33 % and the matrix unit in 22 %: sixteen waves meet at a barrier a step and do the same at the
// same time.  (At 217 us:) without the products of the values it takes 28 us less, without the turned queries' pieces 31, without the conversion of values 18, without
// exponentials 13, without loads 8; 16 are its start and the partial results.  Call by call the same batch takes 365 us and reads 26 times as much.
#include "pc_window.h"
#include "pc_mx4.h"
#include "pc_mx4_products.h"

#include <type_traits>

#define TURNS 4               // rotations that a wave has at hand at once

namespace {

typedef const __attribute__((address_space(3))) win_i32x4 *lds16;
typedef __attribute__((address_space(3))) win_i32x4 *lds16_out;
typedef const __attribute__((address_space(3))) uint32_t *lds4;
typedef uint32_t mx4_u32x2 __attribute__((ext_vector_type(2)));
typedef const __attribute__((address_space(3))) mx4_u32x2 *lds8;
template <int N> __device__ __forceinline__ void wait_vm() { __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | ((N >> 4) << 14)); }
__device__ __forceinline__ void ring_barrier() { asm volatile("s_barrier" ::: "memory"); }
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


constexpr int TILES = PC_WIN_STEP_TILES, RING = 4, AHEAD = RING - 1;
// of a tile in the ring: codes of keys and of values, exponents of keys and of values (256 bytes each: a direct load's lanes)
constexpr int VALUES = PC_MX4_CODES, K_EXPS = 2 * PC_MX4_CODES, V_EXPS = K_EXPS + 256, TILE = V_EXPS + 256, SLOT = TILES * TILE;

}  // namespace

template <int NW> struct SharedLds {
    unsigned char kv[RING][SLOT] __attribute__((aligned(1024)));
    unsigned char v[2][TILES][PC_TILE * PC_D * 2] __attribute__((aligned(1024)));       // values as a bf16 cache has them (or in fp16), of this step and the next
    _Float16 rot[NW][TURNS][2][PC_D / 2] __attribute__((aligned(16)));                  // cosines, sines
    int4 see[NW][16];                                    // what a column's call sees of the wave's visit: pos0, n_tok, sink, lo
    double freq[PC_D / 2];
};
// HALF: probabilities and values in fp16, where no value of the cache is outside it.  A probability of a column's reference is 2^6 then, and the reference
// moves where one would be above 2^15: what is 2^20 below a column's largest still is a normal number, and 2^31 below it one of a few bits.
template <int NW, bool HALF> __device__ __forceinline__ void shared_decode(const PcWin &W, const PcWinShared &S, SharedLds<NW> &lds)
{
    constexpr int LOADS = 16 / NW;
    constexpr float LAZY_LOG2 = HALF ? 15.f : 32.f, ABOVE = HALF ? 6.f : 0.f;         // (2^31 keys of 2^32 x 6 x 2^60 fit 32 bits)
    auto &s_kv = lds.kv;
    auto &s_v = lds.v;
    auto &s_rot = lds.rot;
    auto &s_see = lds.see;
    auto &s_freq = lds.freq;

    const int kh = blockIdx.x % W.n_kv_heads;
    const win_i32x4 i0 = listed4(S.items + blockIdx.x / W.n_kv_heads), i1 = listed4((const char *)(S.items + blockIdx.x / W.n_kv_heads) + 16);
    const int visit0 = i0.x, n_steps = i0.y, call0 = i0.z, n_calls = i0.w, waves = i1.x, split0 = i1.y;
    const int g = W.n_q_heads / W.n_kv_heads, per = 16 / g;          // calls a group of columns
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const int n = lane & 15, a = lane >> 4, sub = n / g;
    const int my = wave % waves, rep = wave / waves, reps = NW / waves;      // its group of columns; its share of the steps

    const unsigned char *kb = (const unsigned char *)W.k_store + (int64_t)kh * (W.slots / PC_TILE) * PC_MX4_TILE;
    const unsigned char *vb = (const unsigned char *)W.v_store + (int64_t)kh * (W.slots / PC_TILE) * PC_MX4_TILE;
    const unsigned ring = (unsigned)(uintptr_t)&s_kv[0][0];

    // the columns' queries, as they came: dims 16 a + 0..15, then 64 up
    const int call = my * per + sub;
    const bool real = sub < per && call < n_calls;
    uint4 q[4];
    int low;                                             // the least position that its call sees but for sinks
    {
        const int row = S.calls[call0 + (real ? call : 0)].row;
        low = win_low(W.q_pos[row], W.window);
        const unsigned char *qp = (const unsigned char *)W.q + ((int64_t)row * W.n_q_heads + kh * g + n % g) * (PC_D * 2) + 32 * a;
#pragma unroll
        for (int i = 0; i < 4; ++i) q[i] = real ? ldg16(qp + 128 * (i >> 1) + 16 * (i & 1)) : make_uint4(0, 0, 0, 0);
    }
    if (wave == 0) s_freq[lane] = W.inv_freq[lane];
    // (all of it is here before the first direct load is asked for: the compiler's wait would be one for all of those)
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
    for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(q[i].x), "+v"(q[i].y), "+v"(q[i].z), "+v"(q[i].w));
    // the row's unit, for every turn (which keeps a pair's norm): its largest value, scaled, between 128 and 256
    float unit;
    {
        float top = 0.f;
        bool fine = true;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t w[4] = {q[i].x, q[i].y, q[i].z, q[i].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) top = mx4_top(top, w[j], fine);
        }
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        unit = mx4_unit(top * W.scale_log2);
        // (a query that holds what is no number: all of it is NaN)
        int all = fine;
        all &= __shfl_xor(all, 16);
        all &= __shfl_xor(all, 32);
        const float by = W.scale_log2 / unit;
#pragma unroll
        for (int i = 0; i < 4; ++i) q[i] = all ? mx4_halves(q[i], by) : make_uint4(0x7E007E00u, 0x7E007E00u, 0x7E007E00u, 0x7E007E00u);
    }
    __syncthreads();

    // (what the walks need of a visit they ask for a visit ahead: a latency each otherwise)
    const int last = visit0 + i1.z - 1;
    int to_visit = visit0, to_tile = 0, to_asked = 0, to_slot = 0, to_has = 0, to_next_slot = 0, to_next_has = 0;
    auto ahead = [&]() __attribute__((always_inline)) {
        const PcWinVisit *v = S.visits + min(to_visit + 1, last);
        to_next_slot = listed(&v->slot0); to_next_has = listed(&v->n_tiles);
    };
    if (n_steps > 0) {
        to_slot = listed(&S.visits[visit0].slot0); to_has = listed(&S.visits[visit0].n_tiles);
        ahead();
    }
    auto request = [&](int place) __attribute__((always_inline)) {
        const int l = lane_again();
        if (to_asked > 0) {
            to_tile += TILES;
            if (to_tile >= to_has) {
                ++to_visit; to_tile = 0;
                to_slot = to_next_slot; to_has = to_next_has;
                ahead();
            }
        }
        ++to_asked;
        // a tile is eight loads: two of codes of keys, two of values, and their exponents (twice, so that every wave asks as often)
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int job = wave + NW * i, t = job >> 3, part = job & 7;
            const bool of_keys = part < 4;
            // (behind a visit's last tile: it again)
            const unsigned char *from = (of_keys ? kb : vb) + (int64_t)(to_slot / PC_TILE + min(to_tile + t, to_has - 1)) * PC_MX4_TILE;
            const unsigned to = (unsigned)uniform((int)(ring + place * SLOT + t * TILE));
            if ((part & 2) == 0) {
                // position p of the keys' codes holds block (p & 3) ^ (key >> 3) of key p >> 2; of the values' half (p & 1) ^ (m >> 3) of m = p / 2 % 16:
                // what the lanes of a fragment read at once hits different banks
                const int p = (part & 1) * 64 + l;
                const unsigned key_at = (unsigned)((p >> 2) * 64 + (((p & 3) ^ (p >> 5)) << 4)), value_at = (unsigned)((p >> 1) * 32 + (((p & 1) ^ (p >> 4 & 1)) << 4));
                mx4_dma16(from, of_keys ? key_at : value_at, to + (of_keys ? 0 : VALUES) + (part & 1) * 1024);
            } else mx4_dma4(from, (unsigned)(PC_MX4_CODES + (l & 31) * 4), to + (of_keys ? K_EXPS : V_EXPS));
        }
    };
    // a step's values: a thread eight slots of a dimension (or of two)
    // (where a thread's part of a step stands is worked out once)
    unsigned conv_codes, conv_exps, conv_to;
    {
        const int thread = wave * 64 + lane_again(), t = thread >> 9, grp = thread >> 7 & 3, d = thread & 127, m = d & 15, db = d >> 4;
        conv_codes = ring + t * TILE + VALUES + grp * 512 + m * 32 + (((db >> 2) ^ (m >> 3)) << 4) + (db & 3) * 4;
        conv_exps = ring + t * TILE + V_EXPS + grp * 32 + (d >> 5) * 8;
        conv_to = (unsigned)(uintptr_t)&s_v[0][0][0] + thread * 16;
        asm volatile("" : "+v"(conv_codes), "+v"(conv_exps), "+v"(conv_to));
    }
    auto convert = [&](int place, int to) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const unsigned at = place * SLOT + (64 * NW * i >> 9) * TILE;
            const uint32_t w = *(lds4)(uintptr_t)(conv_codes + at);
            const mx4_u32x2 ex = *(lds8)(uintptr_t)(conv_exps + at);
            uint4 x;
            x.x = mx4_numbers<HALF>(w, ex.x, std::integral_constant<int, 0>{}); x.y = mx4_numbers<HALF>(w, ex.x, std::integral_constant<int, 1>{});
            x.z = mx4_numbers<HALF>(w, ex.y, std::integral_constant<int, 2>{}); x.w = mx4_numbers<HALF>(w, ex.y, std::integral_constant<int, 3>{});
            *(lds16_out)(uintptr_t)(conv_to + to * (TILES * PC_TILE * PC_D * 2) + 64 * NW * i * 16) = __builtin_bit_cast(win_i32x4, x);
        }
    };
    for (int i = 0; i < min(AHEAD, n_steps); ++i) request(i);
    if (n_steps > 0) {
        if (n_steps >= AHEAD) wait_vm<LOADS * (AHEAD - 1)>();
        else wait_vm<0>();
        ring_barrier();
        convert(0, 0);
    }

    float m_ref = -INFINITY;
    f32x4 sums = {0.f, 0.f, 0.f, 0.f};                   // of the column's probabilities (four times the same)
    f32x4 acc[8];
    mx4_i32x8 q_hi, q_lo;                                // turned and scaled, in two pieces
    int listers = 0;                                     // entries of the group
    int whole_to = 0;                                    // tiles of the visit that the column sees whole, from the first one on; -1: it sees nothing of the visit
#pragma unroll
    for (int db = 0; db < 8; ++db) acc[db] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 8; ++i) q_hi[i] = q_lo[i] = 0;
    const int e_hi = (int)(__float_as_uint(unit) >> 23), e_lo = e_hi - 4;
    int visit = visit0 - 1, tile = 0, has = 0;           // the walk of what is computed
    int next_has = 0, next_e0 = 0, next_first = 0, next_end = 0;
    auto header = [&]() __attribute__((always_inline)) {
        const PcWinVisit *v = S.visits + min(visit + 1, last);
        next_has = listed(&v->n_tiles); next_e0 = listed(&v->e0); next_first = listed(&v->off[my]); next_end = listed(&v->off[my + 1]);
    };
    if (n_steps > 0) header();
#pragma unroll 1
    for (int step = 0, place = 0; step < n_steps; ++step, place = place == RING - 1 ? 0 : place + 1) {
        if (step + AHEAD <= n_steps) wait_vm<LOADS * (AHEAD - 2)>();           // (the next step's tiles too)
        else wait_vm<0>();
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        ring_barrier();
        const int before = place == 0 ? RING - 1 : place - 1;            // (free: the next but one step's)
        tile += TILES;
        if (tile >= has) {
            ++visit; tile = 0;
            has = next_has;
            const int e0 = next_e0, first = next_first, end = next_end;
            header();
            listers = end - first;
            asm volatile("" ::: "memory");               // (a wave's own LDS accesses happen in order)
            if (a == 0) s_see[wave][n] = make_int4(0, 0, 0, 0);
#pragma unroll 1
            for (int e = first; e < end; e += TURNS) {
                int of = -1;                             // which of the rotations is the lane's
                asm volatile("" ::: "memory");
                win_i32x4 x[TURNS];                      // (all at once: one latency)
#pragma unroll
                for (int i = 0; i < TURNS; ++i) {
                    x[i] = listed4((const PcMx4See *)S.sees + e0 + min(e + i, end - 1));
                }
#pragma unroll
                for (int i = 0; i < TURNS; ++i) {
                    if (e + i >= end) break;
                    const uint32_t packed = (uint32_t)x[i].y;
                    const bool mine = sub == (int)(packed >> 28);
                    if (mine && a == 0) s_see[wave][n] = make_int4(x[i].x, (int)(packed & PC_MX4_SEE_TOKENS), x[i].z, low);
                    of = mine ? i : of;
                    const int64_t turn = (int64_t)((uint64_t)(packed >> 26 & 3) << 62 | (uint64_t)(uint32_t)x[i].w << 30) >> 30;
                    const float2 cs = mx4_rotation((double)turn * s_freq[lane]);
                    s_rot[wave][i][0][lane] = (_Float16)cs.x; s_rot[wave][i][1][lane] = (_Float16)cs.y;
                }
                asm volatile("" ::: "memory");
                const uint4 *rot = reinterpret_cast<const uint4 *>(&s_rot[wave][max(of, 0)][0][16 * a]);          // (sines: eight further)
#pragma unroll
                for (int s = 0; s < 4; ++s) {            // dims 16 a + 4 s, and 64 up
                    int u_hi, u_rest, v_hi, v_rest;
                    const uint4 c = rot[s >> 1], t = rot[8 + (s >> 1)];
                    mx4_turned(mx4_two(q[s >> 1], s & 1), mx4_two(q[2 + (s >> 1)], s & 1), mx4_two(c, s & 1), mx4_two(t, s & 1), u_hi, u_rest, v_hi, v_rest);
                    q_hi[s] = of >= 0 ? u_hi : q_hi[s]; q_lo[s] = of >= 0 ? u_rest : q_lo[s];
                    q_hi[4 + s] = of >= 0 ? v_hi : q_hi[4 + s]; q_lo[4 + s] = of >= 0 ? v_rest : q_lo[4 + s];
                }
                asm volatile("" ::: "memory");
            }
            const int4 w = s_see[wave][n];
            whole_to = w.y <= 0 ? -1 : w.w <= w.x ? min(w.y / PC_TILE, has) : 0;
        }
        uint32_t sees[TILES], some = 0, all = ~0u;       // bit: key of a tile; of any tile, of all there are
#pragma unroll
        for (int t = 0; t < TILES; ++t) sees[t] = 0;
        if (listers == 0 || (reps > 1 && step % reps != rep)) {
        } else if (__builtin_amdgcn_ballot_w64(whole_to >= 0 && tile + TILES > whole_to) == 0) {
            some = all = whole_to < 0 ? 0u : ~0u;
        } else {
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
            float sc[8 * TILES];                         // keys 32 t + 8 a + 0..7 of column n, less the column's reference
            const float ref = m_ref == -INFINITY ? 0.f : m_ref;
            {
                const int l = lane_again(), m = l & 15, key = 8 * (m >> 2) + (m & 3);
                const unsigned at = (unsigned)(key * 64 + (((l >> 4) ^ (key >> 3)) << 4));
#pragma unroll
                for (int t = 0; t < TILES; ++t)
#pragma unroll
                    for (int tau = 0; tau < 2; ++tau) {
                        const uint4 codes = __builtin_bit_cast(uint4, *(lds16)(uintptr_t)(kt + t * TILE + at + tau * 256));
                        const int e = (int)(*(lds4)(uintptr_t)(kt + t * TILE + K_EXPS + key * 4 + tau * 16) >> (8 * (l >> 4)));
                        f32x4 s = mx4_scores16(codes, e, q_lo, e_lo, (f32x4){-ref, -ref, -ref, -ref});
                        s = mx4_scores16(codes, e, q_hi, e_hi, s);
#pragma unroll
                        for (int j = 0; j < 4; ++j) sc[8 * t + 4 * tau + j] = s[j];
                    }
            }
            __builtin_amdgcn_sched_barrier(0);
            const bool whole = all == ~0u;
            if (__builtin_amdgcn_ballot_w64(!whole) == 0) {                  // (nothing is masked)
            } else if (__builtin_amdgcn_ballot_w64(some != 0 && !whole) == 0) {          // (all or nothing)
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
            // (on the bit patterns, which take no care of NaN: right wherever some score is above the reference)
            auto fi = [](float x) { return __float_as_int(x); };
            int top = imax3(fi(sc[0]), fi(sc[1]), fi(sc[2]));
#pragma unroll
            for (int j = 3; j < 8 * TILES - 1; j += 2) top = imax3(top, fi(sc[j]), fi(sc[j + 1]));
            top = max(top, fi(sc[8 * TILES - 1]));
            // The reference of a column's exponents moves only where a score is 2^LAZY above it (a column's first always is):
            // probabilities up to that are as exact, and the lanes of a column need not agree on a maximum step by step.
            if (__builtin_expect(__builtin_amdgcn_ballot_w64(top > fi(LAZY_LOG2) || (m_ref == -INFINITY && some != 0)) != 0, 0)) {
                const float limit = m_ref == -INFINITY ? -INFINITY : LAZY_LOG2;
                float mx = sc[0];
#pragma unroll
                for (int j = 1; j < 8 * TILES; ++j) mx = fmaxf(mx, sc[j]);
                mx = fmaxf(mx, __shfl_xor(mx, 16));
                mx = fmaxf(mx, __shfl_xor(mx, 32));
                const bool up = mx > limit;
                const float m_new = up ? ref + mx - ABOVE : m_ref, by = up ? m_new - ref : 0.f, f = !up ? 1.f : m_ref == -INFINITY ? 0.f : ex2(-by);
                m_ref = m_new;
                sums *= f;
#pragma unroll
                for (int db = 0; db < 8; ++db) acc[db] *= f;
#pragma unroll
                for (int j = 0; j < 8 * TILES; ++j) sc[j] -= by;
            }
            bf16x8 p[TILES];
#pragma unroll
            for (int t = 0; t < TILES; ++t) {
                uint32_t pk[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) pk[j] = mx4_pack<HALF>(ex2(sc[8 * t + 2 * j]), ex2(sc[8 * t + 2 * j + 1]));
                p[t] = __builtin_bit_cast(bf16x8, make_uint4(pk[0], pk[1], pk[2], pk[3]));
            }
            // (the denominator: of the probabilities as the products take them, so that their rounding cancels)
            constexpr uint32_t ONES = HALF ? 0x3C003C00u : 0x3F803F80u;
            const bf16x8 ones = __builtin_bit_cast(bf16x8, make_uint4(ONES, ONES, ONES, ONES));
#pragma unroll
            for (int t = 0; t < TILES; ++t) sums = mx4_mfma16<HALF>(ones, p[t], sums);
            __builtin_amdgcn_sched_barrier(0);           // (values read any earlier would not fit the registers)
            const int lv = lane_again();
            const unsigned vt = (unsigned)(uintptr_t)&s_v[step & 1][0][0] + (unsigned)(((lv >> 4) * PC_D + (lv & 15)) * 16);
#pragma unroll
            for (int db = 0; db < 8; ++db)
#pragma unroll
                for (int t = 0; t < TILES; ++t)
                    acc[db] = mx4_mfma16<HALF>(__builtin_bit_cast(bf16x8, *(lds16)(uintptr_t)(vt + t * (PC_TILE * PC_D * 2) + 256 * db)), p[t], acc[db]);
        }
        if (step + 1 < n_steps) convert(place == RING - 1 ? 0 : place + 1, (step + 1) & 1);
        // (what is asked for comes behind this step's products: the waves that have none are at it meanwhile)
        if (step + AHEAD < n_steps) request(before);
    }
    if (!real) return;
    const float l = sums[0];
    const int64_t at = ((int64_t)S.calls[call0 + call].part0 + split0 + rep) * W.n_q_heads + kh * g + n % g;
#pragma unroll
    for (int db = 0; db < 8; ++db) *reinterpret_cast<f32x4 *>(W.part_o + at * PC_D + 16 * db + 4 * a) = acc[db];
    if (a == 0) *reinterpret_cast<float2 *>(W.part_ml + at * 2) = make_float2(l == 0.f ? -INFINITY : m_ref, l);
}

template <int NW> __global__ __launch_bounds__(64 * NW, NW / 4) void pc_mx4_shared_decode_kernel(PcWin W, PcWinShared S)
{
    __shared__ SharedLds<NW> lds;
    if (listed((const int32_t *)S.bf16_only) == 0) shared_decode<NW, true>(W, S, lds);
    else shared_decode<NW, false>(W, S, lds);
}

void pc_launch_win_shared_decode_mx4(const PcWin &W, const PcWinShared &S, hipStream_t st)
{
    if (S.n_items <= 0) return;
    const unsigned grid = (unsigned)S.n_items * W.n_kv_heads;
    if (S.wide) pc_mx4_shared_decode_kernel<16><<<grid, 1024, 0, st>>>(W, S);
    else pc_mx4_shared_decode_kernel<8><<<grid, 512, 0, st>>>(W, S);
}
