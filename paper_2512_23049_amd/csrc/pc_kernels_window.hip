// Attention with a sliding window and sinks, bf16 caches (gfx950): prefill and decode; the rotations and the merge of splits
// that the fp32 kernels share.  What is visible, and how the host states it: pc_window.h.
//
// The problem is the transposed one of the other bf16 kernels: S^T = K . Q^T, O^T = V^T . P^T, keys as stored (turned to
// base + in-message index), queries turned by q_pos - (start - base) for each run whose rotation differs from the one before.
#include "pc_window.h"
#include "pc_mfma_common.h"

#include <type_traits>

#define TILE_BYTES 8192
#define LAZY_LOG2 64.0f
#define MFMA32(a, b, c) __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0)
#define MFMA16(a, b, c) __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0)

namespace {

__device__ __forceinline__ float ex2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ int imax3(int a, int b, int c) { return max(max(a, b), c); }
__device__ __forceinline__ float other_half(float x) { return __shfl_xor(x, 32); }
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
template <int N> __device__ __forceinline__ void wait_vm() { __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | ((N >> 4) << 14)); }
__device__ __forceinline__ void ring_barrier() { asm volatile("s_barrier" ::: "memory"); }
// One 16-byte per lane direct load: lane l's bytes land at lds_wave_base + 16 l; completion is awaited with wait_vm.
__device__ __forceinline__ void dma16(const void *gbase_uniform, unsigned lane_off, unsigned lds_wave_base)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                 ::"s"(lds_wave_base), "v"(lane_off), "s"(gbase_uniform) : "memory", "m0");
}
// a wave's own LDS accesses happen in the order they are issued: the compiler is to keep it
__device__ __forceinline__ void in_order() { asm volatile("" ::: "memory"); }
__device__ __forceinline__ bool finite16(uint32_t bits) { return (bits & 0x7F80u) != 0x7F80u; }
// zeros in the place of what is not finite
__device__ __forceinline__ bf16x8 finite_or_zero(bf16x8 x)
{
    uint4 u = __builtin_bit_cast(uint4, x);
    uint32_t *w = reinterpret_cast<uint32_t *>(&u);
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = (finite16(w[j]) ? w[j] & 0xFFFFu : 0u) | (finite16(w[j] >> 16) ? w[j] & 0xFFFF0000u : 0u);
    return __builtin_bit_cast(bf16x8, u);
}
// PC_WIN_ODD_* for what is not finite, else zeros
__device__ __forceinline__ bf16x8 odd_code(bf16x8 x)
{
    auto code = [](uint32_t b) { return finite16(b) ? 0u : (b & 0x7Fu) ? 0x4780u : (b & 0x8000u) ? 0x4380u : 0x3F80u; };
    uint4 u = __builtin_bit_cast(uint4, x);
    uint32_t *w = reinterpret_cast<uint32_t *>(&u);
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = code(w[j] & 0xFFFFu) | (code(w[j] >> 16) << 16);
    return __builtin_bit_cast(bf16x8, u);
}
__device__ __forceinline__ const __attribute__((address_space(4))) char *arguments()
{
    return (const __attribute__((address_space(4))) char *)__builtin_amdgcn_kernarg_segment_ptr();
}

}  // namespace

// ------------------------------------------------------------------------------------------------------------- turns
// A call's lists to the workspace, and the rotations (in 64 bits, rounded once) of its rows and of its runs.  Lists are read where the
// host put them (arguments, or pinned memory): 160 KB of them take 6.5 us, 8192 rows' rotations 10.5, a short call's 3.6.
__device__ __forceinline__ void win_turns(const char *from, const PcWinTurns &T)
{
    const int half = T.D / 2;
    const int64_t n_copy = from != T.ws ? T.n16 : 0, n_q = (int64_t)T.n_rows * half, n_all = n_copy + n_q + (int64_t)T.n_rot * half;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n_all; i += (int64_t)gridDim.x * 256) {
        if (i < n_copy) {
            reinterpret_cast<uint4 *>(T.ws)[i] = reinterpret_cast<const uint4 *>(from)[i];
        } else if (i < n_copy + n_q) {
            const int64_t R = (i - n_copy) / half;
            const int f = (int)((i - n_copy) % half);
            const float2 cs = rope_turn(reinterpret_cast<const int32_t *>(from + T.off_q_pos)[R], T.inv_freq[f]);
            if (T.rot_q) T.rot_q[R * half + f] = cs;
            if (T.rot_lanes) T.rot_lanes[win_rot_at(R, f)] = pack_f16(cs.x, cs.y);
        } else {
            const int64_t k = (i - n_copy - n_q) / half;
            const int f = (int)((i - n_copy - n_q) % half);
            const float2 cs = rope_angle((double)reinterpret_cast<const int64_t *>(from + T.off_rot)[k] * T.inv_freq[f]);
            T.rot_run[k * half + f] = make_float2(cs.x * T.run_scale, cs.y * T.run_scale);
        }
    }
}

__global__ __launch_bounds__(256) void pc_win_turns_kernel(PcWinTurns T) { win_turns((const char *)T.from, T); }
__global__ __launch_bounds__(256) void pc_win_turns_arg_kernel(PcArgBlob, PcWinTurns T) { win_turns((const char *)arguments(), T); }       // (the blob comes first)

void pc_launch_win_turns(const PcWinTurns &T, const PcArgBlob *blob, hipStream_t st)
{
    const int64_t n = T.n16 + ((int64_t)T.n_rows + T.n_rot) * (T.D / 2);
    const unsigned grid = (unsigned)std::max<int64_t>(1, std::min<int64_t>((n + 255) / 256, 2048));
    if (blob) pc_win_turns_arg_kernel<<<grid, 256, 0, st>>>(*blob, T);
    else pc_win_turns_kernel<<<grid, 256, 0, st>>>(T);
}

// ----------------------------------------------------------------------------------------------------------- prefill
// A workgroup is 4 waves = 4 consecutive units (32 rows x head, heads of a KV head fastest) over the same run of tiles, two
// workgroups a compute unit (256 registers a wave, 64 KB of LDS): the two share no barrier, so one's matrix work runs beside
// the other's softmax, and one's start and end beside the other's walk; a window's walk is short.  K and V tiles come by
// direct loads into a ring of four, three tiles ahead.
//
// Softmax: base 2, the scale folded into the queries, a reference that starts at 0 and moves only when a score exceeds it by
// 2^LAZY_LOG2 or a row's first scores lie that far below it.  Its negative is what the scores' accumulators start from.
//
// Masks are bits, made only for tiles on an edge (a ragged end, the causal limit, the window's end).  What a row does not see
// may be anything there: its score is replaced, not added to, and where a value of such a tile is not finite (asked of the
// matrix unit: 0 x value) the product leaves those values out and the rows that see them get what they make of a sum (win_odd_sum).
//
// What bounds it.  Long walks: the matrix unit and the softmax beside it, with two workgroups of four waves to overlap: 8192 rows,
// 32 heads over 8, window 4096: 600 to 650 us, 0.9 PFLOP/s of visible work (16 matrix instructions, 102 vector and 50 scalar ones a
// tile and wave; the matrix unit is busy 0.7 of the time).  Short walks: starts and turns, whose loads nothing hides: 33 blocks of
// rows over 20 tiles of seven messages, 47 us: a workgroup's first tile 6 us after its start, a turn 3 us, a tile 1 us, its results 2.5 us.
// Tried and dropped, in this one loop with its edges and turns: the next tile's scores beside this one's exponentials (spills: 1171 us;
// pc_attend's packed walk holds both in 210 registers, in a loop of its own over tiles that are seen whole), a row's queries kept in
// registers from turn to turn (spills).
__global__ __launch_bounds__(256, 2) void pc_win_prefill_bf16_kernel(PcWin W)
{
    constexpr int RING = 4, AHEAD = 3;
    __shared__ __attribute__((aligned(1024))) unsigned char s_kv[RING][2 * TILE_BYTES];
    __shared__ __attribute__((aligned(16))) float2 s_rot[4][PC_D / 2];
    __shared__ int s_again;

    const int kh = blockIdx.x % W.n_kv_heads;          // consecutive workgroups (one per XCD) take different KV heads
    const PcWinItem item = W.items[blockIdx.x / W.n_kv_heads];
    const int g = W.n_q_heads / W.n_kv_heads;
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const int n = lane & 31, hh = lane >> 5;
    const int n_units = ((item.n_q + 31) >> 5) * g;
    const bool unit_ok = item.unit0 + wave < n_units;
    const int unit = unit_ok ? item.unit0 + wave : item.unit0;
    const int ub = unit / g, h = kh * g + (unit - ub * g);
    const int last_row = min(32 * ub + 31, item.n_q - 1), row = min(32 * ub + n, last_row);
    const bool row_ok = unit_ok && 32 * ub + n < item.n_q;
    const int64_t R = (int64_t)item.q_off + row;
    const int lim = item.lim0 + row, lim_first = item.lim0 + 32 * ub;       // (lim_first: uniform)
    int lo = 0, lo_max = 0;                              // the least position the row sees; the largest such of the wave's rows
    auto look_up_rows = [&]() __attribute__((always_inline)) {
        lo = win_low(W.q_pos[R], W.window);
        lo_max = lo;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) lo_max = max(lo_max, __shfl_xor(lo_max, o));
        lo_max = uniform(lo_max);
    };

    const unsigned char *kb = (const unsigned char *)W.k_store + (int64_t)kh * W.slots * (PC_D * 2);
    const unsigned char *vb = (const unsigned char *)W.v_store + (int64_t)kh * W.slots * (PC_D * 2);
    // chunk position p of a K tile holds chunk (p & 15) ^ (p >> 4 & 15) of row p >> 4
    const unsigned lds0 = (unsigned)(uintptr_t)&s_kv[0][0] + wave * 1024;
    const unsigned k_src = (threadIdx.x >> 4) * 256 + (((threadIdx.x & 15) ^ (threadIdx.x >> 4 & 15)) << 4), v_src = threadIdx.x * 16;
    auto request = [&](int slot0, int slot) __attribute__((always_inline)) {
        const int64_t at = (int64_t)slot0 * (PC_D * 2);
        const unsigned to = lds0 + slot * (2 * TILE_BYTES);
        dma16(kb + at, k_src, to);
        dma16(kb + at + 4096, k_src, to + 4096);         // (rows 16 up: the same chunk order)
        dma16(vb + at, v_src, to + TILE_BYTES);
        dma16(vb + at + 4096, v_src, to + TILE_BYTES + 4096);
    };

    bf16x8 qop[8];
    // (few: in the walk, what is read for all of it at once would not fit the registers)
    auto turn = [&](int rot, auto few) __attribute__((always_inline)) {
        const uint4 *rq = reinterpret_cast<const uint4 *>(W.rot_lanes) + (R >> 5) * 512 + hh * 32 + (R & 31);
        // (the run's rotation is the same for all rows: one load a lane, and broadcasts from shared memory)
        const float2 own = W.rot_run[(int64_t)rot * (PC_D / 2) + lane];
        asm volatile("" ::: "memory");
        s_rot[wave][lane] = own;
        asm volatile("" ::: "memory");                   // (a wave's own LDS accesses happen in order)
        const float4 *rr = reinterpret_cast<const float4 *>(&s_rot[wave][8 * hh]);
        // the lane's row, as it came (from the cache each time: 32 registers): dims 16 ks + 8 hh + 0..7, then 64 up
        const unsigned char *qp = (const unsigned char *)W.q + (R * W.n_q_heads + h) * (PC_D * 2) + 16 * hh;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            uint4 lq = ldg16(qp + 32 * ks), hq = ldg16(qp + 32 * ks + 128);
            if (!row_ok) lq = hq = make_uint4(0, 0, 0, 0);
            const uint32_t lw[4] = {lq.x, lq.y, lq.z, lq.w}, hw[4] = {hq.x, hq.y, hq.z, hq.w};
            const uint4 p0 = rq[ks * 128], p1 = rq[ks * 128 + 64];
            const uint32_t pw[8] = {p0.x, p0.y, p0.z, p0.w, p1.x, p1.y, p1.z, p1.w};
            uint32_t a[4], b[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float4 p = make_float4(f16_lo(pw[2 * j]), f16_hi(pw[2 * j]), f16_lo(pw[2 * j + 1]), f16_hi(pw[2 * j + 1]));
                const float4 r = rr[8 * ks + j];
                const float c0 = p.x * r.x + p.y * r.y, s0 = p.y * r.x - p.x * r.y, c1 = p.z * r.z + p.w * r.w, s1 = p.w * r.z - p.z * r.w;
                const float x0 = bf_lo(lw[j]), x1 = bf_hi(lw[j]), y0 = bf_lo(hw[j]), y1 = bf_hi(hw[j]);
                a[j] = pack_bf16(x0 * c0 - y0 * s0, x1 * c1 - y1 * s1);
                b[j] = pack_bf16(x0 * s0 + y0 * c0, x1 * s1 + y1 * c1);
            }
            qop[ks] = __builtin_bit_cast(bf16x8, make_uint4(a[0], a[1], a[2], a[3]));
            qop[ks + 4] = __builtin_bit_cast(bf16x8, make_uint4(b[0], b[1], b[2], b[3]));
            if (decltype(few)::value && (ks & 1)) __builtin_amdgcn_sched_barrier(0);
        }
    };

    // K row of the lane's MFMA row: permuted so that score registers 0..7 / 8..15 are keys 8 hh + 0..7 / 16 + 8 hh + 0..7
    const int krow = 16 * (n >> 4) + 8 * ((n >> 2) & 1) + 4 * ((n >> 3) & 1) + (n & 3);
    typedef const __attribute__((address_space(3))) bf16x8 *lds_frag;
    // fragment ks of a tile of keys at k_base ^ 32 ks
    unsigned k_base = (unsigned)(uintptr_t)&s_kv[0][krow * 256 + ((hh ^ (krow & 15)) << 4)];
    asm volatile("" : "+v"(k_base));
    unsigned v_rd = (unsigned)(uintptr_t)&s_kv[0][TILE_BYTES + (hh * PC_D + n) * 16];
    asm volatile("" : "+v"(v_rd));

    float m_ref = 0.f, l_run = 0.f;
    bool seen = false, all_seen = false, shifted = false;          // the row has met a key; every row of the wave has; some row's reference has moved
    f32x16 acc[4];
    const f32x16 zeros = (f32x16){0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int db = 0; db < 4; ++db) acc[db] = zeros;

    auto fi = [](float x) { return __float_as_int(x); };
    auto largest = [&](const f32x16 &s) __attribute__((always_inline)) {        // (on the bit patterns: right wherever some score is positive)
        int m = imax3(fi(s[0]), fi(s[1]), fi(s[2]));
#pragma unroll
        for (int r = 3; r < 15; r += 2) m = imax3(m, fi(s[r]), fi(s[r + 1]));
        return max(m, fi(s[15]));
    };
    // the reference moves, if a row's scores ask for it; s: scores less the reference
    auto rebase = [&](f32x16 &s) __attribute__((always_inline)) {
        float mx = s[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[r]);
        mx = fmaxf(mx, other_half(mx));
        const bool now = mx > -INFINITY, need = mx > LAZY_LOG2 || (!seen && now && mx < -LAZY_LOG2);
        seen |= now;
        all_seen = __builtin_amdgcn_ballot_w64(seen) == ~0ull;
        if (__builtin_amdgcn_ballot_w64(need) != 0) {
            const float shift = need ? mx : 0.f, alpha = ex2(-fmaxf(shift, 0.f));       // (down: nothing has been added yet)
            l_run *= alpha;
#pragma unroll
            for (int db = 0; db < 4; ++db) acc[db] *= alpha;
            m_ref += shift;
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] -= shift;
            shifted = __builtin_amdgcn_ballot_w64(m_ref != 0.f) != 0;
        }
    };
    auto less_reference = [&](f32x16 &s) __attribute__((always_inline)) {
        if (__builtin_expect(shifted, 0)) {
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] -= m_ref;
        }
    };
    const int T = item.n_tiles;
    bool met_odd = false;                                // a value that is not finite, in a tile that some row does not see all of
    // The item's tiles.  ODD: with such values taken care of, as the first walk, which looks for them, does not: what that takes would
    // cost it its registers.
    auto walk_tiles = [&](auto odd_c) __attribute__((always_inline)) {
        constexpr bool ODD = decltype(odd_c)::value;
        // two walks over the same runs: of the tiles that are asked for, and of those that are worked on
        WinWalk ahead(W.runs + item.run0, item.skip, T), walk = ahead;
        int asked = 0;
        auto ask = [&](int slot) __attribute__((always_inline)) {
            if (asked >= T) return;
            request(ahead.a.x, slot);
            if (++asked < T) ahead.next();
        };
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) ask(i);
        int cur = walk.rot;
        turn(cur, std::false_type{});
        look_up_rows();                                  // (behind the first requests: its latency is not theirs)
        int t = 0;
#pragma unroll 1
        while (t < T) {
            // Four tiles of which every row sees everything, the ring's slots as constants: nothing is looked up, masked or turned.
            if (!ODD && (t & (RING - 1)) == 0 && walk.a.z >= RING * PC_TILE && walk.rot == cur && all_seen && !shifted &&
                (lo_max <= walk.a.y || walk.a.w >= RING * PC_TILE) && (!walk.self || lim_first - walk.a.y >= RING * PC_TILE - 1) &&
                T - asked >= RING && ahead.a.z > (RING - 1) * PC_TILE) {
                const int slot0 = ahead.a.x;
#pragma unroll
                for (int u = 0; u < RING; ++u) {
                    const int at = u * 2 * TILE_BYTES;
                    wait_vm<4 * (AHEAD - 1)>();
                    ring_barrier();
                    request(slot0 + PC_TILE * u, (u + AHEAD) & (RING - 1));
                    f32x16 s = zeros;
#pragma unroll
                    for (int ks = 0; ks < 8; ++ks) s = MFMA32(*(lds_frag)((k_base ^ (ks << 5)) + at), qop[ks], s);
                    bf16x8 fr[8];
#pragma unroll
                    for (int f = 0; f < 8; ++f) fr[f] = *(lds_frag)(v_rd + at + ((f >> 2) * 2 * PC_D + 32 * (f & 3)) * 16);
                    less_reference(s);
                    if (__builtin_expect(__builtin_amdgcn_ballot_w64(largest(s) > fi(LAZY_LOG2)) != 0, 0)) rebase(s);
                    uint32_t pk[8];
                    float ps = 0.f;
#pragma unroll
                    for (int r = 0; r < 8; ++r) {
                        const float a = ex2(s[2 * r]), b = ex2(s[2 * r + 1]);
                        ps += a;
                        ps += b;
                        pk[r] = pack_bf16(a, b);
                    }
                    l_run += ps;
                    const bf16x8 p[2] = {__builtin_bit_cast(bf16x8, make_uint4(pk[0], pk[1], pk[2], pk[3])), __builtin_bit_cast(bf16x8, make_uint4(pk[4], pk[5], pk[6], pk[7]))};
#pragma unroll
                    for (int f = 0; f < 8; ++f) acc[f & 3] = MFMA32(fr[f], p[f >> 2], acc[f & 3]);
                }
                asked += RING;
                ahead.pass(RING - 1);
                if (asked < T) ahead.next();
                t += RING;
                walk.pass(RING - 1);
                if (t < T) walk.next();
                continue;
            }
            const int u = t & (RING - 1);
            const unsigned at = u * (2 * TILE_BYTES);
            if (t + AHEAD <= T) wait_vm<4 * (AHEAD - 1)>();        // this wave's share of tile t has landed
            else wait_vm<0>();
            ring_barrier();                              // ... every wave's has, and tile t - 1 is no longer read
            const WinTile e = walk.tile();
            if (__builtin_expect(e.rot != cur, 0)) { cur = e.rot; turn(cur, std::true_type{}); }
            ask((u + AHEAD) & (RING - 1));
            f32x16 s = zeros;
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) s = MFMA32(*(lds_frag)((k_base ^ (ks << 5)) + at), qop[ks], s);
            less_reference(s);
            const bool edge = e.valid < PC_TILE || (e.self && lim_first - e.pos0 < PC_TILE - 1) || (lo_max > e.pos0 && e.sink < PC_TILE);
            uint32_t sees = ~0u;
            bool none = false;
            if (__builtin_expect(edge, 0)) {
                sees = win_sees(e.pos0, e.valid, e.sink, e.self != 0, lo, lim);
                none = __builtin_amdgcn_ballot_w64(sees != 0) == 0;
                const int mine = (int)(sees >> (8 * hh));
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = (mine >> (16 * (r >> 3) + (r & 7))) & 1 ? s[r] : -INFINITY;
            }
            if (!none) {
                if (__builtin_expect(!all_seen || __builtin_amdgcn_ballot_w64(largest(s) > fi(LAZY_LOG2)) != 0, 0)) rebase(s);
                uint32_t pk[8];
                float ps = 0.f;
#pragma unroll
                for (int r = 0; r < 8; ++r) {
                    const float a = ex2(s[2 * r]), b = ex2(s[2 * r + 1]);
                    ps += a;
                    ps += b;
                    pk[r] = pack_bf16(a, b);
                }
                const bf16x8 p[2] = {__builtin_bit_cast(bf16x8, make_uint4(pk[0], pk[1], pk[2], pk[3])), __builtin_bit_cast(bf16x8, make_uint4(pk[4], pk[5], pk[6], pk[7]))};
                bf16x8 fr[8];
#pragma unroll
                for (int f = 0; f < 8; ++f) fr[f] = *(lds_frag)(v_rd + at + ((f >> 2) * 2 * PC_D + 32 * (f & 3)) * 16);
                if (__builtin_expect(edge, 0)) {
                    // (a row of few keys: the sum of the probabilities as the products take them, so that their rounding cancels)
                    ps = 0.f;
#pragma unroll
                    for (int r = 0; r < 8; ++r) ps += bf_lo(pk[r]) + bf_hi(pk[r]);
                    f32x16 z = zeros;                    // 0 x value
                    const bf16x8 zero = __builtin_bit_cast(bf16x8, make_uint4(0, 0, 0, 0));
#pragma unroll
                    for (int f = 0; f < 8; ++f) z = MFMA32(fr[f], zero, z);
                    float odd = 0.f;
#pragma unroll
                    for (int r = 0; r < 16; ++r) odd += z[r];
                    if (__builtin_expect(__builtin_amdgcn_ballot_w64(odd != 0.f) != 0, 0)) {
                        met_odd = true;
                        if constexpr (ODD) {
                            const int mine = (int)(sees >> (8 * hh));
                            bf16x8 one[2];               // the keys the row sees (0 x infinity is not a number: PC_WIN_ODD_NAN)
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
                                uint32_t w[4];
#pragma unroll
                                for (int j = 0; j < 4; ++j) {
                                    const uint32_t x = pk[4 * k + j];
                                    w[j] = ((mine >> (16 * k + 2 * j)) & 1 ? ((x & 0xFFFFu) ? 0x3F80u : 0x4780u) : 0u) |
                                           ((mine >> (16 * k + 2 * j + 1)) & 1 ? ((x >> 16) ? 0x3F800000u : 0x47800000u) : 0u);
                                }
                                one[k] = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
                            }
#pragma unroll
                            for (int db = 0; db < 4; ++db) {
                                z = MFMA32(odd_code(fr[db]), one[0], zeros);
                                z = MFMA32(odd_code(fr[db + 4]), one[1], z);
                                fr[db] = finite_or_zero(fr[db]);
                                fr[db + 4] = finite_or_zero(fr[db + 4]);
#pragma unroll
                                for (int r = 0; r < 16; ++r) acc[db][r] += win_odd_sum(z[r]);
                                __builtin_amdgcn_sched_barrier(0);          // (one after the other: registers)
                            }
                        }
                    }
                }
                l_run += ps;
#pragma unroll
                for (int f = 0; f < 8; ++f) acc[f & 3] = MFMA32(fr[f], p[f >> 2], acc[f & 3]);
            }
            ++t;
            if (t < T) walk.next();
        }
    };
    if (T > 0) {
        if (threadIdx.x == 0) s_again = 0;
        walk_tiles(std::false_type{});
        if (__builtin_expect(met_odd, 0)) s_again = 1;   // (behind at least one barrier of the walk)
        __syncthreads();
        if (__builtin_expect(uniform(s_again), 0)) {
            m_ref = l_run = 0.f;
            seen = all_seen = shifted = false;
#pragma unroll
            for (int db = 0; db < 4; ++db) acc[db] = zeros;
            walk_tiles(std::true_type{});
        }
    }
    ring_barrier();

    // results leave as whole cache lines, turned round in the wave's quarter of the ring: chunk c (16 bytes) of row r at c ^ (r & 15)
    const float l = l_run + other_half(l_run);
    unsigned char *stg = &s_kv[0][0] + wave * TILE_BYTES;
    const int r4 = lane >> 4, c = lane & 15;
    if (item.part < 0) {
        const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
        for (int db = 0; db < 4; ++db)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {
                uint2 w;
                w.x = pack_bf16(acc[db][4 * q4] * inv, acc[db][4 * q4 + 1] * inv);
                w.y = pack_bf16(acc[db][4 * q4 + 2] * inv, acc[db][4 * q4 + 3] * inv);
                *reinterpret_cast<uint2 *>(stg + n * 256 + (((4 * db + q4) ^ (n & 15)) << 4) + 8 * hh) = w;
            }
        in_order();
        unsigned char *dst = (unsigned char *)W.out + ((int64_t)item.q_off * W.n_q_heads + h) * (PC_D * 2) + 16 * c;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = 4 * i + r4, rw = 32 * ub + r;
            const uint4 v = *reinterpret_cast<const uint4 *>(stg + r * 256 + ((c ^ (r & 15)) << 4));
            if (unit_ok && rw < item.n_q) *reinterpret_cast<uint4 *>(dst + (int64_t)rw * W.n_q_heads * (PC_D * 2)) = v;
        }
        if (W.lse && row_ok && hh == 0) W.lse[R * W.n_q_heads + h] = l == 0.f ? -INFINITY : (m_ref + log2f(l)) * 0.6931471805599453f;
        return;
    }
    float *dst = W.part_o + ((int64_t)item.part * W.n_q_heads + h) * PC_D + 4 * c;
#pragma unroll
    for (int half = 0; half < 2; ++half) {               // half a row is 256 bytes
        in_order();
#pragma unroll
        for (int db = 0; db < 2; ++db)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {
                const f32x16 &a = acc[2 * half + db];
                *reinterpret_cast<float4 *>(stg + n * 256 + (((8 * db + 2 * q4 + hh) ^ (n & 15)) << 4)) = make_float4(a[4 * q4], a[4 * q4 + 1], a[4 * q4 + 2], a[4 * q4 + 3]);
            }
        in_order();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = 4 * i + r4, rw = 32 * ub + r;
            const float4 v = *reinterpret_cast<const float4 *>(stg + r * 256 + ((c ^ (r & 15)) << 4));
            if (unit_ok && rw < item.n_q) *reinterpret_cast<float4 *>(dst + (int64_t)rw * W.n_q_heads * PC_D + 64 * half) = v;
        }
    }
    if (row_ok && hh == 0) {
        float *ml = W.part_ml + (((int64_t)item.part + row) * W.n_q_heads + h) * 2;
        ml[0] = l == 0.f ? -INFINITY : m_ref;
        ml[1] = l;
    }
}

void pc_launch_win_prefill_bf16(const PcWin &W, int n_items, hipStream_t st)
{
    if (n_items > 0) pc_win_prefill_bf16_kernel<<<(unsigned)n_items * W.n_kv_heads, 256, 0, st>>>(W);
}

// ------------------------------------------------------------------------------------------------------------ decode
// One query row a call.  A workgroup is 4 waves over one item of one KV head, each with a contiguous share of its tiles;
// the g <= 16 heads of the KV head are the columns of 16x16x32 products.  Tiles come straight from memory into registers, two
// ahead: the kernel lives on bytes in flight.  A wave makes the rotations of its runs itself (a lane a frequency), so that a
// call needs no launch in front of this one but for lists too long for its arguments.  One row: what it sees of a tile is one
// word for the whole wave, and the values of keys it does not see are cleared.  Bound: memory (64 calls of 32 heads over 8, window
// 1024, 2048 shared tokens: 40 us for 210 MB); a few calls: latency (four
// of 17 tiles, 7.7 us, and 3.6 for the merge of their splits).
namespace {
struct WinDecTile {
    uint4 k[2][4];      // [16-key half][d step of 32]: key 8 (m >> 2) + 4 half + (m & 3) of lane m = lane & 15
    uint4 v[8];         // [16-d block]
    WinTile d;
};
__device__ __forceinline__ void win_dec_load(WinDecTile &T, const unsigned char *kb, const unsigned char *vb, int lane)
{
    const int m = lane & 15, a = lane >> 4;
    const unsigned char *kt = kb + (int64_t)T.d.slot0 * (PC_D * 2), *vt = vb + (int64_t)T.d.slot0 * (PC_D * 2);
#pragma unroll
    for (int tau = 0; tau < 2; ++tau) {
        const unsigned at = (unsigned)((8 * (m >> 2) + 4 * tau + (m & 3)) * (PC_D * 2) + 16 * a);
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) T.k[tau][ks] = ldg16(kt + at + 64 * ks);
    }
    const unsigned at = (unsigned)((a * PC_D + m) * 16);
#pragma unroll
    for (int db = 0; db < 8; ++db) T.v[db] = ldg16(vt + at + 256 * db);
}
}  // namespace

__device__ __forceinline__ void win_decode(const PcWin &W, const PcWinItem *items, const PcWinRun *runs, const int32_t *q_pos)
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
        const unsigned char *kb = (const unsigned char *)W.k_store + (int64_t)kh * W.slots * (PC_D * 2);
        const unsigned char *vb = (const unsigned char *)W.v_store + (int64_t)kh * W.slots * (PC_D * 2);
        WinWalk walk(runs + item.run0, skip, n_tiles);
        int asked = 0;
        auto fetch = [&](WinDecTile &T) __attribute__((always_inline)) {
            if (asked > 0 && asked < n_tiles) walk.next();
            ++asked;
            T.d = walk.tile();
            T.d.rot = (int)((walk.run - reinterpret_cast<uintptr_t>(runs)) / sizeof(PcWinRun));       // (the run)
            win_dec_load(T, kb, vb, lane);
        };
        // the column's head, as it came (from the cache each time: registers): dims 32 ks + 8 a + 0..7, then 64 up
        const unsigned char *qp = (const unsigned char *)W.q + ((int64_t)item.q_off * W.n_q_heads + kh * g + min(n, g - 1)) * (PC_D * 2) + 16 * a;
        const double freq = W.inv_freq[lane];
        WinDecTile A, B;
        fetch(A);
        if (n_tiles > 1) fetch(B);
        int cur = -1;
        int64_t cur_turn = 0;
        bf16x8 qop[4];
        auto compute = [&](WinDecTile &T) __attribute__((always_inline)) {
            if (T.d.rot != cur) {                        // another run: another rotation?
                const int64_t turn = pos - T.d.rot_pos;
                const bool fresh = cur < 0 || turn != cur_turn;
                cur = T.d.rot; cur_turn = turn;
                if (fresh) {
                    const float2 cs = rope_angle((double)turn * freq);
                    s_rot[wave][lane] = make_float2(cs.x * W.scale_log2, cs.y * W.scale_log2);
                    in_order();
#pragma unroll
                    for (int ks = 0; ks < 2; ++ks) {
                        uint4 lq = ldg16(qp + 64 * ks), hq = ldg16(qp + 64 * ks + 128);
                        if (n >= g) lq = hq = make_uint4(0, 0, 0, 0);
                        const uint32_t lw[4] = {lq.x, lq.y, lq.z, lq.w}, hw[4] = {hq.x, hq.y, hq.z, hq.w};
                        uint32_t x[4], y[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float4 r = *reinterpret_cast<const float4 *>(&s_rot[wave][32 * ks + 8 * a + 2 * j]);
                            const float x0 = bf_lo(lw[j]), x1 = bf_hi(lw[j]), y0 = bf_lo(hw[j]), y1 = bf_hi(hw[j]);
                            x[j] = pack_bf16(x0 * r.x - y0 * r.y, x1 * r.z - y1 * r.w);
                            y[j] = pack_bf16(x0 * r.y + y0 * r.x, x1 * r.w + y1 * r.z);
                        }
                        qop[ks] = __builtin_bit_cast(bf16x8, make_uint4(x[0], x[1], x[2], x[3]));
                        qop[ks + 2] = __builtin_bit_cast(bf16x8, make_uint4(y[0], y[1], y[2], y[3]));
                    }
                    in_order();
                }
            }
            f32x4 s[2];
#pragma unroll
            for (int tau = 0; tau < 2; ++tau) {
                s[tau] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int ks = 0; ks < 4; ++ks) s[tau] = MFMA16(__builtin_bit_cast(bf16x8, T.k[tau][ks]), qop[ks], s[tau]);
            }
            float sc[8];                                 // keys 8 a + 0..7 of column n
#pragma unroll
            for (int j = 0; j < 8; ++j) sc[j] = s[j >> 2][j & 3];
            const uint32_t sees = win_sees(T.d.pos0, T.d.valid, T.d.sink, false, lo, 0);        // (the only row sees all of the new message)
            if (sees != ~0u) {                           // (uniform)
                const uint32_t mine = sees >> (8 * a);
                uint32_t keep[4];
#pragma unroll
                for (int j = 0; j < 8; ++j) sc[j] = (mine >> j) & 1 ? sc[j] : -INFINITY;
#pragma unroll
                for (int j = 0; j < 4; ++j) keep[j] = ((mine >> (2 * j)) & 1 ? 0xFFFFu : 0u) | ((mine >> (2 * j + 1)) & 1 ? 0xFFFF0000u : 0u);
#pragma unroll
                for (int db = 0; db < 8; ++db) { T.v[db].x &= keep[0]; T.v[db].y &= keep[1]; T.v[db].z &= keep[2]; T.v[db].w &= keep[3]; }
            }
            float mx = fmaxf(fmaxf(fmaxf(sc[0], sc[1]), fmaxf(sc[2], sc[3])), fmaxf(fmaxf(sc[4], sc[5]), fmaxf(sc[6], sc[7])));
            mx = fmaxf(mx, __shfl_xor(mx, 16));
            mx = fmaxf(mx, other_half(mx));
            const float m_new = fmaxf(m_run, mx), m_safe = m_new == -INFINITY ? 0.f : m_new, alpha = ex2(m_run - m_safe);
            uint32_t pk[4];
            float ps = 0.f;                              // (of the probabilities as the products take them: their rounding cancels)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                pk[j] = pack_bf16(ex2(sc[2 * j] - m_safe), ex2(sc[2 * j + 1] - m_safe));
                ps += bf_lo(pk[j]) + bf_hi(pk[j]);
            }
            l_run = l_run * alpha + ps;
            m_run = m_new;
            if (__builtin_amdgcn_ballot_w64(alpha != 1.f) != 0) {           // rare once the running maxima have settled
#pragma unroll
                for (int db = 0; db < 8; ++db) acc[db] *= alpha;
            }
            const bf16x8 p = __builtin_bit_cast(bf16x8, make_uint4(pk[0], pk[1], pk[2], pk[3]));
#pragma unroll
            for (int db = 0; db < 8; ++db) acc[db] = MFMA16(__builtin_bit_cast(bf16x8, T.v[db]), p, acc[db]);
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
    l_run += other_half(l_run);
    if (a == 0) { s_m[wave][n] = m_run; s_l[wave][n] = l_run; }
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

__global__ __launch_bounds__(256, 2) void pc_win_decode_bf16_kernel(PcWin W) { win_decode(W, W.items, W.runs, W.q_pos); }
__global__ __launch_bounds__(256, 2) void pc_win_decode_bf16_arg_kernel(PcArgBlob, PcWinDecode O, PcWin W)
{
    const char *lists = (const char *)arguments();       // (the blob comes first)
    if (blockIdx.x == 0 && (int)threadIdx.x < O.n16) reinterpret_cast<uint4 *>(O.ws)[threadIdx.x] = reinterpret_cast<const uint4 *>(lists)[threadIdx.x];
    win_decode(W, reinterpret_cast<const PcWinItem *>(lists + O.off_items), reinterpret_cast<const PcWinRun *>(lists + O.off_runs),
               reinterpret_cast<const int32_t *>(lists + O.off_q_pos));
}

void pc_launch_win_decode_bf16(const PcWin &W, int n_items, const PcArgBlob *blob, const PcWinDecode &O, hipStream_t st)
{
    if (n_items <= 0) return;
    const unsigned grid = (unsigned)n_items * W.n_kv_heads;
    if (blob) pc_win_decode_bf16_arg_kernel<<<grid, 256, 0, st>>>(*blob, O, W);
    else pc_win_decode_bf16_kernel<<<grid, 256, 0, st>>>(W);
}

// ------------------------------------------------------------------------------------------------------------- merge
// The splits of a row, in their order: out = sum o_s 2^(m_s - m) / sum l_s 2^(m_s - m).  Four dims a thread.  Bound: memory (940 rows of
// 32 heads in two or three splits, 39 MB: 13 us); a few rows: two round trips, 3.6 us.
template <int D, bool BF16>
__global__ __launch_bounds__(256) void pc_win_merge_kernel(const PcMergeRow *__restrict__ rows, int64_t n, PcWin W)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    const int dim = 4 * (int)(i % (D / 4));
    const int64_t pair = i / (D / 4);
    const int h = (int)(pair % W.n_q_heads);
    const PcMergeRow mr = rows[pair / W.n_q_heads];
    float m = -INFINITY, l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s0 = 0; s0 < mr.n_splits; s0 += 8) {        // (eight at a time: the loads' latency is what this costs)
        float2 ml[8];
        float4 x[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            ml[u] = make_float2(-INFINITY, 0.f);
            x[u] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (s0 + u < mr.n_splits) {
                const int64_t at = ((int64_t)mr.part_row0 + (int64_t)(s0 + u) * mr.n_q) * W.n_q_heads + h;
                ml[u] = *reinterpret_cast<const float2 *>(W.part_ml + at * 2);
                x[u] = *reinterpret_cast<const float4 *>(W.part_o + at * D + dim);
            }
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            if (ml[u].y == 0.f) continue;                // saw nothing
            const float m_new = fmaxf(m, ml[u].x), keep = l == 0.f ? 0.f : ex2(m - m_new), f = ex2(ml[u].x - m_new);
            o.x = o.x * keep + x[u].x * f; o.y = o.y * keep + x[u].y * f; o.z = o.z * keep + x[u].z * f; o.w = o.w * keep + x[u].w * f;
            l = l * keep + ml[u].y * f;
            m = m_new;
        }
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int64_t at = ((int64_t)mr.row * W.n_q_heads + h) * D + dim;
    if constexpr (BF16) *reinterpret_cast<uint2 *>((uint16_t *)W.out + at) = make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
    else *reinterpret_cast<float4 *>((float *)W.out + at) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
    if (W.lse && dim == 0) W.lse[(int64_t)mr.row * W.n_q_heads + h] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
}

void pc_launch_win_merge(const PcWin &W, const PcMergeRow *rows, int n_rows, int dtype, int D, hipStream_t st)
{
    if (n_rows <= 0) return;
    const int64_t n = (int64_t)n_rows * W.n_q_heads * (D / 4);
    const unsigned grid = (unsigned)((n + 255) / 256);
    if (dtype == 1) pc_win_merge_kernel<128, true><<<grid, 256, 0, st>>>(rows, n, W);
    else if (D == 64) pc_win_merge_kernel<64, false><<<grid, 256, 0, st>>>(rows, n, W);
    else pc_win_merge_kernel<128, false><<<grid, 256, 0, st>>>(rows, n, W);
}
