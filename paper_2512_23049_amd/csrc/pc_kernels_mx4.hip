// Attention over a PC_MX4 cache: single tokens, and rows of prompts (gfx950).  What a row sees, and how
// the host states it: pc_window.h; how the cache holds keys and values: pc_mx4.h.
#include "pc_window.h"
#include "pc_mx4_products.h"

#include <algorithm>
#include <type_traits>

namespace {

__device__ __forceinline__ const __attribute__((address_space(4))) char *arguments()
{
    return (const __attribute__((address_space(4))) char *)__builtin_amdgcn_kernarg_segment_ptr();
}
typedef const __attribute__((address_space(3))) win_i32x4 *lds16;
typedef const __attribute__((address_space(3))) uint32_t *lds4;
template <int N> __device__ __forceinline__ void wait_vm() { __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | ((N >> 4) << 14)); }

}  // namespace

#define DEC_WAVES 8
// One query row a call.  A workgroup is 8 waves over one item of one KV head, each with a contiguous share of its tiles; the g <= 16
// heads of the KV head are the columns of the products.
//   scores   codes of keys as they are stored, by the turned query as the sum of two e4m3 numbers under one power of two for the row:
//            v_mfma_scale 16x16x128, a key's blocks and exponents where the instruction wants them, nothing is unpacked;
//   values   eight slots of a dimension are a word: four conversions make the operand, in units of the slots' powers.  The powers ride
//            on the probabilities, by block of 32 dimensions: probabilities are held 2^60 times as large, and a saturating
//            subtraction from their exponents takes the powers (-60 to 60) off again.
// Tiles come by direct loads, two places a wave of its own: no registers wait for them (two tiles in registers left room for two waves a
// SIMD: 66 us where this took 50), and no wave for another.  Bound: memory, 4352 bytes a tile and KV head, where there are many (64
// calls of 150 tiles, 32 heads over 8: 334 MB call by call, of which 119 are distinct, in 45 us: 7.4 TB/s out of the caches, and the vector unit half of the time; with a maximum across lanes a
// tile it was 51); latency where
// there are few (4 calls, window 512: 9 us, of which a launch of nothing takes 3).
__device__ __forceinline__ void mx4_decode(const PcWin &W, const PcWinItem *items, const PcWinRun *runs, const int32_t *q_pos)
{
    // of a tile: codes of keys and of values, exponents of keys and of values (256 bytes each: a direct load's lanes)
    constexpr int VALUES = PC_MX4_CODES, K_EXPS = 2 * PC_MX4_CODES, V_EXPS = K_EXPS + 256, TILE = V_EXPS + 256, LOADS = 6;
    constexpr int RING = 2 * TILE, COLUMN = PC_D + 4;
    static_assert(16 * COLUMN * 4 <= RING, "a wave's results take the place of its tiles");
    __shared__ __attribute__((aligned(1024))) unsigned char s_ring[DEC_WAVES][RING];
    __shared__ float s_m[DEC_WAVES][16], s_l[DEC_WAVES][16];
    __shared__ __attribute__((aligned(16))) float2 s_rot[DEC_WAVES][PC_D / 2];

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
    const int share = item.n_tiles / DEC_WAVES, more = item.n_tiles % DEC_WAVES;
    const int n_tiles = share + (wave < more), skip = item.skip + wave * share + min(wave, more);
    const unsigned ring = (unsigned)uniform((int)(unsigned)(uintptr_t)&s_ring[wave][0]);

    // Probabilities are 2^60 times 2^(score - m_ref); the reference moves where one would be above 2^16 of that (a column's first always does): the lanes
    // of a column need not agree on a maximum tile by tile.
    constexpr float LAZY_LOG2 = 16.f;
    float m_ref = -INFINITY, l_run = 0.f;
    f32x4 acc[8];
#pragma unroll
    for (int db = 0; db < 8; ++db) acc[db] = (f32x4){0.f, 0.f, 0.f, 0.f};
    if (n_tiles > 0) {
        const unsigned char *kb = (const unsigned char *)W.k_store + (int64_t)kh * (W.slots / PC_TILE) * PC_MX4_TILE;
        const unsigned char *vb = (const unsigned char *)W.v_store + (int64_t)kh * (W.slots / PC_TILE) * PC_MX4_TILE;
        // position p of the keys' codes holds block (p & 3) ^ (key >> 3) of key p >> 2; of the values' half (p & 1) ^ (m >> 3) of m = p / 2 % 16:
        // what the lanes of a fragment read at once hits different banks (the second 64 positions: 16 keys, and two groups of slots, on)
        const unsigned k_src = (unsigned)((lane >> 2) * 64 + (((lane & 3) ^ (lane >> 5)) << 4)), v_src = (unsigned)((lane >> 1) * 32 + (((lane & 1) ^ (lane >> 4 & 1)) << 4));
        const unsigned e_src = (unsigned)(PC_MX4_CODES + (lane & 31) * 4);
        auto request = [&](int slot0, int place) __attribute__((always_inline)) {
            const unsigned char *kt = kb + (int64_t)(slot0 / PC_TILE) * PC_MX4_TILE, *vt = vb + (int64_t)(slot0 / PC_TILE) * PC_MX4_TILE;
            const unsigned to = ring + place * TILE;
            mx4_dma16(kt, k_src, to);
            mx4_dma16(kt, (k_src ^ 32) + 1024, to + 1024);
            mx4_dma4(kt, e_src, to + K_EXPS);
            mx4_dma16(vt, v_src, to + VALUES);
            mx4_dma16(vt + 1024, v_src, to + VALUES + 1024);
            mx4_dma4(vt, e_src, to + V_EXPS);
        };
        // the column's head, as it came (from the cache each time: registers): dims 16 a + 0..15, then 64 up
        const unsigned char *qp = (const unsigned char *)W.q + ((int64_t)item.q_off * W.n_q_heads + kh * g + min(n, g - 1)) * (PC_D * 2) + 32 * a;
        const double freq = W.inv_freq[lane];
        uint4 raw[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) raw[i] = ldg16(qp + 128 * (i >> 1) + 16 * (i & 1));
        // two walks over the same runs: of the tiles that are asked for, and of those that are worked on
        WinWalk ahead(runs + item.run0, skip, n_tiles), walk = ahead;
        request(ahead.a.x, 0);
        if (n_tiles > 1) {
            ahead.next();
            request(ahead.a.x, 1);
        }
        // the row's unit, the same for every turn; a query that holds what is no number is all NaN
        bool fine = true;
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) top = mx4_top(top, w[j], fine);
        }
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        fine &= __shfl_xor((int)fine, 16) != 0;
        fine &= __shfl_xor((int)fine, 32) != 0;
        const float unit = mx4_unit(top * W.scale_log2);
        const int e_hi = (int)(__float_as_uint(unit) >> 23), e_lo = e_hi - 4;
#pragma unroll
        for (int i = 0; i < 4; ++i) {                    // (columns behind the last head are zeros)
            raw[i].x = n >= g ? 0u : fine ? raw[i].x : 0x7FC07FC0u; raw[i].y = n >= g ? 0u : fine ? raw[i].y : 0x7FC07FC0u;
            raw[i].z = n >= g ? 0u : fine ? raw[i].z : 0x7FC07FC0u; raw[i].w = n >= g ? 0u : fine ? raw[i].w : 0x7FC07FC0u;
        }
        const int key = 8 * (n >> 2) + (n & 3);
        const unsigned k_rd = ring + (unsigned)(key * 64 + ((a ^ (key >> 3)) << 4)), ke_rd = ring + K_EXPS + key * 4;
        const unsigned v_rd = ring + VALUES + (unsigned)(a * 512 + n * 32 + ((n >> 3) << 4)), ve_rd = ring + V_EXPS + a * 32;
        bool turned = false;
        int64_t cur_turn = 0;
        mx4_i32x8 q_hi, q_lo;
#pragma unroll 1
        for (int t = 0; t < n_tiles; ++t) {
            const WinTile e = walk.tile();
            const int64_t turn = pos - e.rot_pos;
            if (!turned || turn != cur_turn) {           // another run: another rotation?
                turned = true; cur_turn = turn;
                const float2 cs = mx4_rotation((double)turn * freq);
                in_order();
                s_rot[wave][lane] = make_float2(cs.x * W.scale_log2, cs.y * W.scale_log2);
                in_order();
#pragma unroll
                for (int i = 0; i < 4; ++i)              // (its 32 numbers, taken apart once and kept, would not fit the registers)
                    asm volatile("" : "+v"(raw[i].x), "+v"(raw[i].y), "+v"(raw[i].z), "+v"(raw[i].w));
#pragma unroll
                for (int s = 0; s < 4; ++s) {            // dims 16 a + 4 s, and 64 up
                    const uint4 lq = raw[s >> 1], hq = raw[2 + (s >> 1)];
                    const uint32_t lw[2] = {s & 1 ? lq.z : lq.x, s & 1 ? lq.w : lq.y}, hw[2] = {s & 1 ? hq.z : hq.x, s & 1 ? hq.w : hq.y};
                    const float4 *r = reinterpret_cast<const float4 *>(&s_rot[wave][16 * a + 4 * s]);
                    const float4 r0 = r[0], r1 = r[1];
                    const float x0 = bf_lo(lw[0]), x1 = bf_hi(lw[0]), x2 = bf_lo(lw[1]), x3 = bf_hi(lw[1]);
                    const float y0 = bf_lo(hw[0]), y1 = bf_hi(hw[0]), y2 = bf_lo(hw[1]), y3 = bf_hi(hw[1]);
                    const float u[4] = {x0 * r0.x - y0 * r0.y, x1 * r0.z - y1 * r0.w, x2 * r1.x - y2 * r1.y, x3 * r1.z - y3 * r1.w};
                    const float v[4] = {x0 * r0.y + y0 * r0.x, x1 * r0.w + y1 * r0.z, x2 * r1.y + y2 * r1.x, x3 * r1.w + y3 * r1.z};
                    int hi, rest;
                    mx4_pieces(u, unit, hi, rest);
                    q_hi[s] = hi; q_lo[s] = rest;
                    mx4_pieces(v, unit, hi, rest);
                    q_hi[4 + s] = hi; q_lo[4 + s] = rest;
                }
                in_order();
            }
            if (t + 1 < n_tiles) wait_vm<LOADS>();       // this tile has landed
            else wait_vm<0>();
            in_order();
            const unsigned at = (t & 1) * TILE;
            f32x4 s[2];
            const float ref = m_ref == -INFINITY ? 0.f : m_ref, start = PC_MX4_E_MAX - ref;
#pragma unroll
            for (int tau = 0; tau < 2; ++tau) {
                const uint4 codes = __builtin_bit_cast(uint4, *(lds16)(uintptr_t)(k_rd + at + tau * 256));
                const int ek = (int)(*(lds4)(uintptr_t)(ke_rd + at + tau * 16) >> (8 * a));
                s[tau] = mx4_scores16(codes, ek, q_lo, e_lo, (f32x4){start, start, start, start});
                s[tau] = mx4_scores16(codes, ek, q_hi, e_hi, s[tau]);
            }
            uint32_t vw[8], ew[8];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const win_i32x4 w = *(lds16)(uintptr_t)((v_rd ^ (half << 4)) + at), x = *(lds16)(uintptr_t)(ve_rd + at + half * 16);
                vw[4 * half] = (uint32_t)w.x; vw[4 * half + 1] = (uint32_t)w.y; vw[4 * half + 2] = (uint32_t)w.z; vw[4 * half + 3] = (uint32_t)w.w;
                ew[4 * half] = (uint32_t)x.x; ew[4 * half + 1] = (uint32_t)x.y; ew[4 * half + 2] = (uint32_t)x.z; ew[4 * half + 3] = (uint32_t)x.w;
            }
            float sc[8];                                 // keys 8 a + 0..7 of column n, less the reference, and 60
#pragma unroll
            for (int j = 0; j < 8; ++j) sc[j] = s[j >> 2][j & 3];
            const uint32_t sees = win_sees(e.pos0, e.valid, e.sink, false, lo, 0);        // (the only row sees all of the new message)
            if (sees != ~0u) {                           // (uniform; values need no mask: codes are finite)
                const uint32_t mine = sees >> (8 * a);
#pragma unroll
                for (int j = 0; j < 8; ++j) sc[j] = (mine >> j) & 1 ? sc[j] : -INFINITY;
            }
            // (on the bit patterns, which take no care of NaN: right wherever some score is above the reference)
            auto fi = [](float x) { return __float_as_int(x); };
            const int top = max(imax3(imax3(fi(sc[0]), fi(sc[1]), fi(sc[2])), fi(sc[3]), fi(sc[4])), imax3(fi(sc[5]), fi(sc[6]), fi(sc[7])));
            if (__builtin_expect(__builtin_amdgcn_ballot_w64(top > fi(PC_MX4_E_MAX + LAZY_LOG2) || m_ref == -INFINITY) != 0, 0)) {
                float mx = fmaxf(fmaxf(fmaxf(sc[0], sc[1]), fmaxf(sc[2], sc[3])), fmaxf(fmaxf(sc[4], sc[5]), fmaxf(sc[6], sc[7])));
                mx = fmaxf(mx, __shfl_xor(mx, 16));
                mx = fmaxf(mx, __shfl_xor(mx, 32)) - PC_MX4_E_MAX;
                const bool up = mx > (m_ref == -INFINITY ? -INFINITY : LAZY_LOG2);
                const float m_new = up ? ref + mx : m_ref, by = up ? m_new - ref : 0.f, f = !up ? 1.f : m_ref == -INFINITY ? 0.f : ex2(-by);
                m_ref = m_new;
                l_run *= f;
#pragma unroll
                for (int db = 0; db < 8; ++db) acc[db] *= f;
#pragma unroll
                for (int j = 0; j < 8; ++j) sc[j] -= by;
            }
            uint32_t pk[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {                // (summed as the products take them: their rounding cancels)
                pk[j] = pack_bf16(ex2(sc[2 * j]), ex2(sc[2 * j + 1]));
                l_run = mx4_sum<false>(pk[j], l_run);
            }
            // (the tile's last numbers are in registers: its place is free)
#pragma unroll
            for (int j = 0; j < 8; ++j) asm volatile("" : "+v"(vw[j]), "+v"(ew[j]));
            if (t + 2 < n_tiles) {
                ahead.next();
                request(ahead.a.x, t & 1);
            }
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const bf16x8 p = __builtin_bit_cast(bf16x8, make_uint4(mx4_lowered<0>(pk[0], ew[2 * b]), mx4_lowered<1>(pk[1], ew[2 * b]),
                                                                       mx4_lowered<0>(pk[2], ew[2 * b + 1]), mx4_lowered<1>(pk[3], ew[2 * b + 1])));
#pragma unroll
                for (int i = 0; i < 2; ++i) acc[2 * b + i] = MFMA16(mx4_of_codes(vw[2 * b + i]), p, acc[2 * b + i]);
            }
            if (t + 1 < n_tiles) walk.next();
        }
    }
    l_run += __shfl_xor(l_run, 16);
    l_run += __shfl_xor(l_run, 32);
    float (*s_acc)[COLUMN] = reinterpret_cast<float (*)[COLUMN]>(&s_ring[wave][0]);      // (no load of its own is on its way to it)
    if (a == 0) { s_m[wave][n] = m_ref; s_l[wave][n] = l_run * 0x1p-60f; }
#pragma unroll
    for (int db = 0; db < 8; ++db) *reinterpret_cast<f32x4 *>(&s_acc[n][16 * db + 4 * a]) = acc[db];
    __syncthreads();
    for (int idx = threadIdx.x; idx < g * (PC_D / 2); idx += 64 * DEC_WAVES) {
        const int col = idx / (PC_D / 2), dim = 2 * (idx % (PC_D / 2)), h = kh * g + col;
        float m = -INFINITY;
#pragma unroll
        for (int w = 0; w < DEC_WAVES; ++w) m = fmaxf(m, s_m[w][col]);
        float o0 = 0.f, o1 = 0.f, l = 0.f;
#pragma unroll
        for (int w = 0; w < DEC_WAVES; ++w) {
            // (a wave whose scores were not numbers has a sum that is none; one that saw nothing has a sum of 0)
            const float f = s_l[w][col] == 0.f ? 0.f : ex2(s_m[w][col] - (m == -INFINITY ? 0.f : m));
            const float2 x = *reinterpret_cast<const float2 *>(&s_ring[w][(col * COLUMN + dim) * 4]);
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

__global__ __launch_bounds__(64 * DEC_WAVES, 4) void pc_mx4_decode_kernel(PcWin W) { mx4_decode(W, W.items, W.runs, W.q_pos); }
__global__ __launch_bounds__(64 * DEC_WAVES, 4) void pc_mx4_decode_arg_kernel(PcArgBlob, PcWinDecode O, PcWin W)
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
    if (blob) pc_mx4_decode_arg_kernel<<<grid, 64 * DEC_WAVES, 0, st>>>(*blob, O, W);
    else pc_mx4_decode_kernel<<<grid, 64 * DEC_WAVES, 0, st>>>(W);
}

// ----------------------------------------------------------------------------------------------------------- prepare
// In front of the attention of rows: the call's lists to the workspace and the rotations of its runs (as win_turns), its queries turned
// by their positions and the unit that their 8-bit pieces are in, and the values of the tiles that rows see, as a bf16 cache has them, in fp16 or bf16 (what the
// codes stand for is exact there; 68 bytes read and 256 written for each, once, where every workgroup of rows would convert them again).
// Bound: latency (77 rows over 5 messages, 32 heads over 8: 5.6 us, with eight heads a block 8.3).
__device__ __forceinline__ void mx4_prepare(const char *from, const PcMx4Prepare &P)
{
    __shared__ __attribute__((aligned(16))) float2 s_rot[PC_D / 2][33];           // [frequency][row]
    if (P.mark && *P.mark != P.mark_value) return;       // (the walk in front of this one served every call)
    int block = blockIdx.x;
    if (block < P.list_blocks) {
        const int64_t n_copy = from != P.ws ? P.n16 : 0, n_all = n_copy + (int64_t)P.n_rot * (PC_D / 2);
        for (int64_t i = (int64_t)block * 256 + threadIdx.x; i < n_all; i += (int64_t)P.list_blocks * 256) {
            if (i < n_copy) { reinterpret_cast<uint4 *>(P.ws)[i] = reinterpret_cast<const uint4 *>(from)[i]; continue; }
            const int64_t k = (i - n_copy) / (PC_D / 2);
            const int f = (int)((i - n_copy) % (PC_D / 2));
            const float2 cs = mx4_rotation((double)reinterpret_cast<const int64_t *>(from + P.off_rot)[k] * P.inv_freq[f]);
            P.rot_run[k * PC_D + f] = (_Float16)cs.x;
            P.rot_run[k * PC_D + PC_D / 2 + f] = (_Float16)-cs.y;
        }
        return;
    }
    block -= P.list_blocks;
    if (block < P.query_blocks) {                        // 32 rows, a head a wave
        const int chunks = (P.n_q_heads + 3) / 4;
        const int64_t group = block / chunks, groups = ((int64_t)P.n_rows + 31) / 32;
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 31, hh = lane >> 5;
        const int64_t R = group * 32 + n, row = R < P.n_rows ? R : P.n_rows - 1;
        const int h = block % chunks * 4 + wave;
        uint4 raw[8];                                    // dims 16 hh, 32 + 16 hh, and 64 up, 16 each (on their way while the rotations are made)
        if (h < P.n_q_heads) {
            const unsigned char *qp = (const unsigned char *)P.q + (row * P.n_q_heads + h) * (PC_D * 2) + 32 * hh;
#pragma unroll
            for (int i = 0; i < 8; ++i) raw[i] = ldg16(qp + (i >> 1) * 64 + (i & 1) * 16);
        }
        {   // a frequency a lane, eight rows a wave
            const double freq = P.inv_freq[lane];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int64_t r = group * 32 + wave * 8 + i;
                if (r < P.n_rows) s_rot[lane][wave * 8 + i] = mx4_rotation((double)reinterpret_cast<const int32_t *>(from + P.off_q_pos)[r] * freq);
            }
        }
        __syncthreads();
        if (h < P.n_q_heads) {
            float top = 0.f;
            bool fine = true;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) top = mx4_top(top, w[j], fine);
            }
            top = fmaxf(top, __shfl_xor(top, 32));
            fine &= __shfl_xor((int)fine, 32) != 0;
            const float unit = mx4_unit(top * P.scale_log2), by = P.scale_log2 / unit;
            if (hh == 0) P.q_unit[(int64_t)h * groups * 32 + R] = unit;
#pragma unroll
            for (int s = 0; s < 8; ++s) {
                const uint4 lo = raw[(s >> 2) * 2 + (s >> 1 & 1)], hi = raw[4 + (s >> 2) * 2 + (s >> 1 & 1)];
                const uint32_t lw[2] = {s & 1 ? lo.z : lo.x, s & 1 ? lo.w : lo.y}, hw[2] = {s & 1 ? hi.z : hi.x, s & 1 ? hi.w : hi.y};
                float x[4], y[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 cs = s_rot[(s >> 2) * 32 + 16 * hh + 4 * (s & 3) + j][n];
                    const float a = j & 1 ? bf_hi(lw[j >> 1]) : bf_lo(lw[j >> 1]), b = j & 1 ? bf_hi(hw[j >> 1]) : bf_lo(hw[j >> 1]);
                    x[j] = fine ? (a * cs.x - b * cs.y) * by : __builtin_nanf("");
                    y[j] = fine ? (a * cs.y + b * cs.x) * by : __builtin_nanf("");
                }
                P.q_abs[mx4_query_at(groups, h, R, hh, s)] = make_uint2(mx4_pack<true>(x[0], x[1]), mx4_pack<true>(x[2], x[3]));
                P.q_abs[mx4_query_at(groups, h, R, hh, s + 8)] = make_uint2(mx4_pack<true>(y[0], y[1]), mx4_pack<true>(y[2], y[3]));
            }
        }
        return;
    }
    const bool half = *P.bf16_only == 0;
    for (int64_t at = block - P.query_blocks; at < (int64_t)P.n_tiles * P.n_kv_heads; at += gridDim.x - P.list_blocks - P.query_blocks) {
        const int kh = (int)(at / P.n_tiles), tile = (int)(at % P.n_tiles);
        const int slot0 = reinterpret_cast<const int32_t *>(from + P.off_tiles)[tile];
        const char *vt = (const char *)P.v_store + ((int64_t)kh * P.slots + slot0) / PC_TILE * PC_MX4_TILE;
        char *to = (char *)P.v_to + ((int64_t)kh * P.n_tiles + tile) * (PC_TILE * PC_D * 2);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int grp = (threadIdx.x >> 7) + 2 * i, d = threadIdx.x & 127;
            const uint32_t w = reinterpret_cast<const uint32_t *>(vt + grp * 512)[mx4_word(d)];
            const uint2 ex = *reinterpret_cast<const uint2 *>(vt + PC_MX4_CODES + grp * 32 + d / 32 * 8);
            uint4 x;
            auto numbers = [&](auto half) __attribute__((always_inline)) {
                constexpr bool HALF = decltype(half)::value;
                x.x = mx4_numbers<HALF>(w, ex.x, std::integral_constant<int, 0>{}); x.y = mx4_numbers<HALF>(w, ex.x, std::integral_constant<int, 1>{});
                x.z = mx4_numbers<HALF>(w, ex.y, std::integral_constant<int, 2>{}); x.w = mx4_numbers<HALF>(w, ex.y, std::integral_constant<int, 3>{});
            };
            if (half) numbers(std::true_type{});
            else numbers(std::false_type{});
            *reinterpret_cast<uint4 *>(to + (grp * 128 + d) * 16) = x;
        }
    }
}

__global__ __launch_bounds__(256) void pc_mx4_prepare_kernel(PcMx4Prepare P) { mx4_prepare((const char *)P.from, P); }
__global__ __launch_bounds__(256) void pc_mx4_prepare_arg_kernel(PcArgBlob, PcMx4Prepare P) { mx4_prepare((const char *)arguments(), P); }       // (the blob comes first)

void pc_launch_mx4_prepare(PcMx4Prepare P, const PcArgBlob *blob, hipStream_t st)
{
    P.list_blocks = (int32_t)std::max<int64_t>(1, std::min<int64_t>((P.n16 + (int64_t)P.n_rot * (PC_D / 2) + 255) / 256, 1024));
    P.query_blocks = (P.n_rows + 31) / 32 * ((P.n_q_heads + 3) / 4);
    const unsigned grid = (unsigned)(P.list_blocks + P.query_blocks + std::min<int64_t>((int64_t)P.n_tiles * P.n_kv_heads, 1 << 20));
    if (blob) pc_mx4_prepare_arg_kernel<<<grid, 256, 0, st>>>(*blob, P);
    else pc_mx4_prepare_kernel<<<grid, 256, 0, st>>>(P);
}

// -------------------------------------------------------------------------------------------------------------- rows
// A workgroup is 4 waves = 4 consecutive units (32 rows x head, heads of a KV head fastest) over the same run of tiles, two
// workgroups a compute unit: the transposed problem of the bf16 kernel (S^T = K . Q^T, O^T = V^T . P^T, see pc_kernels_window.hip, which
// this one follows in its softmax, masks and ring of direct loads).  What is its own:
//   scores   codes of keys straight from the ring to v_mfma_scale 32x32x64, by two e4m3 pieces of the turned queries: as long on the matrix unit
//            as bf16 keys would be (twice the work at twice the rate), a quarter of the reads from shared memory;
//   queries  come turned by their positions (pc_mx4_prepare_kernel) and are turned back by a run's rotation, both in fp16 (2^-11 of a value, an eighth
//            of what pieces are off by; 1 us less of a small prefill), then cut in pieces under one power of two for the row, the same for every turn;
//   values   come from the copy; they are finite, so that a probability of zero takes a key out.
// Bound: the vector unit, 140 instructions a tile and wave of which 49 turned queries (messages of 160 tokens: every fifth tile is another's) before that
// went to fp16, beside
// 512 cycles of matrix work; 64 heads over 8, 1024 rows over 13k tokens of such messages: 573 us, 0.76 PFLOP/s, which is why long prefills go another way.  Small ones
// are chains of latencies: 77 rows over 5 messages 15.3 us, in splits of six tiles (of four, three or two no less, and more to merge).

namespace {
__device__ __forceinline__ void ring_barrier() { asm volatile("s_barrier" ::: "memory"); }
// a tile's place in the ring: codes of keys, values, exponents
constexpr int ROWS_RING = 4, ROWS_SLOT = PC_MX4_CODES + PC_TILE * PC_D * 2 + 256;
}  // namespace

// HALF: probabilities and values in fp16, where no value of the cache is outside it.  A row's first scores put their largest at 2^ABOVE, and the reference
// moves where one would be above 2^LAZY_LOG2: what is 2^20 below a row's largest still is a normal number, and 2^30 below it one of a few bits.  (With a
// reference that stays at zero where a row's first scores are near it, what is 2^21 below a row's largest would be lost; less work, but no less time.)
template <bool HALF> __device__ __forceinline__ void mx4_rows(const PcWin &W, const PcMx4Rows &M, unsigned char *s_kv, uint32_t (*s_rot)[PC_D / 2])
{
    constexpr int RING = ROWS_RING, AHEAD = 3, LOADS = 3;
    constexpr int VALUES = PC_MX4_CODES, EXPS = VALUES + PC_TILE * PC_D * 2, SLOT = ROWS_SLOT;
    constexpr float LAZY_LOG2 = HALF ? 15.f : 32.f, ABOVE = HALF ? 6.f : 0.f;         // (2^31 keys of 2^32 x 6 x 2^60 fit 32 bits)
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
    const int64_t groups = ((int64_t)M.n_rows + 31) / 32;
    const uint2 *q_abs = M.q_abs + mx4_query_at(groups, h, R, hh, 0);
    const float q_unit = M.q_unit[(int64_t)h * groups * 32 + R];
    const int e_hi = (int)(__float_as_uint(q_unit) >> 23), e_lo = e_hi - 4;

    const unsigned char *kb = (const unsigned char *)W.k_store + (int64_t)kh * (W.slots / PC_TILE) * PC_MX4_TILE;
    const unsigned char *vb = (const unsigned char *)M.v_tiles + (int64_t)kh * M.v_slots * (PC_D * 2);
    // position p of a tile's codes (16 bytes each) holds block (p & 3) ^ (p >> 4 & 3) of key p >> 2: four keys fill the banks
    const unsigned lds0 = (unsigned)(uintptr_t)&s_kv[0];
    const unsigned k_src = (unsigned)((threadIdx.x & 127) >> 2) * 64 + (((threadIdx.x & 3) ^ (threadIdx.x >> 4 & 3)) << 4), v_src = threadIdx.x * 16;
    const unsigned e_src = PC_MX4_CODES + (unsigned)(lane & 31) * 4;
    auto request = [&](int slot0, int place, int at) __attribute__((always_inline)) {
        const unsigned char *kt = kb + (int64_t)(slot0 / PC_TILE) * PC_MX4_TILE, *vt = vb + (int64_t)(slot0 + place) * (PC_D * 2);
        const unsigned to = lds0 + at * SLOT;
        if (wave < 2) mx4_dma16(kt, k_src, to + wave * 1024);
        else mx4_dma4(kt, e_src, to + EXPS);                 // (both waves the same: every wave asks as often)
        mx4_dma16(vt, v_src, to + VALUES + wave * 1024);
        mx4_dma16(vt + 4096, v_src, to + VALUES + 4096 + wave * 1024);
    };

    mx4_i32x8 q_hi[2], q_lo[2];
    // (few: in the walk, what is read for all of it at once would not fit the registers)
    auto turn = [&](int rot, auto few) __attribute__((always_inline)) {
        const uint32_t own = M.rot_run[(int64_t)rot * (PC_D / 2) + lane];
        const uint2 *from = q_abs;
        asm volatile("" : "+v"(from));                   // (sixteen addresses, made once and kept, would not fit the registers)
        in_order();
        s_rot[wave][lane] = own;
        in_order();
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            const uint2 *r = reinterpret_cast<const uint2 *>(&s_rot[wave][(s >> 2) * 16 + 8 * hh + 2 * (s & 3)]);        // (sines: 32 words further)
            int u_hi, u_rest, v_hi, v_rest;
            mx4_turned(from[64 * s], from[64 * (s + 8)], r[0], r[16], u_hi, u_rest, v_hi, v_rest);
            q_hi[0][s] = u_hi; q_lo[0][s] = u_rest;
            q_hi[1][s] = v_hi; q_lo[1][s] = v_rest;
            if (decltype(few)::value && (s & 1)) __builtin_amdgcn_sched_barrier(0);
        }
        in_order();
    };

    // K row of the lane's MFMA row: permuted so that score registers 0..7 / 8..15 are keys 8 hh + 0..7 / 16 + 8 hh + 0..7
    const int krow = 16 * (n >> 4) + 8 * ((n >> 2) & 1) + 4 * ((n >> 3) & 1) + (n & 3);
    typedef const __attribute__((address_space(3))) bf16x8 *lds_frag;
    typedef const __attribute__((address_space(3))) int *lds_word;
    unsigned k_rd = lds0 + krow * 64 + ((hh ^ (krow >> 2 & 3)) << 4);          // block hh; block 2 + hh: at k_rd ^ 32
    asm volatile("" : "+v"(k_rd));
    unsigned v_rd = lds0 + VALUES + (hh * PC_D + n) * 16;
    asm volatile("" : "+v"(v_rd));
    unsigned e_rd = lds0 + EXPS + krow * 4;
    asm volatile("" : "+v"(e_rd));

    float m_ref = 0.f, l_run = 0.f;
    bool seen = false, all_seen = false;                 // the row has met a key; every row of the wave has
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
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const bool now = mx > -INFINITY, need = mx > LAZY_LOG2 || (!seen && now);
        seen |= now;
        all_seen = __builtin_amdgcn_ballot_w64(seen) == ~0ull;
        if (__builtin_amdgcn_ballot_w64(need) != 0) {
            const float shift = need ? mx - ABOVE : 0.f, alpha = ex2(-fmaxf(shift, 0.f));       // (down: nothing has been added yet)
            l_run *= alpha;
#pragma unroll
            for (int db = 0; db < 4; ++db) acc[db] *= alpha;
            m_ref += shift;
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] -= shift;
        }
    };
    auto score = [&](unsigned at) __attribute__((always_inline)) {
        const uint4 k0 = __builtin_bit_cast(uint4, *(lds_frag)(k_rd + at)), k1 = __builtin_bit_cast(uint4, *(lds_frag)((k_rd ^ 32) + at));
        const int e = (int)((unsigned)*(lds_word)(e_rd + at) >> (8 * hh));
        f32x16 s = mx4_scores32<0>(k0, e, q_lo[0], e_lo, zeros);
        s = mx4_scores32<2>(k1, e, q_lo[1], e_lo, s);
        s = mx4_scores32<0>(k0, e, q_hi[0], e_hi, s);
        return mx4_scores32<2>(k1, e, q_hi[1], e_hi, s);
    };
    const int T = item.n_tiles;
    if (T > 0) {
        // two walks over the same runs: of the tiles that are asked for, and of those that are worked on
        WinWalk ahead(W.runs + item.run0, item.skip, T), walk = ahead;
        auto place_of = [&](const WinWalk &w) __attribute__((always_inline)) {
            return *reinterpret_cast<const __attribute__((address_space(4))) int32_t *>(reinterpret_cast<uintptr_t>(M.places) +
                                                                                     (w.run - reinterpret_cast<uintptr_t>(W.runs)) / sizeof(PcWinRun) * sizeof(int32_t));
        };
        int asked = 0, place = place_of(ahead);
        auto further = [&]() __attribute__((always_inline)) {
            const bool same = ahead.a.z > PC_TILE;
            ahead.next();
            if (!same) place = place_of(ahead);
        };
        auto ask = [&](int at) __attribute__((always_inline)) {
            if (asked >= T) return;
            request(ahead.a.x, place, at);
            if (++asked < T) further();
        };
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) ask(i);
        int cur = walk.rot;
        turn(cur, std::false_type{});
        look_up_rows();                                  // (behind the first requests: its latency is not theirs)
        int t = 0;
#pragma unroll 1
        while (t < T) {
            const int u = t & (RING - 1);
            const unsigned at = u * SLOT;
            if (t + AHEAD <= T) wait_vm<LOADS * (AHEAD - 1)>();        // this wave's share of tile t has landed
            else wait_vm<0>();
            ring_barrier();                              // ... every wave's has, and tile t - 1 is no longer read
            const WinTile e = walk.tile();
            if (__builtin_expect(e.rot != cur, 0)) { cur = e.rot; turn(cur, std::true_type{}); }
            ask((u + AHEAD) & (RING - 1));
            f32x16 s = score(at);
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] -= m_ref;
            const bool edge = e.valid < PC_TILE || (e.self && lim_first - e.pos0 < PC_TILE - 1) || (lo_max > e.pos0 && e.sink < PC_TILE);
            bool none = false;
            if (__builtin_expect(edge, 0)) {
                const uint32_t sees = win_sees(e.pos0, e.valid, e.sink, e.self != 0, lo, lim);
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
                    pk[r] = mx4_pack<HALF>(ex2(s[2 * r]), ex2(s[2 * r + 1]));
                    ps = mx4_sum<HALF>(pk[r], ps);
                }
                const bf16x8 p[2] = {__builtin_bit_cast(bf16x8, make_uint4(pk[0], pk[1], pk[2], pk[3])), __builtin_bit_cast(bf16x8, make_uint4(pk[4], pk[5], pk[6], pk[7]))};
                bf16x8 fr[8];
#pragma unroll
                for (int f = 0; f < 8; ++f) fr[f] = *(lds_frag)(v_rd + at + ((f >> 2) * 2 * PC_D + 32 * (f & 3)) * 16);
                l_run += ps;
#pragma unroll
                for (int f = 0; f < 8; ++f) acc[f & 3] = mx4_mfma32<HALF>(fr[f], p[f >> 2], acc[f & 3]);
            }
            ++t;
            if (t < T) walk.next();
        }
    }
    ring_barrier();

    // results leave as whole cache lines, turned round in the wave's quarter of the ring: chunk c (16 bytes) of row r at c ^ (r & 15)
    const float l = l_run + __shfl_xor(l_run, 32);
    unsigned char *stg = &s_kv[0] + wave * 8192;
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

// (two waves a SIMD and not three, for which there were registers: 2048 rows of 64 heads over one message of 13k tokens 809 us, so 855; windows of 4096 270 and 300)
__global__ __attribute__((amdgpu_flat_work_group_size(256, 256), amdgpu_waves_per_eu(2, 2))) void pc_mx4_prefill_kernel(PcWin W, PcMx4Rows M)
{
    __shared__ __attribute__((aligned(1024))) unsigned char s_kv[ROWS_RING * ROWS_SLOT];
    __shared__ __attribute__((aligned(16))) uint32_t s_rot[4][PC_D / 2];         // a wave's cosines and sines, in fp16
    if (M.mark && *M.mark != M.mark_value) return;       // (the walk in front of this one served every call)
    if (*M.bf16_only == 0) mx4_rows<true>(W, M, s_kv, s_rot);
    else mx4_rows<false>(W, M, s_kv, s_rot);
}

void pc_launch_win_prefill_mx4(const PcWin &W, const PcMx4Rows &M, int n_items, hipStream_t st)
{
    if (n_items > 0) pc_mx4_prefill_kernel<<<(unsigned)n_items * W.n_kv_heads, 256, 0, st>>>(W, M);
}

// ------------------------------------------------------------------------------------------------------------ gather
// Long prefills (see pc_attend_mx4): the call's keys and values copied token after token into a packed copy, as pc_gather_kernel does it for bf16,
// keys turned to the positions that the call gives them and rounded to fp16 (off by 2^-11 of a value), values as the bf16 that they stand for.
// Values above 7 x 2^24 (times probabilities of 2^64, where that walk's reference need not move, and 2^31 keys, they would not fit 32 bits), keys of a norm
// above 2^10, and those that are no number (which that walk would add to masks), mark the call for the walk behind it: below, what queries under
// fp16's normal numbers are off by, 2^-25, moves a score by 2^-25 x 2^10 x sqrt(128) at most.
// Bound: memory, 136 bytes read and 512 written a token and KV head (9.9k tokens of 8 KV heads: 22 us; the walk behind it, pc_prefill_bf16_kernel, 2048
// rows of 64 heads: 490 us, 1.2 PFLOP/s, where the walk over the cache itself takes 930).
__global__ __launch_bounds__(256) void pc_mx4_gather_kernel(PcLaunch L, const PcGatherItem *__restrict__ items, int n_items, const int32_t *__restrict__ seg_kvoff,
                                                            uint32_t *mark, uint32_t value)
{
    __shared__ int s_slot[PC_TILE], s_seg[PC_TILE];
    __shared__ float s_norm[4];
    const int G = blockIdx.x, kh = blockIdx.y;
    int j = 0;
    while (j + 1 < n_items && items[j + 1].kg_tile0 <= G) ++j;           // few calls gather: a short scan
    const PcGatherItem it = items[j];
    const PcCallDesc cd = L.calls[it.call];
    const int t = G - it.kg_tile0;
    const int p_tiles = (it.n_par + PC_TILE - 1) / PC_TILE;
    if (threadIdx.x < PC_TILE) {
        const int r = threadIdx.x;
        int slot = -1, seg = 0;
        if (t < p_tiles) {
            const int i = PC_TILE * t + r - (p_tiles * PC_TILE - it.n_par);   // token of the parents' part (the padding comes first)
            if (i >= 0) {
                const int32_t *off = seg_kvoff + cd.seg_off;
                int lo = 0, hi = cd.n_sel - 1;
                while (lo < hi) {                          // last parent whose first token is <= i (empty ones share their successor's offset)
                    const int mid = (lo + hi + 1) >> 1;
                    if (off[mid] <= i) lo = mid; else hi = mid - 1;
                }
                seg = lo;
                slot = L.segs[cd.seg_off + lo].slot_start + (i - off[lo]);
            }
        } else {
            const int i = PC_TILE * (t - p_tiles) + r;     // token of the new message
            if (i < cd.self_len) { seg = cd.n_seg - 1; slot = L.segs[cd.seg_off + seg].slot_start + i; }
        }
        s_slot[r] = slot; s_seg[r] = seg;
    }
    __syncthreads();
    const int64_t head = (int64_t)kh * (L.slots / PC_TILE) * PC_MX4_TILE;
    const char *ks = (const char *)L.k_store + head, *vs = (const char *)L.v_store + head;
    {
        const int r = threadIdx.x >> 3, c = threadIdx.x & 7;
        const int slot = s_slot[r];
        uint16_t *dst = (uint16_t *)L.k_gather + ((int64_t)kh * L.kg_slots + (int64_t)G * PC_TILE + r) * PC_D + 8 * c;
        uint4 lo = make_uint4(0, 0, 0, 0), hi = lo;
        float ss = 0.f;
        if (slot >= 0) {
            const char *kt = ks + (int64_t)(slot / PC_TILE) * PC_MX4_TILE;
            const uint32_t a = *reinterpret_cast<const uint32_t *>(kt + slot % PC_TILE * 64 + 4 * c), b = *reinterpret_cast<const uint32_t *>(kt + slot % PC_TILE * 64 + 32 + 4 * c);
            const uint32_t ex = *reinterpret_cast<const uint32_t *>(kt + PC_MX4_CODES + slot % PC_TILE * 4) >> 8 * (c >> 2);
            const uint32_t ea = ex & 255u, eb = ex >> 16 & 255u;
            // (255: no number, which has codes of zero; a block of 2^10 holds one above 2^10, whose square marks the call: larger ones need no more)
            if (max(ea, eb) == (uint32_t)PC_MX4_NAN) *mark = value;
            const float ua = __uint_as_float(min(ea, 127u + 10u) << 23), ub = __uint_as_float(min(eb, 127u + 10u) << 23);
            const float4 *rot = reinterpret_cast<const float4 *>(L.rot_seg + (int64_t)(cd.seg_off + s_seg[r]) * (PC_D / 2) + 8 * c);
            uint32_t *lw = reinterpret_cast<uint32_t *>(&lo), *hw = reinterpret_cast<uint32_t *>(&hi);
            auto pair = [&](auto u) __attribute__((always_inline)) {
                constexpr int U = decltype(u)::value;
                const float4 cs = rot[U];                    // (cos, sin) of pairs 2 U and 2 U + 1
                const auto xs = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(a, 1.f, U), ys = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(b, 1.f, U);
                const float x0 = xs[0] * ua, x1 = xs[1] * ua, y0 = ys[0] * ub, y1 = ys[1] * ub;
                ss += x0 * x0 + x1 * x1 + y0 * y0 + y1 * y1;                 // (a turn keeps it)
                lw[U] = pack_f16(x0 * cs.x - y0 * cs.y, x1 * cs.z - y1 * cs.w);
                hw[U] = pack_f16(x0 * cs.y + y0 * cs.x, x1 * cs.w + y1 * cs.z);
            };
            pair(std::integral_constant<int, 0>{}); pair(std::integral_constant<int, 1>{}); pair(std::integral_constant<int, 2>{}); pair(std::integral_constant<int, 3>{});
        }
        *reinterpret_cast<uint4 *>(dst) = lo;
        *reinterpret_cast<uint4 *>(dst + 64) = hi;
        // The largest squared norm of the tile's keys (see pc_gather_kernel).  Eight lanes hold a row.
        ss += __shfl_xor(ss, 1); ss += __shfl_xor(ss, 2); ss += __shfl_xor(ss, 4);
        if (ss > 0x1p20f) *mark = value;
        ss = fmaxf(ss, __shfl_xor(ss, 8)); ss = fmaxf(ss, __shfl_xor(ss, 16)); ss = fmaxf(ss, __shfl_xor(ss, 32));
        if ((threadIdx.x & 63) == 0) s_norm[threadIdx.x >> 6] = ss;
    }
    __syncthreads();
    if (threadIdx.x == 0)
        L.kg_norm[(int64_t)kh * (L.kg_slots / PC_TILE) + G] = fmaxf(fmaxf(s_norm[0], s_norm[1]), fmaxf(s_norm[2], s_norm[3]));
#pragma unroll
    for (int rep = 0; rep < 2; ++rep) {
        const int idx = threadIdx.x + 256 * rep;
        const int q = idx >> 7, d = idx & 127;             // (q is the same for all lanes of a wave)
        auto word_of = [&](int slot) { return *reinterpret_cast<const uint32_t *>(vs + (int64_t)(slot / PC_TILE) * PC_MX4_TILE + slot % PC_TILE / 8 * 512 + mx4_word(d) * 4); };
        auto exps_of = [&](int slot) { return *reinterpret_cast<const uint64_t *>(vs + (int64_t)(slot / PC_TILE) * PC_MX4_TILE + PC_MX4_CODES + slot % PC_TILE / 8 * 32 + d / 32 * 8); };
        int sl[PC_VGROUP];
        bool run = true;                                   // the group's 8 tokens sit in 8 consecutive slots of the cache
#pragma unroll
        for (int k = 0; k < PC_VGROUP; ++k) {
            sl[k] = s_slot[PC_VGROUP * q + k];
            run = run && sl[0] >= 0 && sl[k] == sl[0] + k;
        }
        uint32_t w = 0;
        uint64_t ex = 0;                                   // (60 less the exponents)
        if (run) {                                         // of two groups of the cache
            const int sh = sl[0] & 7;
            w = word_of(sl[0]) >> 4 * sh;
            ex = exps_of(sl[0]) >> 8 * sh;
            if (sh > 0) {
                w |= word_of(sl[7]) << (32 - 4 * sh);
                ex |= exps_of(sl[7]) << (64 - 8 * sh);
            }
        } else {
#pragma unroll
            for (int k = 0; k < PC_VGROUP; ++k) {
                if (sl[k] >= 0) w |= (word_of(sl[k]) >> 4 * (sl[k] & 7) & 15u) << 4 * k;
                ex |= (sl[k] >= 0 ? exps_of(sl[k]) >> 8 * (sl[k] & 7) & 255u : (uint64_t)PC_MX4_E_MAX) << 8 * k;
            }
        }
        // some exponent of the eight is above PC_MX4_COPIED
        constexpr uint64_t EACH = 0x0101010101010101ull;
        if (~((ex | 0x80 * EACH) - (PC_MX4_E_MAX - PC_MX4_COPIED) * EACH) & 0x80 * EACH) *mark = value;
        const uint32_t e0 = (uint32_t)ex, e1 = (uint32_t)(ex >> 32);
        uint4 x;
        x.x = mx4_values(w, e0, std::integral_constant<int, 0>{}); x.y = mx4_values(w, e0, std::integral_constant<int, 1>{});
        x.z = mx4_values(w, e1, std::integral_constant<int, 2>{}); x.w = mx4_values(w, e1, std::integral_constant<int, 3>{});
        *reinterpret_cast<uint4 *>((uint16_t *)L.v_gather + (((int64_t)kh * L.kg_slots + (int64_t)G * PC_TILE) / PC_VGROUP + q) * PC_D * PC_VGROUP + (int64_t)d * PC_VGROUP) = x;
    }
}

void pc_launch_gather_mx4(const PcLaunch &L, const PcGatherItem *items, int n_items, int64_t n_tiles, const int32_t *seg_kvoff, uint32_t *mark, uint32_t value, hipStream_t st)
{
    if (n_items > 0 && n_tiles > 0) pc_mx4_gather_kernel<<<dim3((unsigned)n_tiles, (unsigned)L.n_kv_heads), 256, 0, st>>>(L, items, n_items, seg_kvoff, mark, value);
}
