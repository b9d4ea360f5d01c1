// Gradient of the windowed attention, bf16 caches (gfx950), and what both types share.
//
// With p = exp(s - LSE) from the forward's LSE, dp = dO . v and Delta = dO . out of a row:
//   ds = p (dp - Delta),  dq = scale sum ds k,  dk = scale sum ds q,  dv = sum p dO.
// p and ds are rounded to bf16 for the second products, as in the forward; what is summed is fp32, and no sum depends on the
// order in which workgroups run: a row's gradient belongs to one item (or to its splits, added up in order), a tile of keys to one
// item (or to its parts, likewise), so that the same call gives the same bits.
//
//   prep   per 32 rows and head: Delta, the queries turned by their positions, output gradients and statistics, laid out for keys
//   dq     rows: the forward's walk, with 24 matrix instructions a tile and unit (scores 8, dp 8, dq 8)
//   keys   four tiles of keys: a walk over the units that see them (32: scores and dv, dp and dk)
//
// Rotations.  dq is collected in the frame of the present run's keys and turned when the rotation changes; dk in the frame of the
// turned queries, in which a call's keys are turned once.
//
// Few keys.  Those keys are rounded once more than in the forward, so that a row's probabilities do not add up to 1: of two
// keys, that is as much as what the gradient is left with when Delta is taken off (dk 5.4e-3 off in the 2-norm; 4e-3 from 50 keys
// up).  Where window and sinks are 32 at most, the queries are turned for each extent as the forward turns them, and keys stay as they
// are stored: the same scores, and dk in the stored keys' frame.  (Not where a run's blocks see more than eight tiles of four, or parts of
// them, in the mean: 5.4e-3 at most of twelve messages of two tokens.)  The first rows of a message without parents see few keys under any
// window: 3.96e-3 over 300 rows.
#include "pc_window.h"
#include "pc_bwd_tiles.h"
#include <type_traits>

namespace {

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
// the lane's number, made where it stands: kept from the kernel's start it would wait in memory, and who fetches a register from
// there waits for all loads before it
__device__ __forceinline__ int lane_again()
{
    int x;
    asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(x));
    return x;
}
__device__ __forceinline__ bool finite16(uint32_t bits) { return (bits & 0x7F80u) != 0x7F80u; }
__device__ __forceinline__ bf16x8 finite_or_zero(bf16x8 x)
{
    uint4 u = __builtin_bit_cast(uint4, x);
    uint32_t *w = reinterpret_cast<uint32_t *>(&u);
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = (finite16(w[j]) ? w[j] & 0xFFFFu : 0u) | (finite16(w[j] >> 16) ? w[j] & 0xFFFF0000u : 0u);
    return __builtin_bit_cast(bf16x8, u);
}
// Accumulators of 32 columns, element (db, r) dim 32 db + 8 (r / 4) + 4 hh + r % 4: every column turned by the angles of `a` less
// those of `b` (rows of (cos, sin), 64 pairs; b null: by those of a), times f.
__device__ __forceinline__ void turn_columns(f32x16 (&acc)[4], const float2 *a, const float2 *b, int hh, float f)
{
#pragma unroll
    for (int db = 0; db < 2; ++db)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
            const int at = 32 * db + 8 * q4 + 4 * hh;
            const float4 a0 = *reinterpret_cast<const float4 *>(a + at), a1 = *reinterpret_cast<const float4 *>(a + at + 2);
            const float ac[4] = {a0.x, a0.z, a1.x, a1.z}, as[4] = {a0.y, a0.w, a1.y, a1.w};
            float4 b0 = make_float4(1.f, 0.f, 1.f, 0.f), b1 = b0;
            if (b) { b0 = *reinterpret_cast<const float4 *>(b + at); b1 = *reinterpret_cast<const float4 *>(b + at + 2); }
            const float bc[4] = {b0.x, b0.z, b1.x, b1.z}, bs[4] = {b0.y, b0.w, b1.y, b1.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float c = (ac[j] * bc[j] + as[j] * bs[j]) * f, s = (as[j] * bc[j] - ac[j] * bs[j]) * f;
                const float x = acc[db][4 * q4 + j], y = acc[db + 2][4 * q4 + j];
                acc[db][4 * q4 + j] = x * c - y * s;
                acc[db + 2][4 * q4 + j] = x * s + y * c;
            }
            __builtin_amdgcn_sched_barrier(0);           // (registers: a few loads at a time)
        }
}

}  // namespace

// -------------------------------------------------------------------------------------------------------------- prep
// bf16: a block of 32 rows of a head, eight threads a row; fp32: 32 (row, head) columns of a KV head.  Bound: memory (940 rows of 32
// heads: 38 MB read and written, 12 us).
// Delta by matrix instructions instead of by the threads' own sums costs nothing there; 160 fp32 rows of 8 heads of 64: 3.5 -> 5.8 us at least (a
// chain of 32 dependent instructions), of a step of 95.
template <int D, bool BF16>
__global__ __launch_bounds__(256) void pc_win_bwd_prep_kernel(PcWin W, PcWinBwd B)
{
    constexpr int HALF = D / 2, PER = HALF / 8;          // pairs a thread takes
    __shared__ int s_lo[32], s_state[32];                // of a row: 0 there is none, 1 it has a gradient, 2 it has none
    const PcWinBlock blk = B.blocks[blockIdx.x];
    const int g = W.n_q_heads / W.n_kv_heads;
    const int r = threadIdx.x >> 3, c = threadIdx.x & 7;
    const int64_t unit = (int64_t)blockIdx.x * gridDim.y + blockIdx.y;
    auto place = [&](int i, int64_t &row, int64_t &h, bool &ok) {
        if constexpr (BF16) {
            row = 32 * (int64_t)blk.block + i; h = blockIdx.y; ok = row < blk.n_q;
            row = min(row, (int64_t)blk.n_q - 1);
        } else {
            int64_t col = 32 * (int64_t)blk.block + i;
            ok = col < (int64_t)blk.n_q * g;
            col = min(col, (int64_t)blk.n_q * g - 1);
            row = col / g; h = (int64_t)blockIdx.y * g + col % g;
        }
    };
    int64_t row, h;
    bool ok;
    place(r, row, h, ok);
    // Behind the last row: its queries again, without a gradient.  What the keys it sees make of it is what they make of the last
    // row, and 0 times that, also where a key is not finite; no tile is masked for its sake.
    const int64_t R = (int64_t)blk.q_off + row, at = (R * W.n_q_heads + h) * D + PER * c;
    const float lse = B.lse[R * W.n_q_heads + h];
    const bool some = lse > -INFINITY, live = ok && some;          // (a row that saw nothing, or whose scores were not numbers, has no gradient)
    // Delta = d_out . out, by the instruction and in the order that dp = d_out . v is made with (the diagonal of a product of the 32 rows, by
    // the first wave): where a row sees one key, out is v, dp - Delta is 0 to the last bit, and so are d_q and d_k.
    if (threadIdx.x < 64) {
        const int lane = threadIdx.x, n = lane & 31, hh = lane >> 5;
        int64_t row_n, h_n;
        bool ok_n;
        place(n, row_n, h_n, ok_n);
        const int64_t at_n = ((int64_t)blk.q_off + row_n) * W.n_q_heads + h_n;
        f32x16 prod;
#pragma unroll
        for (int i = 0; i < 16; ++i) prod[i] = 0.f;
        if constexpr (BF16) {
            const uint16_t *o = (const uint16_t *)B.out + at_n * D + 8 * hh, *d = (const uint16_t *)B.d_out + at_n * D + 8 * hh;
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) prod = MFMA32(__builtin_bit_cast(bf16x8, ldg16(o + 16 * ks)), __builtin_bit_cast(bf16x8, ldg16(d + 16 * ks)), prod);
        } else {
            const float *o = (const float *)B.out + at_n * D + HALF * hh, *d = (const float *)B.d_out + at_n * D + HALF * hh;
#pragma unroll 4
            for (int i = 0; i < HALF; i += 4) {
                const float4 u = *reinterpret_cast<const float4 *>(o + i), v = *reinterpret_cast<const float4 *>(d + i);
                prod = __builtin_amdgcn_mfma_f32_32x32x2f32(u.x, v.x, prod, 0, 0, 0);
                prod = __builtin_amdgcn_mfma_f32_32x32x2f32(u.y, v.y, prod, 0, 0, 0);
                prod = __builtin_amdgcn_mfma_f32_32x32x2f32(u.z, v.z, prod, 0, 0, 0);
                prod = __builtin_amdgcn_mfma_f32_32x32x2f32(u.w, v.w, prod, 0, 0, 0);
            }
        }
        float delta = 0.f;                               // element (row n, column n): register 4 (n / 8) + n % 4 of the lane whose half is n / 4 % 2
#pragma unroll
        for (int i = 0; i < 16; ++i) delta = i == 4 * (n >> 3) + (n & 3) ? prod[i] : delta;
        if (hh == ((n >> 2) & 1)) {
            delta = ok_n && B.lse[at_n] > -INFINITY ? delta : 0.f;
            reinterpret_cast<PcWinStat *>(B.stat + unit * PC_WIN_STAT_BYTES)->delta[n] = delta;
            if (ok_n) B.delta[at_n] = delta;
        }
    }
    float x[PER], y[PER], gx[PER], gy[PER];
    // PER numbers at p: pairs' first halves, or (HALF further) their second
    auto get = [&](const void *p, int64_t i, float (&v)[PER]) {
        if constexpr (BF16) {
            const uint4 w = ldg16((const uint16_t *)p + i);
            const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int k = 0; k < PER / 2; ++k) { v[2 * k] = bf_lo(u[k]); v[2 * k + 1] = bf_hi(u[k]); }
        } else {
#pragma unroll
            for (int k = 0; k < PER; k += 4) *reinterpret_cast<float4 *>(v + k) = *reinterpret_cast<const float4 *>((const float *)p + i + k);
        }
    };
    auto put = [&](void *p, int64_t i, const float (&v)[PER]) {
        if constexpr (BF16) *reinterpret_cast<uint4 *>((uint16_t *)p + i) = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
        else {
#pragma unroll
            for (int k = 0; k < PER; k += 4) *reinterpret_cast<float4 *>((float *)p + i + k) = *reinterpret_cast<const float4 *>(v + k);
        }
    };
    {
        float qx[PER], qy[PER];
        get(W.q, at, qx); get(W.q, at + HALF, qy);
        get(B.d_out, at, gx); get(B.d_out, at + HALF, gy);
        const float4 *rot = reinterpret_cast<const float4 *>(W.rot_q + R * HALF + PER * c);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const float4 cs2 = rot[i / 2];
            const float co = i & 1 ? cs2.z : cs2.x, si = i & 1 ? cs2.w : cs2.y;
            x[i] = some ? qx[i] * co - qy[i] * si : 0.f; y[i] = some ? qx[i] * si + qy[i] * co : 0.f;
            gx[i] = live ? gx[i] : 0.f; gy[i] = live ? gy[i] : 0.f;
        }
    }
    const int64_t to = (unit * 32 + r) * D + PER * c;
    if (!B.turned) { put(B.q_abs, to, x); put(B.q_abs, to + HALF, y); }
    put(B.d_o, to, gx); put(B.d_o, to + HALF, gy);
    const int lo = win_low(W.q_pos[R], W.window);
    char *const st = B.stat + unit * PC_WIN_STAT_BYTES;
    PcWinStat *const to_stat = reinterpret_cast<PcWinStat *>(st);
    if (c == 0) {
        to_stat->lse2[r] = live ? lse * 1.4426950408889634f : INFINITY;
        to_stat->lo[r] = lo; to_stat->lim[r] = blk.lim0 + (int)row;
        s_lo[r] = lo;
        s_state[r] = live ? 1 : ok ? 2 : 0;
    }
    __syncthreads();
    if (threadIdx.x < 64) {                              // (lanes 32 up: the rows again)
        const int at = threadIdx.x & 31, state = s_state[at];
        int lo_min = s_state[at] ? s_lo[at] : INT32_MAX, lo_max = state == 2 ? INT32_MAX : state ? s_lo[at] : INT32_MIN;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { lo_min = min(lo_min, __shfl_xor(lo_min, o)); lo_max = max(lo_max, __shfl_xor(lo_max, o)); }
        const uint32_t live_rows = (uint32_t)__builtin_amdgcn_ballot_w64(state == 1);
        if (threadIdx.x == 0) {
            const int64_t first = BF16 ? 32 * (int64_t)blk.block : 32 * (int64_t)blk.block / g;
            const int64_t last = min((int64_t)blk.n_q - 1, BF16 ? first + 31 : (32 * (int64_t)blk.block + 31) / g);
            to_stat->head = make_int4(lo_min, lo_max, blk.lim0 + (int)first, blk.lim0 + (int)last);
            to_stat->live = (int)live_rows;
        }
    }
}

void pc_launch_win_bwd_prep(const PcWin &W, const PcWinBwd &B, int dtype, int D, hipStream_t st)
{
    if (B.n_blocks <= 0) return;
    const dim3 grid((unsigned)B.n_blocks, (unsigned)(dtype == 1 ? W.n_q_heads : W.n_kv_heads));
    if (dtype == 1) pc_win_bwd_prep_kernel<128, true><<<grid, 256, 0, st>>>(W, B);
    else if (D == 64) pc_win_bwd_prep_kernel<64, false><<<grid, 256, 0, st>>>(W, B);
    else pc_win_bwd_prep_kernel<128, false><<<grid, 256, 0, st>>>(W, B);
}

// The forward's queries of a block for one extent: the same numbers (row by row, scale included) that its scores were made of.
__global__ __launch_bounds__(256) void pc_win_bwd_turned_kernel(PcWin W, PcWinBwd B)
{
    const PcWinTurned t = B.turned[blockIdx.x];
    const PcWinBlock blk = B.blocks[t.block];
    const int r = threadIdx.x >> 3, c = threadIdx.x & 7;             // a row, eight pairs
    const int64_t h = blockIdx.y, R = (int64_t)blk.q_off + min(32 * (int64_t)blk.block + r, (int64_t)blk.n_q - 1);
    const bool some = B.lse[R * W.n_q_heads + h] > -INFINITY;
    const uint16_t *q = (const uint16_t *)W.q + (R * W.n_q_heads + h) * PC_D + 8 * c;
    const uint4 lq = ldg16(q), hq = ldg16(q + 64);
    const uint4 *rq = reinterpret_cast<const uint4 *>(W.rot_lanes) + ((R >> 5) * 16 + (c >> 1) * 4 + (c & 1)) * 32 + (R & 31);
    const uint4 p0 = rq[0], p1 = rq[64];
    const float4 *rr = reinterpret_cast<const float4 *>(W.rot_run + (int64_t)t.rot * (PC_D / 2) + 8 * c);
    const uint32_t lw[4] = {lq.x, lq.y, lq.z, lq.w}, hw[4] = {hq.x, hq.y, hq.z, hq.w}, pw[8] = {p0.x, p0.y, p0.z, p0.w, p1.x, p1.y, p1.z, p1.w};
    uint32_t a[4], b[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float4 p = make_float4(f16_lo(pw[2 * j]), f16_hi(pw[2 * j]), f16_lo(pw[2 * j + 1]), f16_hi(pw[2 * j + 1]));
        float4 r4 = rr[j];
        r4.x *= W.scale_log2; r4.y *= W.scale_log2; r4.z *= W.scale_log2; r4.w *= W.scale_log2;
        const float c0 = p.x * r4.x + p.y * r4.y, s0 = p.y * r4.x - p.x * r4.y, c1 = p.z * r4.z + p.w * r4.w, s1 = p.w * r4.z - p.z * r4.w;
        const float x0 = bf_lo(lw[j]), x1 = bf_hi(lw[j]), y0 = bf_lo(hw[j]), y1 = bf_hi(hw[j]);
        a[j] = some ? pack_bf16(x0 * c0 - y0 * s0, x1 * c1 - y1 * s1) : 0u;
        b[j] = some ? pack_bf16(x0 * s0 + y0 * c0, x1 * s1 + y1 * c1) : 0u;
    }
    uint16_t *to = (uint16_t *)B.q_abs + (((int64_t)blockIdx.x * W.n_q_heads + h) * 32 + r) * PC_D + 8 * c;
    *reinterpret_cast<uint4 *>(to) = make_uint4(a[0], a[1], a[2], a[3]);
    *reinterpret_cast<uint4 *>(to + 64) = make_uint4(b[0], b[1], b[2], b[3]);
}

void pc_launch_win_bwd_turned(const PcWin &W, const PcWinBwd &B, hipStream_t st)
{
    if (B.n_turned > 0) pc_win_bwd_turned_kernel<<<dim3((unsigned)B.n_turned, (unsigned)W.n_q_heads), 256, 0, st>>>(W, B);
}

// ---------------------------------------------------------------------------------------------------------------- dq
// As the forward's prefill kernel: 4 waves = 4 units, two workgroups a compute unit, K and V tiles in a ring of four.  Bound likewise:
// 33 blocks of rows over 20 tiles of seven messages, 66 us.
__global__ __launch_bounds__(256, 2) void pc_win_bwd_dq_bf16_kernel(PcWin W, PcWinBwd B)
{
    constexpr int RING = 4, AHEAD = 3;
    __shared__ __attribute__((aligned(1024))) unsigned char s_kv[RING][2 * TILE_BYTES];
    __shared__ __attribute__((aligned(16))) float2 s_rot[4][PC_D / 2];

    const int kh = blockIdx.x % W.n_kv_heads;
    const PcWinItem item = W.items[blockIdx.x / W.n_kv_heads];
    const int g = W.n_q_heads / W.n_kv_heads;
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const int n = lane & 31, hh = lane >> 5;
    const int n_units = ((item.n_q + 31) >> 5) * g;
    const bool unit_ok = item.unit0 + wave < n_units;
    const int unit = unit_ok ? item.unit0 + wave : item.unit0;
    const int ub = unit / g, h = kh * g + (unit - ub * g);
    const int row = min(32 * ub + n, item.n_q - 1);
    const bool row_ok = unit_ok && 32 * ub + n < item.n_q;
    const int64_t R = (int64_t)item.q_off + row;
    const int lim = item.lim0 + row, lim_first = item.lim0 + 32 * ub;

    const unsigned char *kb = (const unsigned char *)W.k_store + (int64_t)kh * W.slots * (PC_D * 2);
    const unsigned char *vb = (const unsigned char *)W.v_store + (int64_t)kh * W.slots * (PC_D * 2);
    const unsigned ring = (unsigned)(uintptr_t)&s_kv[0][0], lds0 = ring + wave * 1024;
    const unsigned k_src = (threadIdx.x >> 4) * 256 + (((threadIdx.x & 15) ^ swz(threadIdx.x >> 4)) << 4);
    const unsigned v_src = (unsigned)v_src_chunk(threadIdx.x) * 16;
    auto request = [&](const WinTile &d, int slot) __attribute__((always_inline)) {
        const int64_t at = (int64_t)d.slot0 * (PC_D * 2);
        const unsigned to = lds0 + slot * (2 * TILE_BYTES);
        dma16(kb + at, k_src, to);
        dma16(kb + at + 4096, k_src, to + 4096);         // (rows 16 up: the same order of chunks)
        dma16(vb + at, v_src, to + TILE_BYTES);
        dma16(vb + at + 4096, v_src, to + TILE_BYTES + 4096);
    };
    const RowMajor by_key(perm_row(n), lane);
    const ValuesByKey<true> rv(lane);

    const int T = item.n_tiles;
    WinWalk walk(W.runs + item.run0, item.skip, T);         // (not looked at where there is no tile)
    WinTile d[AHEAD + 1];
    int asked = 0;
    auto ask = [&](WinTile &to, int slot) __attribute__((always_inline)) {
        if (asked >= T) return;
        if (asked > 0) walk.next();
        ++asked;
        to = walk.tile();
        request(to, slot);
    };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) ask(d[i], i);
    const float lse = B.lse[R * W.n_q_heads + h], delta_r = B.delta[R * W.n_q_heads + h];
    const int lo = win_low(W.q_pos[R], W.window);
    const bool live = row_ok && lse > -INFINITY;
    const float lse2 = live ? lse * 1.4426950408889634f : INFINITY, delta = live ? delta_r : 0.f;
    int lo_max = live ? lo : INT32_MIN;                  // (a row without a gradient gets zeros at the end)
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) lo_max = max(lo_max, __shfl_xor(lo_max, o));
    lo_max = uniform(lo_max);
    bf16x8 go[8];                                        // the lane's row of output gradients, dims 16 ks + 8 hh + 0..7
    {
        const unsigned char *p = (const unsigned char *)B.d_out + (R * W.n_q_heads + h) * (PC_D * 2) + 16 * hh;
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) go[ks] = __builtin_bit_cast(bf16x8, live ? ldg16(p + 32 * ks) : make_uint4(0, 0, 0, 0));
    }
    bf16x8 qop[8];
    auto turn = [&](int rot) __attribute__((always_inline)) {       // as in the forward: the same bits but for a rounding of the scale
        const uint4 *rq = reinterpret_cast<const uint4 *>(W.rot_lanes) + (R >> 5) * 512 + hh * 32 + (R & 31);
        // (the run's rotation is the same for all rows: one load a lane, and broadcasts from shared memory)
        const float2 own = W.rot_run[(int64_t)rot * (PC_D / 2) + lane];
        asm volatile("" ::: "memory");
        s_rot[wave][lane] = own;
        asm volatile("" ::: "memory");                   // (a wave's own LDS accesses happen in order)
        const float4 *rr = reinterpret_cast<const float4 *>(&s_rot[wave][8 * hh]);
        const unsigned char *qp = (const unsigned char *)W.q + (R * W.n_q_heads + h) * (PC_D * 2) + 16 * hh;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            uint4 lq = ldg16(qp + 32 * ks), hq = ldg16(qp + 32 * ks + 128);
            if (!live) lq = hq = make_uint4(0, 0, 0, 0);
            const uint32_t lw[4] = {lq.x, lq.y, lq.z, lq.w}, hw[4] = {hq.x, hq.y, hq.z, hq.w};
            const uint4 p0 = rq[ks * 128], p1 = rq[ks * 128 + 64];
            const uint32_t pw[8] = {p0.x, p0.y, p0.z, p0.w, p1.x, p1.y, p1.z, p1.w};
            uint32_t a[4], b[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float4 p = make_float4(f16_lo(pw[2 * j]), f16_hi(pw[2 * j]), f16_lo(pw[2 * j + 1]), f16_hi(pw[2 * j + 1]));
                const float4 r = rr[8 * ks + j];
                const float c0 = (p.x * r.x + p.y * r.y) * W.scale_log2, s0 = (p.y * r.x - p.x * r.y) * W.scale_log2;
                const float c1 = (p.z * r.z + p.w * r.w) * W.scale_log2, s1 = (p.w * r.z - p.z * r.w) * W.scale_log2;
                const float x0 = bf_lo(lw[j]), x1 = bf_hi(lw[j]), y0 = bf_lo(hw[j]), y1 = bf_hi(hw[j]);
                a[j] = pack_bf16(x0 * c0 - y0 * s0, x1 * c1 - y1 * s1);
                b[j] = pack_bf16(x0 * s0 + y0 * c0, x1 * s1 + y1 * c1);
            }
            qop[ks] = frag4(a[0], a[1], a[2], a[3]);
            qop[ks + 4] = frag4(b[0], b[1], b[2], b[3]);
            if (ks & 1) __builtin_amdgcn_sched_barrier(0);         // (what is read for all of it at once would not fit the registers)
        }
    };
    f32x16 acc[4];
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[db][r] = 0.f;

    int cur = -1;
    if (T > 0) {
#pragma unroll 1
        for (int t = 0, u = 0; t < T; ++t, u = (u + 1) & (RING - 1)) {
            const unsigned kt = ring + u * (2 * TILE_BYTES), vt = kt + TILE_BYTES;
            if (t + AHEAD <= T) wait_vm<4 * (AHEAD - 1)>();
            else wait_vm<0>();
            ring_barrier();
            const WinTile e = d[0];
            if (__builtin_expect(e.rot != cur, 0)) {
                if (cur >= 0) turn_columns(acc, W.rot_run + (int64_t)cur * (PC_D / 2), W.rot_run + (int64_t)e.rot * (PC_D / 2), hh, 1.f);
                cur = e.rot;
                turn(cur);
            }
            ask(d[AHEAD], (u + AHEAD) & (RING - 1));
            RowMajor rk = by_key;
            asm volatile("" : "+v"(rk.row_at), "+v"(rk.col_at[0]), "+v"(rk.col_at[1]));       // (sixteen addresses made once and kept would not fit the registers)
            f32x16 s, dp;
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = dp[r] = 0.f;
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) s = MFMA32(rk.by_row(kt, ks), qop[ks], s);
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) dp = MFMA32(rv.get(vt, ks), go[ks], dp);
            const bool edge = e.valid < PC_TILE || (e.self && lim_first - e.pos0 < PC_TILE - 1) || (lo_max > e.pos0 && e.sink < PC_TILE);
            bool odd = false;
            uint32_t sees = ~0u;
            if (__builtin_expect(edge, 0)) {
                sees = win_sees(e.pos0, e.valid, e.sink, e.self != 0, lo, lim);
                f32x16 z;
#pragma unroll
                for (int r = 0; r < 16; ++r) z[r] = 0.f;
                const bf16x8 zero = frag4(0, 0, 0, 0);
#pragma unroll
                for (int ks = 0; ks < 8; ++ks) z = MFMA32(rk.by_row(kt, ks), zero, z);
                float sum = 0.f;
#pragma unroll
                for (int r = 0; r < 16; ++r) sum += z[r];
                odd = __builtin_amdgcn_ballot_w64(sum != 0.f) != 0;          // (a key that is not finite)
            }
            uint32_t pk[8];
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = ex2(s[r] - lse2) * (dp[r] - delta);
            if (__builtin_expect(edge, 0)) {
                const int mine = (int)(sees >> (8 * hh));
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = (mine >> (16 * (r >> 3) + (r & 7))) & 1 ? s[r] : 0.f;
            }
#pragma unroll
            for (int r = 0; r < 8; ++r) pk[r] = pack_bf16(s[2 * r], s[2 * r + 1]);
            const bf16x8 ds[2] = {frag4(pk[0], pk[1], pk[2], pk[3]), frag4(pk[4], pk[5], pk[6], pk[7])};
            if (__builtin_expect(odd, 0)) {              // (the rows that see such a key have no gradient, or a probability of 0)
#pragma unroll
                for (int f = 0; f < 8; ++f) acc[f & 3] = MFMA32(finite_or_zero(rk.by_col(kt, f >> 2, f & 3)), ds[f >> 2], acc[f & 3]);
            } else {
#pragma unroll
                for (int f = 0; f < 8; ++f) acc[f & 3] = MFMA32(rk.by_col(kt, f >> 2, f & 3), ds[f >> 2], acc[f & 3]);
            }
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) d[i] = d[i + 1];
        }
    }
    // back from the last run's frame and the row's position, and out as whole lines (in two halves of a row, 256 bytes each)
    if (cur >= 0) turn_columns(acc, W.rot_run + (int64_t)cur * (PC_D / 2), W.rot_q + R * (PC_D / 2), hh, B.scale);
    ring_barrier();
    unsigned char *stg = &s_kv[0][0] + wave * TILE_BYTES;
    const int r4 = lane >> 4, c = lane & 15;
    float *dst = (item.part < 0 ? B.d_q + (int64_t)item.q_off * W.n_q_heads * PC_D : W.part_o + (int64_t)item.part * W.n_q_heads * PC_D) + (int64_t)h * PC_D + 4 * c;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        asm volatile("" ::: "memory");
#pragma unroll
        for (int db = 0; db < 2; ++db)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {
                const f32x16 &a = acc[2 * half + db];
                *reinterpret_cast<float4 *>(stg + n * 256 + (((8 * db + 2 * q4 + hh) ^ (n & 15)) << 4)) = live ? make_float4(a[4 * q4], a[4 * q4 + 1], a[4 * q4 + 2], a[4 * q4 + 3]) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
        asm volatile("" ::: "memory");
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = 4 * i + r4, rw = 32 * ub + r;
            const float4 v = *reinterpret_cast<const float4 *>(stg + r * 256 + ((c ^ (r & 15)) << 4));
            if (unit_ok && rw < item.n_q) *reinterpret_cast<float4 *>(dst + (int64_t)rw * W.n_q_heads * PC_D + 64 * half) = v;
        }
    }
}

void pc_launch_win_bwd_dq_bf16(const PcWin &W, const PcWinBwd &B, int n_items, hipStream_t st)
{
    if (n_items > 0) pc_win_bwd_dq_bf16_kernel<<<(unsigned)n_items * W.n_kv_heads, 256, 0, st>>>(W, B);
}

__global__ __launch_bounds__(256) void pc_win_bwd_rows_kernel(const PcMergeRow *__restrict__ rows, int64_t n, int row16, const float *__restrict__ part, float *__restrict__ d_q)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    const PcMergeRow mr = rows[i / row16];
    const int64_t at = i % row16;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s = 0; s < mr.n_splits; ++s) {
        const float4 x = reinterpret_cast<const float4 *>(part)[((int64_t)mr.part_row0 + (int64_t)s * mr.n_q) * row16 + at];
        sum.x += x.x; sum.y += x.y; sum.z += x.z; sum.w += x.w;
    }
    reinterpret_cast<float4 *>(d_q)[(int64_t)mr.row * row16 + at] = sum;
}

void pc_launch_win_bwd_rows(const PcWin &W, const PcWinBwd &B, const PcMergeRow *rows, int n_rows, int D, hipStream_t st)
{
    if (n_rows <= 0) return;
    const int row16 = W.n_q_heads * D / 4;
    const int64_t n = (int64_t)n_rows * row16;
    pc_win_bwd_rows_kernel<<<(unsigned)((n + 255) / 256), 256, 0, st>>>(rows, n, row16, W.part_o, B.d_q);
}

// -------------------------------------------------------------------------------------------------------------- keys
// A workgroup is 8 waves over four tiles of keys: waves 0 to 3 make the probabilities of a tile and collect its dv, waves 4 to 7
// collect its dk, a unit behind: they find the probabilities in shared memory (fp32).  A wave then has 16 matrix instructions a unit
// and room for two waves a SIMD; with everything in one wave it would need 330 registers.  The units' turned queries, output
// gradients and statistics come by direct loads into a ring of five.
//
// What bounds it: 33 blocks of rows, 32 heads over 8, over 4800 listed tokens, 76 us, in steps of a unit of 1.3 us: with all four
// tiles at work shared memory (210 KB a step: 1.7 thousand of 2.8 thousand cycles), with the sinks' one tile a wave's own chain; and
// 8 us an item to start and to write 128 KB.  Before: scores in both halves of the waves 122 us; probabilities handed over, operands
// read as they were needed 97; read ahead 79; items spread by the host 76.
__global__ __launch_bounds__(512, 2) void pc_win_bwd_keys_bf16_kernel(PcWin W, PcWinBwd B)
{
    constexpr int RING = 5, AHEAD = 3, SLOT = 2 * TILE_BYTES + PC_WIN_STAT_BYTES;
    __shared__ __attribute__((aligned(1024))) unsigned char s_ring[RING][SLOT];
    __shared__ __attribute__((aligned(1024))) unsigned char s_v[PC_WIN_KEY_TILES][TILE_BYTES];        // the call's values, in the store's order
    __shared__ float4 s_p[2][PC_WIN_KEY_TILES][4][64];   // a unit's probabilities, in the lanes' order

    const int kh = blockIdx.x % W.n_kv_heads;
    const int bin = blockIdx.x / W.n_kv_heads;
    const int g = W.n_q_heads / W.n_kv_heads;
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const int n = lane & 31, hh = lane >> 5;
    const int tile = wave & 3;
    const bool is_k = wave >= 4;
    const unsigned ring = (unsigned)(uintptr_t)&s_ring[0][0];
    const unsigned src = (threadIdx.x >> 4) * 256 + (((threadIdx.x & 15) ^ swz(threadIdx.x >> 4)) << 4);
    const RowMajor by_row(perm_row(n), lane), by_col(n, lane);
    const ValuesByKey<false> values(lane);               // by key, the lane's one
    const int item_end = B.bins[bin + 1];
#pragma unroll 1
    for (int i_item = B.bins[bin]; i_item < item_end; ++i_item) {
    const PcWinKeyItem item = B.key_items[i_item];
    const int my_keys = item.n_keys - PC_TILE * tile;    // of the wave's tile
    f32x16 acc[4];
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[db][r] = 0.f;
    int cur = -1;
    auto collect = [&](auto role) __attribute__((always_inline)) {
    constexpr bool K = decltype(role)::value;
    for (int a = 0; a < item.n_apps; ++a) {
        const PcWinApp app = B.apps[item.app0 + a];
        const int pos0 = app.pos0 + PC_TILE * tile, valid = min(app.n_tok - PC_TILE * tile, PC_TILE), sink = min(max(app.sink - PC_TILE * tile, 0), PC_TILE);
        const bool active = valid > 0;
        const int U = app.n_blocks * g;
        int64_t next = (int64_t)app.block0 * W.n_q_heads + kh * g;       // the unit to ask for, and its head within the group
        const int64_t q_ahead = ((int64_t)app.q0 - app.block0) * W.n_q_heads;
        int next_j = 0, next_slot = 0;
        auto request = [&]() __attribute__((always_inline)) {
            const unsigned to = ring + next_slot * SLOT + wave * 1024;
            dma16((const unsigned char *)B.q_abs + (next + q_ahead) * TILE_BYTES, src, to);
            dma16((const unsigned char *)B.d_o + next * TILE_BYTES, src, to + TILE_BYTES);
            if (!K && wave == 0) dma16(B.stat + next * PC_WIN_STAT_BYTES, lane * 16, to + 2 * TILE_BYTES);
            ++next; ++next_j;
            if (next_j == g) { next_j = 0; next += W.n_q_heads - g; }
            next_slot = next_slot == RING - 1 ? 0 : next_slot + 1;
        };
        // all but the last N units that were asked for are there
        auto landed = [&](auto N) __attribute__((always_inline)) {
            constexpr int units = decltype(N)::value;
            if (!K && wave == 0) wait_vm<3 * units>();
            else wait_vm<2 * units>();
        };
        ring_barrier();                                  // (the last call's units and values are no longer read)
        if (!K && active) {
            const unsigned char *v = (const unsigned char *)W.v_store + ((int64_t)kh * W.slots + item.slot0 + PC_TILE * tile) * (PC_D * 2);
            const unsigned to = (unsigned)(uintptr_t)&s_v[tile][0];
#pragma unroll
            for (int i = 0; i < 8; ++i) dma16(v, (unsigned)v_src_chunk(64 * i + lane) * 16, to + 1024 * i);
        }
        for (int i = 0; i < min(AHEAD, U); ++i) request();
        bf16x8 op[8];                                    // the lane's key, turned and scaled, or its value: dims 16 ks + 8 hh + 0..7
        if constexpr (K) {
            // dk, kept in the frame of the queries: from the last call's to this one's
            if (active) {
                if (cur >= 0 && cur != app.rot) turn_columns(acc, W.rot_run + (int64_t)app.rot * (PC_D / 2), W.rot_run + (int64_t)cur * (PC_D / 2), hh, 1.f);
                cur = app.rot;
            }
        } else {
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) op[ks] = frag4(0, 0, 0, 0);
            if (active) {
                const int64_t slot = (int64_t)kh * W.slots + item.slot0 + PC_TILE * tile + n;
                const unsigned char *kp = (const unsigned char *)W.k_store + slot * (PC_D * 2) + 16 * hh;
                const float4 *rr = reinterpret_cast<const float4 *>(W.rot_run + (int64_t)app.rot * (PC_D / 2) + 8 * hh);
#pragma unroll
                for (int ks = 0; ks < 4; ++ks) {
                    const uint4 lk = ldg16(kp + 32 * ks), hk = ldg16(kp + 32 * ks + 128);
                    const uint32_t lw[4] = {lk.x, lk.y, lk.z, lk.w}, hw[4] = {hk.x, hk.y, hk.z, hk.w};
                    uint32_t x[4], y[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        float4 r = rr[8 * ks + j];
                        r.x *= B.k_factor; r.y *= B.k_factor; r.z *= B.k_factor; r.w *= B.k_factor;
                        const float x0 = bf_lo(lw[j]), x1 = bf_hi(lw[j]), y0 = bf_lo(hw[j]), y1 = bf_hi(hw[j]);
                        x[j] = pack_bf16(x0 * r.x - y0 * r.y, x1 * r.z - y1 * r.w);
                        y[j] = pack_bf16(x0 * r.y + y0 * r.x, x1 * r.w + y1 * r.z);
                    }
                    op[ks] = frag4(x[0], x[1], x[2], x[3]);
                    op[ks + 4] = frag4(y[0], y[1], y[2], y[3]);
                    if (ks & 1) __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
        if (U >= AHEAD) landed(std::integral_constant<int, AHEAD - 1>());
        else wait_vm<0>();
        ring_barrier();
        bf16x8 rows[8];                                  // the left operand of the wave's next unit, and that unit's limits
        int4 head = make_int4(0, 0, 0, 0);
        auto fetch = [&](int place) __attribute__((always_inline)) {
            const unsigned left = ring + place * SLOT + (K ? TILE_BYTES : 0);
            RowMajor at = by_row;
            asm volatile("" : "+v"(at.row_at));          // (eight addresses made once and kept would not fit the registers)
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) rows[ks] = at.by_row(left, ks);
            head = reinterpret_cast<const PcWinStat *>(&s_ring[place][2 * TILE_BYTES])->head;
        };
        if constexpr (K) {                               // (the values were asked for in front of the first unit)
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) op[ks] = values.get((unsigned)(uintptr_t)&s_v[tile][0], ks);
        }
        fetch(0);
        // Step i: dv of unit i, dk of unit i - 1; unit i + 1 is there, and the left operand of the wave's next unit is read while the
        // present one's second product runs (between two barriers all waves would else read first and multiply then).
        auto step = [&](int i) __attribute__((always_inline)) {
            if (i + AHEAD <= U) landed(std::integral_constant<int, AHEAD - 2>());
            else wait_vm<0>();
            if constexpr (!K) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");        // (the last unit's probabilities are written)
            ring_barrier();
            if (i + AHEAD < U) request();
        };
        if constexpr (K) step(0);
        int mine = 0, j = 0;                             // the unit's place in the ring, its head within the group
        uint32_t seen = 0;                               // of the unit's block, where some row does not see some key: bit: register
        bool have = false;
#pragma unroll 1
        for (int i = 0; i < U; ++i) {
            step(K ? i + 1 : i);
            const int lo_min = uniform(head.x), lo_max = uniform(head.y), lim_first = uniform(head.z), lim_last = uniform(head.w);
            // something of the tile is seen by the unit; some row of it does not see all
            const bool some = active && !(app.self && lim_last < pos0) && !(sink == 0 && lo_min > pos0 && (unsigned)lo_min - (unsigned)pos0 > PC_TILE - 1u);
            const unsigned other = ring + mine * SLOT + (K ? 0 : TILE_BYTES);
            const PcWinStat *stat = reinterpret_cast<const PcWinStat *>(&s_ring[mine][2 * TILE_BYTES]);
            mine = mine == RING - 1 ? 0 : mine + 1;
            bf16x8 cols[8], x[2];
            if (some) {
                const bool edge = valid < PC_TILE || (app.self && lim_first - pos0 < PC_TILE - 1) || lo_max == INT32_MAX || (lo_max > pos0 && sink < PC_TILE);
                float4 *const probs = &s_p[i & 1][tile][0][lane];
                f32x16 s;                                // scores or dp
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = 0.f;
                RowMajor at = by_col;
                asm volatile("" : "+v"(at.col_at[0]), "+v"(at.col_at[1]));
#pragma unroll
                for (int f = 0; f < 8; ++f) cols[f] = at.by_col(other, f >> 2, f & 3);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int ks = 0; ks < 8; ++ks) s = MFMA32(rows[ks], op[ks], s);
                __builtin_amdgcn_sched_barrier(0);
                // register r: row 16 (r / 8) + 8 hh + r % 8, column: the lane's key
                const float4 *const st = reinterpret_cast<const float4 *>(K ? stat->delta : stat->lse2) + 2 * hh;
#pragma unroll
                for (int q4 = 0; q4 < 4; ++q4) {
                    const float4 l = st[4 * (q4 >> 1) + (q4 & 1)];
                    if constexpr (K) {
                        const float4 p = probs[64 * q4];
                        s[4 * q4] = p.x * (s[4 * q4] - l.x); s[4 * q4 + 1] = p.y * (s[4 * q4 + 1] - l.y);
                        s[4 * q4 + 2] = p.z * (s[4 * q4 + 2] - l.z); s[4 * q4 + 3] = p.w * (s[4 * q4 + 3] - l.w);
                    } else {
                        s[4 * q4] = ex2(s[4 * q4] - l.x); s[4 * q4 + 1] = ex2(s[4 * q4 + 1] - l.y); s[4 * q4 + 2] = ex2(s[4 * q4 + 2] - l.z); s[4 * q4 + 3] = ex2(s[4 * q4 + 3] - l.w);
                        probs[64 * q4] = make_float4(s[4 * q4], s[4 * q4 + 1], s[4 * q4 + 2], s[4 * q4 + 3]);
                    }
                }
                if (__builtin_expect(edge, 0)) {
                    const int at_lane = lane_again(), n = at_lane & 31, hh = at_lane >> 5;
                    if (!have) {                         // (the heads of a group see the same)
                        const int pos = pos0 + min(n, valid - 1), from = n < sink ? INT32_MAX : pos, upto = app.self ? pos : INT32_MIN;
                        seen = 0;
#pragma unroll
                        for (int q4 = 0; q4 < 4; ++q4) {
                            const int at = 4 * (q4 >> 1) + (q4 & 1) + 2 * hh;
                            const int4 lo = reinterpret_cast<const int4 *>(stat->lo)[at], lim = reinterpret_cast<const int4 *>(stat->lim)[at];
                            seen |= (uint32_t)((lo.x <= from) & (lim.x >= upto)) << (4 * q4) | (uint32_t)((lo.y <= from) & (lim.y >= upto)) << (4 * q4 + 1) |
                                    (uint32_t)((lo.z <= from) & (lim.z >= upto)) << (4 * q4 + 2) | (uint32_t)((lo.w <= from) & (lim.w >= upto)) << (4 * q4 + 3);
                        }
                        if (n >= valid) seen = 0;
                        have = true;
                    }
                    // (what is masked need not be finite: its bits are taken away)
                    const uint32_t live = (uint32_t)stat->live >> (8 * hh), both = seen & ((live & 0xFFu) | (live >> 8 & 0xFF00u));
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[r] = __uint_as_float(__float_as_uint(s[r]) & (uint32_t)((int32_t)(both << (31 - r)) >> 31));
                }
                uint32_t pk[8];
#pragma unroll
                for (int r = 0; r < 8; ++r) pk[r] = pack_bf16(s[2 * r], s[2 * r + 1]);
                x[0] = frag4(pk[0], pk[1], pk[2], pk[3]); x[1] = frag4(pk[4], pk[5], pk[6], pk[7]);
            }
            if (i + 1 < U) fetch(mine);
            if (some) {
#pragma unroll
                for (int f = 0; f < 8; ++f) acc[f & 3] = MFMA32(cols[f], x[f >> 2], acc[f & 3]);
            }
            if (++j == g) { j = 0; have = false; }
        }
        if constexpr (!K) step(U);
    }
    };
    if (is_k) collect(std::true_type());
    else collect(std::false_type());
    ring_barrier();                                      // (dk is a unit behind: the ring is free only now)
    if (my_keys <= 0) continue;
    if (is_k && cur >= 0) {                              // back by the run's rotation (keys as they are stored)
        const float2 *rr = W.rot_run + (int64_t)cur * (PC_D / 2);
#pragma unroll
        for (int db = 0; db < 2; ++db)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {
                const int at = 32 * db + 8 * q4 + 4 * hh;
                const float4 a0 = *reinterpret_cast<const float4 *>(rr + at), a1 = *reinterpret_cast<const float4 *>(rr + at + 2);
                const float c[4] = {a0.x, a0.z, a1.x, a1.z}, s[4] = {a0.y, a0.w, a1.y, a1.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float x = acc[db][4 * q4 + j] * B.key_scale, y = acc[db + 2][4 * q4 + j] * B.key_scale;
                    acc[db][4 * q4 + j] = x * c[j] + y * s[j];
                    acc[db + 2][4 * q4 + j] = y * c[j] - x * s[j];
                }
            }
    }
    // out as whole lines, in two halves of a row, over the ring
    unsigned char *stg = &s_ring[0][0] + wave * TILE_BYTES;
    const int at_lane = lane_again(), n = at_lane & 31, hh = at_lane >> 5, r4 = at_lane >> 4, c = at_lane & 15;
    const bool whole = item.part < 0;
    float *to = whole ? (is_k ? B.d_k : B.d_v) + (((int64_t)item.slot0 + PC_TILE * tile) * W.n_kv_heads + kh) * PC_D + 4 * c
                      : B.key_part + ((((int64_t)item.part * W.n_kv_heads + kh) * 2 + (is_k ? 0 : 1)) * (PC_WIN_KEY_TILES * PC_TILE) + PC_TILE * tile) * PC_D + 4 * c;
    const int64_t stride = whole ? (int64_t)W.n_kv_heads * PC_D : PC_D;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        asm volatile("" ::: "memory");
#pragma unroll
        for (int db = 0; db < 2; ++db)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {
                const f32x16 &a = acc[2 * half + db];
                *reinterpret_cast<float4 *>(stg + n * 256 + (((8 * db + 2 * q4 + hh) ^ (n & 15)) << 4)) = make_float4(a[4 * q4], a[4 * q4 + 1], a[4 * q4 + 2], a[4 * q4 + 3]);
            }
        asm volatile("" ::: "memory");
        float4 was[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) was[i] = whole && 4 * i + r4 < my_keys ? *reinterpret_cast<const float4 *>(to + (4 * i + r4) * stride + 64 * half) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = 4 * i + r4;
            float4 v = *reinterpret_cast<const float4 *>(stg + r * 256 + ((c ^ (r & 15)) << 4));
            v.x += was[i].x; v.y += was[i].y; v.z += was[i].z; v.w += was[i].w;
            if (r < my_keys) *reinterpret_cast<float4 *>(to + r * stride + 64 * half) = v;
        }
    }
    wait_vm<0>();                                        // (what is counted from here on are the next item's loads alone)
    }
}

void pc_launch_win_bwd_keys_bf16(const PcWin &W, const PcWinBwd &B, hipStream_t st)
{
    if (B.n_bins > 0) pc_win_bwd_keys_bf16_kernel<<<(unsigned)B.n_bins * W.n_kv_heads, 512, 0, st>>>(W, B);
}

// The parts of tiles that several items collect, added up in their order and to what is there: a thread four numbers, eight parts a
// round of loads.
template <int D>
__global__ __launch_bounds__(256) void pc_win_bwd_sums_kernel(PcWinBwd B, int H)
{
    const PcWinSum sm = B.sums[blockIdx.x];
    const int kh = blockIdx.y, which = blockIdx.z % 2;   // keys, values
    constexpr int KEYS = PC_WIN_KEY_TILES * PC_TILE;
    const int i = (int)(blockIdx.z / 2) * 256 + threadIdx.x, key = i / (D / 4), d4 = i % (D / 4);
    if (key >= sm.n_keys) return;
    float4 *p = reinterpret_cast<float4 *>((which ? B.d_v : B.d_k) + (((int64_t)sm.slot0 + key) * H + kh) * D) + d4, v = *p;
    const float4 *part = reinterpret_cast<const float4 *>(B.key_part + ((((int64_t)sm.part0 * H + kh) * 2 + which) * KEYS + key) * D) + d4;
    const int64_t step = (int64_t)H * 2 * KEYS * D / 4;
    for (int s0 = 0; s0 < sm.n_parts; s0 += 8) {
        float4 x[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) x[u] = s0 + u < sm.n_parts ? part[(s0 + u) * step] : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int u = 0; u < 8; ++u) { v.x += x[u].x; v.y += x[u].y; v.z += x[u].z; v.w += x[u].w; }
    }
    *p = v;
}

void pc_launch_win_bwd_sums(const PcWin &W, const PcWinBwd &B, int D, hipStream_t st)
{
    if (B.n_sums <= 0) return;
    const dim3 grid((unsigned)B.n_sums, (unsigned)W.n_kv_heads, (unsigned)(2 * PC_WIN_KEY_TILES * PC_TILE * D / 4 / 256));
    if (D == 64) pc_win_bwd_sums_kernel<64><<<grid, 256, 0, st>>>(B, W.n_kv_heads);
    else pc_win_bwd_sums_kernel<128><<<grid, 256, 0, st>>>(B, W.n_kv_heads);
}
