// Gradient of the windowed attention, fp32 caches (gfx950), on the fp32 matrix instruction; the formulas and what is
// computed where: pc_kernels_window_bwd.hip.  Columns are (row, head) pairs of a KV head, 32 a unit, as in the forward; the
// order of a summed index is free, so that a lane half holds half of the rotation's pairs (scores), half of the dims
// (dp), and results are operands of the next product as they are.
#include "pc_window.h"
#include "pc_pieces.h"

#define MFMA_F32(a, b, c) __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0)

namespace {

__device__ __forceinline__ float ex2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ void in_order() { asm volatile("" ::: "memory"); }       // a wave's own LDS accesses are
__device__ __forceinline__ bool finite(float x) { return __builtin_fabsf(x) < INFINITY; }
template <int W> struct Vec;
template <> struct Vec<2> { using type = f32x2; };
template <> struct Vec<4> { using type = f32x4; };
__device__ __forceinline__ f32x16 zeros()
{
    f32x16 z;
#pragma unroll
    for (int r = 0; r < 16; ++r) z[r] = 0.f;
    return z;
}
// four floats of chunk c of a row of a RowTile
template <int D> __device__ __forceinline__ f32x4 chunk(unsigned lds, int row, int c) { return from_lds<f32x4>(lds + row * (D * 4) + ((c ^ (row % (D / 4))) << 4)); }
// floats VW m .. VW m + VW - 1 of a row of a RowTile
template <int D> __device__ __forceinline__ typename Vec<D / 32>::type part(unsigned lds, int row, int m)
{
    using VV = typename Vec<D / 32>::type;
    const int at = D / 32 * m;
    return from_lds<VV>(lds + row * (D * 4) + (((at / 4) ^ (row % (D / 4))) << 4) + (at % 4) * 4);
}
// accumulators whose element (i, r) is dim VW (8 (r / 4) + 4 hh + r % 4) + i of the lane's column: turned by the angles of a less those of b
template <int D> __device__ __forceinline__ void turn_columns(f32x16 (&acc)[D / 32], const float2 *a, const float2 *b, int hh)
{
    constexpr int VW = D / 32;
#pragma unroll
    for (int r = 0; r < 8; ++r)
#pragma unroll
        for (int i = 0; i < VW; ++i) {
            const int f = VW * (8 * (r >> 2) + 4 * hh + (r & 3)) + i;
            const float2 u = a[f], v = b ? b[f] : make_float2(1.f, 0.f);
            const float c = u.x * v.x + u.y * v.y, s = u.y * v.x - u.x * v.y, x = acc[i][r], y = acc[i][r + 8];
            acc[i][r] = x * c - y * s;
            acc[i][r + 8] = x * s + y * c;
        }
}

}  // namespace

// dq: 4 waves over the same 32 columns, each with a share of the item's tiles, whose sums meet in LDS.
template <int D>
__global__ __launch_bounds__(256, 1) void pc_win_bwd_dq_f32_kernel(PcWin W, PcWinBwd B)
{
    constexpr int HALF = D / 2, P = D / 4, VW = D / 32, PITCH = D + 4, NW = 4;
    constexpr int MEM = NW * 32 * PITCH * 4 > NW * 2 * RowTile<D>::BYTES ? NW * 32 * PITCH * 4 : NW * 2 * RowTile<D>::BYTES;
    __shared__ __attribute__((aligned(1024))) unsigned char s_mem[MEM];     // the waves' tiles of keys and values, then their sums
    __shared__ __attribute__((aligned(16))) float2 s_rot[NW][HALF];
    float (*const s_acc)[32 * PITCH] = reinterpret_cast<float (*)[32 * PITCH]>(s_mem);

    const int kh = blockIdx.x % W.n_kv_heads;
    const PcWinItem item = W.items[blockIdx.x / W.n_kv_heads];
    const int g = W.n_q_heads / W.n_kv_heads;
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const int n = lane & 31, hh = lane >> 5;
    const int64_t col0 = (int64_t)item.unit0 * 32, n_cols = (int64_t)item.n_q * g;
    const bool col_ok = col0 + n < n_cols;
    const int64_t col = col_ok ? col0 + n : n_cols - 1;
    const int row = (int)(col / g), h = kh * g + (int)(col % g);
    const int64_t R = (int64_t)item.q_off + row, at = R * W.n_q_heads + h;
    const float lse = B.lse[at];
    const bool live = col_ok && lse > -INFINITY;
    const float lse2 = live ? lse * 1.4426950408889634f : INFINITY, delta = live ? B.delta[at] : 0.f;
    const int lo = win_low(W.q_pos[R], W.window), lim = item.lim0 + row;
    float qx[P], qy[P], go[HALF];                        // the column's query, turned (pairs P hh + i), and output gradients (dims HALF hh + i)
    {
        const float *q = (const float *)W.q + at * D + P * hh, *d = (const float *)B.d_out + at * D + HALF * hh;
        const float2 *rot = W.rot_q + R * HALF + P * hh;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const float x = q[i], y = q[i + HALF];
            const float2 cs = rot[i];
            qx[i] = live ? x * cs.x - y * cs.y : 0.f;
            qy[i] = live ? x * cs.y + y * cs.x : 0.f;
        }
#pragma unroll
        for (int i = 0; i < HALF; ++i) go[i] = live ? d[i] : 0.f;
    }
    const int share = item.n_tiles / NW, more = item.n_tiles % NW;
    const int n_tiles = share + (wave < more), skip = item.skip + wave * share + min(wave, more);
    f32x16 acc[VW];
#pragma unroll
    for (int i = 0; i < VW; ++i) acc[i] = zeros();
    using VV = typename Vec<VW>::type;
    const float *kb = (const float *)W.k_store + (int64_t)kh * W.slots * D, *vb = (const float *)W.v_store + (int64_t)kh * W.slots * D;
    int cur = -1;
    if (n_tiles > 0) {
        unsigned char *const mine = s_mem + wave * 2 * RowTile<D>::BYTES;
        const RowTile<D> keys(mine, lane), values(mine + RowTile<D>::BYTES, lane);
        WinWalk walk(W.runs + item.run0, skip, n_tiles);
        WinTile d = walk.tile();
        keys.request(kb + (int64_t)d.slot0 * D);
#pragma unroll 1
        for (int t = 0; t < n_tiles; ++t) {
            const WinTile e = d;
            values.request(vb + (int64_t)e.slot0 * D);
            if (e.rot != cur) {
                const float2 *to = W.rot_run + (int64_t)e.rot * HALF;
                if (cur >= 0) turn_columns<D>(acc, W.rot_run + (int64_t)cur * HALF, to, hh);       // (collected in the keys' frame)
                cur = e.rot;
                for (int i = lane; i < HALF; i += 64) s_rot[wave][i] = to[i];
                in_order();
            }
            wait_vm0();
            f32x16 s = zeros(), dp = zeros();
            float odd = 0.f;
#pragma unroll
            for (int i = 0; i < P; i += 4) {
                const f32x4 kx = chunk<D>(keys.lds, n, (P * hh + i) / 4), ky = chunk<D>(keys.lds, n, (P * hh + i + HALF) / 4);
                const float4 c0 = *reinterpret_cast<const float4 *>(&s_rot[wave][P * hh + i]), c1 = *reinterpret_cast<const float4 *>(&s_rot[wave][P * hh + i + 2]);
                const float cs[4] = {c0.x, c0.z, c1.x, c1.z}, sn[4] = {c0.y, c0.w, c1.y, c1.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    s = MFMA_F32(kx[j] * cs[j] - ky[j] * sn[j], qx[i + j], s);
                    dp = MFMA_F32(kx[j] * sn[j] + ky[j] * cs[j], qy[i + j], dp);
                    odd += (kx[j] + ky[j]) * 0.f;
                }
            }
            s += dp;                                     // (two chains round less than one)
            dp = zeros();
#pragma unroll
            for (int i = 0; i < HALF; i += 4) {
                const f32x4 x = chunk<D>(values.lds, n, (HALF * hh + i) / 4);
#pragma unroll
                for (int j = 0; j < 4; ++j) dp = MFMA_F32(x[j], go[i + j], dp);
            }
            const uint32_t sees = live ? win_sees(e.pos0, e.valid, e.sink, e.self != 0, lo, lim) : 0u;
            const int bits = (int)(sees >> (4 * hh));
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float x = ex2(__builtin_fmaf(s[r], W.scale_log2, -lse2)) * (dp[r] - delta);
                s[r] = (bits >> (8 * (r >> 2) + (r & 3))) & 1 ? x : 0.f;
            }
            const bool some = __builtin_amdgcn_ballot_w64(odd != 0.f) != 0;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                VV k = part<D>(keys.lds, 8 * (r >> 2) + 4 * hh + (r & 3), n);
                if (some) {                              // (a key that is not finite: the columns that see it have no gradient)
#pragma unroll
                    for (int i = 0; i < VW; ++i) k[i] = finite(k[i]) ? k[i] : 0.f;
                }
#pragma unroll
                for (int i = 0; i < VW; ++i) acc[i] = MFMA_F32(k[i], s[r], acc[i]);
            }
            if (t + 1 < n_tiles) {
                walk.next();
                d = walk.tile();
                __builtin_amdgcn_s_waitcnt(0xC07F);      // lgkmcnt(0): nothing of the tile's place is still to be read
                keys.request(kb + (int64_t)d.slot0 * D);
            }
            __builtin_amdgcn_s_waitcnt(0xC07F);          // (nor of the values')
        }
        turn_columns<D>(acc, W.rot_run + (int64_t)cur * HALF, nullptr, hh);
    }
    __syncthreads();                                     // (nobody reads a tile any more)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        VV z;
#pragma unroll
        for (int i = 0; i < VW; ++i) z[i] = acc[i][r];
        *reinterpret_cast<VV *>(&s_acc[wave][n * PITCH + VW * (8 * (r >> 2) + 4 * hh + (r & 3))]) = z;
    }
    __syncthreads();
    for (int e = threadIdx.x; e < 32 * HALF; e += 256) {
        const int cn = e / HALF, f = e % HALF;
        const int64_t cc = col0 + cn;
        if (cc >= n_cols) continue;
        const int hc = kh * g + (int)(cc % g), rc = (int)(cc / g);
        float x = 0.f, y = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) { x += s_acc[w][cn * PITCH + f]; y += s_acc[w][cn * PITCH + f + HALF]; }
        const float2 cs = W.rot_q[((int64_t)item.q_off + rc) * HALF + f];
        float *to = item.part < 0 ? B.d_q + (((int64_t)item.q_off + rc) * W.n_q_heads + hc) * D : W.part_o + (((int64_t)item.part + rc) * W.n_q_heads + hc) * D;
        to[f] = (x * cs.x + y * cs.y) * B.scale;
        to[f + HALF] = (y * cs.x - x * cs.y) * B.scale;
    }
}

void pc_launch_win_bwd_dq_f32(const PcWin &W, const PcWinBwd &B, int n_items, int D, hipStream_t st)
{
    if (n_items <= 0) return;
    const unsigned grid = (unsigned)n_items * W.n_kv_heads;
    if (D == 64) pc_win_bwd_dq_f32_kernel<64><<<grid, 256, 0, st>>>(W, B);
    else pc_win_bwd_dq_f32_kernel<128><<<grid, 256, 0, st>>>(W, B);
}

// dk and dv: a tile of keys a wave, four a workgroup, which share the units' turned queries and output gradients (two at a time in LDS).
template <int D>
__global__ __launch_bounds__(256, 1) void pc_win_bwd_keys_f32_kernel(PcWin W, PcWinBwd B)
{
    constexpr int HALF = D / 2, P = D / 4, VW = D / 32, SLOT = 2 * RowTile<D>::BYTES + PC_WIN_STAT_BYTES;
    __shared__ __attribute__((aligned(1024))) unsigned char s_ring[2][SLOT];
    const int kh = blockIdx.x % W.n_kv_heads;
    const int bin = blockIdx.x / W.n_kv_heads, item_end = B.bins[bin + 1];
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const int n = lane & 31, hh = lane >> 5;
#pragma unroll 1
    for (int i_item = B.bins[bin]; i_item < item_end; ++i_item) {
    const PcWinKeyItem item = B.key_items[i_item];
    const int my_keys = item.n_keys - PC_TILE * wave;
    f32x16 dk[VW], dv[VW];
#pragma unroll
    for (int i = 0; i < VW; ++i) dk[i] = dv[i] = zeros();
    using VV = typename Vec<VW>::type;
    int cur = -1;
    for (int a = 0; a < item.n_apps; ++a) {
        const PcWinApp app = B.apps[item.app0 + a];
        const int pos0 = app.pos0 + PC_TILE * wave, valid = min(app.n_tok - PC_TILE * wave, PC_TILE), sink = min(max(app.sink - PC_TILE * wave, 0), PC_TILE);
        const bool active = valid > 0;
        auto request = [&](int i, int slot) __attribute__((always_inline)) {       // a wave an operand
            const int64_t u = (int64_t)(app.block0 + i) * W.n_kv_heads + kh;
            unsigned char *to = &s_ring[slot][0];
            if (wave == 0) RowTile<D>(to, lane).request((const float *)B.q_abs + u * 32 * D);
            if (wave == 1) RowTile<D>(to + RowTile<D>::BYTES, lane).request((const float *)B.d_o + u * 32 * D);
            if (wave == 2) dma16(B.stat + u * PC_WIN_STAT_BYTES, lane * 16, (unsigned)(uintptr_t)(to + 2 * RowTile<D>::BYTES));
        };
        __syncthreads();                                 // (the last call's units are no longer read)
        if (app.n_blocks > 0) request(0, 0);
        float kx[P], ky[P], v[HALF];                     // the lane's key, turned (pairs P hh + i), and its value (dims HALF hh + i)
#pragma unroll
        for (int i = 0; i < P; ++i) kx[i] = ky[i] = 0.f;
#pragma unroll
        for (int i = 0; i < HALF; ++i) v[i] = 0.f;
        if (active) {
            const int64_t slot = (int64_t)kh * W.slots + item.slot0 + PC_TILE * wave + n;
            const float *k = (const float *)W.k_store + slot * D + P * hh, *vp = (const float *)W.v_store + slot * D + HALF * hh;
            const float2 *rot = W.rot_run + (int64_t)app.rot * HALF;
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const float2 cs = rot[P * hh + i];
                const float x = k[i], y = k[i + HALF];
                kx[i] = x * cs.x - y * cs.y;
                ky[i] = x * cs.y + y * cs.x;
            }
#pragma unroll
            for (int i = 0; i < HALF; ++i) v[i] = vp[i];
            if (cur >= 0 && cur != app.rot) turn_columns<D>(dk, rot, W.rot_run + (int64_t)cur * HALF, hh);      // (kept in the frame of the queries)
            cur = app.rot;
        }
#pragma unroll 1
        for (int i = 0; i < app.n_blocks; ++i) {
            wait_vm0();
            __syncthreads();
            if (i + 1 < app.n_blocks) request(i + 1, (i + 1) & 1);
            const unsigned qt = (unsigned)(uintptr_t)&s_ring[i & 1][0], gt = qt + RowTile<D>::BYTES;
            const PcWinStat *stat = reinterpret_cast<const PcWinStat *>(&s_ring[i & 1][2 * RowTile<D>::BYTES]);
            const int4 hd = stat->head;
            const int lo_min = uniform(hd.x), lo_max = uniform(hd.y), lim_first = uniform(hd.z), lim_last = uniform(hd.w);
            if (!active || (app.self && lim_last < pos0) || (sink == 0 && lo_min > pos0 && (unsigned)lo_min - (unsigned)pos0 > PC_TILE - 1u)) continue;
            f32x16 s = zeros(), dp = zeros();
#pragma unroll
            for (int j = 0; j < P; j += 4) {
                const f32x4 x = chunk<D>(qt, n, (P * hh + j) / 4), y = chunk<D>(qt, n, (P * hh + j + HALF) / 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s = MFMA_F32(x[e], kx[j + e], s);
                    dp = MFMA_F32(y[e], ky[j + e], dp);
                }
            }
            s += dp;
            dp = zeros();
#pragma unroll
            for (int j = 0; j < HALF; j += 4) {
                const f32x4 x = chunk<D>(gt, n, (HALF * hh + j) / 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) dp = MFMA_F32(x[e], v[j + e], dp);
            }
            // register r: column 8 (r / 4) + 4 hh + r % 4 of the unit; the lane's key
            auto col_of = [&](int r) { return 8 * (r >> 2) + 4 * hh + (r & 3); };
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const float4 l = *reinterpret_cast<const float4 *>(&stat->lse2[col_of(r)]), d = *reinterpret_cast<const float4 *>(&stat->delta[col_of(r)]);
                const float lse2[4] = {l.x, l.y, l.z, l.w}, delta[4] = {d.x, d.y, d.z, d.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[r + e] = ex2(__builtin_fmaf(s[r + e], W.scale_log2, -lse2[e]));
                    dp[r + e] = s[r + e] * (dp[r + e] - delta[e]);
                }
            }
            if (valid < PC_TILE || (app.self && lim_first - pos0 < PC_TILE - 1) || lo_max == INT32_MAX || (lo_max > pos0 && sink < PC_TILE)) {
                const int pos = pos0 + min(n, valid - 1);
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int c = col_of(r);
                    const bool see = (n < valid) & (stat->lse2[c] < INFINITY) & ((pos >= stat->lo[c]) | (n < sink)) & (!app.self | (pos <= stat->lim[c]));
                    s[r] = see ? s[r] : 0.f;
                    dp[r] = see ? dp[r] : 0.f;
                }
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int rw = 8 * (r >> 2) + 4 * hh + (r & 3);
                const VV q = part<D>(qt, rw, n), d = part<D>(gt, rw, n);
#pragma unroll
                for (int j = 0; j < VW; ++j) {
                    dv[j] = MFMA_F32(d[j], s[r], dv[j]);
                    dk[j] = MFMA_F32(q[j], dp[r], dk[j]);
                }
            }
        }
    }
    if (my_keys <= 0) continue;
    if (cur >= 0) {                                      // back by the run's rotation (keys as they are stored): less its angles
        const float2 *rot = W.rot_run + (int64_t)cur * HALF;
#pragma unroll
        for (int r = 0; r < 8; ++r)
#pragma unroll
            for (int i = 0; i < VW; ++i) {
                const float2 u = rot[VW * (8 * (r >> 2) + 4 * hh + (r & 3)) + i];
                const float x = dk[i][r] * B.scale, y = dk[i][r + 8] * B.scale;
                dk[i][r] = x * u.x + y * u.y;
                dk[i][r + 8] = y * u.x - x * u.y;
            }
    }
    const bool whole = item.part < 0;
    if (whole && n >= my_keys) continue;
    const int64_t in_part = (int64_t)PC_TILE * wave + n;
    float *to_k, *to_v;
    if (whole) {
        const int64_t at = (((int64_t)item.slot0 + in_part) * W.n_kv_heads + kh) * D;
        to_k = B.d_k + at; to_v = B.d_v + at;
    } else {
        to_k = B.key_part + ((((int64_t)item.part * W.n_kv_heads + kh) * 2) * (PC_WIN_KEY_TILES * PC_TILE) + in_part) * D;
        to_v = to_k + (int64_t)PC_WIN_KEY_TILES * PC_TILE * D;
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int m = VW * (8 * (r >> 2) + 4 * hh + (r & 3));
        VV x, y;
#pragma unroll
        for (int i = 0; i < VW; ++i) { x[i] = dk[i][r]; y[i] = dv[i][r]; }
        VV *pk = reinterpret_cast<VV *>(to_k + m), *pv = reinterpret_cast<VV *>(to_v + m);
        if (whole) { x += *pk; y += *pv; }
        *pk = x; *pv = y;
    }
    }
}

void pc_launch_win_bwd_keys_f32(const PcWin &W, const PcWinBwd &B, int D, hipStream_t st)
{
    if (B.n_bins <= 0) return;
    const unsigned grid = (unsigned)B.n_bins * W.n_kv_heads;
    if (D == 64) pc_win_bwd_keys_f32_kernel<64><<<grid, 256, 0, st>>>(W, B);
    else pc_win_bwd_keys_f32_kernel<128><<<grid, 256, 0, st>>>(W, B);
}
