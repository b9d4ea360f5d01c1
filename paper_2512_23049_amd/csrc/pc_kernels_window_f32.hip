// Attention with a sliding window and sinks, fp32 caches (gfx950), on the fp32 matrix instruction.
//
// S^T = K . Q^T and O^T = V^T . P^T with 32 keys and 32 columns, a column being a (query row, head) pair of one KV head:
// v_mfma_f32_32x32x2_f32 takes one number a lane of each operand, lane (n, hh) those of summed index hh.  The order of a
// summed index is free as long as both operands agree, so lane half hh holds half of the rotation's pairs (of its key, of its
// column), and register r of the scores, key 8 (r / 4) + 4 hh + r % 4, is the right operand of a step of the second product as it is.
// Keys are turned by (start - stored base), queries by their positions.  Every rounding is fp32's.
#include "pc_window.h"
#include "pc_pieces.h"

#define MFMA_F32(a, b, c) __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0)

namespace {

__device__ __forceinline__ float ex2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float other_half(float x) { return __shfl_xor(x, 32); }
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ void in_order() { asm volatile("" ::: "memory"); }       // a wave's own LDS accesses are
__device__ __forceinline__ bool finite(float x) { return __builtin_fabsf(x) < INFINITY; }
template <int W> struct Vec;                                                // W consecutive floats of a row
template <> struct Vec<2> { using type = f32x2; };
template <> struct Vec<4> { using type = f32x4; };

}  // namespace

// A workgroup is 4 waves over the same 32 columns, each with a contiguous share of the item's tiles; their results meet in LDS.
template <int D>
__global__ __launch_bounds__(256, 2) void pc_win_attend_f32_kernel(PcWin W)
{
    constexpr int HALF = D / 2, P = D / 4, VW = D / 32, PITCH = D + 4, NW = 4;
    constexpr int MEM = NW * 32 * PITCH * 4 > NW * RowTile<D>::BYTES ? NW * 32 * PITCH * 4 : NW * RowTile<D>::BYTES;
    __shared__ __attribute__((aligned(1024))) unsigned char s_mem[MEM];     // the waves' tiles of keys, then their results
    __shared__ __attribute__((aligned(16))) float2 s_rot[NW][HALF];
    __shared__ float s_m[NW][32], s_l[NW][32];
    float (*const s_acc)[32 * PITCH] = reinterpret_cast<float (*)[32 * PITCH]>(s_mem);

    const int kh = blockIdx.x % W.n_kv_heads;          // consecutive workgroups (one per XCD) take different KV heads
    const PcWinItem item = W.items[blockIdx.x / W.n_kv_heads];
    const int g = W.n_q_heads / W.n_kv_heads;
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const int n = lane & 31, hh = lane >> 5;
    const int64_t col0 = (int64_t)item.unit0 * 32, n_cols = (int64_t)item.n_q * g;
    const bool col_ok = col0 + n < n_cols;
    const int64_t col = col_ok ? col0 + n : n_cols - 1;
    const int row = (int)(col / g), h = kh * g + (int)(col % g);
    const int64_t R = (int64_t)item.q_off + row;
    const int lo = win_low(W.q_pos[R], W.window), lim = item.lim0 + row;
    int lo_max = lo;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) lo_max = max(lo_max, __shfl_xor(lo_max, o));
    lo_max = uniform(lo_max);
    const int lim_first = item.lim0 + (int)(col0 / g);

    float qx[P], qy[P];                                  // dims P hh + i of the column's query, turned, and their partners
    {
        const float *q = (const float *)W.q + (R * W.n_q_heads + h) * D + P * hh;
        const float2 *rot = W.rot_q + R * HALF + P * hh;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const float x = q[i], y = q[i + HALF];
            const float2 cs = rot[i];
            qx[i] = col_ok ? x * cs.x - y * cs.y : 0.f;
            qy[i] = col_ok ? x * cs.y + y * cs.x : 0.f;
        }
    }
    const int share = item.n_tiles / NW, more = item.n_tiles % NW;
    const int n_tiles = share + (wave < more), skip = item.skip + wave * share + min(wave, more);
    float m_run = -INFINITY, l_run = 0.f;
    f32x16 acc[VW];
#pragma unroll
    for (int i = 0; i < VW; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][r] = 0.f;
    using VV = typename Vec<VW>::type;
    const float *kb = (const float *)W.k_store + (int64_t)kh * W.slots * D, *vb = (const float *)W.v_store + (int64_t)kh * W.slots * D;
    if (n_tiles > 0) {
        unsigned char *const mine = s_mem + wave * RowTile<D>::BYTES;
        const RowTile<D> keys(mine, lane);
        const unsigned row_at = keys.lds + n * (D * 4);
        WinWalk walk(W.runs + item.run0, skip, n_tiles);
        WinTile d = walk.tile();
        keys.request(kb + (int64_t)d.slot0 * D);
        int cur = -1;
#pragma unroll 1
        for (int t = 0; t < n_tiles; ++t) {
            const WinTile e = d;
            if (e.rot != cur) {
                cur = e.rot;
                for (int i = lane; i < HALF; i += 64) s_rot[wave][i] = W.rot_run[(int64_t)cur * HALF + i];
                in_order();
            }
            const float *vt = vb + (int64_t)e.slot0 * D;
            VV v[8];                                     // of register r, key 8 (r / 4) + 4 hh + r % 4: dims VW n + 0..VW-1; eight registers at a time
            auto load_v = [&](int part) __attribute__((always_inline)) {
#pragma unroll
                for (int r = 0; r < 8; ++r) v[r] = *reinterpret_cast<const VV *>(vt + (16 * part + 8 * (r >> 2) + 4 * hh + (r & 3)) * D + VW * n);
            };
            load_v(0);
            wait_vm0();
            f32x16 s, s1;                                // (two chains round less than one)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = s1[r] = 0.f;
#pragma unroll
            for (int i = 0; i < P; i += 4) {
                const int c = (P * hh + i) / 4;
                const f32x4 kx = from_lds<f32x4>(row_at + ((c ^ (n % RowTile<D>::CHUNKS)) << 4));
                const f32x4 ky = from_lds<f32x4>(row_at + (((c + HALF / 4) ^ (n % RowTile<D>::CHUNKS)) << 4));
                const float4 c0 = *reinterpret_cast<const float4 *>(&s_rot[wave][P * hh + i]), c1 = *reinterpret_cast<const float4 *>(&s_rot[wave][P * hh + i + 2]);
                const float cs[4] = {c0.x, c0.z, c1.x, c1.z}, sn[4] = {c0.y, c0.w, c1.y, c1.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    s = MFMA_F32(kx[j] * cs[j] - ky[j] * sn[j], qx[i + j], s);
                    s1 = MFMA_F32(kx[j] * sn[j] + ky[j] * cs[j], qy[i + j], s1);
                }
            }
            s += s1;
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] *= W.scale_log2;
            const bool edge = e.valid < PC_TILE || (e.self && lim_first - e.pos0 < PC_TILE - 1) || (lo_max > e.pos0 && e.sink < PC_TILE);
            uint32_t sees = ~0u;
            if (edge) {
                sees = win_sees(e.pos0, e.valid, e.sink, e.self != 0, lo, lim);
                const int bits = (int)(sees >> (4 * hh));
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = (bits >> (8 * (r >> 2) + (r & 3))) & 1 ? s[r] : -INFINITY;
            }
            float mx = s[0];
#pragma unroll
            for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[r]);
            mx = fmaxf(mx, other_half(mx));
            const float m_new = fmaxf(m_run, mx), m_safe = m_new == -INFINITY ? 0.f : m_new, alpha = ex2(m_run - m_safe);
            m_run = m_new;
            float ps = 0.f;
#pragma unroll
            for (int r = 0; r < 16; ++r) { s[r] = ex2(s[r] - m_safe); ps += s[r]; }
            l_run = l_run * alpha + ps;
            if (__builtin_amdgcn_ballot_w64(alpha != 1.f) != 0) {
#pragma unroll
                for (int i = 0; i < VW; ++i) acc[i] *= alpha;
            }
            const bool more_tiles = t + 1 < n_tiles;
            if (more_tiles) {
                walk.next();
                d = walk.tile();
            }
#pragma unroll
            for (int part = 0; part < 2; ++part) {
                if (part == 1) load_v(1);
                if (part == 1 && more_tiles) {           // (behind the values: they are not to wait for it)
                    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0): nothing of the tile's place is still to be read
                    keys.request(kb + (int64_t)d.slot0 * D);
                }
                if (edge) {
                    float odd = 0.f;                     // (see win_odd_sum)
#pragma unroll
                    for (int r = 0; r < 8; ++r)
#pragma unroll
                        for (int i = 0; i < VW; ++i) odd += v[r][i] * 0.f;
                    if (__builtin_amdgcn_ballot_w64(odd != 0.f) != 0) {
                        const int bits = (int)(sees >> (4 * hh + 16 * part));
#pragma unroll
                        for (int i = 0; i < VW; ++i) {
                            f32x16 z;
#pragma unroll
                            for (int r = 0; r < 16; ++r) z[r] = 0.f;
#pragma unroll
                            for (int r = 0; r < 8; ++r) {
                                const float x = v[r][i];
                                z = MFMA_F32(finite(x) ? 0.f : x != x ? PC_WIN_ODD_NAN : x < 0.f ? PC_WIN_ODD_NEG : PC_WIN_ODD_INF, (bits >> (8 * (r >> 2) + (r & 3))) & 1 ? (s[8 * part + r] == 0.f ? PC_WIN_ODD_NAN : 1.f) : 0.f, z);
                                v[r][i] = finite(x) ? x : 0.f;
                            }
#pragma unroll
                            for (int r = 0; r < 16; ++r) acc[i][r] += win_odd_sum(z[r]);
                            __builtin_amdgcn_sched_barrier(0);              // (one after the other: registers)
                        }
                    }
                }
#pragma unroll
                for (int r = 0; r < 8; ++r)
#pragma unroll
                    for (int i = 0; i < VW; ++i) acc[i] = MFMA_F32(v[r][i], s[8 * part + r], acc[i]);
            }
        }
    }
    l_run += other_half(l_run);
    if (hh == 0) { s_m[wave][n] = m_run; s_l[wave][n] = l_run; }
    __syncthreads();                                     // (nobody reads a tile any more)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        VV z;
#pragma unroll
        for (int i = 0; i < VW; ++i) z[i] = acc[i][r];
        *reinterpret_cast<VV *>(&s_acc[wave][n * PITCH + VW * (8 * (r >> 2) + 4 * hh + (r & 3))]) = z;
    }
    __syncthreads();
    for (int e = threadIdx.x; e < 32 * (D / 4); e += 256) {
        const int cn = e / (D / 4), dim = 4 * (e % (D / 4));
        const int64_t cc = col0 + cn;
        if (cc >= n_cols) continue;
        const int hc = kh * g + (int)(cc % g), rc = (int)(cc / g);
        float m = -INFINITY, l = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) m = fmaxf(m, s_m[w][cn]);
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            if (s_l[w][cn] == 0.f) continue;             // saw nothing (a sum that is not a number stays one)
            const float f = ex2(s_m[w][cn] - (m == -INFINITY ? 0.f : m));
            o += *reinterpret_cast<const f32x4 *>(&s_acc[w][cn * PITCH + dim]) * f;
            l += s_l[w][cn] * f;
        }
        if (item.part < 0) {
            const float inv = l == 0.f ? 0.f : 1.f / l;
            *reinterpret_cast<f32x4 *>((float *)W.out + (((int64_t)item.q_off + rc) * W.n_q_heads + hc) * D + dim) = o * inv;
            if (W.lse && dim == 0) W.lse[((int64_t)item.q_off + rc) * W.n_q_heads + hc] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
        } else {
            const int64_t at = ((int64_t)item.part + rc) * W.n_q_heads + hc;
            *reinterpret_cast<f32x4 *>(W.part_o + at * D + dim) = o;
            if (dim == 0) *reinterpret_cast<float2 *>(W.part_ml + at * 2) = make_float2(l == 0.f ? -INFINITY : m, l);
        }
    }
}

void pc_launch_win_attend_f32(const PcWin &W, int n_items, int D, hipStream_t st)
{
    if (n_items <= 0) return;
    const unsigned grid = (unsigned)n_items * W.n_kv_heads;
    if (D == 64) pc_win_attend_f32_kernel<64><<<grid, 256, 0, st>>>(W);
    else pc_win_attend_f32_kernel<128><<<grid, 256, 0, st>>>(W);
}
