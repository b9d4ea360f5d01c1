// The cache's own copies (gfx950): forks of messages, and the cache closing up.
#include "pc_copies.h"
#include "pc_mx4.h"
#include "pc_mfma_common.h"

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// the slot of a fork's token, whose pieces are in token order
__device__ __forceinline__ int fork_slot(const PcForkPiece *pieces, int n, int token)
{
    int i = 0;
    while (i + 1 < n && token >= pieces[i + 1].first) ++i;
    return pieces[i].slot + (token - pieces[i].first);
}

}  // namespace

// -------------------------------------------------------------------------------------------------------------- fork
// A workgroup copies four tiles of one fork and KV head.  Keys, stored turned to base + token, are turned by one angle a
// frequency (whose 64 or 32 rotations the workgroup makes once); values of a bf16 cache lie in groups of eight tokens by
// dimension, so that eight tokens from the middle of a group are two 16-byte reads and a shift.  Bound: memory; 16-byte
// accesses of consecutive lanes, all loads of a tile in front of its first store: 32 forks of 950 tokens, 8 KV heads, 250 MB
// read and written in 62 us (4.0 TB/s; a large copy 4.95); one fork of 200 tokens 5.4 us.
#define FORK_TILES 4

template <bool TURN>
__device__ __forceinline__ void fork_keys_bf16(const PcForkItem &it, const PcForkPiece *pieces, int tile0, int tile1, const uint16_t *src, uint16_t *dst, const float2 *rot)
{
    const int r = threadIdx.x >> 3, c = threadIdx.x & 7;             // a row, 8 dims and their partners
    uint4 lo[FORK_TILES], hi[FORK_TILES];
#pragma unroll
    for (int t = 0; t < FORK_TILES; ++t) {
        const int token = (tile0 + t) * PC_TILE + r;
        lo[t] = hi[t] = make_uint4(0, 0, 0, 0);
        if (token < it.len) {                            // (tiles behind the last hold no tokens)
            const uint16_t *p = src + (int64_t)fork_slot(pieces, it.n_pieces, token) * PC_D + 8 * c;
            lo[t] = ldg16(p); hi[t] = ldg16(p + 64);
        }
    }
#pragma unroll
    for (int t = 0; t < FORK_TILES; ++t) {
        if (tile0 + t >= tile1) break;
        if constexpr (TURN) {
            uint32_t *lw = reinterpret_cast<uint32_t *>(&lo[t]), *hw = reinterpret_cast<uint32_t *>(&hi[t]);
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const float4 cs = *reinterpret_cast<const float4 *>(&rot[8 * c + 2 * u]);
                const float x0 = bf_lo(lw[u]), x1 = bf_hi(lw[u]), y0 = bf_lo(hw[u]), y1 = bf_hi(hw[u]);
                lw[u] = pack_bf16(x0 * cs.x - y0 * cs.y, x1 * cs.z - y1 * cs.w);
                hw[u] = pack_bf16(x0 * cs.y + y0 * cs.x, x1 * cs.w + y1 * cs.z);
            }
        }
        uint16_t *q = dst + ((int64_t)it.slot0 + (tile0 + t) * PC_TILE + r) * PC_D + 8 * c;
        *reinterpret_cast<uint4 *>(q) = lo[t];
        *reinterpret_cast<uint4 *>(q + 64) = hi[t];
    }
}

// Eight consecutive groups of a fork that comes from one piece: what its tokens are shifted by within a group is the same everywhere, so
// that a group of the source, read once, ends one group of the fork and begins the next.
template <int WORDS>
__device__ __forceinline__ void shifted_groups(const uint4 (&x)[9], unsigned bits, int len, int g0, int g1, uint16_t *dst)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t y[9] = {x[j].x, x[j].y, x[j].z, x[j].w, x[j + 1].x, x[j + 1].y, x[j + 1].z, x[j + 1].w, 0u};
        const int n = len - 8 * (g0 + j);
        uint32_t w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            w[k] = __builtin_amdgcn_alignbit(y[k + WORDS + 1], y[k + WORDS], bits);
            if (n < 8) w[k] &= (2 * k < n ? 0xFFFFu : 0u) | (2 * k + 1 < n ? 0xFFFF0000u : 0u);         // what lies behind the last token is another's
        }
        if (g0 + j < g1) *reinterpret_cast<uint4 *>(dst + (int64_t)j * PC_D * PC_VGROUP) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

__device__ __forceinline__ void fork_values_bf16(const PcForkItem &it, const PcForkPiece *pieces, int tile0, int tile1, const uint16_t *src, uint16_t *dst)
{
    const int d = threadIdx.x & 127, half = threadIdx.x >> 7;       // a dimension; (the group is the same for all lanes of a wave)
    if (it.n_pieces == 1) {
        static_assert(FORK_TILES == 4, "a half of the workgroup takes eight groups");
        const int g0 = 4 * tile0 + 8 * half, sh = pieces[0].slot & 7;
        const uint16_t *p = src + ((int64_t)((pieces[0].slot >> 3) + g0) * PC_D + d) * PC_VGROUP;
        uint16_t *q = dst + ((int64_t)(it.slot0 / PC_VGROUP + g0) * PC_D + d) * PC_VGROUP;
        uint4 x[9];
#pragma unroll
        for (int j = 0; j < 9; ++j) {                    // (a group's first token that is wanted: 8 (g0 + j) - sh)
            x[j] = make_uint4(0, 0, 0, 0);
            if (j == 0 ? 8 * g0 < it.len : 8 * (g0 + j) - sh < it.len && (j < 8 || sh > 0)) x[j] = ldg16(p + (int64_t)j * PC_D * PC_VGROUP);
        }
        const unsigned bits = 16u * (unsigned)(sh & 1);
        switch (sh >> 1) {
        case 0: shifted_groups<0>(x, bits, it.len, g0, 4 * tile1, q); break;
        case 1: shifted_groups<1>(x, bits, it.len, g0, 4 * tile1, q); break;
        case 2: shifted_groups<2>(x, bits, it.len, g0, 4 * tile1, q); break;
        default: shifted_groups<3>(x, bits, it.len, g0, 4 * tile1, q); break;
        }
        return;
    }
    for (int g = 4 * tile0 + half; g < 4 * tile1; g += 2) {
        const int t0 = 8 * g, n = min(8, it.len - t0);
        uint32_t w[4] = {0u, 0u, 0u, 0u};
        if (n > 0) {
            const int s0 = fork_slot(pieces, it.n_pieces, t0), s1 = fork_slot(pieces, it.n_pieces, t0 + n - 1);
            if (s1 - s0 == n - 1) {
                const int sh = s0 & 7;
                const uint16_t *p = src + ((int64_t)(s0 >> 3) * PC_D + d) * PC_VGROUP;
                const uint4 lo = ldg16(p);
                uint4 hi = make_uint4(0, 0, 0, 0);
                if (sh + n > 8) hi = ldg16(p + PC_D * PC_VGROUP);
                const uint32_t x[9] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w, 0u};
                const unsigned bits = 16u * (unsigned)(sh & 1);
                switch (sh >> 1) {
                case 0:
#pragma unroll
                    for (int j = 0; j < 4; ++j) w[j] = __builtin_amdgcn_alignbit(x[j + 1], x[j], bits);
                    break;
                case 1:
#pragma unroll
                    for (int j = 0; j < 4; ++j) w[j] = __builtin_amdgcn_alignbit(x[j + 2], x[j + 1], bits);
                    break;
                case 2:
#pragma unroll
                    for (int j = 0; j < 4; ++j) w[j] = __builtin_amdgcn_alignbit(x[j + 3], x[j + 2], bits);
                    break;
                default:
#pragma unroll
                    for (int j = 0; j < 4; ++j) w[j] = __builtin_amdgcn_alignbit(x[j + 4], x[j + 3], bits);
                    break;
                }
                if (n < 8) {                             // what lies behind the last token is another's
#pragma unroll
                    for (int j = 0; j < 4; ++j) w[j] &= (2 * j < n ? 0xFFFFu : 0u) | (2 * j + 1 < n ? 0xFFFF0000u : 0u);
                }
            } else {                                     // a group over the border of two extents
                for (int k = 0; k < n; ++k) {
                    const int s = fork_slot(pieces, it.n_pieces, t0 + k);
                    const uint32_t v = src[((int64_t)(s >> 3) * PC_D + d) * PC_VGROUP + (s & 7)];
#pragma unroll
                    for (int j = 0; j < 4; ++j) w[j] |= (k >> 1) == j ? v << (16 * (k & 1)) : 0u;
                }
            }
        }
        *reinterpret_cast<uint4 *>(dst + ((int64_t)(it.slot0 / PC_VGROUP + g) * PC_D + d) * PC_VGROUP) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

template <int D>
__device__ __forceinline__ void fork_f32(const PcForkItem &it, const PcForkPiece *pieces, int tile0, int tile1, const float *ks, float *kd, const float *vs, float *vd, const float2 *rot)
{
    constexpr int HALF = D / 2, PER = D / 8, STEP = 256 / PER;       // threads a row (4 dims and their partners), rows a step
    const int r = threadIdx.x / PER, c = 4 * (threadIdx.x % PER);
    for (int token = tile0 * PC_TILE + r; token < tile1 * PC_TILE; token += STEP) {
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f), y = x, a = x, b = x;
        if (token < it.len) {
            const int64_t at = (int64_t)fork_slot(pieces, it.n_pieces, token) * D + c;
            x = *reinterpret_cast<const float4 *>(ks + at); y = *reinterpret_cast<const float4 *>(ks + at + HALF);
            a = *reinterpret_cast<const float4 *>(vs + at); b = *reinterpret_cast<const float4 *>(vs + at + HALF);
        }
        if (it.turn != 0) {
            const float4 u = *reinterpret_cast<const float4 *>(&rot[c]), v = *reinterpret_cast<const float4 *>(&rot[c + 2]);
            const float4 p = x, q = y;
            x = make_float4(p.x * u.x - q.x * u.y, p.y * u.z - q.y * u.w, p.z * v.x - q.z * v.y, p.w * v.z - q.w * v.w);
            y = make_float4(p.x * u.y + q.x * u.x, p.y * u.w + q.y * u.z, p.z * v.y + q.z * v.x, p.w * v.w + q.w * v.z);
        }
        const int64_t to = ((int64_t)it.slot0 + token) * D + c;
        *reinterpret_cast<float4 *>(kd + to) = x; *reinterpret_cast<float4 *>(kd + to + HALF) = y;
        *reinterpret_cast<float4 *>(vd + to) = a; *reinterpret_cast<float4 *>(vd + to + HALF) = b;
    }
}

// Four bits: codes and exponents as they are; a word of values is put together from the places its eight tokens have where they come from.
__device__ __forceinline__ void fork_mx4(const PcForkItem &it, const PcForkPiece *pieces, int tile0, int tile1, char *k, char *v)
{
    __shared__ int s_from[PC_TILE];                      // where each token of the tile comes from, -1: there is none
    for (int tile = tile0; tile < tile1; ++tile) {
        __syncthreads();
        if (threadIdx.x < PC_TILE) {
            const int t = tile * PC_TILE + threadIdx.x;
            int from = -1;
            if (t < it.len) {
                int p = 0;
                while (p + 1 < it.n_pieces && pieces[p + 1].first <= t) ++p;
                from = pieces[p].slot + t - pieces[p].first;
            }
            s_from[threadIdx.x] = from;
        }
        __syncthreads();
        char *kt = k + ((int64_t)it.slot0 / PC_TILE + tile) * PC_MX4_TILE, *vt = v + ((int64_t)it.slot0 / PC_TILE + tile) * PC_MX4_TILE;
        auto place = [](char *store, int slot) { return store + (int64_t)(slot / PC_TILE) * PC_MX4_TILE; };
        {
            const int row = threadIdx.x >> 3, part = threadIdx.x & 7, from = s_from[row];
            uint2 x = make_uint2(0, 0);
            if (from >= 0) x = *reinterpret_cast<const uint2 *>(place(k, from) + from % PC_TILE * 64 + 8 * part);
            *reinterpret_cast<uint2 *>(kt + row * 64 + 8 * part) = x;
        }
        if (threadIdx.x < PC_TILE) {
            const int from = s_from[threadIdx.x];
            *reinterpret_cast<uint32_t *>(kt + PC_MX4_CODES + threadIdx.x * 4) = from < 0 ? 0u : *reinterpret_cast<const uint32_t *>(place(k, from) + PC_MX4_CODES + from % PC_TILE * 4);
        } else if (threadIdx.x < PC_TILE + 128) {
            const int b = threadIdx.x - PC_TILE, from = s_from[b / 32 * 8 + b % 8];        // byte b: group, block, slot
            vt[PC_MX4_CODES + b] = from < 0 ? 0 : place(v, from)[PC_MX4_CODES + from % PC_TILE / 8 * 32 + b / 8 % 4 * 8 + from % 8];
        }
        for (int e = threadIdx.x; e < 512; e += 256) {
            uint32_t w = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int from = s_from[e / 128 * 8 + j];
                if (from >= 0) w |= (reinterpret_cast<const uint32_t *>(place(v, from) + from % PC_TILE / 8 * 512)[e % 128] >> 4 * (from % 8) & 15u) << 4 * j;
            }
            reinterpret_cast<uint32_t *>(vt)[e] = w;
        }
    }
}

template <int D, bool BF16>
__device__ __forceinline__ void fork_copy(const PcForkItem *items, const PcForkPiece *all_pieces, int64_t slots, const double *__restrict__ inv_freq, void *k_store,
                                          void *v_store, PcMsgEntry *table)
{
    __shared__ __attribute__((aligned(16))) float2 s_rot[D / 2];
    const PcForkItem it = items[blockIdx.z];
    const int tile0 = blockIdx.x * FORK_TILES, tiles = (it.rows + PC_TILE - 1) / PC_TILE, tile1 = min(tile0 + FORK_TILES, tiles);
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) table[it.msg] = PcMsgEntry{it.slot0, it.len, it.base, 0};
    if (tile0 >= tiles) return;
    const PcForkPiece *pieces = all_pieces + it.piece0;
    if (it.turn != 0) {
        if (threadIdx.x < D / 2) s_rot[threadIdx.x] = rope_angle((double)it.turn * inv_freq[threadIdx.x]);
        __syncthreads();
    }
    const int64_t head = (int64_t)blockIdx.y * slots * D;
    if constexpr (BF16) {
        uint16_t *k = (uint16_t *)k_store + head, *v = (uint16_t *)v_store + head;
        if (it.turn != 0) fork_keys_bf16<true>(it, pieces, tile0, tile1, k, k, s_rot);
        else fork_keys_bf16<false>(it, pieces, tile0, tile1, k, k, s_rot);
        fork_values_bf16(it, pieces, tile0, tile1, v, v);
    } else {
        float *k = (float *)k_store + head, *v = (float *)v_store + head;
        fork_f32<D>(it, pieces, tile0, tile1, k, k, v, v, s_rot);
    }
}

template <int D, bool BF16>
__global__ __launch_bounds__(256) void pc_fork_kernel(const PcForkItem *items, const PcForkPiece *pieces, int64_t slots, const double *inv_freq, void *k_store,
                                                      void *v_store, PcMsgEntry *table)
{
    fork_copy<D, BF16>(items, pieces, slots, inv_freq, k_store, v_store, table);
}
template <int D, bool BF16>
__global__ __launch_bounds__(256) void pc_fork_arg_kernel(PcArgBlob, int n, int64_t slots, const double *inv_freq, void *k_store, void *v_store, PcMsgEntry *table)
{
    const PcForkItem *items = (const PcForkItem *)__builtin_amdgcn_kernarg_segment_ptr();          // (the blob comes first)
    fork_copy<D, BF16>(items, reinterpret_cast<const PcForkPiece *>(items + n), slots, inv_freq, k_store, v_store, table);
}

__device__ __forceinline__ void fork_copy_mx4(const PcForkItem *items, const PcForkPiece *all_pieces, int64_t slots, char *k_store, char *v_store, PcMsgEntry *table)
{
    const PcForkItem it = items[blockIdx.z];
    const int tile0 = blockIdx.x * FORK_TILES, tiles = (it.rows + PC_TILE - 1) / PC_TILE, tile1 = min(tile0 + FORK_TILES, tiles);
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) table[it.msg] = PcMsgEntry{it.slot0, it.len, it.base, 0};
    const int64_t head = (int64_t)blockIdx.y * (slots / PC_TILE) * PC_MX4_TILE;
    fork_mx4(it, all_pieces + it.piece0, tile0, tile1, k_store + head, v_store + head);
}
__global__ __launch_bounds__(256) void pc_fork_mx4_kernel(const PcForkItem *items, const PcForkPiece *pieces, int64_t slots, char *k_store, char *v_store, PcMsgEntry *table)
{
    fork_copy_mx4(items, pieces, slots, k_store, v_store, table);
}
__global__ __launch_bounds__(256) void pc_fork_mx4_arg_kernel(PcArgBlob, int n, int64_t slots, char *k_store, char *v_store, PcMsgEntry *table)
{
    const PcForkItem *items = (const PcForkItem *)__builtin_amdgcn_kernarg_segment_ptr();          // (the blob comes first)
    fork_copy_mx4(items, reinterpret_cast<const PcForkPiece *>(items + n), slots, k_store, v_store, table);
}

void pc_launch_fork(int dtype, const PcArgBlob *blob, const PcForkItem *items, const PcForkPiece *pieces, int n, int max_rows, int n_kv_heads, int D, int64_t slots,
                    const double *inv_freq, void *k_store, void *v_store, PcMsgEntry *table, hipStream_t st)
{
    const int tiles = (max_rows + PC_TILE - 1) / PC_TILE;
    if (blob) {
        const dim3 grid((unsigned)((tiles + FORK_TILES - 1) / FORK_TILES), (unsigned)n_kv_heads, (unsigned)n);
        if (dtype == 2) pc_fork_mx4_arg_kernel<<<grid, 256, 0, st>>>(*blob, n, slots, (char *)k_store, (char *)v_store, table);
        else if (dtype == 1) pc_fork_arg_kernel<128, true><<<grid, 256, 0, st>>>(*blob, n, slots, inv_freq, k_store, v_store, table);
        else if (D == 64) pc_fork_arg_kernel<64, false><<<grid, 256, 0, st>>>(*blob, n, slots, inv_freq, k_store, v_store, table);
        else pc_fork_arg_kernel<128, false><<<grid, 256, 0, st>>>(*blob, n, slots, inv_freq, k_store, v_store, table);
        return;
    }
    for (int at = 0; at < n; at += 65535) {              // (the limit of a grid's third dimension)
        const dim3 grid((unsigned)((tiles + FORK_TILES - 1) / FORK_TILES), (unsigned)n_kv_heads, (unsigned)std::min(n - at, 65535));
        if (dtype == 2) pc_fork_mx4_kernel<<<grid, 256, 0, st>>>(items + at, pieces, slots, (char *)k_store, (char *)v_store, table);
        else if (dtype == 1) pc_fork_kernel<128, true><<<grid, 256, 0, st>>>(items + at, pieces, slots, inv_freq, k_store, v_store, table);
        else if (D == 64) pc_fork_kernel<64, false><<<grid, 256, 0, st>>>(items + at, pieces, slots, inv_freq, k_store, v_store, table);
        else pc_fork_kernel<128, false><<<grid, 256, 0, st>>>(items + at, pieces, slots, inv_freq, k_store, v_store, table);
    }
}

// ----------------------------------------------------------------------------------------------------------- compact
// Extents slide down over the gaps in front of them, in one launch and one pass: read once, written once.  A workgroup takes a
// chunk of tiles of one head's keys or values, reads all of it into registers, says so, and writes once the chunks whose tiles lie
// where it writes have said so.
//
// Why every wait ends.  Chunks are numbered by the slots they come from and everything moves down, so what lies where a chunk
// writes belongs to chunks of lower numbers or to itself.  A workgroup takes its number from its store's counter when it starts: the
// holders of all lower numbers have started, and each says that it has read before it waits for anything.  What is passed on is no data,
// only that loads have returned (the wait in front of the flag); the tiles written are whole cache lines that nobody
// reads in this launch any more.
// Bound: memory.  512 messages of 160 tokens, 8 KV heads: 650 MB read and written in 145 us (4.5 TB/s); 64 KB a workgroup and one counter
// for all stores 174 us, 32 KB 330 (a counter gives 70 numbers a microsecond); kept in the caches like other data 5 % more.
// Flags hold the launch's number and the counter goes on from launch to launch, so that nothing has to be cleared.
// TILE: pieces of 16 bytes in a tile that do not fill a step of the workgroup (4 bits), 0: those that do
template <int TILE> __device__ __forceinline__ void compact_chunk(const PcCompact &C)
{
    __shared__ uint32_t s_ticket;
    const int store = (int)(blockIdx.x % (unsigned)C.n_stores), H = C.n_stores / 2;
    if (threadIdx.x == 0) s_ticket = __hip_atomic_fetch_add(C.ticket + store * PC_COMPACT_COUNTER, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) - C.ticket0;
    __syncthreads();
    const int chunk = __builtin_amdgcn_readfirstlane((int)s_ticket);
    const int per = PC_COMPACT_BYTES / C.tile_bytes, tile0 = chunk * per, n = min(per, C.n_tiles - tile0);
    if (chunk == 0 && store == 0)
        for (int i = threadIdx.x; i < C.n_moves; i += PC_COMPACT_THREADS) C.table[C.moves[i].rec].slot_start = C.moves[i].slot_start;
    char *base = store < H ? C.k_store + store * C.head_bytes : C.v_store + (store - H) * C.head_bytes;
    constexpr int PIECE = 16 * PC_COMPACT_THREADS, PIECES = PC_COMPACT_BYTES / PIECE;
    const int steps = TILE ? 1 : C.tile_bytes / PIECE;   // (1 or 2)
    // piece j of the thread: of which tile, and where in it
    auto tile_of = [&](int j) { return TILE ? (j * PC_COMPACT_THREADS + (int)threadIdx.x) / (TILE ? TILE : 1) : j / steps; };
    auto byte_of = [&](int j) { return TILE ? (j * PC_COMPACT_THREADS + (int)threadIdx.x) % (TILE ? TILE : 1) * 16 : (j % steps) * PIECE + (int)threadIdx.x * 16; };
    u32x4 x[PIECES];
#pragma unroll
    for (int j = 0; j < PIECES; ++j) {
        const int t = tile_of(j);
        x[j] = (u32x4){0u, 0u, 0u, 0u};
        if (t < n) {
            const int src = C.tiles[tile0 + t].src;
            if (src >= 0) x[j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(base + (int64_t)src * C.tile_bytes + byte_of(j)));
        }
    }
#pragma unroll
    for (int j = 0; j < PIECES; ++j) asm volatile("" : "+v"(x[j]));      // every load has returned ...
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();                                     // ... in every wave
    uint32_t *read = C.read + (int64_t)store * C.n_chunks;
    if (threadIdx.x == 0) __hip_atomic_store(read + chunk, C.epoch, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if ((int)threadIdx.x < n) {
        const int after = C.tiles[tile0 + threadIdx.x].after;
        if (after >= 0 && after != chunk)
            while (__hip_atomic_load(read + after, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != C.epoch) __builtin_amdgcn_s_sleep(1);
    }
    asm volatile("" ::: "memory");
    __syncthreads();
#pragma unroll
    for (int j = 0; j < PIECES; ++j) {
        const int t = tile_of(j);
        if (t < n) __builtin_nontemporal_store(x[j], reinterpret_cast<u32x4 *>(base + (int64_t)C.tiles[tile0 + t].dst * C.tile_bytes + byte_of(j)));
    }
}

template <int TILE> __global__ __launch_bounds__(PC_COMPACT_THREADS) void pc_compact_kernel(PcCompact C) { compact_chunk<TILE>(C); }
template <int TILE> __global__ __launch_bounds__(PC_COMPACT_THREADS) void pc_compact_arg_kernel(PcArgBlob, PcCompact C)
{
    const char *lists = (const char *)__builtin_amdgcn_kernarg_segment_ptr();          // (the blob comes first)
    C.tiles = reinterpret_cast<const PcCompactTile *>(lists);
    C.moves = reinterpret_cast<const PcCompactMove *>(C.tiles + C.n_tiles);
    compact_chunk<TILE>(C);
}

void pc_launch_compact(const PcCompact &C, const PcArgBlob *blob, hipStream_t st)
{
    if (C.n_chunks <= 0) return;
    const unsigned grid = (unsigned)(C.n_chunks * C.n_stores);
    constexpr int MX4 = PC_MX4_TILE / 16;
    if (C.tile_bytes == PC_MX4_TILE) {
        if (blob) pc_compact_arg_kernel<MX4><<<grid, PC_COMPACT_THREADS, 0, st>>>(*blob, C);
        else pc_compact_kernel<MX4><<<grid, PC_COMPACT_THREADS, 0, st>>>(C);
    } else if (blob) pc_compact_arg_kernel<0><<<grid, PC_COMPACT_THREADS, 0, st>>>(*blob, C);
    else pc_compact_kernel<0><<<grid, PC_COMPACT_THREADS, 0, st>>>(C);
}
