// Structures and launch wrappers of the windowed attention (internal to the library).
//
// Visibility.  A row at position p of a call sees a key at position x if the call lists the key (own tokens: up to the row's
// own one) and x > p - window, or the key is one of the first n_sink tokens of the call's list.  The host turns that into
// runs: for each group of rows and each listed extent the tiles that some row of the group sees (a suffix of the extent, its
// sinks in front), so that the kernels walk what is needed and mask at its edges only.
#ifndef PC_WINDOW_H_
#define PC_WINDOW_H_

#include "pc_internal.h"

// Consecutive tiles of one extent.
struct PcWinRun {
    int32_t slot0;            // first slot (multiple of PC_TILE)
    int32_t pos0;             // position the call gives the token in that slot
    int32_t n_tok;            // tokens from there on that count
    int32_t sink;             // the first of them that are visible at any distance
    int32_t rot;              // row of the rotation table
    int32_t self;             // 1: the new message (causal limit)
    int64_t rot_pos;          // the extent's start - the position its keys are stored at: what the queries are turned back by
};

// One workgroup's share of a launch, for each KV head.
struct PcWinItem {
    int32_t q_off, n_q;       // the call's packed rows
    int32_t unit0;            // bf16: first of four units (32 rows x head of the KV head, head fastest); fp32: block of 32 (row, head) columns
    int32_t lim0;             // position of the last own token that row 0 of the call sees (row r: lim0 + r)
    int32_t run0, skip;       // the first run, and its tiles that belong to the split before
    int32_t n_tiles;
    int32_t part;             // -1, or the partial row of the call's row 0 in this split
};

// What every launch of a call needs.
struct PcWin {
    const PcWinRun  *runs;
    const PcWinItem *items;
    const int32_t   *q_pos;   // [rows]
    const float2    *rot_q;   // [rows][D/2]: (cos, sin)(q_pos theta_i)
    const uint32_t  *rot_lanes;       // the same as fp16 in the lanes' order (see win_rot_at)
    const float2    *rot_run; // [rot][D/2]: (cos, sin)(rot_pos theta_i)
    const double    *inv_freq;
    const void      *k_store, *v_store, *q;
    void            *out;
    float           *lse;     // or null
    float           *part_o;  // [part rows][H_q][D], not normalised
    float           *part_ml; // [part rows][H_q][2]
    int64_t          slots;
    int32_t          n_q_heads, n_kv_heads;
    int32_t          window;
    float            scale_log2;
};
// Offsets of a decode launch's lists, where they travel in its arguments.
struct PcWinDecode { int32_t off_items, off_runs, off_q_pos, n16; void *ws; };      // n16 > 0: so many pieces of 16 bytes are left in the workspace for the merge

// ---- single tokens of calls that list the same messages ----
#define PC_WIN_STEP_TILES 2   // tiles of a visit that are multiplied between two barriers
#define PC_WIN_GROUPS 16      // groups of 16 columns (calls x heads of the KV head) a workgroup takes at most
struct PcWinVisit {           // consecutive tiles, and who sees some of them
    int32_t slot0, n_tiles;
    int32_t e0;               // the first of its entries
    int32_t off[PC_WIN_GROUPS + 1];   // of them: the first of each group of columns
};
struct PcWinSee {             // a call's view of a visit
    int32_t pos0;             // position the call gives the visit's first token
    int32_t n_tok;            // tokens from there on that count
    int32_t sink, lo;         // as in PcWinRun; the least position that is visible but for the sinks
    int64_t turn;             // the row's position less the run's rotation: what its queries are turned by
    int32_t sub;              // the call's place in its group of columns
    int32_t pad;
};
struct PcWinSharedItem {      // one workgroup's tiles, for each KV head
    int32_t visit0, n_steps;  // (a step: PC_WIN_STEP_TILES tiles of a visit)
    int32_t call0, n_calls;   // its set of calls
    int32_t waves;            // that hold all groups of columns (a power of two); the others share its steps
    int32_t split0;
    int32_t pad[2];
};
struct PcWinSharedCall { int32_t row, part0; };         // packed row, partial row of split 0
struct PcWinShared {
    const PcWinSharedItem *items;
    const PcWinVisit      *visits;
    const PcWinSee        *sees;
    const PcWinSharedCall *calls;
    int32_t n_items;
    int32_t wide;             // 1: 16 waves (groups of columns) a workgroup, 0: 8
};

// ---- the gradient ----
// 32 rows (fp32: 32 (row, head) columns of a KV head) of a call.
struct PcWinBlock { int32_t q_off, n_q, lim0, block; };
// A call that lists the extent a key item's tiles belong to.
struct PcWinApp {
    int32_t pos0;             // position the call gives the item's first token
    int32_t n_tok;            // the call's tokens from there on
    int32_t sink;             // the first of them that are visible at any distance
    int32_t rot;              // row of the rotation table
    int32_t self;             // 1: the call's new message
    int32_t block0, n_blocks; // the blocks that may see some of the item's tokens
    int32_t q0;               // their queries, in units' blocks: block0, or the first of those turned for this call's rotation
};
#define PC_WIN_FEW 32
// Rows of few keys (window and sinks, PC_WIN_FEW at most): a block's queries turned for one listed extent, as the forward turns them.
struct PcWinTurned { int32_t block, rot; };
#define PC_WIN_KEY_TILES 4
struct PcWinKeyItem {         // up to four tiles of an extent, and calls (or some of their blocks) that see them
    int32_t slot0;
    int32_t n_keys;           // tokens of the extent from there on (at most 128)
    int32_t app0, n_apps;
    int32_t part;             // -1: the only item of its tiles; else where its sums go
    int32_t pad[3];
};
struct PcWinSum { int32_t slot0, n_keys, part0, n_parts; };       // tiles whose items' sums are added up
struct PcWinStat {            // of a unit's rows
    float lse2[32], delta[32];        // lse log2 e (+inf: no gradient), Delta
    int32_t lo[32], lim[32];          // the positions a row sees: from, up to (own)
    int4 head;                // least lo; largest lo (INT32_MAX if some row that is there has no gradient); first and last lim
    int32_t live;             // bits of the rows with a gradient
};
#define PC_WIN_STAT_BYTES 1024
static_assert(sizeof(PcWinStat) <= PC_WIN_STAT_BYTES, "");
struct PcWinBwd {
    const PcWinBlock   *blocks;
    const PcWinApp     *apps;
    const PcWinKeyItem *key_items;
    const PcWinSum     *sums;
    const int32_t      *bins; // [n_bins + 1] the first of each workgroup's items
    int32_t n_blocks, n_bins, n_sums, n_turned;
    const PcWinTurned *turned;        // null: queries are turned by their positions, keys by their extents'
    const void  *out, *d_out;
    const float *lse;
    float       *delta;       // [rows][H_q]
    void        *q_abs;       // [unit][32][D] queries turned by their positions, in the cache's type; unit: (block, head), fp32: (block, KV head)
    void        *d_o;         // [unit][32][D] the output gradients, zeros for rows without
    char        *stat;        // [unit][PC_WIN_STAT_BYTES]: PcWinStat
    float       *key_part;    // [part][KV head][keys, values][128][D]
    float       *d_q, *d_k, *d_v;
    float        scale;
    float        k_factor, key_scale;         // bf16 keys: what rides on the keys for the scores, and on their gradients
};
void pc_launch_win_bwd_prep(const PcWin &W, const PcWinBwd &B, int dtype, int D, hipStream_t st);
void pc_launch_win_bwd_turned(const PcWin &W, const PcWinBwd &B, hipStream_t st);
void pc_launch_win_bwd_dq_bf16(const PcWin &W, const PcWinBwd &B, int n_items, hipStream_t st);
void pc_launch_win_bwd_dq_f32(const PcWin &W, const PcWinBwd &B, int n_items, int D, hipStream_t st);
// the splits of a row's gradient, added up in their order
void pc_launch_win_bwd_rows(const PcWin &W, const PcWinBwd &B, const PcMergeRow *rows, int n_rows, int D, hipStream_t st);
void pc_launch_win_bwd_keys_bf16(const PcWin &W, const PcWinBwd &B, hipStream_t st);
void pc_launch_win_bwd_keys_f32(const PcWin &W, const PcWinBwd &B, int D, hipStream_t st);
void pc_launch_win_bwd_sums(const PcWin &W, const PcWinBwd &B, int D, hipStream_t st);

// index of pair i of packed row R in the lanes' order of the bf16 kernels that turn queries (D = 128): 16 bytes a lane, lanes of
// consecutive rows side by side.  (cos, sin) are fp16 there, off by 2^-12 at most, an eighth of what the turned query's own rounding
// may take: a run's first tile waits for these bytes.
__host__ __device__ __forceinline__ int64_t win_rot_at(int64_t R, int i)
{
    return ((R / 32 * 16 + i / 16 * 4 + i % 8 / 4 * 2 + i / 8 % 2) * 32 + R % 32) * 4 + i % 4;
}

// the least position a row at p sees (but for the sinks)
__host__ __device__ __forceinline__ int32_t win_low(int32_t p, int32_t window)
{
    const int64_t low = (int64_t)p - window + 1;
    return low < INT32_MIN ? INT32_MIN : (int32_t)low;
}

// lists (n16 pieces of 16 bytes, at `from`, or in the arguments where blob is not null) to ws, and the rotations of rows and runs
struct PcWinTurns {
    const void *from; void *ws; int n16;
    int off_q_pos, n_rows, off_rot, n_rot;        // within the lists: int32 positions, int64 positions
    int D;
    float run_scale;                              // rides on the runs' rotations
    float2 *rot_q, *rot_run;                      // rot_q, rot_lanes: null where nobody reads them
    uint32_t *rot_lanes;
    const double *inv_freq;
};
void pc_launch_win_turns(const PcWinTurns &T, const PcArgBlob *blob, hipStream_t st);

void pc_launch_win_prefill_bf16(const PcWin &W, int n_items, hipStream_t st);
// blob: its lists (W.items, W.runs and W.q_pos are not read then), or null
void pc_launch_win_decode_bf16(const PcWin &W, int n_items, const PcArgBlob *blob, const PcWinDecode &O, hipStream_t st);
void pc_launch_win_attend_f32(const PcWin &W, int n_items, int D, hipStream_t st);
void pc_launch_win_shared_decode_bf16(const PcWin &W, const PcWinShared &S, hipStream_t st);
void pc_launch_win_merge(const PcWin &W, const PcMergeRow *rows, int n_rows, int dtype, int D, hipStream_t st);

#ifdef __HIPCC__
__device__ __forceinline__ float f16_lo(uint32_t w) { return (float)__builtin_bit_cast(_Float16, (uint16_t)w); }
__device__ __forceinline__ float f16_hi(uint32_t w) { return (float)__builtin_bit_cast(_Float16, (uint16_t)(w >> 16)); }
// A walk over the tiles of an item, run after run (uniform over the wave: everything stays in scalar registers).
struct WinTile { int slot0, pos0, valid, sink, rot, self; int64_t rot_pos; };
typedef int win_i32x4 __attribute__((ext_vector_type(4)));
struct WinWalk {
    uintptr_t run;            // the present run
    win_i32x4 a;              // slot0, pos0, n_tok, sink of what is left of it
    int rot, self;
    int64_t rot_pos;
    __device__ __forceinline__ void load()
    {
        const auto *p = reinterpret_cast<const __attribute__((address_space(4))) win_i32x4 *>(run);
        a = p[0];
        const win_i32x4 b = p[1];
        rot = b.x; self = b.y;
        rot_pos = (int64_t)(((uint64_t)(uint32_t)b.w << 32) | (uint32_t)b.z);
    }
    __device__ __forceinline__ void pass(int tiles)      // tiles of the present run (fewer than it has)
    {
        a.x += PC_TILE * tiles; a.y += PC_TILE * tiles; a.z -= PC_TILE * tiles; a.w -= PC_TILE * tiles;
    }
    // tiles: of the walk; where there is none there may be no run either, and nothing is read
    __device__ __forceinline__ WinWalk(const void *runs, int skip, int tiles) : run(reinterpret_cast<uintptr_t>(runs)), a((win_i32x4){0, 0, 0, 0}), rot(0), self(0), rot_pos(0)
    {
        if (tiles <= 0) return;
        load();
        for (;;) {                                       // (a wave's or a split's share may begin some runs further on)
            const int n = (a.z + PC_TILE - 1) / PC_TILE;
            if (skip < n) break;
            skip -= n;
            run += sizeof(PcWinRun);
            load();
        }
        pass(skip);
    }
    __device__ __forceinline__ WinTile tile() const { return WinTile{a.x, a.y, min(a.z, PC_TILE), min(max(a.w, 0), PC_TILE), rot, self, rot_pos}; }
    __device__ __forceinline__ void next()               // (not behind the item's last tile: there may be no further run)
    {
        if (a.z > PC_TILE) { pass(1); return; }
        run += sizeof(PcWinRun);
        load();
    }
};
// Values that are not finite, in a tile of which some row does not see every key: a probability of 0 would not take them out of
// the product.  They are left out of it, and a second product adds up, over the keys a row sees, a number for each of them: its
// digits say which there were, and with that what they make of the sum.
#define PC_WIN_ODD_INF 1.f
#define PC_WIN_ODD_NEG 256.f  // (at most 32 keys: no carry)
#define PC_WIN_ODD_NAN 65536.f
__device__ __forceinline__ float win_odd_sum(float z)
{
    const float neg = __builtin_truncf(z * (1.f / PC_WIN_ODD_NEG)), pos = z - neg * PC_WIN_ODD_NEG;
    const bool none = (z >= PC_WIN_ODD_NAN) | ((neg > 0.f) & (pos > 0.f));
    const float some = neg > 0.f ? -INFINITY : INFINITY, what = none ? __builtin_nanf("") : some;
    return z == 0.f ? 0.f : what;
}
// bit j: the row with those limits sees key j of the tile (lo: its least position, lim: the last own position it sees)
__device__ __forceinline__ uint32_t win_sees(int pos0, int valid, int sink, bool self, int lo, int lim)
{
    auto first = [](unsigned n) { return n >= 32u ? ~0u : (1u << n) - 1u; };          // bits 0 .. n - 1
    const unsigned below = lo <= pos0 ? 0u : (unsigned)lo - (unsigned)pos0;             // (positions may lie 2^32 apart)
    const unsigned own = !self ? 32u : lim < pos0 ? 0u : min((unsigned)lim - (unsigned)pos0, 31u) + 1u;
    return first(min(own, (unsigned)valid)) & (~first(below) | first((unsigned)sink));
}
#endif

#endif
