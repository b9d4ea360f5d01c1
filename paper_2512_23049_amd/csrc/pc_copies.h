// Structures and launch wrappers of the cache's own copies: forks of messages, and the cache closing up (internal to the library).
#ifndef PC_COPIES_H_
#define PC_COPIES_H_

#include "pc_internal.h"

// One fork (staged by the host): tokens of a message's extents, one after the other, as a message of one extent.
struct PcForkItem {
    int32_t msg;              // the new message
    int32_t slot0;
    int32_t len;
    int32_t rows;             // >= len: slots written; those behind the last token get zeros
    int32_t base;             // positions its keys are turned to: base + token
    int32_t piece0, n_pieces; // where its tokens come from
    int32_t pad;
    int64_t turn;             // positions the keys are turned by on the way (0: copied bit for bit)
    int64_t pad2;
};
// Tokens [first, first + n) of the new message lie from this slot on.
struct PcForkPiece { int32_t first, n, slot, pad; };

#define PC_COMPACT_THREADS 512
#define PC_COMPACT_BYTES (256 * PC_COMPACT_THREADS)       // what a workgroup moves: it holds all of it in registers
#define PC_COMPACT_COUNTER 64     // words: a counter's cache lines are its own
// A tile that moves; the tiles are in the order of their slots.
struct PcCompactTile {
    int32_t src;              // slot / PC_TILE, -1: no tokens there, zeros are written
    int32_t dst;
    int32_t after;            // the chunk of tiles that has to be read before dst is written, -1: none
    int32_t pad;
};
struct PcCompactMove { int32_t rec, slot_start; };        // a table row's new place
struct PcCompact {
    const PcCompactTile *tiles;
    const PcCompactMove *moves;
    int32_t n_tiles, n_moves, n_chunks, n_stores;     // n_stores: KV heads, times two (keys, then values)
    uint32_t epoch, ticket0;
    uint32_t *ticket;         // [n_stores], PC_COMPACT_COUNTER words apart: count a store's workgroups of every launch
    uint32_t *read;           // [n_stores][n_chunks]: epoch once the chunk has been read
    char *k_store, *v_store;
    int64_t head_bytes;       // a head's share of a store
    int32_t tile_bytes;
    PcMsgEntry *table;
};

// items, pieces: staged, or (blob not null) in the arguments, the pieces behind the items; max_rows: the longest fork's
void pc_launch_fork(int dtype, const PcArgBlob *blob, const PcForkItem *items, const PcForkPiece *pieces, int n, int max_rows, int n_kv_heads, int D, int64_t slots,
                    const double *inv_freq, void *k_store, void *v_store, PcMsgEntry *table, hipStream_t st);
// blob: its lists, the moves behind the tiles (C.tiles and C.moves are not read then), or null
void pc_launch_compact(const PcCompact &C, const PcArgBlob *blob, hipStream_t st);

#endif
