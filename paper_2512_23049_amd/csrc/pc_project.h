// Structures and launch wrappers of rows on their way into the cache: norms of heads, rotation, the stored form; the gradient of that
// way; and messages read back (internal to the library).
#ifndef PC_PROJECT_H_
#define PC_PROJECT_H_

#include "pc_internal.h"

// Consecutive tokens that go to consecutive slots of one extent (staged by the host).
struct PcRowsItem {
    const void *q, *k, *v;    // the first token's rows
    int64_t q_row;            // its row of q_out
    int32_t slot0, pos0;      // its slot, and the position its key is turned to
    int32_t n;                // tokens
    int32_t rows;             // fresh: slots written, >= n; those behind the last token get zeros (a 4-bit cache needs none)
    int32_t msg, len;         // the table's row, and the tokens it holds then
    int32_t block0;           // the item's first block of the launch
    int32_t fresh;            // 1: a new message (the table's row is written whole)
};
static_assert(sizeof(PcRowsItem) == 64, "");
#define PC_ROWS_GROUP 8       // slots (a group of them, aligned) that a block takes
#define PC_ROWS_HEADS 8       // heads that a block takes

struct PcRows {
    const PcRowsItem *items;
    int32_t n_items, n_blocks, block0;        // (block0: the launch's first)
    int64_t q_stride, k_stride, v_stride;     // elements from a row to the next
    const float *q_weight, *k_weight;         // [D] or null: ones
    float   eps;
    int32_t norm;                             // 0: keys as they come (and no queries)
    void   *q_out;                            // [rows][n_q_heads][D], null: no queries
    int32_t n_q_heads, n_kv_heads, D;
    int64_t slots;
    const double *inv_freq;
    void   *k_store, *v_store;
    PcMsgEntry *table;
    uint32_t *wide;                           // (4 bits) set where a value is outside what PC_MX4_HALF says
};
// blob: the items in the arguments (R.items is not read then), or null
void pc_launch_rows(int dtype, PcRows R, const PcArgBlob *blob, hipStream_t st);

// The gradient.
struct PcRowsBwdItem {
    int64_t row0;             // the first token's row
    int32_t slot0, pos0, n;
    int32_t block0;
};
struct PcRowsBwd {
    const PcRowsBwdItem *items;
    int32_t n_items, n_blocks;
    int32_t block_rows;                       // rows that a block takes
    const void *q, *k;
    int64_t q_stride, k_stride;
    const float *q_weight, *k_weight;
    float   eps;
    int32_t n_q_heads, n_kv_heads, D;
    const float *d_q, *d_k, *d_v;
    void   *to_q, *to_k, *to_v;
    int64_t to_q_stride, to_k_stride, to_v_stride;
    float  *q_part, *k_part;                  // a block's sums for the weights: [block][chunk of heads][D]
    float  *to_q_weight, *to_k_weight;        // null: not asked for
    uint32_t *done, n_done;                   // n_done > 0: the last of so many blocks adds the sums up
    const double *inv_freq;
};
void pc_launch_rows_backward(int dtype, const PcRowsBwd &B, const PcArgBlob *blob, hipStream_t st);

// Extents read back: tokens [0, n) from slot0 on become rows row0 and on.
struct PcReadItem { int64_t row0; int32_t slot0, n, block0, pad; };
struct PcRead {
    const PcReadItem *items;
    int32_t n_items, n_blocks, n_kv_heads, D;
    int64_t slots;
    const void *k_store, *v_store;
    void *k, *v;              // [rows][n_kv_heads][D]
};
void pc_launch_read(int dtype, const PcRead &R, const PcArgBlob *blob, hipStream_t st);

#endif
