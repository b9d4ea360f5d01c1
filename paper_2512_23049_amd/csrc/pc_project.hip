// Host side of rows on their way into the cache (norms of heads, rotation, append), of the gradient of that way, and of messages read
// back.
#include "pc_host.h"
#include "pc_project.h"

namespace {

constexpr int64_t FEW_SUMS = 64;
constexpr int64_t MOST_BLOCKS = (1 << 24) - 1;           // of 256 threads, in one dimension of a launch

bool aligned(const void *p, size_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

// a strided tensor of rows of heads, each 16-byte aligned
int32_t check_rows(pc_cache *c, const char *what, const char *name, const void *p, int64_t stride, int heads)
{
    if (!p) return pc_fail(c, PC_ERR_INVALID_ARG, "%s: null %s", what, name);
    if (!aligned(p, 16) || stride % (int64_t)(16 / c->esize)) return pc_fail(c, PC_ERR_INVALID_ARG, "%s: the rows of %s must be 16-byte aligned", what, name);
    if (stride < (int64_t)heads * c->D) return pc_fail(c, PC_ERR_SHAPE, "%s: rows of %s are %lld elements apart, %d heads take %lld", what, name, (long long)stride, heads,
                                                       (long long)heads * c->D);
    return PC_OK;
}

int32_t check_projected(pc_cache *c, const char *what, const pc_projected *p, bool values)
{
    if (!p) return pc_fail(c, PC_ERR_INVALID_ARG, "%s: null rows", what);
    if (!(p->eps >= 0.f) || !(p->eps < INFINITY)) return pc_fail(c, PC_ERR_INVALID_ARG, "%s: eps must be finite and not negative", what);
    if (c->host_only) return PC_OK;
    if (p->q) {
        const int32_t rc = check_rows(c, what, "q", p->q, p->q_stride, c->cfg.n_q_heads);
        if (rc != PC_OK) return rc;
    }
    int32_t rc = check_rows(c, what, "k", p->k, p->k_stride, c->cfg.n_kv_heads);
    if (rc == PC_OK && values) rc = check_rows(c, what, "v", p->v, p->v_stride, c->cfg.n_kv_heads);
    if (rc == PC_OK && (!aligned(p->q_weight, 4) || !aligned(p->k_weight, 4))) rc = pc_fail(c, PC_ERR_INVALID_ARG, "%s: weights must be 4-byte aligned", what);
    return rc;
}

// The launch for some items: what they bring is in the arguments, or staged.
template <class Item> int32_t stage(pc_cache *c, const std::vector<Item> &items, PcArgBlob &blob, bool &in_args, hipStream_t st)
{
    const size_t bytes = sizeof(Item) * items.size();
    in_args = bytes <= PC_ARG_BYTES;
    if (!in_args) {
        if (pc_recorded(st)) return pc_fail(c, PC_ERR_INVALID_ARG, "lists of %zu bytes: the stream is being captured, and a replay would find others in their place", bytes);
        return pc_stage_items(c, items.data(), bytes, st);
    }
    std::memcpy(blob.w, items.data(), bytes);
    return PC_OK;
}

const void *row_of(const void *p, int64_t row, int64_t stride, size_t esize) { return p ? (const char *)p + row * stride * (int64_t)esize : nullptr; }

PcRows launch_of(const pc_cache *c, const pc_projected *p, void *q_out)
{
    PcRows R{};
    R.q_stride = p->q_stride; R.k_stride = p->k_stride; R.v_stride = p->v_stride;
    R.q_weight = p->q_weight; R.k_weight = p->k_weight;
    R.eps = p->eps; R.norm = 1;
    R.q_out = q_out;
    return R;
}

int32_t check_q_out(pc_cache *c, const char *what, const pc_projected *p, const void *q_out)
{
    if (c->host_only) return PC_OK;
    if (!p->q != !q_out) return pc_fail(c, PC_ERR_INVALID_ARG, "%s: q and q_out come together, or not at all", what);
    if (!aligned(q_out, 16)) return pc_fail(c, PC_ERR_INVALID_ARG, "%s: q_out must be 16-byte aligned", what);
    return PC_OK;
}

int32_t append_projected(pc_cache *c, const pc_projected *p, int32_t n, const int32_t *lens, const int32_t *reserves, int32_t *msg_ids, void *q_out, hipStream_t st)
{
    const char *what = "append_projected";
    if (n < 0 || (n > 0 && (!lens || !msg_ids))) return pc_fail(c, PC_ERR_INVALID_ARG, "%s: bad lists", what);
    if (n == 0) return PC_OK;
    int32_t rc = check_projected(c, what, p, true);
    if (rc == PC_OK) rc = check_q_out(c, what, p, q_out);
    if (rc != PC_OK) return rc;
    if ((int64_t)c->msgs.size() + n > c->cfg.max_messages) return pc_fail(c, PC_ERR_NO_SPACE, "%s: message table full (%d)", what, c->cfg.max_messages);
    if (!c->host_only && pc_recorded(st)) return pc_fail(c, PC_ERR_INVALID_ARG, "%s: the stream is being captured", what);
    std::vector<FreeSpan> spans = c->free_spans;         // all or nothing: on copies first
    int64_t next = c->next_slot, row = 0;
    std::vector<PcRowsItem> items((size_t)n);
    std::vector<HostMsg> fresh((size_t)n);
    for (int j = 0; j < n; ++j) {
        if (lens[j] < 1) return pc_fail(c, PC_ERR_INVALID_ARG, "%s: message %d has len = %d", what, j, lens[j]);
        const int32_t res = std::max(reserves ? reserves[j] : 0, lens[j]);
        int64_t start = 0;
        if (!pc_take_slots(spans, next, c->slots, res, start))
            return pc_fail(c, PC_ERR_NO_SPACE, "%s: message %d (%d slots) does not fit, capacity %lld", what, j, res, (long long)c->slots);
        fresh[(size_t)j] = HostMsg{start, lens[j], res, 0, true};
        items[(size_t)j] = PcRowsItem{row_of(p->q, row, p->q_stride, c->esize), row_of(p->k, row, p->k_stride, c->esize), row_of(p->v, row, p->v_stride, c->esize), row,
                                      (int32_t)start, 0, lens[j], pc_rows_to_write(c, start, lens[j], res), (int32_t)c->msgs.size() + j, lens[j], 0, 1};
        row += lens[j];
    }
    c->msgs.reserve(c->msgs.size() + (size_t)n);         // (nothing may fail behind the launch)
    if (!c->host_only) {
        rc = pc_write_rows(c, launch_of(c, p, q_out), items, st);
        if (rc != PC_OK) return rc;
    }
    for (int j = 0; j < n; ++j) {
        msg_ids[j] = (int32_t)c->msgs.size();
        if (!c->msgs.empty() && fresh[(size_t)j].slot_start < c->msgs.back().slot_start) c->slots_in_id_order = false;
        c->msgs.push_back(fresh[(size_t)j]);
    }
    c->free_spans.swap(spans);
    c->next_slot = next;
    return PC_OK;
}

int32_t append_projected_tokens(pc_cache *c, const pc_projected *p, const int32_t *msg_ids, int32_t n_msgs, void *q_out, hipStream_t st)
{
    const char *what = "append_projected_tokens";
    if (n_msgs < 0 || (n_msgs > 0 && !msg_ids)) return pc_fail(c, PC_ERR_INVALID_ARG, "%s: bad id list", what);
    if (n_msgs == 0) return PC_OK;
    int32_t rc = check_projected(c, what, p, true);
    if (rc == PC_OK) rc = check_q_out(c, what, p, q_out);
    if (rc == PC_OK) rc = pc_check_token_batch(c, msg_ids, n_msgs, p->k, p->v);
    if (rc != PC_OK) return rc;
    PcDeviceScope on(c);
    if (!c->host_only && !on.ok) return pc_fail(c, PC_ERR_HIP, "%s: the cache's device cannot be made current", what);
    if (!c->host_only && pc_recorded(st)) return pc_fail(c, PC_ERR_INVALID_ARG, "%s: the stream is being captured", what);
    const PcRows R = launch_of(c, p, q_out);
    return pc_append_token_items(c, std::vector<int32_t>(msg_ids, msg_ids + n_msgs), p->k, p->v, st, nullptr, &R, p->q);
}

int32_t projected_backward(pc_cache *c, const pc_projected *p, int32_t n, const int32_t *msg_ids, const int32_t *lens, const float *d_q, const float *d_k, const float *d_v,
                           const pc_projected_grad *to, hipStream_t st)
{
    const char *what = "projected_backward";
    if (n < 0 || (n > 0 && (!msg_ids || !lens))) return pc_fail(c, PC_ERR_INVALID_ARG, "%s: bad lists", what);
    if (c->cfg.dtype == PC_MX4) return pc_fail(c, PC_ERR_INVALID_ARG, "%s: a PC_MX4 cache has no gradient", what);
    if (!to) return pc_fail(c, PC_ERR_INVALID_ARG, "%s: null gradients", what);
    int32_t rc = check_projected(c, what, p, false);
    if (rc != PC_OK) return rc;
    if (!c->host_only) {
        if (!p->q != !d_q || !p->q != !to->q || (!p->q && to->q_weight)) return pc_fail(c, PC_ERR_INVALID_ARG, "%s: q, d_q and their gradients come together, or not at all", what);
        if (!d_k || !d_v) return pc_fail(c, PC_ERR_INVALID_ARG, "%s: null d_k or d_v", what);
        if (!aligned(d_q, 16) || !aligned(d_k, 16) || !aligned(d_v, 16)) return pc_fail(c, PC_ERR_INVALID_ARG, "%s: d_q, d_k and d_v must be 16-byte aligned", what);
        if (to->q) rc = check_rows(c, what, "the gradient of q", to->q, to->q_stride, c->cfg.n_q_heads);
        if (rc == PC_OK) rc = check_rows(c, what, "the gradient of k", to->k, to->k_stride, c->cfg.n_kv_heads);
        if (rc == PC_OK) rc = check_rows(c, what, "the gradient of v", to->v, to->v_stride, c->cfg.n_kv_heads);
        if (rc != PC_OK) return rc;
        if (!aligned(to->q_weight, 4) || !aligned(to->k_weight, 4)) return pc_fail(c, PC_ERR_INVALID_ARG, "%s: weights must be 4-byte aligned", what);
    }
    std::vector<PcRowsBwdItem> items((size_t)n);
    int64_t row = 0, blocks = 0;
    for (int j = 0; j < n; ++j) {
        if (!known(c, msg_ids[j])) return pc_fail(c, PC_ERR_BAD_MSG_ID, "%s: unknown message %d", what, msg_ids[j]);
        const HostMsg &m = c->msgs[(size_t)msg_ids[j]];
        if (lens[j] < 1 || lens[j] > m.len) return pc_fail(c, PC_ERR_SHAPE, "%s: %d rows of message %d, whose first extent holds %d tokens", what, lens[j], msg_ids[j], m.len);
        items[(size_t)j] = PcRowsBwdItem{row, (int32_t)m.slot_start, m.base_pos, lens[j], 0};
        row += lens[j];
    }
    if (row > INT32_MAX) return pc_fail(c, PC_ERR_SHAPE, "%s: too many rows", what);
    if (c->host_only || n == 0) return PC_OK;
    PcDeviceScope on(c);
    if (!on.ok) return pc_fail(c, PC_ERR_HIP, "%s: the cache's device cannot be made current", what);
    if (pc_recorded(st)) return pc_fail(c, PC_ERR_INVALID_ARG, "%s: the stream is being captured, and the cache's workspace may move", what);
    // A block's rows, four at a time: few where there are few (a wave's steps follow each other: 160 rows of fp32 take 9.5 us in blocks
    // of 32 rows), more where blocks fill the chip anyway, so that there are fewer sums to add up behind it.
    const int64_t chunks = (p->q ? (c->cfg.n_q_heads + 7) / 8 : 0) + 2 * ((c->cfg.n_kv_heads + 7) / 8);
    const int32_t block_rows = (int32_t)std::max<int64_t>(4, std::min<int64_t>(64, row * chunks / 2048 / 4 * 4));
    for (PcRowsBwdItem &it : items) {
        it.block0 = (int32_t)blocks;
        blocks += (it.n + block_rows - 1) / block_rows;
    }
    if (blocks > MOST_BLOCKS) return pc_fail(c, PC_ERR_SHAPE, "%s: too many rows", what);
    PcRowsBwd B{};
    B.block_rows = block_rows;
    B.n_items = n; B.n_blocks = (int32_t)blocks;
    B.q = p->q; B.k = p->k; B.q_stride = p->q_stride; B.k_stride = p->k_stride;
    B.q_weight = p->q_weight; B.k_weight = p->k_weight; B.eps = p->eps;
    B.n_q_heads = c->cfg.n_q_heads; B.n_kv_heads = c->cfg.n_kv_heads; B.D = c->D;
    B.d_q = d_q; B.d_k = d_k; B.d_v = d_v;
    B.to_q = to->q; B.to_k = to->k; B.to_v = to->v;
    B.to_q_stride = to->q_stride; B.to_k_stride = to->k_stride; B.to_v_stride = to->v_stride;
    B.to_q_weight = to->q_weight; B.to_k_weight = to->k_weight;
    B.inv_freq = c->inv_freq_dev;
    // A few sums are added up by the block that is done last (a launch of its own is 4 us with what lies between the two), many by a second launch: one
    // block would read them one latency after the other.
    const int64_t q_chunks = to->q_weight ? (c->cfg.n_q_heads + 7) / 8 : 0, k_chunks = to->k_weight ? (c->cfg.n_kv_heads + 7) / 8 : 0;
    if (blocks * std::max(q_chunks, k_chunks) <= FEW_SUMS) { B.done = c->counters_dev + PC_ROWS_DONE; B.n_done = (uint32_t)(blocks * (q_chunks + k_chunks)); }
    const size_t part = sizeof(float) * (size_t)c->D * (size_t)blocks;
    const size_t q_bytes = align_up(part * (((size_t)c->cfg.n_q_heads + 7) / 8), 256), k_bytes = part * (((size_t)c->cfg.n_kv_heads + 7) / 8);
    rc = pc_ensure_ws(c, q_bytes + k_bytes, st);
    if (rc != PC_OK) return rc;
    B.q_part = (float *)c->ws; B.k_part = (float *)((char *)c->ws + q_bytes);
    PcArgBlob blob;
    bool in_args = false;
    rc = stage(c, items, blob, in_args, st);
    if (rc != PC_OK) return rc;
    B.items = (const PcRowsBwdItem *)c->tok_dev;
    ProfScope ps(c, 5, st);
    pc_forget_error();
    pc_launch_rows_backward(c->cfg.dtype, B, in_args ? &blob : nullptr, st);
    PC_HIP(c, hipGetLastError());
    return PC_OK;
}

int32_t messages_read(pc_cache *c, int32_t n, const int32_t *msg_ids, void *k, void *v, hipStream_t st)
{
    const char *what = "messages_read";
    if (n < 0 || (n > 0 && !msg_ids)) return pc_fail(c, PC_ERR_INVALID_ARG, "%s: bad id list", what);
    if (!c->host_only && (!aligned(k, 16) || !aligned(v, 16))) return pc_fail(c, PC_ERR_INVALID_ARG, "%s: k and v must be 16-byte aligned", what);
    std::vector<PcReadItem> items;
    int64_t row = 0, blocks = 0;
    for (int j = 0; j < n; ++j) {
        if (!known(c, msg_ids[j])) return pc_fail(c, PC_ERR_BAD_MSG_ID, "%s: unknown message %d", what, msg_ids[j]);
        for (int32_t r = msg_ids[j]; r >= 0; r = c->msgs[(size_t)r].next) {
            const HostMsg &m = c->msgs[(size_t)r];
            if (m.len == 0) continue;
            items.push_back(PcReadItem{row, (int32_t)m.slot_start, m.len, (int32_t)blocks, 0});
            row += m.len;
            blocks += (m.len + 7) / 8;
            if (blocks > MOST_BLOCKS) return pc_fail(c, PC_ERR_SHAPE, "%s: too many tokens", what);
        }
    }
    if (c->host_only || items.empty() || (!k && !v)) return PC_OK;
    PcDeviceScope on(c);
    if (!on.ok) return pc_fail(c, PC_ERR_HIP, "%s: the cache's device cannot be made current", what);
    if (pc_recorded(st)) return pc_fail(c, PC_ERR_INVALID_ARG, "%s: the stream is being captured", what);
    PcArgBlob blob;
    bool in_args = false;
    const int32_t rc = stage(c, items, blob, in_args, st);
    if (rc != PC_OK) return rc;
    const PcRead R{(const PcReadItem *)c->tok_dev, (int32_t)items.size(), (int32_t)blocks, c->cfg.n_kv_heads, c->D, c->slots, c->k_store, c->v_store, k, v};
    ProfScope ps(c, 0, st);
    pc_forget_error();
    pc_launch_read(c->cfg.dtype, R, in_args ? &blob : nullptr, st);
    PC_HIP(c, hipGetLastError());
    return PC_OK;
}

}  // namespace

int32_t pc_write_rows(pc_cache *c, PcRows R, std::vector<PcRowsItem> &items, hipStream_t st)
{
    PcDeviceScope on(c);
    if (!on.ok) return pc_fail(c, PC_ERR_HIP, "append: the cache's device cannot be made current");
    int64_t blocks = 0;
    for (PcRowsItem &it : items) {
        if (c->cfg.dtype == PC_MX4) it.rows = it.n;      // (nothing has to be cleared: see pc_mx4.h)
        const int32_t upto = it.fresh ? std::max(it.n, it.rows) : it.n;
        it.block0 = (int32_t)blocks;
        blocks += (it.slot0 % PC_ROWS_GROUP + upto + PC_ROWS_GROUP - 1) / PC_ROWS_GROUP;
    }
    R.n_items = (int32_t)items.size(); R.n_blocks = (int32_t)blocks;
    R.n_q_heads = c->cfg.n_q_heads; R.n_kv_heads = c->cfg.n_kv_heads; R.D = c->D;
    R.slots = c->slots; R.inv_freq = c->inv_freq_dev; R.k_store = c->k_store; R.v_store = c->v_store; R.table = c->table_dev; R.wide = c->counters_dev + PC_MX4_WIDE;
    PcArgBlob blob;
    bool in_args = false;
    const int32_t rc = stage(c, items, blob, in_args, st);
    if (rc != PC_OK) return rc;
    R.items = (const PcRowsItem *)c->tok_dev;
    ProfScope ps(c, 0, st);
    pc_forget_error();
    pc_launch_rows(c->cfg.dtype, R, in_args ? &blob : nullptr, st);
    PC_HIP(c, hipGetLastError());
    return PC_OK;
}

extern "C" {

int32_t pc_append_projected(pc_cache *c, const pc_projected *rows, int32_t n, const int32_t *lens, const int32_t *reserves, int32_t *msg_ids, void *q_out, void *stream)
{
    if (!c) return PC_ERR_INVALID_ARG;
    return pc_guarded(c, [&] { return append_projected(c, rows, n, lens, reserves, msg_ids, q_out, (hipStream_t)stream); });
}

int32_t pc_append_projected_tokens(pc_cache *c, const pc_projected *rows, const int32_t *msg_ids, int32_t n_msgs, void *q_out, void *stream)
{
    if (!c) return PC_ERR_INVALID_ARG;
    return pc_guarded(c, [&] { return append_projected_tokens(c, rows, msg_ids, n_msgs, q_out, (hipStream_t)stream); });
}

int32_t pc_projected_backward(pc_cache *c, const pc_projected *rows, int32_t n, const int32_t *msg_ids, const int32_t *lens, const float *d_q, const float *d_k,
                              const float *d_v, const pc_projected_grad *to, void *stream)
{
    if (!c) return PC_ERR_INVALID_ARG;
    return pc_guarded(c, [&] { return projected_backward(c, rows, n, msg_ids, lens, d_q, d_k, d_v, to, (hipStream_t)stream); });
}

int32_t pc_messages_read(pc_cache *c, int32_t n, const int32_t *msg_ids, void *k, void *v, void *stream)
{
    if (!c) return PC_ERR_INVALID_ARG;
    return pc_guarded(c, [&] { return messages_read(c, n, msg_ids, k, v, (hipStream_t)stream); });
}

}  // extern "C"
