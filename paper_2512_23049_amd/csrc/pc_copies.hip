// Host side of the cache's own copies: forks of messages, and the cache closing up.
#include "pc_host.h"
#include "pc_copies.h"
#include "pc_window.h"

namespace {

// A call's items (a multiple of 16 bytes) to tok_dev, read from the staging slot by a kernel: a copy by the copy engine, between two
// kernels of the stream, costs 12 us more.
int32_t fetch_items(pc_cache *c, const void *items, size_t bytes, hipStream_t st)
{
    int32_t rc = pc_items_room(c, bytes, st);
    if (rc != PC_OK) return rc;
    StageSlot *slot = nullptr;
    rc = pc_stage_acquire(c, bytes, &slot);
    if (rc != PC_OK) return rc;
    std::memcpy(slot->host, items, bytes);
    PcWinTurns T{};
    T.from = slot->host; T.ws = c->tok_dev; T.n16 = (int)(bytes / 16); T.D = c->D;
    pc_forget_error();                                   // (or the slot would not be released, with its reader enqueued)
    pc_launch_win_turns(T, nullptr, st);
    PC_HIP(c, hipGetLastError());
    return pc_stage_release(c, slot, st);
}

int32_t message_fork(pc_cache *c, const pc_fork *forks, int32_t n, int32_t *msg_ids, hipStream_t st)
{
    if (n < 0 || (n > 0 && (!forks || !msg_ids))) return pc_fail(c, PC_ERR_INVALID_ARG, "message_fork: bad lists");
    if (n == 0) return PC_OK;
    if ((int64_t)c->msgs.size() + n > c->cfg.max_messages)
        return pc_fail(c, PC_ERR_NO_SPACE, "message_fork: message table full (%d)", c->cfg.max_messages);
    // all or nothing: allocated on copies first
    std::vector<FreeSpan> spans = c->free_spans;
    int64_t next = c->next_slot;
    std::vector<PcForkItem> items((size_t)n);
    std::vector<PcForkPiece> pieces;
    std::vector<HostMsg> fresh((size_t)n);
    int max_rows = 0;
    for (int j = 0; j < n; ++j) {
        const pc_fork &f = forks[j];
        if (!known(c, f.msg_id)) return pc_fail(c, PC_ERR_BAD_MSG_ID, "message_fork: fork %d names unknown message %d", j, f.msg_id);
        const int64_t len = chain_len(c, f.msg_id);
        if (f.first < 0 || f.len < 1 || (int64_t)f.first + f.len > len)
            return pc_fail(c, PC_ERR_INVALID_ARG, "message_fork: fork %d takes tokens [%d, %lld) of the %lld of message %d", j, f.first,
                        (long long)f.first + f.len, (long long)len, f.msg_id);
        const int64_t stored = (int64_t)c->msgs[(size_t)f.msg_id].base_pos + f.first, base = f.base == PC_POS_AUTO ? stored : f.base;
        if (base > c->cfg.max_position || base < -(int64_t)c->cfg.max_position)
            return pc_fail(c, PC_ERR_INVALID_ARG, "message_fork: fork %d: position %lld outside [-%d, %d]", j, (long long)base, c->cfg.max_position,
                        c->cfg.max_position);
        const int32_t res = std::max(f.reserve, f.len);
        int64_t start = 0;
        if (!pc_take_slots(spans, next, c->slots, res, start))
            return pc_fail(c, PC_ERR_NO_SPACE, "message_fork: fork %d (%d slots) does not fit, capacity %lld", j, res, (long long)c->slots);
        fresh[(size_t)j] = HostMsg{start, f.len, res, (int32_t)base, true};
        PcForkItem &it = items[(size_t)j];
        // (whole tiles are written: what lies behind the last token of a fork's last tile is zero)
        it = PcForkItem{(int32_t)c->msgs.size() + j, (int32_t)start, f.len, (int32_t)align_up((size_t)pc_rows_to_write(c, start, f.len, res), PC_TILE), (int32_t)base,
                        (int32_t)pieces.size(), 0, 0, base - stored, 0};
        int64_t at = 0;                                  // the source's tokens in front of the extent
        for (int32_t r = f.msg_id; r >= 0; r = c->msgs[(size_t)r].next) {
            const HostMsg &m = c->msgs[(size_t)r];
            const int64_t from = std::max<int64_t>(at, f.first), to = std::min<int64_t>(at + m.len, (int64_t)f.first + f.len);
            if (from < to) pieces.push_back(PcForkPiece{(int32_t)(from - f.first), (int32_t)(to - from), (int32_t)(m.slot_start + (from - at)), 0});
            at += m.len;
        }
        it.n_pieces = (int32_t)pieces.size() - it.piece0;
        max_rows = std::max(max_rows, it.rows);
    }
    if (!c->host_only) {
        PcDeviceScope on(c);
        if (!on.ok) return pc_fail(c, PC_ERR_HIP, "message_fork: the cache's device cannot be made current");
        if (pc_recorded(st)) return pc_fail(c, PC_ERR_INVALID_ARG, "message_fork: the stream is being captured");
        const size_t n_items = sizeof(PcForkItem) * items.size(), bytes = n_items + sizeof(PcForkPiece) * pieces.size();
        const bool in_args = bytes <= PC_ARG_BYTES;
        PcArgBlob blob;
        std::vector<char> lists(in_args ? 0 : bytes);
        char *at = in_args ? (char *)blob.w : lists.data();
        std::memcpy(at, items.data(), n_items);
        std::memcpy(at + n_items, pieces.data(), sizeof(PcForkPiece) * pieces.size());
        const int32_t rc = in_args ? PC_OK : fetch_items(c, lists.data(), bytes, st);
        if (rc != PC_OK) return rc;
        c->msgs.reserve(c->msgs.size() + (size_t)n);     // (nothing may fail behind the launch)
        ProfScope ps(c, 0, st);
        pc_forget_error();
        pc_launch_fork(c->cfg.dtype, in_args ? &blob : nullptr, (const PcForkItem *)c->tok_dev, (const PcForkPiece *)((char *)c->tok_dev + n_items), n, max_rows, c->cfg.n_kv_heads, c->D,
                       c->slots, c->inv_freq_dev, c->k_store, c->v_store, c->table_dev, st);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) {                           // (of several launches some may have written: nobody's tokens, in slots that stay free)
            c->dirty_end = std::max(c->dirty_end, next);
            return pc_fail(c, PC_ERR_HIP, "message_fork: %s", hipGetErrorString(e));
        }
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

// The extents that hold slots, in slot order.  The last call's list is kept: what was freed since drops out, and what came since
// stands behind it in the table (a message that was swapped in again does not: then all of the table is looked through).
void live_extents(pc_cache *c, std::vector<int32_t> &order)
{
    size_t from = 0;
    if (!c->order_stale) { order = c->slot_order; from = c->order_seen; }
    order.erase(std::remove_if(order.begin(), order.end(), [&](int32_t r) { return !c->msgs[(size_t)r].live; }), order.end());
    for (size_t r = from; r < c->msgs.size(); ++r) if (c->msgs[r].live) order.push_back((int32_t)r);
    std::sort(order.begin(), order.end(), [&](int32_t a, int32_t b) { return c->msgs[(size_t)a].slot_start < c->msgs[(size_t)b].slot_start; });
}

int64_t span_of(const HostMsg &m) { return (int64_t)align_up((size_t)m.reserve, PC_SLOT_ALIGN); }

int32_t compact(pc_cache *c, int64_t max_slots, int64_t *slots_moved, hipStream_t st)
{
    if (max_slots < 0) return pc_fail(c, PC_ERR_INVALID_ARG, "cache_compact: max_slots = %lld must be >= 0", (long long)max_slots);
    if (!c->host_only && pc_recorded(st)) return pc_fail(c, PC_ERR_INVALID_ARG, "cache_compact: the stream is being captured");
    if (slots_moved) *slots_moved = 0;
    std::vector<int32_t> order;
    live_extents(c, order);
    std::vector<PcCompactMove> moves;
    int64_t next = 0, moved = 0;
    for (int32_t r : order) {
        const HostMsg &m = c->msgs[(size_t)r];
        const int64_t span = span_of(m);
        if (m.slot_start != next) {
            if (max_slots > 0 && moved > 0 && moved + span > max_slots) break;
            moves.push_back(PcCompactMove{r, (int32_t)next});
            moved += span;
        }
        next += span;
    }
    c->free_spans.reserve(order.size() + 1);             // (nothing may fail behind the launch)
    if (!moves.empty() && !c->host_only) {
        PcDeviceScope on(c);
        if (!on.ok) return pc_fail(c, PC_ERR_HIP, "cache_compact: the cache's device cannot be made current");
        const int32_t tile_bytes = (int32_t)(PC_TILE * c->D * c->esize), per = PC_COMPACT_BYTES / tile_bytes;
        // a list of tiles in slot order, the table's moves behind it
        const size_t n_tiles = (size_t)(moved / PC_TILE), at_moves = sizeof(PcCompactTile) * n_tiles;
        std::vector<char> lists(align_up(at_moves + sizeof(PcCompactMove) * moves.size(), 16));
        PcCompactTile *tiles = (PcCompactTile *)lists.data();
        size_t t = 0, behind = 0;                        // behind: the first tile whose source lies at or behind the place being written
        std::vector<int32_t> place(n_tiles);             // where each tile lies now, whether or not it holds tokens
        for (const PcCompactMove &mv : moves) {
            const HostMsg &m = c->msgs[(size_t)mv.rec];
            const int32_t n = (int32_t)(span_of(m) / PC_TILE), used = (m.len + PC_TILE - 1) / PC_TILE;
            for (int32_t i = 0; i < n; ++i, ++t) {
                const int32_t src = (int32_t)(m.slot_start / PC_TILE) + i, dst = mv.slot_start / PC_TILE + i;
                place[t] = src;
                while (behind < t && place[behind] < dst) ++behind;
                const bool over = behind < t && place[behind] == dst && tiles[behind].src >= 0;
                tiles[t] = PcCompactTile{i < used ? src : -1, dst, over ? (int32_t)(behind / (size_t)per) : -1, 0};
            }
        }
        std::memcpy(lists.data() + at_moves, moves.data(), sizeof(PcCompactMove) * moves.size());
        PcCompact C{};
        C.n_tiles = (int32_t)n_tiles; C.n_moves = (int32_t)moves.size();
        C.n_chunks = (int32_t)((n_tiles + per - 1) / per); C.n_stores = 2 * c->cfg.n_kv_heads;
        const size_t counters = (size_t)PC_COMPACT_COUNTER * C.n_stores, words = counters + (size_t)C.n_chunks * C.n_stores;
        if (words > c->flag_words) {                     // a counter for every store, then a flag for every chunk and store
            if (c->flags_dev) {
                PC_HIP(c, hipStreamSynchronize(st));
                PC_HIP(c, hipDeviceSynchronize());
                PC_HIP(c, hipFree(c->flags_dev));
            }
            c->flags_dev = nullptr; c->flag_words = 0; c->tickets = 0; c->flag_epoch = 0;
            const size_t cap = std::max<size_t>(2 * words, 1 << 14);
            PC_HIP(c, hipMalloc((void **)&c->flags_dev, sizeof(uint32_t) * cap));
            PC_HIP(c, hipMemsetAsync(c->flags_dev, 0, sizeof(uint32_t) * cap, st));
            c->flag_words = cap;                         // (cleared: not before, or a further call would take what is there for its flags)
        } else if (c->flag_epoch == UINT32_MAX) {        // the launches' numbers begin anew
            PC_HIP(c, hipMemsetAsync(c->flags_dev, 0, sizeof(uint32_t) * c->flag_words, st));
            c->tickets = 0; c->flag_epoch = 0;
        }
        const bool in_args = lists.size() <= PC_ARG_BYTES;
        PcArgBlob blob;
        if (in_args) std::memcpy(blob.w, lists.data(), lists.size());
        const int32_t rc = in_args ? PC_OK : fetch_items(c, lists.data(), lists.size(), st);
        if (rc != PC_OK) return rc;
        C.tiles = (const PcCompactTile *)c->tok_dev; C.moves = (const PcCompactMove *)((char *)c->tok_dev + at_moves);
        C.epoch = c->flag_epoch + 1; C.ticket0 = c->tickets;
        C.ticket = c->flags_dev; C.read = c->flags_dev + counters;
        C.k_store = (char *)c->k_store; C.v_store = (char *)c->v_store;
        C.head_bytes = c->slots * c->D * (int64_t)c->esize; C.tile_bytes = tile_bytes;
        C.table = c->table_dev;
        ProfScope ps(c, 7, st);
        pc_forget_error();
        pc_launch_compact(C, in_args ? &blob : nullptr, st);
        PC_HIP(c, hipGetLastError());                    // (the launch's own: nothing has moved)
        c->flag_epoch = C.epoch;
        c->tickets += (uint32_t)C.n_chunks;
    }
    if (!moves.empty()) c->dirty_end = std::max(c->dirty_end, c->next_slot);      // (what moved leaves itself behind)
    for (const PcCompactMove &mv : moves) c->msgs[(size_t)mv.rec].slot_start = mv.slot_start;
    c->free_spans.clear();
    int64_t end = 0;
    for (int32_t r : order) {
        const HostMsg &m = c->msgs[(size_t)r];
        if (m.slot_start > end) c->free_spans.push_back(FreeSpan{end, m.slot_start - end});
        end = m.slot_start + span_of(m);
    }
    c->next_slot = end;
    c->slot_order.swap(order);
    c->order_seen = c->msgs.size();
    c->order_stale = false;
    if (slots_moved) *slots_moved = moved;
    return PC_OK;
}

}  // namespace

extern "C" {

int32_t pc_message_fork(pc_cache *c, const pc_fork *forks, int32_t n, int32_t *msg_ids, void *stream)
{
    if (!c) return PC_ERR_INVALID_ARG;
    return pc_guarded(c, [&] { return message_fork(c, forks, n, msg_ids, (hipStream_t)stream); });
}

int32_t pc_cache_compact(pc_cache *c, int64_t max_slots, int64_t *slots_moved, void *stream)
{
    if (!c) return PC_ERR_INVALID_ARG;
    return pc_guarded(c, [&] { return compact(c, max_slots, slots_moved, (hipStream_t)stream); });
}

}  // extern "C"
