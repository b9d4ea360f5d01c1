// Host side of the windowed attention: what each group of rows sees as runs of tiles, work items, staging, entry points.
#include "pc_host.h"
#include "pc_window.h"

#include <new>
#include <queue>

namespace {

// One listed extent of a call, in list order.
struct Seg {
    int64_t rot_pos;
    int64_t before;           // tokens of the call's list in front of it
    int32_t slot0, start, len;
    int32_t rot;              // its row of the rotation table, -1: none yet
    bool self;
};
struct WinCall {
    int32_t q_off, n_q, lim0, own_first;      // own_first: index (within the last extent of the new message) of row 0's token
    size_t seg0, n_seg;
    int32_t row0, row1;                       // the rows that are planned for
};
struct WinPlan {
    std::vector<Resolved> res;
    std::vector<WinCall> calls;
    std::vector<Seg> segs;
    std::vector<int32_t> q_pos;
    std::vector<PcWinItem> pre, dec;
    std::vector<PcWinRun> runs;
    std::vector<size_t> run_seg;              // of each run: the entry it is a part of, in segs
    std::vector<int64_t> rots;
    std::vector<PcMergeRow> merge;
    int64_t part_rows = 0, part_first = 0;    // partial rows [part_first, part_rows) are used
    std::vector<int32_t> tiles, places;       // PC_MX4: first slots of the tiles that rows of prompts see, each once; of each of their runs, what is added to a slot
                                              // for its place among these
    int32_t window = 0, n_sink = 0;
    // single tokens of calls that list the same messages
    std::vector<PcWinSharedItem> sh_items;
    std::vector<PcWinVisit> sh_visits;
    std::vector<PcWinSee> sh_sees;
    std::vector<PcMx4See> sh_sees4;           // (PC_MX4) in their place
    std::vector<PcWinSharedCall> sh_calls;
    bool sh_wide = false;

    void clear()
    {
        each([](auto &v) { v.clear(); });
        part_rows = part_first = 0;
        sh_wide = false;
    }
    // what is not worth keeping from one call to the next
    void trim()
    {
        size_t held = 0;
        for (const Resolved &r : res) held += sizeof(Resolved) + 8 * (r.sel.capacity() + r.entry_start.capacity()) + 4 * r.q_pos.capacity();
        if (held > KEPT_BYTES) std::vector<Resolved>().swap(res);
        each([](auto &v) { keep(v); });
    }

private:
    template <typename F> void each(F &&f)               // (not res: its lists are written over)
    {
        f(calls); f(segs); f(q_pos); f(pre); f(dec); f(runs); f(run_seg); f(rots); f(merge); f(tiles); f(places); f(sh_items); f(sh_visits); f(sh_sees); f(sh_sees4); f(sh_calls);
    }
};

// (first: the number of calls[0] in the caller's list)
int32_t resolve_all(pc_cache *c, const pc_call *calls, int32_t n_calls, WinPlan &P, int32_t first = 0)
{
    P.res.resize((size_t)n_calls);
    P.calls.resize((size_t)n_calls);
    int64_t total_q = 0;
    size_t entries = 0;
    for (int i = 0; i < n_calls; ++i) entries += (size_t)std::max(calls[i].n_sel, 0) + 1;
    P.segs.reserve(entries);
    for (int i = 0; i < n_calls; ++i) {
        const int32_t rc = pc_resolve(c, &calls[i], first + i, P.res[(size_t)i]);
        if (rc != PC_OK) return rc;
        const Resolved &r = P.res[(size_t)i];
        WinCall &wc = P.calls[(size_t)i];
        wc.q_off = (int32_t)total_q; wc.n_q = r.n_q;
        wc.row0 = 0; wc.row1 = r.n_q;
        wc.own_first = r.self_msg >= 0 ? r.self_len - r.n_q : 0;
        wc.lim0 = r.self_msg >= 0 ? r.self_start + wc.own_first : 0;
        wc.seg0 = P.segs.size();
        int64_t before = 0;
        auto add = [&](int32_t rec, int32_t start, int32_t len, bool self) {
            const HostMsg &m = c->msgs[(size_t)rec];
            P.segs.push_back(Seg{(int64_t)start - m.base_pos, before, (int32_t)m.slot_start, start, len, -1, self});
            before += len;
        };
        for (const int2 &s : r.sel) add(s.x, s.y, c->msgs[(size_t)s.x].len, false);
        if (r.self_msg >= 0) add(r.self_msg, r.self_start, r.self_len, true);
        wc.n_seg = P.segs.size() - wc.seg0;
        P.q_pos.insert(P.q_pos.end(), r.q_pos.begin(), r.q_pos.end());
        total_q += r.n_q;
        if (total_q > INT32_MAX / 2) return pc_fail(c, PC_ERR_SHAPE, "attend_window: too many query rows");
    }
    return PC_OK;
}

// The runs that rows [row0, row1) of a call see, behind those there are; the number of their tiles.  rotations: their rows of the
// rotation table (single tokens' kernels make them themselves).
int32_t add_runs(WinPlan &P, const WinCall &wc, int32_t row0, int32_t row1, bool rotations = true)
{
    int32_t p_min = P.q_pos[(size_t)wc.q_off + row0];
    for (int32_t r = row0 + 1; r < row1; ++r) p_min = std::min(p_min, P.q_pos[(size_t)wc.q_off + r]);
    const int64_t low = win_low(p_min, P.window);
    int64_t tiles = 0;
    for (size_t i = wc.seg0; i < wc.seg0 + wc.n_seg; ++i) {
        Seg &s = P.segs[i];
        const int32_t end = s.self ? std::min(s.len, wc.own_first + row1) : s.len;
        const int64_t skip = std::max<int64_t>(0, low - s.start);       // tokens in front of the window
        const int32_t sinks = (int32_t)std::min<int64_t>(std::max<int64_t>(0, P.n_sink - s.before), end);
        if (skip >= end && sinks == 0) continue;
        if (s.rot < 0 && rotations) {
            if (P.rots.empty() || P.rots.back() != s.rot_pos) P.rots.push_back(s.rot_pos);
            s.rot = (int32_t)P.rots.size() - 1;
        }
        auto run = [&](int32_t first, int32_t n_tok) {                  // (first: a multiple of the tile)
            P.runs.push_back(PcWinRun{s.slot0 + first, s.start + first, n_tok, std::max(0, sinks - first), s.rot, s.self ? 1 : 0, s.rot_pos});
            P.run_seg.push_back(i);
            tiles += (n_tok + PC_TILE - 1) / PC_TILE;
        };
        const int32_t t0 = skip >= end ? end : (int32_t)skip / PC_TILE * PC_TILE, sink_end = (sinks + PC_TILE - 1) / PC_TILE * PC_TILE;
        if (skip < end && t0 <= sink_end) {
            run(0, end);                                 // (sinks and window touch, or there are no tokens in front of the window)
        } else {
            if (sinks > 0) run(0, sinks);
            if (skip < end) run(t0, end - t0);
        }
    }
    return (int32_t)tiles;
}

// A call's work for one group of rows, to be cut into splits.
struct Group { int32_t call, unit0, run0, tiles; };

// target: workgroups (of all KV heads) that fill the chip; least: tiles a split is worth
void make_items(const pc_cache *c, WinPlan &P, const std::vector<Group> &groups, std::vector<PcWinItem> &items, int64_t target, int32_t least, bool may_split, bool fit, bool tokens)
{
    const int H_kv = c->cfg.n_kv_heads;
    int64_t all = 0;
    for (const Group &gr : groups) all += gr.tiles;
    // a split's tiles: what brings the launch to its target (groups that are many already stay whole)
    int64_t chunk = may_split ? std::max<int64_t>(least, (all * H_kv + target - 1) / target) : INT32_MAX;            // (INT32_MAX: one)
    // (many groups: to the nearest, as one a little longer than the others is not worth a merge of its own)
    bool nearest = true;
    auto splits = [&](int32_t tiles) {
        if (tokens && tiles <= least + least / 2) return 1;           // (bf16: 10 tiles whole 8.0 us, halved 9.5, with the merge)
        return (int32_t)std::max<int64_t>(1, std::min<int64_t>((tiles + (nearest ? chunk / 2 : chunk - 1)) / chunk, MAX_SPLITS));
    };
    // fit: where whole groups have room at once, their splits get it too, and the longest is as short as that allows (fp32, two
    // calls of 100 to 500 rows, window 333, 2 KV heads: 17.2 -> 14.2 us; four single tokens of 17 tiles: 8.7 -> 7.7 us).  Not the bf16 blocks of rows, whose splits
    // pay for every run they touch: 33 groups of 20 tiles, 8 KV heads, take 47 us as 528 workgroups where 512 have room, 51 as 368.
    if (fit && may_split && (int64_t)groups.size() * H_kv <= target) {
        nearest = false;
        for (;; ++chunk) {
            int64_t n = 0;
            for (size_t a = 0; a < groups.size();) {
                size_t b = a;
                int32_t most = 0;
                while (b < groups.size() && groups[b].call == groups[a].call) most = std::max(most, groups[b++].tiles);
                n += (int64_t)(b - a) * splits(most);
                a = b;
            }
            if (n * H_kv <= target) break;
            chunk += chunk / 32;
        }
    }
    for (size_t a = 0; a < groups.size();) {
        size_t b = a;
        int32_t most = 0;
        while (b < groups.size() && groups[b].call == groups[a].call) most = std::max(most, groups[b++].tiles);
        const WinCall &wc = P.calls[(size_t)groups[a].call];
        const int32_t n = splits(most), n_rows = wc.row1 - wc.row0;
        const int64_t part0 = P.part_rows;               // (of row row0: part_rows start at part_first, or row 0's could be negative)
        for (int32_t s = 0; s < n; ++s)
            for (size_t i = a; i < b; ++i) {
                const Group &gr = groups[i];
                const int32_t t0 = (int32_t)((int64_t)gr.tiles * s / n), t1 = (int32_t)((int64_t)gr.tiles * (s + 1) / n);
                int32_t run = gr.run0, skip = t0;
                while (t0 < t1) {                        // (found here: a workgroup would look the runs up one after the other)
                    const int32_t has = (P.runs[(size_t)run].n_tok + PC_TILE - 1) / PC_TILE;
                    if (skip < has) break;
                    skip -= has; ++run;
                }
                items.push_back(PcWinItem{wc.q_off, wc.n_q, gr.unit0, wc.lim0, run, skip, t1 - t0, n == 1 ? -1 : (int32_t)(part0 + (int64_t)s * n_rows - wc.row0)});
            }
        if (n > 1) {
            for (int32_t r = wc.row0; r < wc.row1; ++r) P.merge.push_back(PcMergeRow{wc.q_off + r, (int32_t)(part0 + (r - wc.row0)), n, n_rows});
            P.part_rows += (int64_t)n * n_rows;
        }
        a = b;
    }
}

PcMx4See mx4_see(const PcWinSee &e)
{
    return PcMx4See{e.pos0, (uint32_t)std::min(e.n_tok, PC_MX4_SEE_TOKENS) | (uint32_t)((uint64_t)e.turn >> 32 & 3) << 26 | (uint32_t)e.sub << 28, e.sink, (uint32_t)e.turn};
}

// Single tokens by what they see together: the tiles that the calls of a set see, each once, in as many ranges as workgroups run at
// once.  False (and nothing is planned) where reading every call's own tiles is less, or a call lists a message twice.
bool plan_shared(const pc_cache *c, WinPlan &P, const std::vector<Group> &dec)
{
    const int H = c->cfg.n_kv_heads, g = c->g, per = 16 / g;
    const int32_t n_calls = (int32_t)dec.size(), n_groups = (n_calls + per - 1) / per;
    // (with two groups, waves would have every fourth step at most: 8 heads over 8, calls over 410 of 512 messages as below, call by call and
    // shared, 8 calls 84 and 160 us, 16 155 and 204, but 24 236 and 196, which are not taken)
    if (c->decode_sharing == 1 || n_calls < 2 || (c->decode_sharing == 0 && n_groups < 3)) return false;
    const bool wide = n_groups > PC_WIN_GROUPS / 2;
    const int32_t set_calls = std::min(n_groups, wide ? PC_WIN_GROUPS : PC_WIN_GROUPS / 2) * per, n_sets = (n_calls + set_calls - 1) / set_calls;
    // Microseconds of both ways, of the tiles that calls see on their own and of those that are distinct, and of the host: 7 ns for an
    // entry of a list, whichever way, and 15 for a run of tiles, of which the plan below makes visits.  At their prices before the
    // tiles are counted it is known of most small batches that sharing cannot gain.  Measured, call by call and shared:
    //   64 heads over 8, 410 of 512 messages of 160 tokens, window 16 384: 8 calls 83 and 120, 12 118 and 129, 16 155 and 141, 24 239 and 159,
    //   32 281 and 179; 24 of 48 messages, window 4096: 16 calls 35 and 40, 32 51 and 53, 64 84 and 64;
    //   32 heads over 8: 16 calls 155 and 147, 32 294 and 162; of 24 messages 32 calls 49 and 45;
    //   128 over 8: 12 calls 119 and 136, 16 156 and 153, 24 242 and 260, 32 291 and 267;
    //   16 over 2 (the host's time): 16 calls 66 and 93, 32 111 and 158, 64 203 and 305; 64 calls over 16 messages of 640 tokens 62 and 59.
    // 4 bits: a call's own tiles cost a quarter, a shared one what its waves need for it (call by call and shared, of 410 of 512 messages: 64 heads
    // over 8, 8 calls 102 and 142, 12 145 and 153, 16 181 and 160, 32 334 and 226, 64 614 and 448; 128 over 8, 32 calls 341 and 346; of 24 messages 16 calls 28
    // and 43, 64 calls 45 and 55; 64 calls over 32 of 64 messages of 400 tokens 115 and 102, 16 calls 44 and 73; a message of 2048 tokens and 8 of 512, 16 calls
    // 32 and 83, 64 calls 53 and 191).
    // By the caller's word: pc_set_decode_sharing.
    int64_t own = 0, listed = 0, shared = 0;
    for (const Group &gr : dec) { own += gr.tiles; listed += (int64_t)P.calls[(size_t)gr.call].n_seg; }
    const bool mx4 = c->cfg.dtype == PC_MX4;
    const double heads = H / 8.0, host = 12 + (mx4 ? 0.009 : 0.007) * (double)listed, planned = host + (mx4 ? 0.0075 : 0.015) * (double)(P.runs.size() - (size_t)dec[0].run0);
    const double alone = std::max(mx4 ? 20 + 0.0043 * (double)own * heads : 8 + 0.0175 * (double)own * heads, host);
    auto together = [&](int64_t tiles) {
        return std::max(mx4 ? 45 + (0.036 * (double)tiles + 0.0006 * (double)own) * heads : 48 + (0.0227 * (double)tiles + 0.0055 * (double)own) * heads, planned);
    };
    if (c->decode_sharing == 0 && alone <= together(own / set_calls)) return false;
    struct Piece { int32_t slot0, tiles; uint32_t run; int32_t call; };
    struct Visit { int32_t slot0, tiles; size_t p0, p1; };           // a range of consecutive tiles, and the pieces of it
    struct SetOf { size_t visit0; int64_t total; };                  // a set of calls: its first visit, and their tiles
    struct Seen { int32_t call; uint32_t seg; };                     // (call: within the set)
    struct Caller { int32_t q_pos, low, group, sub; };               // a call's place among the columns of its set
    struct Lists {
        std::vector<Piece> pieces, scratch;
        std::vector<uint32_t> digits;
        std::vector<SetOf> of_set;
        std::vector<Seen> seen;                          // who sees the visit at hand, and from which entry of its list; its views: P.sh_sees from e0 on
        std::vector<Visit> visits;
        std::vector<Caller> callers;
    };
    static thread_local Lists kept;
    struct Kept { ~Kept() { keep(kept.pieces); keep(kept.scratch); keep(kept.of_set); keep(kept.seen); keep(kept.visits); } } trim;
    auto &pieces = kept.pieces, &scratch = kept.scratch;
    auto &digits = kept.digits;
    auto &of_set = kept.of_set;
    auto &seen = kept.seen;
    auto &visits = kept.visits;
    auto &callers = kept.callers;
    pieces.clear(); of_set.clear(); visits.clear();
    pieces.reserve(P.runs.size() - (size_t)dec[0].run0);
    // pieces [first, size) by their slots, in the calls' order where those are the same: a pass for 13 bits of a tile's number
    constexpr uint32_t DIGIT = 13;
    digits.resize(1u << DIGIT);
    constexpr uint32_t MASK = (1u << DIGIT) - 1;
    auto by_slot = [&](size_t first, uint32_t most) {    // (digits: how often the lowest ones occur)
        scratch.resize(pieces.size());
        for (uint32_t shift = 0; shift == 0 || (shift < 32 && most >> shift); shift += DIGIT) {
            const uint32_t used = std::min(MASK, most >> shift);
            if (shift > 0) {
                std::fill(digits.begin(), digits.begin() + used + 1, 0u);
                for (size_t k = first; k < pieces.size(); ++k) ++digits[((uint32_t)pieces[k].slot0 / PC_TILE >> shift) & MASK];
            }
            uint32_t next = (uint32_t)first;
            for (uint32_t d = 0; d <= used; ++d) { const uint32_t count = digits[d]; digits[d] = next; next += count; }
            for (size_t k = first; k < pieces.size(); ++k) scratch[digits[((uint32_t)pieces[k].slot0 / PC_TILE >> shift) & MASK]++] = pieces[k];
            if (first == 0) pieces.swap(scratch);
            else std::memcpy(pieces.data() + first, scratch.data() + first, sizeof(Piece) * (pieces.size() - first));
        }
    };
    for (int32_t s = 0; s < n_sets; ++s) {
        const size_t first = pieces.size();
        uint32_t most = 0;
        std::fill(digits.begin(), digits.end(), 0u);
        for (int32_t j = s * set_calls; j < std::min(n_calls, (s + 1) * set_calls); ++j) {
            int32_t left = dec[(size_t)j].tiles;
            for (size_t r = (size_t)dec[(size_t)j].run0; left > 0; ++r) {
                const int32_t t = (P.runs[r].n_tok + PC_TILE - 1) / PC_TILE;
                const uint32_t tile = (uint32_t)P.runs[r].slot0 / PC_TILE;
                pieces.push_back(Piece{P.runs[r].slot0, t, (uint32_t)r, j});
                ++digits[tile & MASK];
                most = std::max(most, tile);
                left -= t;
            }
        }
        by_slot(first, most);
        // ranges of consecutive tiles
        const size_t visit0 = visits.size();
        int64_t total = 0;
        for (size_t k = first; k < pieces.size();) {
            Visit v{pieces[k].slot0, 0, k, k};
            for (; v.p1 < pieces.size() && (v.p1 == v.p0 || pieces[v.p1].slot0 < v.slot0 + PC_TILE * v.tiles); ++v.p1)
                v.tiles = std::max(v.tiles, (pieces[v.p1].slot0 - v.slot0) / PC_TILE + pieces[v.p1].tiles);
            total += v.tiles;
            visits.push_back(v);
            k = v.p1;
        }
        shared += total;
        of_set.push_back(SetOf{visit0, total});
    }
    const int64_t bins = std::max<int64_t>(1, std::min<int64_t>(256 / (H * n_sets), shared / n_sets / 8));
    if (shared == 0 || (c->decode_sharing == 0 && alone <= together(shared))) return false;
    if (mx4) P.sh_sees4.reserve(pieces.size() + pieces.size() / 4);
    else P.sh_sees.reserve(pieces.size() + pieces.size() / 4);
    for (int32_t s = 0; s < n_sets; ++s) {
        const int32_t call0 = s * set_calls, in_set = std::min(n_calls - call0, set_calls), groups = (in_set + per - 1) / per;
        int32_t waves = 1;
        while (waves < groups) waves *= 2;
        const int32_t reps = (wide ? 16 : 8) / waves;
        callers.clear();
        for (int32_t j = 0; j < in_set; ++j) {
            const int32_t q_pos = P.q_pos[(size_t)P.calls[(size_t)dec[(size_t)(call0 + j)].call].q_off];
            callers.push_back(Caller{q_pos, win_low(q_pos, P.window), j / per, j % per});
        }
        const int64_t total = of_set[(size_t)s].total;
        const int64_t n_bins = std::max<int64_t>(1, std::min(bins, total));
        const int32_t splits = (int32_t)n_bins * reps;
        size_t at = of_set[(size_t)s].visit0;
        int32_t done = 0;                                // tiles of visits[at] that earlier workgroups have
        for (int64_t b = 0; b < n_bins; ++b) {
            int32_t left = (int32_t)(total * (b + 1) / n_bins - total * b / n_bins);
            P.sh_items.push_back(PcWinSharedItem{(int32_t)P.sh_visits.size(), 0, call0, in_set, waves, (int32_t)b * reps, 0, 0});
            while (left > 0) {
                const Visit &v = visits[at];
                const int32_t n = std::min(left, v.tiles - done);
                if (mx4 && n > PC_MX4_SEE_TOKENS / PC_TILE) return false;
                const int32_t slot0 = v.slot0 + PC_TILE * done, slot1 = slot0 + PC_TILE * n;
                seen.clear();
                const size_t e0 = mx4 ? P.sh_sees4.size() : P.sh_sees.size();
                for (size_t k = v.p0; k < v.p1; ++k) {
                    const Piece pc = pieces[k];
                    if (k + 12 < pieces.size()) __builtin_prefetch(&P.runs[pieces[k + 12].run]);     // (they lie in the calls' order)
                    if (pc.slot0 >= slot1 || pc.slot0 + PC_TILE * pc.tiles <= slot0) continue;
                    const PcWinRun &r = P.runs[pc.run];
                    const int32_t d = slot0 - r.slot0;   // (what lies in front of a run is left out by its window)
                    const int32_t j = pc.call - call0;
                    const Caller &from = callers[(size_t)j];
                    const PcWinSee e{r.pos0 + d, r.n_tok - d, std::max(0, r.sink > 0 ? r.sink - d : 0), from.low, (int64_t)from.q_pos - r.rot_pos, from.sub, 0};
                    const uint32_t seg = (uint32_t)P.run_seg[pc.run];
                    if (seen.empty() || seen.back().call < j) {          // (in order, mostly)
                        seen.push_back(Seen{j, seg});
                        if (mx4) P.sh_sees4.push_back(mx4_see(e));
                        else P.sh_sees.push_back(e);
                        continue;
                    }
                    size_t i = seen.size();
                    while (i > 0 && seen[i - 1].call > j) --i;
                    if (i > 0 && seen[i - 1].call == j) {                // the sinks of an extent and its end: one view
                        if (seen[i - 1].seg != seg) return false;        // listed twice: two views, and a column has room for one
                        if (mx4) {
                            PcMx4See &o = P.sh_sees4[e0 + i - 1];
                            const PcMx4See w = mx4_see(e);
                            if ((w.packed & PC_MX4_SEE_TOKENS) > (o.packed & PC_MX4_SEE_TOKENS)) o.packed = w.packed;          // (a call's views of an extent are alike but for that)
                            o.sink = std::max(o.sink, w.sink);
                        } else {
                            PcWinSee &o = P.sh_sees[e0 + i - 1];
                            o.n_tok = std::max(o.n_tok, e.n_tok); o.sink = std::max(o.sink, e.sink);
                        }
                    } else {
                        seen.insert(seen.begin() + (ptrdiff_t)i, Seen{j, seg});
                        if (mx4) P.sh_sees4.insert(P.sh_sees4.begin() + (ptrdiff_t)(e0 + i), mx4_see(e));
                        else P.sh_sees.insert(P.sh_sees.begin() + (ptrdiff_t)(e0 + i), e);
                    }
                }
                PcWinVisit pv{slot0, n, (int32_t)e0, {}};
                size_t k = 0;
                for (int32_t gr = 0; gr <= PC_WIN_GROUPS; ++gr) {
                    while (k < seen.size() && callers[(size_t)seen[k].call].group < gr) ++k;
                    pv.off[gr] = (int32_t)k;
                }
                P.sh_visits.push_back(pv);
                ++P.sh_items.back().n_visits;
                P.sh_items.back().n_steps += (n + PC_WIN_STEP_TILES - 1) / PC_WIN_STEP_TILES;
                left -= n; done += n;
                if (done == v.tiles) { ++at; done = 0; }
            }
        }
        for (int32_t j = call0; j < call0 + in_set; ++j) {
            const WinCall &wc = P.calls[(size_t)dec[(size_t)j].call];
            P.sh_calls.push_back(PcWinSharedCall{wc.q_off, (int32_t)P.part_rows});
            P.merge.push_back(PcMergeRow{wc.q_off, (int32_t)P.part_rows, splits, 1});
            P.part_rows += splits;
        }
    }
    P.sh_wide = wide;
    return true;
}

// The tiles that the runs name, each once, in slot order, and the runs' places among these (consecutive tiles stay consecutive).
void list_tiles(WinPlan &P)
{
    P.tiles.clear(); P.places.clear();
    std::vector<std::pair<int32_t, int32_t>> spans;      // slots [first, second)
    for (const PcWinRun &r : P.runs) spans.push_back({r.slot0, r.slot0 + (r.n_tok + PC_TILE - 1) / PC_TILE * PC_TILE});
    std::sort(spans.begin(), spans.end());
    std::vector<std::pair<int32_t, int32_t>> first;      // a joined span's first slot, and its place
    int32_t end = -1;
    for (const auto &s : spans) {
        if (s.first > end || first.empty()) { first.push_back({s.first, (int32_t)P.tiles.size() * PC_TILE}); end = s.first; }
        for (; end < s.second; end += PC_TILE) P.tiles.push_back(end);
    }
    for (const PcWinRun &r : P.runs) {
        const auto it = std::upper_bound(first.begin(), first.end(), std::make_pair(r.slot0, INT32_MAX)) - 1;
        P.places.push_back(it->second - it->first);
    }
}

// Everything a forward call launches: rows of prompts in groups of four units (bf16: 32 rows x head; fp32: blocks of 32 columns, single
// tokens too), with the runs that each group sees, then single tokens, shared or call by call.  may_split: or every group is one
// item; least: tiles that a split of a single token is worth.
void plan_items(const pc_cache *c, WinPlan &P, bool may_split, int32_t least = 0)
{
    if (least == 0) least = c->cfg.dtype == PC_MX4 ? 24 : 8;             // (a workgroup of a 4-bit cache's tokens is eight waves: three tiles each)
    const int g = c->g;
    P.pre.clear(); P.dec.clear(); P.runs.clear(); P.run_seg.clear(); P.rots.clear(); P.merge.clear();
    auto no_shared = [&] { P.sh_items.clear(); P.sh_visits.clear(); P.sh_sees.clear(); P.sh_sees4.clear(); P.sh_calls.clear(); };
    no_shared();
    P.part_rows = 0;
    for (Seg &s : P.segs) s.rot = -1;
    std::vector<Group> pre, dec;
    for (size_t i = 0; i < P.calls.size(); ++i) {
        const WinCall &wc = P.calls[i];
        if (c->cfg.dtype == PC_F32) {
            const int64_t cols = (int64_t)wc.n_q * g;
            for (int64_t u = 0; u * 32 < cols; ++u) {
                const int32_t run0 = (int32_t)P.runs.size(), row0 = (int32_t)(32 * u / g), row1 = (int32_t)(std::min(32 * u + 31, cols - 1) / g) + 1;
                const int32_t tiles = add_runs(P, wc, row0, row1);
                pre.push_back(Group{(int32_t)i, (int32_t)u, run0, tiles});
            }
        } else if (wc.n_q > 1) {
            const int32_t n_units = (wc.n_q + 31) / 32 * g;
            int32_t b0 = -1, b1 = -1, run0 = 0, tiles = 0;
            for (int32_t u = 0; u < n_units; u += 4) {
                const int32_t first = u / g, last = std::min(u + 3, n_units - 1) / g;
                if (first != b0 || last != b1) {         // (workgroups over the same rows share a list)
                    b0 = first; b1 = last;
                    run0 = (int32_t)P.runs.size();
                    tiles = add_runs(P, wc, 32 * first, std::min(32 * (last + 1), wc.n_q));
                }
                pre.push_back(Group{(int32_t)i, u, run0, tiles});
            }
        }
    }
    make_items(c, P, pre, P.pre, 512, c->cfg.dtype == PC_F32 ? 4 : 6, may_split, c->cfg.dtype == PC_F32, false);
    if (c->cfg.dtype == PC_F32) return;
    const size_t runs = P.runs.size(), rots = P.rots.size(), merge = P.merge.size();
    const int64_t part_rows = P.part_rows;
    if (c->cfg.dtype == PC_MX4) list_tiles(P);
    size_t entries = 0;
    for (const WinCall &wc : P.calls) if (wc.n_q == 1) entries += wc.n_seg;
    P.runs.reserve(runs + entries); P.run_seg.reserve(runs + entries);           // (a little more where calls have sinks in front of their windows)
    for (size_t i = 0; i < P.calls.size(); ++i) {
        if (P.calls[i].n_q != 1) continue;
        const int32_t run0 = (int32_t)P.runs.size(), tiles = add_runs(P, P.calls[i], 0, 1, false);
        dec.push_back(Group{(int32_t)i, 0, run0, tiles});
    }
    P.rots.resize(rots);                                 // (single tokens' kernels make their rotations themselves)
    if (may_split && plan_shared(c, P, dec)) { P.runs.resize(runs); P.run_seg.resize(runs); return; }
    no_shared();
    P.merge.resize(merge); P.part_rows = part_rows;
    make_items(c, P, dec, P.dec, 512, least, may_split, true, true);
}

// lists as they are staged, then what the device makes of them
struct WinLayout { size_t pre, dec, runs, merge, q_pos, rots, sh_items, sh_visits, sh_sees, sh_calls, tiles, places, lists, rot_q, rot_run, part_o, part_ml, q_abs, q_unit, v_tiles, total; };

WinLayout lay_out(const pc_cache *c, const WinPlan &P)
{
    WinLayout L;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t a = at; at = align_up(at + bytes, 16); return a; };
    L.pre = take(sizeof(PcWinItem) * P.pre.size());
    L.dec = take(sizeof(PcWinItem) * P.dec.size());
    L.runs = take(sizeof(PcWinRun) * P.runs.size());
    L.merge = take(sizeof(PcMergeRow) * P.merge.size());
    L.q_pos = take(sizeof(int32_t) * P.q_pos.size());
    L.rots = take(sizeof(int64_t) * P.rots.size());
    L.sh_items = take(sizeof(PcWinSharedItem) * P.sh_items.size());
    L.sh_visits = take(sizeof(PcWinVisit) * P.sh_visits.size());
    L.sh_sees = take(sizeof(PcWinSee) * P.sh_sees.size() + sizeof(PcMx4See) * P.sh_sees4.size());         // (one of them)
    L.sh_calls = take(sizeof(PcWinSharedCall) * P.sh_calls.size());
    L.tiles = take(sizeof(int32_t) * P.tiles.size());
    L.places = take(sizeof(int32_t) * P.places.size());
    L.lists = at;
    auto big = [&](size_t bytes) { const size_t a = align_up(at, 256); at = a + bytes; return a; };
    const size_t rot = P.pre.empty() ? 0 : sizeof(float2) * (size_t)c->half;
    const bool mx4 = c->cfg.dtype == PC_MX4;
    L.rot_q = big(mx4 ? 0 : (c->cfg.dtype == PC_BF16 ? rot / 2 : rot) * align_up(P.q_pos.size(), 32));         // (bf16: rot_lanes)
    L.rot_run = big(rot * P.rots.size());
    L.part_o = big(sizeof(float) * (size_t)P.part_rows * (size_t)c->cfg.n_q_heads * (size_t)c->D);
    L.part_ml = big(sizeof(float) * 2 * (size_t)P.part_rows * (size_t)c->cfg.n_q_heads);
    const size_t turned = mx4 && !P.pre.empty() ? align_up(P.q_pos.size(), 32) * (size_t)c->cfg.n_q_heads : 0;
    L.q_abs = big(sizeof(uint16_t) * (size_t)c->D * turned);
    L.q_unit = big(sizeof(float) * turned);
    L.v_tiles = big((size_t)PC_TILE * (size_t)c->D * c->esize * (size_t)c->cfg.n_kv_heads * P.tiles.size());
    L.total = align_up(at, 256);
    return L;
}

void write_lists(const WinPlan &P, const WinLayout &L, char *to)
{
    auto put = [&](size_t at, const auto &v) { if (!v.empty()) std::memcpy(to + at, v.data(), sizeof(v[0]) * v.size()); };
    put(L.pre, P.pre); put(L.dec, P.dec); put(L.runs, P.runs); put(L.merge, P.merge); put(L.q_pos, P.q_pos); put(L.rots, P.rots);
    put(L.sh_items, P.sh_items); put(L.sh_visits, P.sh_visits); put(L.sh_sees, P.sh_sees); put(L.sh_sees, P.sh_sees4); put(L.sh_calls, P.sh_calls); put(L.tiles, P.tiles); put(L.places, P.places);
}

// ---- the gradient -------------------------------------------------------------------------------------------------
constexpr size_t BWD_BYTES = (size_t)256 << 20;          // workspace that a run's blocks may take

struct BwdPlan {
    std::vector<PcWinBlock> blocks;
    std::vector<PcWinApp> apps;
    std::vector<PcWinKeyItem> keys;
    std::vector<PcWinSum> sums;
    std::vector<PcWinTurned> turned;
    std::vector<int32_t> bins;                           // the first of each workgroup's items of keys, and their end
    int32_t parts = 0;
};

// One run over some blocks of the calls: call i's [range[i].x, range[i].y).
void plan_backward(const pc_cache *c, WinPlan &P, BwdPlan &B, const std::vector<int2> &range)
{
    const int g = c->g, H_kv = c->cfg.n_kv_heads;
    const bool f32 = c->cfg.dtype == PC_F32;
    P.pre.clear(); P.dec.clear(); P.runs.clear(); P.run_seg.clear(); P.rots.clear(); P.merge.clear();
    for (Seg &s : P.segs) s.rot = -1;
    B = BwdPlan{};
    std::vector<Group> groups;
    std::vector<int32_t> block0(P.calls.size()), low;     // a call's first block in the run; the least position each block sees
    auto rows_of = [&](const WinCall &wc, int32_t b) {
        return f32 ? make_int2((int)((int64_t)32 * b / g), (int)std::min<int64_t>(wc.n_q, ((int64_t)32 * b + 31) / g + 1)) : make_int2(32 * b, std::min(32 * b + 32, wc.n_q));
    };
    for (size_t i = 0; i < P.calls.size(); ++i) {
        WinCall &wc = P.calls[i];
        block0[i] = (int32_t)B.blocks.size();
        if (range[i].x >= range[i].y) { wc.row0 = wc.row1 = 0; continue; }
        wc.row0 = rows_of(wc, range[i].x).x; wc.row1 = rows_of(wc, range[i].y - 1).y;
        for (int32_t b = range[i].x; b < range[i].y; ++b) {
            const int2 r = rows_of(wc, b);
            int32_t p_min = INT32_MAX;
            for (int32_t k = r.x; k < r.y; ++k) p_min = std::min(p_min, P.q_pos[(size_t)wc.q_off + k]);
            low.push_back(win_low(p_min, P.window));
            B.blocks.push_back(PcWinBlock{wc.q_off, wc.n_q, wc.lim0, b});
            if (f32) {
                const int32_t run0 = (int32_t)P.runs.size(), tiles = add_runs(P, wc, r.x, r.y);
                groups.push_back(Group{(int32_t)i, b, run0, tiles});
            }
        }
        if (!f32) {
            const int32_t n_units = range[i].y * g;
            int32_t b0 = -1, b1 = -1, run0 = 0, tiles = 0;
            for (int32_t u = range[i].x * g; u < n_units; u += 4) {
                const int32_t first = u / g, last = std::min(u + 3, n_units - 1) / g;
                if (first != b0 || last != b1) {
                    b0 = first; b1 = last;
                    run0 = (int32_t)P.runs.size();
                    tiles = add_runs(P, wc, 32 * first, std::min(32 * (last + 1), wc.n_q));
                }
                groups.push_back(Group{(int32_t)i, u, run0, tiles});
            }
        }
    }
    P.part_first = 0;                                    // (a run's first call alone can begin behind its row 0)
    for (const WinCall &wc : P.calls) P.part_first = std::max<int64_t>(P.part_first, wc.row0);
    P.part_rows = P.part_first;
    make_items(c, P, groups, P.pre, 512, 6, true, f32, false);

    // keys: who lists each extent, extents in slot order
    struct Listed { int32_t slot0; uint32_t call, seg; };
    std::vector<Listed> listed;
    for (size_t i = 0; i < P.calls.size(); ++i)
        if (range[i].x < range[i].y)
            for (size_t k = P.calls[i].seg0; k < P.calls[i].seg0 + P.calls[i].n_seg; ++k) listed.push_back(Listed{P.segs[k].slot0, (uint32_t)i, (uint32_t)k});
    std::stable_sort(listed.begin(), listed.end(), [](const Listed &a, const Listed &b) { return a.slot0 < b.slot0; });
    struct Tiles { int32_t slot0, n_keys; size_t app0, n_apps; int64_t blocks; };
    std::vector<Tiles> all;
    std::vector<PcWinApp> apps;
    constexpr int32_t KEYS = PC_WIN_KEY_TILES * PC_TILE;
    for (size_t a = 0; a < listed.size();) {
        size_t b = a;
        while (b < listed.size() && listed[b].slot0 == listed[a].slot0) ++b;
        const int32_t len = P.segs[listed[a].seg].len;
        for (int32_t first = 0; first < len; first += KEYS) {
            Tiles t{listed[a].slot0 + first, std::min(KEYS, len - first), apps.size(), 0, 0};
            for (size_t k = a; k < b; ++k) {
                const WinCall &wc = P.calls[listed[k].call];
                Seg &s = P.segs[listed[k].seg];
                const int32_t end = s.self ? std::min(s.len, wc.own_first + wc.row1) : s.len;
                if (first >= end) continue;
                const int32_t sinks = (int32_t)std::min<int64_t>(std::max<int64_t>(0, P.n_sink - s.before - first), end - first);
                const int32_t last_pos = s.start + std::min(first + KEYS, end) - 1;
                const int2 rg = range[listed[k].call];
                int32_t b0 = -1, b1 = -1;
                for (int32_t bl = rg.x; bl < rg.y; ++bl) {
                    const bool sees = (sinks > 0 || low[(size_t)(block0[listed[k].call] + bl - rg.x)] <= last_pos) && (!s.self || wc.own_first + rows_of(wc, bl).y - 1 >= first);
                    if (!sees) continue;
                    if (b0 < 0) b0 = bl;
                    b1 = bl + 1;
                }
                if (b0 < 0) continue;
                if (s.rot < 0) {
                    if (P.rots.empty() || P.rots.back() != s.rot_pos) P.rots.push_back(s.rot_pos);
                    s.rot = (int32_t)P.rots.size() - 1;
                }
                apps.push_back(PcWinApp{s.start + first, end - first, sinks, s.rot, s.self ? 1 : 0, block0[listed[k].call] + b0 - rg.x, b1 - b0, block0[listed[k].call] + b0 - rg.x});
                t.blocks += b1 - b0;
            }
            t.n_apps = apps.size() - t.app0;
            if (t.n_apps > 0) all.push_back(t);
        }
        a = b;
    }
    // Rows of few keys: the forward's queries for every extent (see the kernels), if they are eight times a block's own at most (8 KB each; with
    // more extents a row mostly sees more keys, and has less need of them).
    int64_t visits = 0;
    for (const PcWinApp &a : apps) visits += a.n_blocks;
    if (!f32 && (int64_t)P.window + P.n_sink <= PC_WIN_FEW && visits <= 8 * (int64_t)B.blocks.size()) {
        const int32_t none = (int32_t)P.rots.size();
        P.rots.push_back(0);                             // (keys as they are stored: turned by nothing)
        for (PcWinApp &a : apps) {
            a.q0 = (int32_t)B.turned.size();
            for (int32_t b = 0; b < a.n_blocks; ++b) B.turned.push_back(PcWinTurned{a.block0 + b, a.rot});
            a.rot = none;
        }
    }
    // The items go to as many workgroups as run at once (a further one would wait for a place in a part of the chip that is not the
    // first to have one): the longest first, each to the workgroup with the least.  Tiles with more than a share of the work (those
    // that every row sees, messages that many calls list) are cut and their parts added up; smaller shares balance better and cost
    // more starts, so the best of a few is taken.  Work is counted in units of bf16 (32 columns of fp32 take four
    // times as long); an item's start and end are worth six, a call's two.
    const int64_t per_block = f32 ? 4 : g, bins = std::max<int64_t>(1, 256 / H_kv);
    auto cost = [&](int64_t n_blocks, int64_t n_apps) { return n_blocks * per_block + 2 * n_apps + 6; };
    int64_t total = 0;
    for (const Tiles &t : all) total += cost(t.blocks, (int64_t)t.n_apps);
    struct Keys { std::vector<PcWinApp> apps; std::vector<PcWinKeyItem> items; std::vector<PcWinSum> sums; std::vector<int32_t> bins; int32_t parts = 0; int64_t worst = INT64_MAX; } best;
    for (int64_t cut = 1; cut <= 3; ++cut) {
        const int64_t share = std::max<int64_t>(16, (total + bins * cut - 1) / (bins * cut));
        Keys K;
        std::vector<int64_t> size;
        for (const Tiles &t : all) {
            const int64_t n = std::min<int64_t>({(cost(t.blocks, (int64_t)t.n_apps) + share - 1) / share, std::max<int64_t>(1, t.blocks / 2), 1024});
            const int32_t part0 = K.parts;
            size_t k = t.app0;
            int32_t taken = 0;                           // blocks of app k that earlier parts have
            int64_t done = 0;
            for (int64_t part = 0; part < n; ++part) {
                const int64_t first = done, upto = t.blocks * (part + 1) / n;
                PcWinKeyItem it{t.slot0, t.n_keys, (int32_t)K.apps.size(), 0, n == 1 ? -1 : part0 + (int32_t)part, {0, 0, 0}};
                while (done < upto) {
                    const int32_t m = (int32_t)std::min<int64_t>(apps[k].n_blocks - taken, upto - done);
                    PcWinApp app = apps[k];
                    app.block0 += taken; app.q0 += taken; app.n_blocks = m;
                    K.apps.push_back(app);
                    done += m; taken += m;
                    if (taken == apps[k].n_blocks) { ++k; taken = 0; }
                }
                it.n_apps = (int32_t)K.apps.size() - it.app0;
                K.items.push_back(it);
                size.push_back(cost(done - first, it.n_apps));
            }
            if (n > 1) {                                 // (parts stand where their numbers say, whatever their order)
                K.sums.push_back(PcWinSum{t.slot0, t.n_keys, part0, (int32_t)n});
                K.parts += (int32_t)n;
            }
        }
        std::vector<uint32_t> by(K.items.size());
        for (size_t i = 0; i < by.size(); ++i) by[i] = (uint32_t)i;
        std::stable_sort(by.begin(), by.end(), [&](uint32_t x, uint32_t y) { return size[x] > size[y]; });
        const size_t n_bins = std::min<size_t>(by.size(), (size_t)bins);
        std::vector<std::vector<uint32_t>> in(n_bins);
        std::priority_queue<std::pair<int64_t, uint32_t>, std::vector<std::pair<int64_t, uint32_t>>, std::greater<>> least;
        for (size_t i = 0; i < n_bins; ++i) least.push({0, (uint32_t)i});
        K.worst = 0;
        for (uint32_t i : by) {
            const auto [load, bin] = least.top();
            least.pop();
            in[bin].push_back(i);
            K.worst = std::max(K.worst, load + size[i]);
            least.push({load + size[i], bin});
        }
        if (K.worst >= best.worst) continue;
        std::vector<PcWinKeyItem> sorted;
        for (const auto &list : in) {
            K.bins.push_back((int32_t)sorted.size());
            for (uint32_t i : list) sorted.push_back(K.items[i]);
        }
        K.bins.push_back((int32_t)sorted.size());
        K.items.swap(sorted);
        best = std::move(K);
    }
    B.apps.swap(best.apps); B.keys.swap(best.items); B.sums.swap(best.sums); B.bins.swap(best.bins);
    B.parts = best.parts;
}

int32_t check(pc_cache *c, const char *what, const pc_call *calls, int32_t n_calls, int32_t window, int32_t n_sink)
{
    if (n_calls < 0 || (n_calls > 0 && !calls)) return pc_fail(c, PC_ERR_INVALID_ARG, "%s: bad call list", what);
    if (window < 1) return pc_fail(c, PC_ERR_INVALID_ARG, "%s: window = %d must be >= 1", what, window);
    if (n_sink < 0) return pc_fail(c, PC_ERR_INVALID_ARG, "%s: n_sink = %d must be >= 0", what, n_sink);
    return PC_OK;
}

// What the resolved calls launch, and where it stands in the workspace.  marked: for a walk that mostly does nothing: no splits, and with them no merge.
int32_t plan_window(pc_cache *c, const char *what, const void *fixed_ws, bool recorded, bool marked, WinPlan &P, WinLayout &L)
{
    plan_items(c, P, !marked);
    L = lay_out(c, P);
    // Lists of single tokens that their launch's arguments do not hold cost a launch in front of it and the event behind that, 7 us: a few
    // longer splits are better where that helps (4 calls of 130 tiles: 22.5 -> 16.5 us; 16 of 17: 19 -> 12).
    const size_t whole = sizeof(PcWinRun) * P.runs.size() + (sizeof(PcWinItem) + sizeof(int32_t)) * P.calls.size();
    if (L.lists > PC_ARG_BYTES && whole + 64 <= PC_ARG_BYTES && P.pre.empty() && P.sh_items.empty()) {
        for (int32_t least = 16; least <= 40 && L.lists > PC_ARG_BYTES; least += 8) {
            plan_items(c, P, true, least);
            L = lay_out(c, P);
        }
        if (L.lists > PC_ARG_BYTES) {
            plan_items(c, P, true);
            L = lay_out(c, P);
        }
    }
    // (what cannot grow holds the plan without splits, if not the one with them)
    if (fixed_ws && (L.total > PC_STATIC_WS_BYTES || (!recorded && L.lists > STAGE_BYTES))) {
        plan_items(c, P, false);
        L = lay_out(c, P);
        if (L.total > PC_STATIC_WS_BYTES)
            return pc_fail(c, PC_ERR_NO_SPACE, "%s: needs a workspace of %zu bytes, the fixed one has %zu", what, L.total, PC_STATIC_WS_BYTES);
    }
    return PC_OK;
}

// The launches of a planned call.  mark: 0, or: nothing is done unless the cache's mark is that (PC_MX4, calls of many rows)
int32_t launch_window(pc_cache *c, const char *what, const WinPlan &P, const WinLayout &L, const void *q, void *out, float *lse, hipStream_t st, void *fixed_ws,
                      bool recorded, uint32_t mark)
{
    int32_t rc = PC_OK;
    const bool in_args = L.lists <= PC_ARG_BYTES;
    StageSlot *slot = nullptr;
    std::vector<char> held;                              // lists of a call that is recorded (see pc_recorded)
    PcArgBlob blob;
    if (!in_args && !recorded && fixed_ws && L.lists > STAGE_BYTES)
        return pc_fail(c, PC_ERR_NO_SPACE, "%s: lists of %zu bytes, a staging slot has %zu", what, L.lists, STAGE_BYTES);
    if (!in_args && recorded) held.resize(align_up(L.lists, 16));
    if (!fixed_ws) {
        rc = pc_ensure_ws(c, L.total, st);
        if (rc != PC_OK) return rc;
    }
    if (!in_args && !recorded) {
        rc = pc_stage_acquire(c, L.lists, &slot);
        if (rc != PC_OK) return rc;
    }
    char *ws = (char *)(fixed_ws ? fixed_ws : c->ws);
    char *from = in_args ? (char *)blob.w : recorded ? held.data() : (char *)slot->host;
    write_lists(P, L, from);

    const bool bf16 = c->cfg.dtype != PC_F32, mx4 = c->cfg.dtype == PC_MX4;
    PcWin W{};
    W.runs = (const PcWinRun *)(ws + L.runs);
    W.q_pos = (const int32_t *)(ws + L.q_pos);
    W.rot_q = (const float2 *)(ws + L.rot_q); W.rot_lanes = (const uint32_t *)(ws + L.rot_q); W.rot_run = (const float2 *)(ws + L.rot_run);
    W.inv_freq = c->inv_freq_dev;
    W.k_store = c->k_store; W.v_store = c->v_store; W.q = q; W.out = out; W.lse = lse;
    W.part_o = (float *)(ws + L.part_o); W.part_ml = (float *)(ws + L.part_ml);
    W.slots = c->slots; W.n_q_heads = c->cfg.n_q_heads; W.n_kv_heads = c->cfg.n_kv_heads;
    W.window = P.window;
    W.scale_log2 = c->scale * 1.4426950408889634f;
    // Lists in the arguments of the decode launch are read there; everything else reads them from the workspace.
    const bool direct = in_args && P.pre.empty() && P.sh_items.empty();
    pc_forget_error();
    if (!direct) {
        ProfScope ps(c, 1, st);
        if (recorded && !in_args) pc_launch_store_args(from, L.lists, ws, st);
        const bool turns = !P.pre.empty();
        if (mx4 && turns) {
            PcMx4Prepare T{};
            T.from = in_args || recorded ? ws : slot->host; T.ws = ws; T.n16 = (int)(L.lists / 16);
            T.off_q_pos = (int)L.q_pos; T.off_rot = (int)L.rots; T.off_tiles = (int)L.tiles;
            T.n_rows = (int)P.q_pos.size(); T.n_rot = (int)P.rots.size(); T.n_tiles = (int)P.tiles.size();
            T.n_q_heads = W.n_q_heads; T.n_kv_heads = W.n_kv_heads; T.scale_log2 = W.scale_log2;
            T.rot_run = (_Float16 *)(ws + L.rot_run);
            T.q = q; T.q_abs = (uint2 *)(ws + L.q_abs); T.q_unit = (float *)(ws + L.q_unit);
            T.inv_freq = c->inv_freq_dev; T.slots = c->slots; T.v_store = c->v_store; T.v_to = ws + L.v_tiles;
            T.bf16_only = c->counters_dev + PC_MX4_WIDE;
            if (mark) { T.mark = c->counters_dev + PC_MX4_MARK; T.mark_value = mark; }
            pc_launch_mx4_prepare(T, in_args ? &blob : nullptr, st);
        } else {
        PcWinTurns T{};
        T.from = in_args || recorded ? ws : slot->host; T.ws = ws; T.n16 = (int)(L.lists / 16);
        T.off_q_pos = (int)L.q_pos; T.n_rows = turns ? (int)P.q_pos.size() : 0;
        T.off_rot = (int)L.rots; T.n_rot = turns ? (int)P.rots.size() : 0;
        T.D = c->D;
        T.run_scale = bf16 ? W.scale_log2 : 1.f;
        if (bf16) T.rot_lanes = (uint32_t *)(ws + L.rot_q);
        else T.rot_q = (float2 *)(ws + L.rot_q);
        T.rot_run = (float2 *)(ws + L.rot_run);
        T.inv_freq = c->inv_freq_dev;
        if (!(recorded && !in_args) || turns) pc_launch_win_turns(T, in_args ? &blob : nullptr, st);
        }
        PC_HIP(c, hipGetLastError());
        if (slot) { rc = pc_stage_release(c, slot, st); if (rc != PC_OK) return rc; }
    }
    if (!P.dec.empty()) {
        ProfScope ps(c, 3, st);
        W.items = (const PcWinItem *)(ws + L.dec);
        const PcWinDecode O{(int32_t)L.dec, (int32_t)L.runs, (int32_t)L.q_pos, direct && !P.merge.empty() ? (int32_t)(L.lists / 16) : 0, ws};
        static_assert(PC_ARG_BYTES / 16 <= 256, "a thread for every 16 bytes");
        if (mx4) pc_launch_win_decode_mx4(W, (int)P.dec.size(), direct ? &blob : nullptr, O, st);
        else pc_launch_win_decode_bf16(W, (int)P.dec.size(), direct ? &blob : nullptr, O, st);
        PC_HIP(c, hipGetLastError());
    }
    if (!P.sh_items.empty()) {
        ProfScope ps(c, 3, st);
        const PcWinShared S{(const PcWinSharedItem *)(ws + L.sh_items), (const PcWinVisit *)(ws + L.sh_visits), (const PcWinSee *)(ws + L.sh_sees),
                            (const PcWinSharedCall *)(ws + L.sh_calls), (int32_t)P.sh_items.size(), P.sh_wide, c->counters_dev + PC_MX4_WIDE};
        if (mx4) pc_launch_win_shared_decode_mx4(W, S, st);
        else pc_launch_win_shared_decode_bf16(W, S, st);
        PC_HIP(c, hipGetLastError());
    }
    if (!P.pre.empty()) {
        ProfScope ps(c, bf16 ? 2 : 5, st);
        W.items = (const PcWinItem *)(ws + L.pre);
        const PcMx4Rows M{(const uint2 *)(ws + L.q_abs), (const uint32_t *)(ws + L.rot_run), (const float *)(ws + L.q_unit), (const int32_t *)(ws + L.places), ws + L.v_tiles,
                          (int64_t)PC_TILE * (int64_t)P.tiles.size(), (int32_t)P.q_pos.size(), mark, mark ? c->counters_dev + PC_MX4_MARK : nullptr, c->counters_dev + PC_MX4_WIDE};
        if (mx4) pc_launch_win_prefill_mx4(W, M, (int)P.pre.size(), st);
        else if (bf16) pc_launch_win_prefill_bf16(W, (int)P.pre.size(), st);
        else pc_launch_win_attend_f32(W, (int)P.pre.size(), c->D, st);
        PC_HIP(c, hipGetLastError());
    }
    if (!P.merge.empty()) {
        ProfScope ps(c, 4, st);
        pc_launch_win_merge(W, (const PcMergeRow *)(ws + L.merge), (int)P.merge.size(), bf16 ? PC_BF16 : PC_F32, c->D, st);
        PC_HIP(c, hipGetLastError());
    }
    return PC_OK;
}

int32_t attend_window(pc_cache *c, const char *what, const pc_call *calls, int32_t n_calls, int32_t window, int32_t n_sink, const void *q, void *out,
                      float *lse, hipStream_t st, void *fixed_ws)
{
    int32_t rc = check(c, what, calls, n_calls, window, n_sink);
    if (rc != PC_OK || n_calls == 0) return rc;
    if (!c->host_only && (!q || !out)) return pc_fail(c, PC_ERR_INVALID_ARG, "%s: null q or out", what);
    if (!c->host_only && ((((uintptr_t)q | (uintptr_t)out) & 15) || ((uintptr_t)lse & 3)))
        return pc_fail(c, PC_ERR_INVALID_ARG, "%s: q and out must be 16-byte aligned, lse 4-byte", what);
    static thread_local WinPlan P;                       // (32 calls over 410 messages, 64 heads: 264 us a call with fresh lists, 256 with these)
    struct Kept { ~Kept() { P.trim(); } } kept;
    P.clear();
    P.window = window; P.n_sink = n_sink;
    rc = resolve_all(c, calls, n_calls, P);
    if (rc != PC_OK || c->host_only) return rc;
    PcDeviceScope on(c);
    if (!on.ok) return pc_fail(c, PC_ERR_HIP, "%s: the cache's device cannot be made current", what);
    const bool recorded = pc_recorded(st);
    if (recorded && !fixed_ws)
        return pc_fail(c, PC_ERR_INVALID_ARG, "%s: the stream is being captured, and the cache's workspace may move: use pc_attend_window_static", what);
    WinLayout L;
    rc = plan_window(c, what, fixed_ws, recorded, false, P, L);
    if (rc != PC_OK) return rc;
    return launch_window(c, what, P, L, q, out, lse, st, fixed_ws, recorded, 0);
}

int32_t backward_run(pc_cache *c, WinPlan &P, const std::vector<int2> &range, PcWin W, PcWinBwd G, hipStream_t st)
{
    const bool bf16 = c->cfg.dtype == PC_BF16;
    const int Hq = c->cfg.n_q_heads, H = c->cfg.n_kv_heads;
    BwdPlan B;
    plan_backward(c, P, B, range);
    // the rows of the run (they follow each other), from a multiple of 32 on as the lanes' order asks for
    int64_t row0 = INT64_MAX, row1 = 0;
    for (const WinCall &wc : P.calls)
        if (wc.row1 > wc.row0) { row0 = std::min<int64_t>(row0, wc.q_off + wc.row0); row1 = std::max<int64_t>(row1, wc.q_off + wc.row1); }
    row0 -= row0 % 32;
    const size_t rows = (size_t)(row1 - row0);
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t a = at; at = align_up(at + bytes, 16); return a; };
    auto of = [](const auto &v) { return sizeof(v[0]) * v.size(); };
    const size_t items = take(of(P.pre)), runs = take(of(P.runs)), merge = take(of(P.merge)), q_pos = take(sizeof(int32_t) * rows), rots = take(of(P.rots));
    const size_t blocks = take(of(B.blocks)), apps = take(of(B.apps)), keys = take(of(B.keys)), sums = take(of(B.sums)), bins = take(of(B.bins)), turned = take(of(B.turned)), lists = at;
    auto big = [&](size_t bytes) { const size_t a = align_up(at, 256); at = a + bytes; return a; };
    const size_t rot = sizeof(float2) * (size_t)c->half, units = B.blocks.size() * (size_t)(bf16 ? Hq : H), unit = 32 * (size_t)c->D * c->esize;
    const size_t rot_lanes = big(bf16 ? rot / 2 * align_up(rows, 32) : 0), rot_q = big(rot * rows), rot_run = big(rot * P.rots.size()), delta = big(sizeof(float) * rows * (size_t)Hq);
    const size_t q_abs = big(B.turned.empty() ? unit * units : unit * B.turned.size() * (size_t)Hq), d_o = big(unit * units), stat = big(PC_WIN_STAT_BYTES * units);
    const size_t part_row = sizeof(float) * (size_t)Hq * (size_t)c->D, part_o = big(part_row * (size_t)(P.part_rows - P.part_first));
    const size_t key_part = big(sizeof(float) * 2 * PC_WIN_KEY_TILES * PC_TILE * (size_t)B.parts * (size_t)H * (size_t)c->D);
    int32_t rc = pc_ensure_ws(c, align_up(at, 256), st);
    if (rc != PC_OK) return rc;
    char *ws = (char *)c->ws;
    PcArgBlob blob;
    StageSlot *slot = nullptr;
    const bool in_args = lists <= PC_ARG_BYTES;
    if (!in_args) {
        rc = pc_stage_acquire(c, lists, &slot);
        if (rc != PC_OK) return rc;
    }
    char *from = in_args ? (char *)blob.w : (char *)slot->host;
    auto put = [&](size_t to, const auto &v) { if (!v.empty()) std::memcpy(from + to, v.data(), of(v)); };
    put(items, P.pre); put(runs, P.runs); put(merge, P.merge); put(rots, P.rots);
    std::memcpy(from + q_pos, P.q_pos.data() + row0, sizeof(int32_t) * rows);
    put(blocks, B.blocks); put(apps, B.apps); put(keys, B.keys); put(sums, B.sums); put(bins, B.bins); put(turned, B.turned);

    W.items = (const PcWinItem *)(ws + items); W.runs = (const PcWinRun *)(ws + runs);
    // (tables of rows: the kernels index them by the batch's rows)
    auto behind = [&](size_t table, size_t row_bytes) { return (uintptr_t)(ws + table) - row_bytes * (size_t)row0; };
    W.q_pos = (const int32_t *)behind(q_pos, sizeof(int32_t));
    W.rot_q = (const float2 *)behind(rot_q, rot); W.rot_lanes = (const uint32_t *)behind(rot_lanes, rot / 2); W.rot_run = (const float2 *)(ws + rot_run);
    W.part_o = (float *)((uintptr_t)(ws + part_o) - part_row * (size_t)P.part_first);
    G.blocks = (const PcWinBlock *)(ws + blocks); G.apps = (const PcWinApp *)(ws + apps);
    G.key_items = (const PcWinKeyItem *)(ws + keys); G.sums = (const PcWinSum *)(ws + sums); G.bins = (const int32_t *)(ws + bins);
    G.n_blocks = (int32_t)B.blocks.size(); G.n_bins = std::max<int32_t>(0, (int32_t)B.bins.size() - 1); G.n_sums = (int32_t)B.sums.size();
    G.turned = B.turned.empty() ? nullptr : (const PcWinTurned *)(ws + turned); G.n_turned = (int32_t)B.turned.size();
    G.k_factor = G.turned ? 1.f : W.scale_log2;
    G.key_scale = G.turned ? 0.6931471805599453f : c->scale;              // (the queries bring the scale, and log2 e)
    G.delta = (float *)behind(delta, sizeof(float) * (size_t)Hq); G.q_abs = ws + q_abs; G.d_o = ws + d_o; G.stat = ws + stat; G.key_part = (float *)(ws + key_part);
    PcWinTurns T{};
    T.from = in_args ? ws : slot->host; T.ws = ws; T.n16 = (int)(lists / 16);
    T.off_q_pos = (int)q_pos; T.n_rows = (int)rows; T.off_rot = (int)rots; T.n_rot = (int)P.rots.size();
    T.D = c->D; T.run_scale = 1.f;
    if (bf16) T.rot_lanes = (uint32_t *)(ws + rot_lanes);
    T.rot_q = (float2 *)(ws + rot_q); T.rot_run = (float2 *)(ws + rot_run); T.inv_freq = c->inv_freq_dev;
    ProfScope ps(c, 5, st);
    pc_forget_error();
    pc_launch_win_turns(T, in_args ? &blob : nullptr, st);
    PC_HIP(c, hipGetLastError());
    if (slot) { rc = pc_stage_release(c, slot, st); if (rc != PC_OK) return rc; }
    pc_launch_win_bwd_prep(W, G, c->cfg.dtype, c->D, st);
    pc_launch_win_bwd_turned(W, G, st);
    if (bf16) pc_launch_win_bwd_dq_bf16(W, G, (int)P.pre.size(), st);
    else pc_launch_win_bwd_dq_f32(W, G, (int)P.pre.size(), c->D, st);
    pc_launch_win_bwd_rows(W, G, (const PcMergeRow *)(ws + merge), (int)P.merge.size(), c->D, st);
    if (bf16) pc_launch_win_bwd_keys_bf16(W, G, st);
    else pc_launch_win_bwd_keys_f32(W, G, c->D, st);
    pc_launch_win_bwd_sums(W, G, c->D, st);
    PC_HIP(c, hipGetLastError());
    return PC_OK;
}

int32_t attend_window_backward(pc_cache *c, const pc_call *calls, int32_t n_calls, int32_t window, int32_t n_sink, const void *q, const void *out,
                               const float *lse, const void *d_out, float *d_q, float *d_k, float *d_v, hipStream_t st)
{
    const char *what = "attend_window_backward";
    if (c->cfg.dtype == PC_MX4) return pc_fail(c, PC_ERR_INVALID_ARG, "%s: a PC_MX4 cache has no gradient", what);
    int32_t rc = check(c, what, calls, n_calls, window, n_sink);
    if (rc != PC_OK || n_calls == 0) return rc;
    if (!c->host_only) {
        if (!q || !out || !lse || !d_out || !d_q || !d_k || !d_v) return pc_fail(c, PC_ERR_INVALID_ARG, "%s: null argument", what);
        const uintptr_t all = (uintptr_t)q | (uintptr_t)out | (uintptr_t)d_out | (uintptr_t)d_q | (uintptr_t)d_k | (uintptr_t)d_v;
        if ((all & 15) || ((uintptr_t)lse & 3)) return pc_fail(c, PC_ERR_INVALID_ARG, "%s: tensors must be 16-byte aligned, lse 4-byte", what);
    }
    WinPlan P;
    P.window = window; P.n_sink = n_sink;
    rc = resolve_all(c, calls, n_calls, P);
    if (rc != PC_OK || c->host_only) return rc;
    PcDeviceScope on(c);
    if (!on.ok) return pc_fail(c, PC_ERR_HIP, "%s: the cache's device cannot be made current", what);
    if (pc_recorded(st)) return pc_fail(c, PC_ERR_INVALID_ARG, "%s: the stream is being captured, and the cache's workspace may move", what);
    const bool bf16 = c->cfg.dtype == PC_BF16;
    PcWin W{};
    W.inv_freq = c->inv_freq_dev;
    W.k_store = c->k_store; W.v_store = c->v_store; W.q = q;
    W.slots = c->slots; W.n_q_heads = c->cfg.n_q_heads; W.n_kv_heads = c->cfg.n_kv_heads;
    W.window = window;
    W.scale_log2 = c->scale * 1.4426950408889634f;
    PcWinBwd G{};
    G.out = out; G.d_out = d_out; G.lse = lse; G.d_q = d_q; G.d_k = d_k; G.d_v = d_v; G.scale = c->scale;
    // Runs of blocks whose workspace fits.  A run ends with a call, or where units and rows end together: after four blocks of 32 rows
    // (a workgroup's units), or the columns of 32 rows.
    const int64_t per_unit = 2 * 32 * c->D * (int64_t)c->esize + PC_WIN_STAT_BYTES, per_row = (bf16 ? 12 : 8) * c->half + 4 * c->cfg.n_q_heads;     // (rotations, Delta)
    const int64_t per_block = (bf16 ? c->cfg.n_q_heads : c->cfg.n_kv_heads) * per_unit + (bf16 ? 32 : (32 + c->g - 1) / c->g) * per_row;
    const int64_t step = bf16 ? 4 : c->g, most = std::max<int64_t>(step, (int64_t)BWD_BYTES / per_block / (bf16 && (int64_t)window + n_sink <= PC_WIN_FEW ? 4 : 1) / step * step);
    std::vector<int2> range(P.calls.size(), make_int2(0, 0));
    int64_t in_run = 0;
    for (size_t i = 0; i < P.calls.size(); ++i) {
        const int64_t n = bf16 ? (P.calls[i].n_q + 31) / 32 : ((int64_t)P.calls[i].n_q * c->g + 31) / 32;
        for (int64_t b = 0; b < n;) {
            const int64_t room = (most - in_run) / step * step, m = std::min(n - b, room);
            if (m > 0) {
                range[i] = make_int2((int)b, (int)(b + m));
                b += m; in_run += m;
            }
            if (b < n || m == 0) {
                rc = backward_run(c, P, range, W, G, st);
                if (rc != PC_OK) return rc;
                std::fill(range.begin(), range.end(), make_int2(0, 0));
                in_run = 0;
            }
        }
    }
    return in_run > 0 ? backward_run(c, P, range, W, G, st) : PC_OK;
}

}  // namespace

// What a call lists is all in a window of 2^31 - 1 (positions are below 2^30 in magnitude: pc_cache_create).
//
// Long prefills (whose rows a window leaves all that they list) go over a packed copy, as in a bf16 cache: there a message's turn costs its keys once, and not every row and head once a
// message.  The copy's keys and the queries are fp16 for the matrix instructions, whose range keys and queries of models are in; where one is not, the
// device marks the call, and the walk over the cache itself, which takes any, follows and does nothing otherwise.
// Taken by calls of LONG_ROWS rows x query heads of a KV head (each copied token is read that often), where those that stand together have
// LONG_SCORES scores in all (two more launches are to be earned back).  In place and copied, us, over messages of 64 to 256 tokens, by rows x query heads of
// a KV head:
//   512: 8 calls of 64 rows over 12064 tokens, 64 heads on 8, 326 and 347; one over 7.7k 55 and 66, over 30k 130 and 136; 128 rows of 32 heads over 12064 71 and 86;
//   1024: 128 rows of 64 heads over 12064 105 and 103, over 30k 206 and 187, 8 calls of it over 12064 546 and 489; 4 over 5000 150 and 139; 256 rows of 32 heads 106 and 103;
//   2048 and more: 256 rows of 64 heads over 2256 (3.7e7 scores) 60 and 67, two calls of it 87 and 82, eight 228 and 191; over 5000 92 and 85; 384 rows over 2256 92 and 73;
//     512 over 1024 (3.4e7) 60 and 51; 1024 over 13024 573 and 398, 8 calls of it 4450 and 2960.
// By the caller's word: pc_set_key_gather.
constexpr int64_t LONG_ROWS = 1024;
constexpr double LONG_SCORES = 3e7;
constexpr int64_t LONG_TOKENS = (int64_t)1 << 22;        // a copy's, where it has more calls than one: 16 GiB of 8 KV heads
int32_t pc_attend_mx4(pc_cache *c, const char *what, const pc_call *calls, int32_t n_calls, int32_t window, int32_t n_sink, const void *q, void *out, float *lse,
                      hipStream_t st, void *fixed_ws)
{
    {
        const int32_t rc = check(c, what, calls, n_calls, window, n_sink);
        if (rc != PC_OK) return rc;
    }
    // every row of the call sees all that it lists (and of the new message what is not behind it)
    auto sees_all = [&](const pc_call &call) {
        if (window == INT32_MAX) return true;
        Resolved r;
        if (pc_resolve(c, &call, 0, r) != PC_OK) return false;           // (refused where it is planned)
        const int32_t low = win_low(*std::max_element(r.q_pos.begin(), r.q_pos.end()), window);
        for (const int2 &s : r.sel) if (s.y < low) return false;
        return r.self_msg < 0 || r.self_start >= low;
    };
    // tokens that a call lists, if it is long
    auto long_tokens = [&](const pc_call &call) -> int64_t {
        if (fixed_ws || c->host_only || call.n_q <= 1 || c->key_gather == 1 || call.n_q * (int64_t)c->g < (c->key_gather == 2 ? 17 : LONG_ROWS) || call.n_sel < 0 || (call.n_sel > 0 && !call.sel)) return 0;
        int64_t tokens = 0;
        auto add = [&](int32_t m) { if (known(c, m)) tokens += chain_len(c, m); };
        for (int32_t e = 0; e < call.n_sel; ++e) add(call.sel[e].msg_id);
        add(call.self_msg);
        return tokens < 100000000 && sees_all(call) ? tokens : 0;
    };
    std::vector<int64_t> tokens((size_t)std::max(n_calls, 0));
    for (int32_t i = 0; i < n_calls; ++i) tokens[(size_t)i] = long_tokens(calls[i]);
    // runs of long calls; each ends the launches that the calls before and behind it would share: several have to earn more
    int runs = 0;
    for (size_t i = 0; i < tokens.size(); ++i) runs += tokens[i] > 0 && (i == 0 || tokens[i - 1] == 0);
    bool some = false;
    for (size_t i = 0; i < tokens.size();) {
        size_t e = i;
        double scores = 0;
        for (; e < tokens.size() && tokens[e] > 0; ++e) scores += (double)tokens[e] * calls[e].n_q * c->cfg.n_q_heads;
        const bool kept = c->key_gather == 2 ? scores > 0 : scores >= (runs > 1 ? 4 : 1) * LONG_SCORES;
        some |= kept;
        if (!kept) std::fill(tokens.begin() + (ptrdiff_t)i, tokens.begin() + (ptrdiff_t)e, 0);
        i = std::max(e, i + 1);
    }
    if (!some) return attend_window(c, what, calls, n_calls, window, n_sink, q, out, lse, st, fixed_ws);
    // Runs of calls of a kind follow each other.  Nothing may be refused behind the first: all are planned, and have room for the walk over the cache, before it.
    if (!q || !out) return pc_fail(c, PC_ERR_INVALID_ARG, "%s: null q or out", what);
    if ((((uintptr_t)q | (uintptr_t)out) & 15) || ((uintptr_t)lse & 3)) return pc_fail(c, PC_ERR_INVALID_ARG, "%s: q and out must be 16-byte aligned, lse 4-byte", what);
    struct Run { int32_t first, n; int64_t row; bool copied; WinPlan P; WinLayout L; };
    static thread_local std::vector<Run> kept;           // (lists as in attend_window)
    struct Kept { ~Kept() { for (Run &r : kept) r.P.trim(); if (kept.size() > 4) kept.resize(4); } } trim;
    size_t n_runs = 0;
    int64_t row = 0;
    for (int32_t a = 0; a < n_calls; ++n_runs) {
        if (n_runs == kept.size()) kept.emplace_back();
        Run &r = kept[n_runs];
        r.first = a; r.row = row; r.copied = tokens[(size_t)a] > 0;
        int32_t b = a;
        int64_t copied = 0;
        for (; b < n_calls && (tokens[(size_t)b] > 0) == r.copied && (b == a || copied + tokens[(size_t)b] <= LONG_TOKENS); ++b) {
            row += std::max(calls[b].n_q, 0);
            copied += tokens[(size_t)b];
        }
        r.n = b - a;
        r.P.clear();
        r.P.window = window; r.P.n_sink = n_sink;
        const int32_t rc = resolve_all(c, calls + a, r.n, r.P, a);
        if (rc != PC_OK) return rc;
        a = b;
    }
    if (row > INT32_MAX / 2) return pc_fail(c, PC_ERR_SHAPE, "%s: too many query rows", what);
    PcDeviceScope on(c);
    if (!on.ok) return pc_fail(c, PC_ERR_HIP, "%s: the cache's device cannot be made current", what);
    if (pc_recorded(st)) return pc_fail(c, PC_ERR_INVALID_ARG, "%s: the stream is being captured, and the cache's workspace may move", what);
    size_t need = 0;
    for (size_t i = 0; i < n_runs; ++i) {
        const int32_t rc = plan_window(c, what, nullptr, false, kept[i].copied, kept[i].P, kept[i].L);
        if (rc != PC_OK) return rc;
        need = std::max(need, kept[i].L.total);
    }
    {
        const int32_t rc = pc_ensure_ws(c, need, st);
        if (rc != PC_OK) return rc;
    }
    for (size_t i = 0; i < n_runs; ++i) {
        Run &r = kept[i];
        const int64_t at = r.row * c->cfg.n_q_heads;
        const uint16_t *rq = (const uint16_t *)q + at * c->D;
        uint16_t *ro = (uint16_t *)out + at * c->D;
        float *rl = lse ? lse + at : nullptr;
        uint32_t mark = 0;
        if (r.copied) {
            if (++c->mark_epoch_mx4 == 0) c->mark_epoch_mx4 = 1;
            mark = c->mark_epoch_mx4;
            if (pc_attend_gathered_mx4(c, calls + r.first, r.n, rq, ro, rl, st, mark) != PC_OK) {
                mark = 0;                                // (no room for the copy: what else may have failed fails again)
                WinPlan P;                               // in splits, if the workspace holds them
                WinLayout L;
                P.window = window; P.n_sink = n_sink;
                if (resolve_all(c, calls + r.first, r.n, P) == PC_OK && plan_window(c, what, nullptr, false, false, P, L) == PC_OK && L.total <= c->ws_cap) {
                    std::swap(r.P, P);
                    r.L = L;
                }
            }
        }
        const int32_t rc = launch_window(c, what, r.P, r.L, rq, ro, rl, st, nullptr, false, mark);
        if (rc != PC_OK) return rc;
    }
    return PC_OK;
}

extern "C" {

int32_t pc_attend_window_backward(pc_cache *c, const pc_call *calls, int32_t n_calls, int32_t window, int32_t n_sink, const void *q, const void *out,
                                  const float *lse, const void *d_out, float *d_q, float *d_k, float *d_v, void *stream)
{
    if (!c) return PC_ERR_INVALID_ARG;
    return pc_guarded(c, [&] {
        return attend_window_backward(c, calls, n_calls, window, n_sink, q, out, lse, d_out, d_q, d_k, d_v, (hipStream_t)stream);
    });
}

int32_t pc_attend_window(pc_cache *c, const pc_call *calls, int32_t n_calls, int32_t window, int32_t n_sink, const void *q, void *out, float *lse,
                         void *stream)
{
    if (!c) return PC_ERR_INVALID_ARG;
    return pc_guarded(c, [&] {
        if (c->cfg.dtype == PC_MX4) return pc_attend_mx4(c, "attend_window", calls, n_calls, window, n_sink, q, out, lse, (hipStream_t)stream, nullptr);
        return attend_window(c, "attend_window", calls, n_calls, window, n_sink, q, out, lse, (hipStream_t)stream, nullptr);
    });
}

int32_t pc_attend_window_static(pc_cache *c, const pc_call *calls, int32_t n_calls, int32_t window, int32_t n_sink, const void *q, void *out, float *lse,
                                void *stream)
{
    if (!c) return PC_ERR_INVALID_ARG;
    if (!c->host_only && !c->static_ws) return pc_fail(c, PC_ERR_HIP, "attend_window_static: the fixed scratch array was not found on this device");
    const bool prof = c->prof;                           // kernel timing takes events from a pool that may have to grow
    c->prof = false;
    const int32_t rc = pc_guarded(c, [&] {
        return attend_window(c, "attend_window_static", calls, n_calls, window, n_sink, q, out, lse, (hipStream_t)stream, c->static_ws);
    });
    c->prof = prof;
    return rc;
}

}  // extern "C"
