// Work lists of the two attentions of one iteration (host code, no GPU).
#include "attn_plan.h"

#include <algorithm>
#include <functional>

#include "common.h"
#include "kernels.h"

namespace slw {

namespace {

// Decode attention runs one wave per work-group, two per SIMD (its register
// use allows no more): kDecodeWaves of them fill a 256-CU part once.  Their
// keys are cut into equal runs (at least kDecodeMinKeys each), so that every
// wave of the launch finishes at about the same time.
constexpr int kDecodeWaves = 2048;
constexpr int kDecodeMinKeys = 128;
// The cache kernels' decodes with no chunk beside them: runs for this many
// waves, or one for each decode where the longest is at most 1.5 runs + 128
// keys, which leaves nothing to merge.  us a layer with its append and merge
// for 2048 / 768 / 512 waves: 64 chat decodes (8-bit) 44.9 / 44.3 / 44.7, 256
// 114.4 / 108.0 / 116.5, 4 of 1 K to 10 K 35.2 / 28.7 / 28.7, 32 of 0.5 K to 2 K
// 32.9 / 28.4 / 31.0; in bf16, 32 in a window of 1024 43.2 / 41.3 / 40.4, 256 chat
// decodes 197.6 / 188.8 / 186.7.  768 waves / one run a decode, decodes of equal
// length, two layers: one of 190 tokens 29.9 / 25.3, of 250 27.8 / 26.8, of 380
// 27.8 / 31.7; 32 of 250 32.4 / 29.8, of 830 49.4 / 53.5; 64 of 380 47.1 / 37.9,
// of 830 72.2 / 57.1; 128 of 1200 137.5 / 119.2; 256 of 830 217.8 / 189.7.
// Beside a chunk, eight waves share a CU, and fewer waves are fewer CUs: 256
// decodes beside 64 rows 116.1 / 159.6 with 2048 / 768.
constexpr int kCacheDecodeWaves = 768;
// Beside a chunk that needs no merge, decodes of up to so many keys get one run
// each: 5 beside 77 rows, split / one run, of 120 tokens 25.4 / 21.7, of 190
// 25.3 / 22.8, of 250 24.9 / 26.1.
constexpr int64_t kBesideWhole = 3 * 64;
// Chunk attention runs one work-group per CU (its register use allows no
// more), so a launch of kChunkSlots work-groups with equal work finishes in
// one round on a 256-CU part.  A work-group takes at least kChunkMinTiles
// 64-key tiles, which keeps its fixed costs (Q load, partial write) small.
constexpr int kChunkSlots = 256;
constexpr int kChunkMinTiles = 4;
// Whole query tiles per work-group when the largest group's load is within
// 11/10 of an equal share.
constexpr int64_t kChunkWholeSlackNum = 11, kChunkWholeSlackDen = 10;
// Cache kernels: what splitting query tiles costs, in 64-key tiles (plan_chunk);
// an item costs kItemTiles5 / 5 for every 1024 values of a row.
constexpr int64_t kMergeTiles = 4, kItemTiles5 = 2;
// Work items of at least kTwoPhaseTiles + kTwoPhaseTilesPer64 (positions of a
// query tile, at least 64, / 64) 64-key tiles on average run the two-phase
// chunk kernel at head dim 128.  Its fill and extra phases are paid per item,
// and every wave computes all tiles of the item, which wastes a few more where
// a query tile holds many positions (few heads a group).  Below the line it
// loses; at head dim 64 it nearly always did (half the products under the same
// softmax).  One-phase / two-phase us at n tiles per item:
//   8B layer (4 heads a group): 1: 11.2 / 13.3, 2 (77 rows at 50): 18.6 / 23.5,
//   3.5: 28.6 / 34.1, 9.5: 33.1 / 34.9, 17.5: 48.1 / 47.8, 20.2: 63.9 / 64.7,
//   25.5: 61.8 / 62.6, 27.2: 81.4 / 79.6, 33.5: 76.8 / 75.8, 73: 292 / 272;
//   2 heads: 28: 77.4 / 80.2, 35: 77.7 / 76.7, 50: 107 / 101;
//   1 head: 31: 73.6 / 77.0, 36: 81.3 / 85.4, 51: 109.5 / 109.4, 84: 310 / 293;
//   head dim 64: 1 head, 59: 102 / 108; 8 heads, 72: 108 / 110; 16 heads, 464: 1130 / 1152.
constexpr int64_t kTwoPhaseTiles = 21, kTwoPhaseTilesPer64 = 5;
// The cache kernels' line; one-phase / two-phase us at n tiles per item, 4096
// rows at 8192 under windows:
//   4 heads a group: 9: 63.3 / 68.5, 12: 76.9 / 79.8, 15: 90.1 / 90.0,
//   18: 104.9 / 102.5; 256 rows at 8192 over the whole context, 8: 59.0 / 56.2;
//   8 heads: 11.5: 159 / 149; 2 heads: 19: 109.2 / 108.6, 28: 157 / 147;
//   1 head: 21: 118 / 130, 45: 225.6 / 224.6.
constexpr int64_t kCacheTwoPhaseTiles = 5, kCacheTwoPhaseTilesPer64 = 10;

inline int64_t span64(int64_t keys) { return (keys + 63) & ~static_cast<int64_t>(63); }

}  // namespace

int decode_slot_cap(const slw_model_cfg& c) { return std::max(1, kDecodeWaves / c.n_kv_heads); }
// A run crosses at most one decode boundary more than it has runs: items <= slots + B - 1.
int decode_work_cap(const slw_model_cfg& c, int B) { return decode_slot_cap(c) + B + 1; }

// Query tiles of the chunk rows: each prefill's rows are tiled on their own,
// so up to SLW_MAX_PREFILLS - 1 tiles more than one prefill of C rows needs.
int chunk_tiles(const slw_model_cfg& c, int C) {
    if (C <= 0) return 0;
    return static_cast<int>(ceil_div(C, chunk_tile_positions(c.n_q_heads / c.n_kv_heads))) +
           std::min(C, static_cast<int>(SLW_MAX_PREFILLS)) - 1;
}
int chunk_slot_cap(const slw_model_cfg& c) { return std::max(1, kChunkSlots / c.n_kv_heads); }
int chunk_item_cap(const slw_model_cfg& c, int C) {
    return C > 0 ? chunk_tiles(c, C) + chunk_slot_cap(c) : 0;
}

int32_t window_skip(const Window& w, int32_t first_pos) {
    if (w.window <= 0) return 0;
    const int64_t lo = static_cast<int64_t>(first_pos) - w.window + 1;  // first key of the window
    const int64_t skip = lo / 64 * 64 - sink_end(w);
    return lo > 0 && skip > 0 ? static_cast<int32_t>(skip) : 0;
}

// Query tiles of the chunk rows: each prefill's rows cut into tiles of
// chunk_tile_positions(group) positions (a tile never mixes sequences).
// Tile q: first chunk row, rows, first position and, when wanted, the offset
// of its sequence's block table (bt_of_prefill[i] for prefill i).
void query_tiles(const slw_model_cfg& c, const std::vector<Prefill>& pre, std::vector<int32_t>& row0,
                 std::vector<int32_t>& rows, std::vector<int32_t>& pos0, std::vector<int32_t>* bt,
                 const std::vector<int32_t>& bt_of_prefill) {
    const int pwg = chunk_tile_positions(c.n_q_heads / c.n_kv_heads);
    row0.clear();
    rows.clear();
    pos0.clear();
    if (bt) bt->clear();
    for (size_t i = 0; i < pre.size(); ++i)
        for (int j = 0; j < pre[i].c; j += pwg) {
            row0.push_back(pre[i].row0 + j);
            rows.push_back(std::min(pwg, pre[i].c - j));
            pos0.push_back(pre[i].prefix + j);
            if (bt) bt->push_back(bt_of_prefill[i]);
        }
}

// Decode attention work.  The keys of all decodes (decode b attends to
// context_lens[b] + 1 of them, or those left by the window), laid end to end
// with each decode's range padded to a multiple of 64, are cut into equal runs
// (multiples of 64 keys, so that every item starts on a page pair; at least
// kDecodeMinKeys each, at most decode_slot_cap(c) runs), one per wave of each
// kv head; a run that crosses decodes becomes one item per decode it touches,
// and padding alone makes no item.  Items come out in decode order, so each
// decode's items are contiguous for the merge.
//
// Layers on the cache kernels (kind) write a decode of one item without a
// merge, and decodes of similar length get one run each (kCacheDecodeWaves).
int plan_decode(const slw_model_cfg& c, const Window& w, DecodeKind kind, int B, const int32_t* context_lens,
                DecodePlan& p) {
    p.b.clear();
    p.kb.clear();
    p.ke.clear();
    p.off.assign(B + 1, 0);
    p.slot_off.assign(1, 0);
    p.skip.resize(std::max(B, 0));
    p.keys.resize(std::max(B, 0));
    if (B <= 0) return SLW_OK;
    int64_t padded = 0;
    int32_t longest = 0;
    for (int b = 0; b < B; ++b) {
        p.skip[b] = window_skip(w, context_lens[b]);
        p.keys[b] = context_lens[b] + 1 - p.skip[b];
        padded += span64(p.keys[b]);
        longest = std::max(longest, p.keys[b]);
    }
    const int cap = decode_work_cap(c, B), slot_cap = decode_slot_cap(c);
    const int64_t slots = kind == DecodeKind::cache_alone ? std::max(1, kCacheDecodeWaves / c.n_kv_heads) : slot_cap;
    const int64_t want = std::min<int64_t>(slots, std::max<int64_t>(1, padded / kDecodeMinKeys));
    const int64_t per = span64(ceil_div(padded, want));
    const bool whole = B <= slot_cap && ((kind == DecodeKind::cache_alone && 2 * span64(longest) <= 3 * per + 4 * 64) ||
                                         (kind == DecodeKind::cache_beside && longest <= kBesideWhole));
    const int n_slots = whole ? B : static_cast<int>(ceil_div(padded, per));
    if (n_slots > slot_cap) return fail(SLW_EINVAL, "internal: %d decode slots above cap", n_slots);
    // at most one item for each end of a slot or of a decode: n_slots + B
    p.b.resize(n_slots + B);
    p.kb.resize(n_slots + B);
    p.ke.resize(n_slots + B);
    p.slot_off.resize(n_slots + 1);
    int n = 0, sl = 0;
    int64_t room = 0;  // keys that the slot can still take
    for (int b = 0; b < B; ++b) {
        const int32_t len = p.keys[b];
        const int64_t span = span64(len);
        for (int64_t k = 0; k < span;) {
            if (room == 0) {
                p.slot_off[sl++] = n;
                room = whole ? span : per;
            }
            const int64_t take = std::min(room, span - k);
            p.b[n] = b;
            p.kb[n] = static_cast<int32_t>(k);
            p.ke[n] = static_cast<int32_t>(std::min<int64_t>(k + take, len));
            ++n;
            k += take;
            room -= take;
        }
        p.off[b + 1] = n;
    }
    p.slot_off[sl] = n;
    p.b.resize(n);
    p.kb.resize(n);
    p.ke.resize(n);
    if (n > cap || sl != n_slots) return fail(SLW_EINVAL, "internal: decode work %d above cap, or %d slots of %d", n, sl, n_slots);
    for (int d = 0; d < B; ++d) {  // the items of each decode tile its keys
        int64_t at = 0;
        for (int i = p.off[d]; i < p.off[d + 1]; ++i) {
            if (p.b[i] != d || p.kb[i] != at || p.ke[i] <= at) return fail(SLW_EINVAL, "internal: decode plan");
            at = p.ke[i];
        }
        if (at != p.keys[d]) return fail(SLW_EINVAL, "internal: decode plan");
    }
    return SLW_OK;
}

// Chunk attention work over query tiles q (first position qt_pos0[q],
// qt_rows[q] rows, keys 0 .. qt_pos0[q] + qt_rows[q] - 1, or those left by the
// window).  Whole query tiles
// where they balance: the tiles, longest first, each go to the least loaded
// of `want` work-groups (LPT); when the largest load stays within
// kChunkWholeSlack of an equal share, no tile is split and nothing is merged
// (long prompts: many tiles of similar length).  Otherwise (fewer tiles than
// work-groups, or tiles of very different lengths, as at the start of a
// prompt) the 64-key tiles of every query tile, laid end to end, are cut into
// equal runs, one per work-group of each kv head; a run that crosses query
// tiles becomes one item per query tile it touches.  Items stay in query-tile
// order; slot_items lists each work-group's items.
//
// Layers on the cache kernels (`cache`) weigh the two instead: whole query
// tiles on up to one work-group each against equal runs, whose partial sums are
// written and merged.  In units of a 64-key tile (1.9 us where few CUs work,
// 2.3 where all do), the rule counts 4 for the merge's launch and 0.4 for an
// item of 1024 values a row (all kv heads).  The two numbers were chosen on two
// shapes, whose both sides they get right, and are no fit: four prompts of 1500
// rows under a window of 512 took 40 + 16 us (merge) in equal runs and 35 + 4 us
// whole; 77 rows at 50, two query tiles, 14 whole against 20.
int plan_chunk(const slw_model_cfg& c, const Window& w, bool cache, int C, const std::vector<int32_t>& qt_pos0,
               const std::vector<int32_t>& qt_rows, ChunkPlan& p) {
    const int n_qt = static_cast<int>(qt_pos0.size());
    p.items.clear();
    p.slot_off.clear();
    p.slot_items.clear();
    p.whole = false;
    p.qt_skip.resize(n_qt);
    for (int q = 0; q < n_qt; ++q) p.qt_skip[q] = window_skip(w, qt_pos0[q]);
    auto key_end = [&](int q) { return static_cast<int64_t>(qt_pos0[q]) + qt_rows[q] - p.qt_skip[q]; };  // virtual
    std::vector<int64_t> tile_end(n_qt + 1, 0);
    for (int q = 0; q < n_qt; ++q) tile_end[q + 1] = tile_end[q] + ceil_div(key_end(q), 64);
    const int64_t total_tiles = tile_end[n_qt];
    std::vector<int32_t>& it = p.items;
    int n_slots = 0;
    if (n_qt > 0) {
        const int64_t want = std::min<int64_t>(chunk_slot_cap(c), std::max<int64_t>(1, total_tiles / kChunkMinTiles));
        const int64_t per = ceil_div(total_tiles, want);
        const int64_t spread = cache ? std::min<int64_t>(n_qt, chunk_slot_cap(c)) : want;  // work-groups for whole tiles
        if (cache || n_qt >= want) {
            std::vector<int32_t> order(n_qt);
            for (int q = 0; q < n_qt; ++q) order[q] = q;
            auto len = [&](int q) { return tile_end[q + 1] - tile_end[q]; };
            std::stable_sort(order.begin(), order.end(), [&](int x, int y) { return len(x) > len(y); });
            // (load, work-group) heap: the least loaded on top, the lowest of equals
            std::vector<std::pair<int64_t, int32_t>> load(spread);
            for (int64_t g = 0; g < spread; ++g) load[g] = {0, static_cast<int32_t>(g)};
            std::vector<int32_t> owner(n_qt);
            int64_t mx = 0;
            for (int q : order) {
                std::pop_heap(load.begin(), load.end(), std::greater<>());
                load.back().first += len(q);
                owner[q] = load.back().second;
                mx = std::max(mx, load.back().first);
                std::push_heap(load.begin(), load.end(), std::greater<>());
            }
            bool whole = mx * kChunkWholeSlackDen <= per * kChunkWholeSlackNum;
            if (cache) {
                const int64_t runs = ceil_div(total_tiles, per);
                whole = mx <= per + kMergeTiles + kItemTiles5 * (n_qt + runs - 1) * c.n_kv_heads * c.head_dim / (5 * 1024);
            }
            if (whole) {
                p.whole = true;
                n_slots = static_cast<int>(spread);
                for (int q = 0; q < n_qt; ++q) {
                    it.push_back(q);
                    it.push_back(0);
                    it.push_back(static_cast<int32_t>(key_end(q)));
                }
                p.slot_off.assign(n_slots + 1, 0);
                for (int q = 0; q < n_qt; ++q) ++p.slot_off[owner[q] + 1];
                for (int g = 0; g < n_slots; ++g) p.slot_off[g + 1] += p.slot_off[g];
                p.slot_items.resize(n_qt);
                std::vector<int32_t> fill(p.slot_off.begin(), p.slot_off.end() - 1);
                for (int q = 0; q < n_qt; ++q) p.slot_items[fill[owner[q]]++] = q;
            }
        }
        if (!p.whole) {
            n_slots = static_cast<int>(ceil_div(total_tiles, per));
            p.slot_off.resize(n_slots + 1);
            int q = 0;
            for (int sl = 0; sl < n_slots; ++sl) {
                p.slot_off[sl] = static_cast<int32_t>(it.size() / 3);
                int64_t t0 = sl * per;
                const int64_t t1 = std::min(total_tiles, t0 + per);
                while (t0 < t1) {
                    while (tile_end[q + 1] <= t0) ++q;
                    const int64_t seg_end = std::min(t1, tile_end[q + 1]);
                    it.push_back(q);
                    it.push_back(static_cast<int32_t>((t0 - tile_end[q]) * 64));
                    it.push_back(static_cast<int32_t>(std::min(key_end(q), (seg_end - tile_end[q]) * 64)));
                    t0 = seg_end;
                }
            }
            p.slot_off[n_slots] = static_cast<int32_t>(it.size() / 3);
            p.slot_items.resize(it.size() / 3);
            for (size_t i = 0; i < p.slot_items.size(); ++i) p.slot_items[i] = static_cast<int32_t>(i);
        }
    } else {
        p.slot_off.assign(1, 0);
    }
    const int n_items = static_cast<int>(it.size() / 3);
    const int64_t blocks64 = std::max(1, chunk_tile_positions(c.n_q_heads / c.n_kv_heads) / 64);
    p.two_phase = c.head_dim == 128 && n_items > 0 &&
                  total_tiles >= (cache ? kCacheTwoPhaseTiles + kCacheTwoPhaseTilesPer64 * blocks64
                                        : kTwoPhaseTiles + kTwoPhaseTilesPer64 * blocks64) * n_items;
    p.qt_off.assign(n_qt + 1, 0);
    for (int q = 0, i = 0; q <= n_qt; ++q) {
        while (i < n_items && it[3 * i] < q) ++i;
        p.qt_off[q] = i;
    }
    if (n_items > chunk_item_cap(c, C) || n_slots > chunk_slot_cap(c))
        return fail(SLW_EINVAL, "internal: chunk items %d / slots %d above cap", n_items, n_slots);
    for (int q = 0; q < n_qt; ++q) {  // the items of each query tile tile its key range
        int64_t at = 0;
        for (int i = p.qt_off[q]; i < p.qt_off[q + 1]; ++i) {
            if (it[3 * i + 1] != at || it[3 * i + 2] <= at) return fail(SLW_EINVAL, "internal: chunk plan");
            at = it[3 * i + 2];
        }
        if (at != key_end(q)) return fail(SLW_EINVAL, "internal: chunk plan");
    }
    return SLW_OK;
}

}  // namespace slw
