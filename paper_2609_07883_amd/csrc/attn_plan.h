// Work lists of the two attentions of one iteration (host code, no GPU).
#pragma once

#include <cstdint>
#include <vector>

#include "sloweave.h"

namespace slw {

// One prefill of an iteration: `c` chunk rows from row `row0` on, at positions
// prefix .. prefix + c - 1 of sequence `seq`.
struct Prefill {
    int64_t seq;
    int32_t prefix;
    int32_t c;
    int32_t row0;
};

// Attention window of a layer: a row at position p sees keys t <= p with
// t > p - window or t < sinks; window 0: every key t <= p.
struct Window {
    int32_t window = 0;
    int32_t sinks = 0;
};
// Keys that no row from position first_pos on sees lie between the sinks and
// the window.  Work lists count in virtual keys, which leave out the whole
// 64-key tiles of that gap: virtual key v is key v below sink_end(w) and key
// v + window_skip(w, first_pos) from there on (both are multiples of 64).
inline int32_t sink_end(const Window& w) { return w.window > 0 ? (w.sinks + 63) / 64 * 64 : 0; }
int32_t window_skip(const Window& w, int32_t first_pos);

struct DecodePlan {
    std::vector<int32_t> b, kb, ke;  // items: decode, first virtual key (a multiple of 64), virtual key past the last
    std::vector<int32_t> off;        // [B + 1] first item of each decode
    std::vector<int32_t> slot_off;   // [slots + 1] first item of each wave slot
    std::vector<int32_t> skip;       // [B] keys between each decode's sinks and its window that are left out
    std::vector<int32_t> keys;       // [B] virtual keys of each decode
};
struct ChunkPlan {
    std::vector<int32_t> items;       // [3 n]: query tile, first virtual key, virtual key past the last
    std::vector<int32_t> slot_off;    // [slots + 1] first entry of each work-group in slot_items
    std::vector<int32_t> slot_items;  // [n] the items of each work-group in turn
    std::vector<int32_t> qt_off;      // [n_qt + 1] first item of each query tile
    std::vector<int32_t> qt_skip;     // [n_qt] keys of each query tile that are left out
    bool whole = false;               // whole query tiles per work-group
    bool two_phase = false;           // the two-phase kernel
};

int decode_slot_cap(const slw_model_cfg& c);
int decode_work_cap(const slw_model_cfg& c, int B);
int chunk_tiles(const slw_model_cfg& c, int C);
int chunk_slot_cap(const slw_model_cfg& c);
int chunk_item_cap(const slw_model_cfg& c, int C);

void query_tiles(const slw_model_cfg& c, const std::vector<Prefill>& pre, std::vector<int32_t>& row0,
                 std::vector<int32_t>& rows, std::vector<int32_t>& pos0, std::vector<int32_t>* bt,
                 const std::vector<int32_t>& bt_of_prefill);
// Which kernels the decodes run on, and beside what: a chunk whose query tiles
// are split is merged by a launch that the decodes then share.
enum class DecodeKind { bf16, cache_alone, cache_beside, cache_split };
inline DecodeKind decode_kind(bool cache, const ChunkPlan& chunk) {
    if (!cache) return DecodeKind::bf16;
    if (chunk.items.empty()) return DecodeKind::cache_alone;
    return chunk.items.size() / 3 + 1 > chunk.qt_off.size() ? DecodeKind::cache_split : DecodeKind::cache_beside;
}
int plan_decode(const slw_model_cfg& c, const Window& w, DecodeKind kind, int B, const int32_t* context_lens,
                DecodePlan& p);
int plan_chunk(const slw_model_cfg& c, const Window& w, bool cache, int C, const std::vector<int32_t>& qt_pos0,
               const std::vector<int32_t>& qt_rows, ChunkPlan& p);

}  // namespace slw
