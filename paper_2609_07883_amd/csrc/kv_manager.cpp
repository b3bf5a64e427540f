// Host-side paged-KV block manager (Table 1, "KV manager").
#include "kv_manager.h"

#include <algorithm>
#include <unordered_map>

#include "common.h"

namespace slw {

void KvManager::reset(int32_t num_blocks, int32_t block_size) {
    num_blocks_ = num_blocks;
    block_size_ = block_size;
    seqs_.clear();
    std::vector<int32_t> ids(num_blocks);
    for (int32_t i = 0; i < num_blocks; ++i) ids[i] = i;
    free_ = decltype(free_)(std::greater<int32_t>(), std::move(ids));
}

int KvManager::create(int64_t id) {
    if (seqs_.count(id)) return fail(SLW_EINVAL, "sequence %lld already exists", (long long)id);
    seqs_.emplace(id, Seq{});
    return SLW_OK;
}

int KvManager::release(int64_t id) {
    auto it = seqs_.find(id);
    if (it == seqs_.end()) return fail(SLW_EINVAL, "sequence %lld unknown", (long long)id);
    for (int32_t b : it->second.blocks) free_.push(b);
    seqs_.erase(it);
    return SLW_OK;
}

// Room for the blocks is there (reserve_batch), so nothing here can fail.
void KvManager::grow(Seq& s, int32_t len, Undo* undo) {
    if (len < s.reserved) len = s.reserved;
    const int64_t need = ceil_div(len, block_size_) - static_cast<int64_t>(s.blocks.size());
    if (undo) undo->grown.push_back({&s, s.blocks.size(), s.reserved});
    for (int64_t i = 0; i < need; ++i) {
        s.blocks.push_back(free_.top());
        free_.pop();
    }
    s.reserved = len;
}

int KvManager::reserve_all(const std::vector<std::pair<int64_t, int32_t>>& req, Undo* undo) {
    if (undo) undo->grown.clear();
    // Largest request per sequence, in request order so block ids are deterministic.
    std::vector<std::pair<Seq*, int32_t>> want;
    std::unordered_map<Seq*, size_t> at;
    for (const auto& r : req) {
        Seq* s = find(r.first);
        if (!s) return fail(SLW_EINVAL, "sequence %lld unknown", (long long)r.first);
        if (r.second < 0) return fail(SLW_EINVAL, "negative length for sequence %lld", (long long)r.first);
        const auto w = at.emplace(s, want.size());
        if (w.second) want.emplace_back(s, r.second);
        else if (r.second > want[w.first->second].second) want[w.first->second].second = r.second;
    }
    return reserve_batch(want, undo);
}

int KvManager::reserve_batch(const std::vector<std::pair<Seq*, int32_t>>& req, Undo* undo) {
    if (undo) undo->grown.clear();
    int64_t total = 0;
    for (const auto& r : req) {
        const int64_t len = r.second > r.first->reserved ? r.second : r.first->reserved;
        const int64_t need = ceil_div(len, block_size_) - static_cast<int64_t>(r.first->blocks.size());
        if (need > 0) total += need;
    }
    if (total > static_cast<int64_t>(free_.size()))
        return fail(SLW_ENOMEM, "KV pool exhausted: need %lld blocks, %d free", (long long)total,
                    free_count());
    // every allocation before the first block is taken
    if (undo) undo->grown.reserve(req.size());
    for (const auto& r : req) {
        std::vector<int32_t>& blocks = r.first->blocks;
        const size_t need = static_cast<size_t>(ceil_div(std::max(r.second, r.first->reserved), block_size_));
        if (need > blocks.capacity()) blocks.reserve(std::max(need, 2 * blocks.capacity()));
    }
    for (const auto& r : req) grow(*r.first, r.second, undo);
    return SLW_OK;
}

void KvManager::rollback(const Undo& undo) {
    for (auto e = undo.grown.rbegin(); e != undo.grown.rend(); ++e) {
        while (e->seq->blocks.size() > e->blocks) {
            free_.push(e->seq->blocks.back());
            e->seq->blocks.pop_back();
        }
        e->seq->reserved = e->reserved;
    }
}

}  // namespace slw
