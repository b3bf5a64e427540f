// Host-side paged-KV block manager (Table 1, "KV manager").
//
// Blocks of 16 positions; a sequence grows by whole blocks taking the
// lowest-numbered free block first; a group of reservations is all or nothing.
#pragma once

#include <cstdint>
#include <functional>
#include <queue>
#include <unordered_map>
#include <utility>
#include <vector>

namespace slw {

class KvManager {
public:
    struct Seq {
        std::vector<int32_t> blocks;
        int32_t reserved = 0;
        uint64_t batch = 0;  // the last batch that named it (next_batch)
        int32_t slot(int32_t pos, int32_t block_size) const {
            return blocks[pos / block_size] * block_size + pos % block_size;
        }
    };
    void reset(int32_t num_blocks, int32_t block_size);
    int32_t num_blocks() const { return num_blocks_; }
    int32_t block_size() const { return block_size_; }
    int32_t free_count() const { return static_cast<int32_t>(free_.size()); }

    bool exists(int64_t id) const { return seqs_.count(id) != 0; }
    // The sequence, or null.  Stays where it is until it is released.
    Seq* find(int64_t id) {
        const auto it = seqs_.find(id);
        return it == seqs_.end() ? nullptr : &it->second;
    }
    uint64_t next_batch() { return ++batch_; }
    // Each returns an SLW_* code (and sets the error message on failure).
    int create(int64_t id);
    int release(int64_t id);
    // What a reservation changed: per grown sequence, its block count and
    // reserved length before the call.
    struct Undo {
        struct Entry {
            Seq* seq;
            size_t blocks;
            int32_t reserved;
        };
        std::vector<Entry> grown;
    };
    // Grows every (id, new_len) in order; all or nothing, also where host memory
    // runs out.  With `undo`, the changes are recorded so that rollback() can
    // return them.
    int reserve_all(const std::vector<std::pair<int64_t, int32_t>>& req, Undo* undo = nullptr);
    // The same for distinct sequences already looked up.
    int reserve_batch(const std::vector<std::pair<Seq*, int32_t>>& req, Undo* undo);
    // Returns the blocks a reservation took and restores the lengths; the
    // free set, and so every later allocation, is as before the reservation.
    void rollback(const Undo& undo);
    // A reservation for a call that may still fail: returned when the call
    // leaves without keep(), by an exception too.
    class Reservation {
    public:
        explicit Reservation(KvManager& kv) : kv_(kv) {}
        Reservation(const Reservation&) = delete;
        Reservation& operator=(const Reservation&) = delete;
        ~Reservation() {
            if (!kept_) kv_.rollback(undo_);
        }
        int reserve(const std::vector<std::pair<Seq*, int32_t>>& req) { return kv_.reserve_batch(req, &undo_); }
        void keep() { kept_ = true; }

    private:
        KvManager& kv_;
        Undo undo_;
        bool kept_ = false;
    };

    const std::vector<int32_t>& table(int64_t id) const { return seqs_.at(id).blocks; }

private:
    void grow(Seq& s, int32_t len, Undo* undo);
    uint64_t batch_ = 0;
    int32_t num_blocks_ = 0;
    int32_t block_size_ = 16;
    std::priority_queue<int32_t, std::vector<int32_t>, std::greater<int32_t>> free_;
    std::unordered_map<int64_t, Seq> seqs_;
};

}  // namespace slw
