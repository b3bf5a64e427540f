"""The block manager where host memory runs out: a reservation that fails on any of its allocations leaves the manager
as it was, and one whose caller fails later returns its blocks (a C++ program built here; CPU)."""
import os
import subprocess

from paper_2609_07883_amd import build

SOURCE = r"""
#include <cstdio>
#include <cstdlib>
#include <new>

#include "kv_manager.h"

static long countdown = -1;  // allocations until one fails; negative: none does
void* operator new(size_t n) {
    if (countdown == 0) throw std::bad_alloc();
    if (countdown > 0) --countdown;
    if (void* p = std::malloc(n)) return p;
    throw std::bad_alloc();
}
void operator delete(void* p) noexcept { std::free(p); }
void operator delete(void* p, size_t) noexcept { std::free(p); }

using slw::KvManager;

static void start(KvManager& kv) {
    kv.reset(400, 16);
    for (int id = 1; id <= 4; ++id) kv.create(id);
    kv.reserve_all({{1, 40}, {2, 16}, {3, 100}});
}
static bool as_started(const KvManager& kv) {
    KvManager fresh;
    start(fresh);
    bool ok = kv.free_count() == fresh.free_count();
    for (int id = 1; id <= 4; ++id) ok = ok && kv.table(id) == fresh.table(id);
    return ok;
}
static int bad(const char* what, long n) {
    std::printf("%s, allocation %ld\n", what, n);
    return 1;
}

int main() {
    const std::vector<std::pair<int64_t, int32_t>> want = {{1, 41}, {2, 900}, {4, 2000}, {3, 1700}};
    for (int way = 0; way < 2; ++way) {  // every allocation of a reservation in turn, by both ways in
        long n = 0;
        for (;; ++n) {
            KvManager kv;
            start(kv);
            std::vector<std::pair<KvManager::Seq*, int32_t>> seqs;
            for (const auto& w : want) seqs.emplace_back(kv.find(w.first), w.second);
            KvManager::Undo undo;
            countdown = n;
            try {
                const int rc = way ? kv.reserve_all(want) : kv.reserve_batch(seqs, &undo);
                countdown = -1;
                if (rc) return bad("refused", n);
                break;
            } catch (const std::bad_alloc&) {
                countdown = -1;
            }
            if (!as_started(kv)) return bad("changed by a reservation that failed", n);
        }
        if (n < 4) return bad("no allocation failed", n);
    }
    KvManager kv;  // a caller that fails after it reserved, and one that does not
    start(kv);
    std::vector<std::pair<KvManager::Seq*, int32_t>> seqs;
    for (const auto& w : want) seqs.emplace_back(kv.find(w.first), w.second);
    try {
        KvManager::Reservation r(kv);
        if (r.reserve(seqs)) return bad("refused", -1);
        throw std::bad_alloc();
    } catch (const std::bad_alloc&) {
    }
    if (!as_started(kv)) return bad("blocks of a call that failed are gone", -1);
    {
        KvManager::Reservation r(kv);
        if (r.reserve(seqs)) return bad("refused", -1);
        r.keep();
    }
    if (kv.find(2)->reserved != 900 || kv.find(4)->blocks.size() != 125) return bad("a reservation that was kept is gone", -1);
    std::puts("ok");
    return 0;
}
"""


def test_reservations_without_memory(tmp_path):
    (tmp_path / "t.cpp").write_text(SOURCE)
    exe = str(tmp_path / "t")
    r = subprocess.run(["g++", *build.CXX_FLAGS, str(tmp_path / "t.cpp"), os.path.join(build.CSRC, "kv_manager.cpp"),
                        os.path.join(build.CSRC, "errors.cpp"), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout + r.stderr
