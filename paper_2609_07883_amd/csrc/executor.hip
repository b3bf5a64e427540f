// Context, paged-KV bookkeeping, the mixed iteration and the cost profiler.
//
// A mixed iteration (Sec. 3: one prefill chunk plus one token for every
// active decode; Sec. 5.1: the chunk arrives through ordinary sequence
// metadata) is: host-side reservation and slot mapping, one upload of the
// per-iteration metadata through a pinned staging ring, a RoPE table for the
// iteration's positions, then per layer: RMSNorm, QKV GEMM (RoPE and KV
// append in its epilogue; over 8-bit pools the append is a kernel of its own),
// chunk and decode attention, output GEMM into an fp32 residual, RMSNorm,
// gate/up GEMM (SiLU*mul epilogue), down GEMM.
#include <algorithm>
#include <atomic>
#include <chrono>
#include <cmath>
#include <cstring>
#include <limits>
#include <memory>
#include <mutex>
#include <random>
#include <vector>

#include "attn_plan.h"
#include "common.h"
#include "cost_table.h"
#include "hip_try.h"
#include "kernels.h"
#include "kv_manager.h"

using namespace slw;

namespace {

constexpr int kRing = 4;                 // pinned staging buffers in flight
constexpr size_t kAlign = 256;
constexpr int64_t kLastLevelCache = 256 << 20;

size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

}  // namespace

struct slw_ctx {
    slw_model_cfg cfg{};
    std::vector<slw_layer_weights> w;
    std::vector<char> have_w;
    void* k_pool = nullptr;
    void* v_pool = nullptr;
    float* k_scale = nullptr;   // e4m3 pools: their scales (null: bf16 pools)
    float* v_scale = nullptr;
    KvManager kv;
    bool kv_ready = false;
    uint64_t kv_id = 0;         // changes with every attachment of pools, and differs between contexts
    Window win;                 // attention window of the layers flagged in `windowed`
    std::vector<char> windowed;
    bool any_windowed = false, any_full = true;
    std::vector<int32_t> last_slots;
    std::vector<int32_t> slots_build;  // slots of the iteration being built
    std::vector<Prefill> prefills;     // the iteration's prefills in row order
    // the batch's sequences and the lengths they need: prefills, then decodes
    std::vector<std::pair<KvManager::Seq*, int32_t>> batch_seqs;
    std::vector<int32_t> meta;  // host build area
    DecodePlan dplan;           // attention work of one class of layers (host build areas)
    ChunkPlan cplan;

    // HIP resources, created on first device use
    bool hip_ready = false;
    int32_t* staging[kRing] = {};      // coherent pinned host memory
    int32_t* staging_dev[kRing] = {};  // the same memory's device address
    size_t staging_cap[kRing] = {};
    hipEvent_t staged[kRing] = {};
    int ring = 0;

    // stage telemetry: a ring of `stage_depth` event sets, each [layer][stage boundary]
    int stage_depth = 0;
    std::vector<hipEvent_t> stage_ev;
    std::vector<uint32_t> stage_mask;  // per set: stages that iteration ran (0: none recorded)
    int64_t stage_iter = 0;            // iterations recorded so far

    ~slw_ctx() {
        if (!hip_ready) return;
        for (int i = 0; i < kRing; ++i) {
            if (staged[i]) {
                (void)hipEventSynchronize(staged[i]);
                (void)hipEventDestroy(staged[i]);
            }
            if (staging[i]) (void)hipHostFree(staging[i]);
        }
        for (hipEvent_t e : stage_ev) (void)hipEventDestroy(e);
    }
};

namespace {

int qkv_width(const slw_model_cfg& c) { return (c.n_q_heads + 2 * c.n_kv_heads) * c.head_dim; }
int max_blocks(const slw_model_cfg& c) { return static_cast<int>(ceil_div(c.max_pos, 16)); }
// Blocks a batch of C chunk rows and B decodes appends to: each prompt may
// begin and end inside a block.
size_t append_cap(int C, int B) {
    const size_t np = std::min(C, static_cast<int>(SLW_MAX_PREFILLS));
    return std::min<size_t>(C, C / 16 + 2 * np) + B;
}

// Metadata of the two attentions and, where wanted, the append (32-bit words):
// block tables, query tiles, blocks to append to, and the work lists of each
// class of layers (full attention, windowed).
size_t attn_meta_ints(const slw_ctx& ctx, int C, int B, bool append) {
    const slw_model_cfg& c = ctx.cfg;
    const size_t mb = static_cast<size_t>(max_blocks(c));
    const size_t np = C > 0 ? static_cast<size_t>(std::min(C, static_cast<int>(SLW_MAX_PREFILLS))) : 0;
    const size_t work = decode_work_cap(c, B), items = chunk_item_cap(c, C);
    const size_t per_class = (B + 1) + decode_slot_cap(c) + 1 + static_cast<size_t>(chunk_tiles(c, C)) + 1 + chunk_slot_cap(c) + 1;
    const size_t cache_classes = ctx.any_windowed + (ctx.any_full && ctx.k_scale);
    return B + (B + 1) + static_cast<size_t>(B) * mb + np * mb + 4 * static_cast<size_t>(chunk_tiles(c, C)) +
           (append ? 4 * append_cap(C, B) : 0) + per_class * (ctx.any_full + ctx.any_windowed) +
           (ctx.any_full && !ctx.k_scale ? 3 * work + 4 * items : 0) + 8 * (work + items) * cache_classes;
}

// An iteration appends to bf16 pools in the QKV projection's epilogue.
bool iteration_appends(const slw_ctx& ctx) { return ctx.k_scale != nullptr; }

size_t meta_ints(const slw_ctx& ctx, int C, int B) {
    return 2 * (static_cast<size_t>(C) + B) + attn_meta_ints(ctx, C, B, iteration_appends(ctx));
}

// Partial sums of the two attentions, after `off`.
struct PartLayout {
    size_t part_o, part_ml, cpart_o, cpart_ml, end;
};
PartLayout part_layout(const slw_model_cfg& c, int C, int B, size_t off) {
    PartLayout P{};
    auto take = [&](size_t bytes) {
        size_t at = off;
        off += align_up(bytes);
        return at;
    };
    const int W = decode_work_cap(c, B);
    P.part_o = take(B > 0 ? static_cast<size_t>(W) * c.n_q_heads * c.head_dim * 4 : 0);
    P.part_ml = take(B > 0 ? static_cast<size_t>(W) * c.n_q_heads * 2 * 4 : 0);
    const size_t crows = static_cast<size_t>(chunk_item_cap(c, C)) * c.n_kv_heads * 256;
    P.cpart_o = take(crows * c.head_dim * 4);
    P.cpart_ml = take(crows * 2 * 4);
    P.end = off;
    return P;
}

struct Layout {
    size_t xn, qkv, attn, h, act, rope, meta, gemm_part, end_fixed;
    PartLayout part;
    size_t gemm_part_bytes;  // from gemm_part on; set where the workspace is known
};

Layout layout(const slw_ctx& ctx, int C, int B) {
    const slw_model_cfg& c = ctx.cfg;
    const size_t M = static_cast<size_t>(C) + B;
    Layout L{};
    size_t off = 0;
    auto take = [&](size_t bytes) {
        size_t at = off;
        off += align_up(bytes);
        return at;
    };
    L.xn = take(M * c.d_model * 2);
    L.qkv = take(M * qkv_width(c) * 2);
    L.attn = take(M * c.n_q_heads * c.head_dim * 2);
    L.h = take(M * c.d_model * 4);  // fp32 residual stream inside the layer
    L.act = take(M * c.ffn_dim * 2);
    L.rope = take(M * (c.head_dim / 2) * 8);
    L.meta = take(meta_ints(ctx, C, B) * 4);
    L.part = part_layout(c, C, B, off);
    off = L.part.end;
    L.gemm_part = off;  // split-K partials take the rest of the workspace
    L.end_fixed = off;
    return L;
}

// GEMM plans of a layer's four projections at M rows.
struct LayerPlans {
    GemmPlan qkv, o, gu, d;
    size_t partial_bytes() const {
        return std::max(std::max(qkv.partial_bytes, o.partial_bytes), std::max(gu.partial_bytes, d.partial_bytes));
    }
    bool ok(const slw_model_cfg& c, int M) const {
        return gemm_plan_ok(qkv, M, qkv_width(c), c.d_model, false) &&
               gemm_plan_ok(o, M, c.d_model, c.n_q_heads * c.head_dim, false) &&
               gemm_plan_ok(gu, M, 2 * c.ffn_dim, c.d_model, true) && gemm_plan_ok(d, M, c.d_model, c.ffn_dim, false);
    }
};

LayerPlans plan_layer(const slw_model_cfg& c, int M) {
    return {plan_gemm(M, qkv_width(c), c.d_model, false), plan_gemm(M, c.d_model, c.n_q_heads * c.head_dim, false),
            plan_gemm(M, 2 * c.ffn_dim, c.d_model, true), plan_gemm(M, c.d_model, c.ffn_dim, false)};
}

int check_cfg(const slw_model_cfg& c) {
    if (c.n_layers < 1) return fail(SLW_EINVAL, "n_layers must be >= 1");
    if (c.head_dim != 64 && c.head_dim != 128) return fail(SLW_EUNSUPPORTED, "head_dim must be 64 or 128");
    if (c.n_q_heads < 1 || c.n_kv_heads < 1 || c.n_q_heads % c.n_kv_heads)
        return fail(SLW_EINVAL, "n_q_heads must be a positive multiple of n_kv_heads");
    const int group = c.n_q_heads / c.n_kv_heads;
    if (group > 16 || (group & (group - 1))) return fail(SLW_EUNSUPPORTED, "GQA group must be 1, 2, 4, 8 or 16");
    if (c.d_model < 128 || c.d_model % 128 || c.d_model > 8192)
        return fail(SLW_EUNSUPPORTED, "d_model must be a multiple of 128 in [128, 8192]");
    if (c.ffn_dim < 64 || c.ffn_dim % 64) return fail(SLW_EUNSUPPORTED, "ffn_dim must be a multiple of 64");
    if (qkv_width(c) % 128) return fail(SLW_EUNSUPPORTED, "(Hq + 2 Hkv) * hd must be a multiple of 128");
    if ((c.n_q_heads * c.head_dim) % 64) return fail(SLW_EUNSUPPORTED, "Hq * hd must be a multiple of 64");
    if (c.block_size != 16) return fail(SLW_EUNSUPPORTED, "block_size must be 16");
    if (c.max_pos < 1 || c.max_pos > (1 << 20)) return fail(SLW_EINVAL, "max_pos out of range");
    if (!(c.rms_eps > 0.f) || !(c.rope_theta > 0.f)) return fail(SLW_EINVAL, "rms_eps and rope_theta must be > 0");
    return SLW_OK;
}

int check_window(const slw_model_cfg& c, int32_t window, int32_t sinks) {
    if (window < 0) return fail(SLW_EINVAL, "negative window");
    if (sinks < 0 || sinks > c.max_pos) return fail(SLW_EINVAL, "sinks must be in [0, max_pos]");
    if (window == 0 && sinks > 0) return fail(SLW_EINVAL, "sinks without a window");
    return SLW_OK;
}

// The staging events order work on this device only: an event
// tells the host that the set-up kernel has finished reading a pinned buffer
// (nothing the GPU wrote has to reach the host).  Without the system-scope
// fence an event record does no cache write-back and invalidation (the CUs sat idle
// for 6-11 us at each record): 8B-layer sweep +1.4%, chat mix +1.6%.
constexpr unsigned kSyncEventFlags = hipEventDisableTiming | hipEventDisableSystemFence;

int ensure_hip(slw_ctx* ctx) {
    if (ctx->hip_ready) return SLW_OK;
    for (int i = 0; i < kRing; ++i) HIP_TRY(hipEventCreateWithFlags(&ctx->staged[i], kSyncEventFlags));
    ctx->hip_ready = true;
    return SLW_OK;
}

// Pinned buffer of the next ring slot with room for n ints (waits for its
// last copy).  The buffers are coherent and mapped: the iteration's first
// kernel reads them over the bus, so the upload needs no copy engine.
int next_staging(slw_ctx* ctx, size_t n, int32_t** buf, int* slot_out) {
    const int slot = ctx->ring;
    ctx->ring = (ctx->ring + 1) % kRing;
    HIP_TRY(hipEventSynchronize(ctx->staged[slot]));
    if (ctx->staging_cap[slot] < n) {
        if (ctx->staging[slot]) HIP_TRY(hipHostFree(ctx->staging[slot]));
        ctx->staging[slot] = nullptr;
        ctx->staging_dev[slot] = nullptr;
        ctx->staging_cap[slot] = 0;
        size_t cap = std::max<size_t>(n, 1 << 16);
        void* p = nullptr;
        HIP_TRY(hipHostMalloc(&p, cap * 4, hipHostMallocMapped | hipHostMallocCoherent));
        ctx->staging[slot] = static_cast<int32_t*>(p);
        void* dp = nullptr;
        HIP_TRY(hipHostGetDevicePointer(&dp, p, 0));
        ctx->staging_dev[slot] = static_cast<int32_t*>(dp);
        ctx->staging_cap[slot] = cap;
    }
    *buf = ctx->staging[slot];
    *slot_out = slot;
    return SLW_OK;
}

constexpr int kStages = SLW_N_STAGES;

int ensure_stage_events(slw_ctx* ctx) {
    const size_t need = static_cast<size_t>(ctx->stage_depth) * ctx->cfg.n_layers * (kStages + 1);
    while (ctx->stage_ev.size() < need) {
        hipEvent_t e;
        HIP_TRY(hipEventCreate(&e));
        ctx->stage_ev.push_back(e);
    }
    return SLW_OK;
}

// Validates a batch with rows: ctx->prefills receives its prefills in row
// order, ctx->batch_seqs its sequences and the lengths to reserve.
int check_batch(slw_ctx* ctx, const slw_batch* bt) {
    const slw_model_cfg& c = ctx->cfg;
    const int C = bt->C, B = bt->B;
    if (B > 0 && (!bt->decode_seqs || !bt->context_lens)) return fail(SLW_EINVAL, "null decode arrays");
    std::vector<Prefill>& pre = ctx->prefills;
    pre.clear();
    if (bt->n_prefill > 1) {
        if (bt->n_prefill > SLW_MAX_PREFILLS) return fail(SLW_ERANGE, "n_prefill %d above %d", bt->n_prefill, SLW_MAX_PREFILLS);
        if (!bt->prefill_seqs || !bt->prefix_lens || !bt->chunk_lens) return fail(SLW_EINVAL, "null prefill arrays");
        int64_t rows = 0;
        for (int i = 0; i < bt->n_prefill; ++i) {
            if (bt->chunk_lens[i] < 1) return fail(SLW_EINVAL, "prefill %d has chunk_len %d", i, bt->chunk_lens[i]);
            pre.push_back({bt->prefill_seqs[i], bt->prefix_lens[i], bt->chunk_lens[i], static_cast<int32_t>(rows)});
            rows += bt->chunk_lens[i];
        }
        if (rows != C) return fail(SLW_EINVAL, "chunk_lens add up to %lld, C is %d", (long long)rows, C);
    } else if (C > 0) {
        pre.push_back({bt->prefill_seq, bt->prefix_len, C, 0});
    }
    auto& seqs = ctx->batch_seqs;
    seqs.clear();
    seqs.reserve(B + pre.size());
    const uint64_t batch = ctx->kv.next_batch();  // a sequence that carries it was named before
    for (const Prefill& f : pre) {
        if (f.prefix < 0) return fail(SLW_EINVAL, "negative prefix_len");
        if (static_cast<int64_t>(f.prefix) + f.c > c.max_pos) return fail(SLW_ERANGE, "prefix_len + chunk exceeds max_pos");
        KvManager::Seq* q = ctx->kv.find(f.seq);
        if (!q) return fail(SLW_EINVAL, "prefill sequence %lld unknown", (long long)f.seq);
        if (q->batch == batch) return fail(SLW_EINVAL, "sequence %lld appears twice in the batch", (long long)f.seq);
        q->batch = batch;
        if (q->reserved < f.prefix)
            return fail(SLW_EINVAL, "prefill sequence %lld holds %d positions, prefix_len is %d", (long long)f.seq,
                        q->reserved, f.prefix);
        seqs.emplace_back(q, f.prefix + f.c);
    }
    for (int b = 0; b < B; ++b) {
        const int64_t id = bt->decode_seqs[b];
        const int32_t L = bt->context_lens[b];
        KvManager::Seq* q = ctx->kv.find(id);
        if (!q) return fail(SLW_EINVAL, "decode sequence %lld unknown", (long long)id);
        if (q->batch == batch) return fail(SLW_EINVAL, "sequence %lld appears twice in the batch", (long long)id);
        q->batch = batch;
        if (L < 0 || L + 1 > c.max_pos) return fail(SLW_ERANGE, "context_len %d out of range", L);
        if (q->reserved < L)
            return fail(SLW_EINVAL, "decode sequence %lld holds %d positions, context_len is %d", (long long)id,
                        q->reserved, L);
        seqs.emplace_back(q, L + 1);
    }
    return SLW_OK;
}

int enqueue_iteration(slw_ctx* ctx, const slw_batch* bt, const void* x_in, void* x_out, void* ws,
                      const Layout& L, const LayerPlans& plans, hipStream_t stream, bool no_alloc);

// One iteration: validation, KV reservation (all or nothing), then the
// metadata, its upload and the kernels.  A failure after the reservation, an
// exception too, returns the reserved blocks, so a failed call leaves the block
// manager as it found it.  no_alloc: the workspace is the static array, the
// metadata is copied with hipMemcpyAsync from host memory the context holds,
// both attentions run on `stream` and no stage events are recorded, so the call
// creates no HIP object and allocates no memory of any kind on the device or
// pinned on the host.
int mixed_iteration_impl(slw_ctx* ctx, const slw_batch* bt, const void* x_in, void* x_out, void* ws,
                         size_t ws_bytes, hipStream_t stream, bool no_alloc = false) {
    const slw_model_cfg& c = ctx->cfg;
    if (!bt) return fail(SLW_EINVAL, "null batch");
    const int C = bt->C, B = bt->B;
    if (C < 0 || B < 0) return fail(SLW_EINVAL, "negative C or B");
    if (C == 0 && B == 0) {
        ctx->last_slots.clear();
        return SLW_OK;
    }
    if (!ctx->kv_ready) return fail(SLW_EINVAL, "KV pools not attached (slw_kv_init)");
    for (int l = 0; l < c.n_layers; ++l)
        if (!ctx->have_w[l]) return fail(SLW_EINVAL, "weights of layer %d not set", l);
    if (!x_in || !x_out || !ws) return fail(SLW_EINVAL, "null device buffer");
    int rc = check_batch(ctx, bt);
    if (rc) return rc;
    Layout L = layout(*ctx, C, B);
    const LayerPlans plans = plan_layer(c, C + B);
    if (!plans.ok(c, C + B)) return fail(SLW_EINVAL, "internal: GEMM plan");
    size_t need = L.end_fixed + plans.partial_bytes();
    // The static array also takes an iteration whose split-K partials alone
    // would not fit: they then share the room of the attention partials, which
    // no product runs beside, and the products run in blocks of as many rows
    // as fit there, with the same plans and so the same results.
    if (no_alloc && ws_bytes < need) {
        L.gemm_part = L.part.part_o;
        need = std::max(L.end_fixed, L.gemm_part + plans.partial_bytes() / (C + B));
    }
    if (ws_bytes < need)
        return fail(SLW_ENOMEM, "%s holds %zu bytes, this iteration needs %zu",
                    no_alloc ? "the static workspace (SLW_STATIC_WS_BYTES)" : "the workspace", ws_bytes, need);
    L.gemm_part_bytes = ws_bytes - L.gemm_part;
    if (!no_alloc) {
        rc = ensure_hip(ctx);
        if (rc) return rc;
        if (ctx->stage_depth > 0) {
            rc = ensure_stage_events(ctx);
            if (rc) return rc;
        }
    }
    KvManager::Reservation room(ctx->kv);
    if ((rc = room.reserve(ctx->batch_seqs))) return rc;
    if ((rc = enqueue_iteration(ctx, bt, x_in, x_out, ws, L, plans, stream, no_alloc))) return rc;
    room.keep();
    return SLW_OK;
}

// Where a batch's attention metadata lies (32-bit words from its start) and
// how long its lists are.
struct AttnMeta {
    int C = 0, B = 0, n_qt = 0, n_app = 0;
    size_t kvlen = 0, btoff = 0, bt = 0, pre = 0, qt = 0, app = 0;
    struct Class {  // the work lists of full ([0]) or windowed ([1]) layers
        int n_work = 0, n_dslots = 0, n_items = 0, n_slots = 0;
        size_t work = 0, work_off = 0, decode_slot = 0, item = 0, slot = 0, slot_items = 0, qtoff = 0;
        bool two_phase = false;
        int64_t decode_keys = 0;
    } cls[2];
};

// Appends the metadata of both attentions and, with `append`, of the append to
// m; offsets count from m's start.
int build_attn_meta(slw_ctx* ctx, const slw_batch* bt, bool append, std::vector<int32_t>& m, AttnMeta& am) {
    const slw_model_cfg& c = ctx->cfg;
    const int C = bt->C, B = bt->B;
    const std::vector<Prefill>& pre = ctx->prefills;
    int rc = SLW_OK;
    auto put = [&](const std::vector<int32_t>& v) {
        const size_t at = m.size();
        m.insert(m.end(), v.begin(), v.end());
        return at;
    };
    am.C = C;
    am.B = B;
    am.kvlen = m.size();
    for (int b = 0; b < B; ++b) m.push_back(bt->context_lens[b] + 1);
    am.btoff = m.size();
    m.resize(m.size() + B + 1);
    am.bt = m.size();
    for (int b = 0; b < B; ++b) {
        m[am.btoff + b] = static_cast<int32_t>(m.size() - am.bt);
        const auto& t = ctx->batch_seqs[pre.size() + b].first->blocks;
        const int nb = static_cast<int>(ceil_div(bt->context_lens[b] + 1, 16));
        m.insert(m.end(), t.begin(), t.begin() + nb);
    }
    m[am.btoff + B] = static_cast<int32_t>(m.size() - am.bt);
    // block tables of the prefills, one after the other
    am.pre = m.size();
    std::vector<int32_t> pre_bt(pre.size());
    for (size_t i = 0; i < pre.size(); ++i) {
        pre_bt[i] = static_cast<int32_t>(m.size() - am.pre);
        const auto& t = ctx->batch_seqs[i].first->blocks;
        const int nb = static_cast<int>(ceil_div(pre[i].prefix + pre[i].c, 16));
        m.insert(m.end(), t.begin(), t.begin() + nb);
    }
    // Each prefill's rows are cut into query tiles (a tile never mixes
    // sequences); query tile q covers chunk rows qt_row0 .. + qt_rows at
    // positions from qt_pos0 on and reads the block table at qt_bt, over keys
    // 0 .. qt_pos0 + qt_rows - 1.
    std::vector<int32_t> qt_row0, qt_rows, qt_pos0, qt_bt;
    query_tiles(c, pre, qt_row0, qt_rows, qt_pos0, &qt_bt, pre_bt);
    const int n_qt = static_cast<int>(qt_row0.size());
    if (n_qt > chunk_tiles(c, C)) return fail(SLW_EINVAL, "internal: %d query tiles above cap", n_qt);
    am.n_qt = n_qt;
    am.qt = put(qt_row0);  // [4][n_qt]: first row, rows, first position, block-table offset
    put(qt_rows);
    put(qt_pos0);
    put(qt_bt);
    if (append) {  // [4][n_app]: block, first new token, new tokens, first row of each block appended to
        std::vector<int32_t> app[4];
        for (auto& v : app) v.reserve(append_cap(C, B));
        auto add = [&](const KvManager::Seq* q, int at, int n, int row) {
            const auto& t = q->blocks;
            for (const int end = at + n; at < end;) {
                const int k = std::min(16 - at % 16, end - at);
                app[0].push_back(t[at / 16]);
                app[1].push_back(at % 16);
                app[2].push_back(k);
                app[3].push_back(row);
                at += k;
                row += k;
            }
        };
        for (size_t i = 0; i < pre.size(); ++i) add(ctx->batch_seqs[i].first, pre[i].prefix, pre[i].c, pre[i].row0);
        for (int b = 0; b < B; ++b) add(ctx->batch_seqs[pre.size() + b].first, bt->context_lens[b], 1, C + b);
        am.n_app = static_cast<int>(app[0].size());
        if (app[0].size() > append_cap(C, B)) return fail(SLW_EINVAL, "internal: %d blocks to append to above cap", am.n_app);
        am.app = m.size();
        for (const auto& v : app) put(v);
    }

    for (int k = 0; k < 2; ++k) {
        if (!(k ? ctx->any_windowed : ctx->any_full)) continue;
        AttnMeta::Class& cl = am.cls[k];
        const Window w = k ? ctx->win : Window{};
        const bool cache = k || ctx->k_scale;
        // plan_chunk hands the query tiles out to the work-groups.  A tile
        // covered by one item is written directly, one covered by several is
        // combined by the merge kernel.
        ChunkPlan& cp = ctx->cplan;
        if ((rc = plan_chunk(c, w, cache, C, qt_pos0, qt_rows, cp))) return rc;
        cl.n_items = static_cast<int>(cp.items.size() / 3);
        cl.n_slots = static_cast<int>(cp.slot_off.size()) - 1;
        cl.slot = put(cp.slot_off);
        cl.qtoff = put(cp.qt_off);
        cl.item = m.size();
        if (!cache) {
            m.resize(m.size() + cp.items.size());
            for (int i = 0; i < cl.n_items; ++i)
                for (int j = 0; j < 3; ++j) m[cl.item + static_cast<size_t>(j) * cl.n_items + i] = cp.items[3 * i + j];
            cl.slot_items = put(cp.slot_items);
        } else {  // CacheAttnArgs::chunk_items
            m.resize(m.size() + 8 * cp.slot_items.size());
            int32_t* at = m.data() + cl.item;
            for (const int32_t i : cp.slot_items) {
                const int q = cp.items[3 * i];
                const bool whole = cp.qt_off[q + 1] - cp.qt_off[q] == 1;
                const int32_t rec[8] = {whole ? ~i : i, cp.items[3 * i + 1], cp.items[3 * i + 2], qt_row0[q],
                                        qt_rows[q], qt_pos0[q], cp.qt_skip[q], qt_bt[q]};
                at = std::copy(rec, rec + 8, at);
            }
        }
        cl.two_phase = cp.two_phase;
        DecodePlan& dp = ctx->dplan;
        if ((rc = plan_decode(c, w, decode_kind(cache, cp), B, bt->context_lens, dp))) return rc;
        cl.n_work = static_cast<int>(dp.b.size());
        cl.n_dslots = static_cast<int>(dp.slot_off.size()) - 1;
        cl.work_off = put(dp.off);
        cl.decode_slot = put(dp.slot_off);
        if (!cache) {
            cl.work = put(dp.b);
            put(dp.kb);
            put(dp.ke);
        } else {  // CacheAttnArgs::decode_items
            cl.work = m.size();
            m.resize(m.size() + 8 * dp.b.size());
            int32_t* at = m.data() + cl.work;
            for (int i = 0; i < cl.n_work; ++i) {
                const int b = dp.b[i];
                const int32_t rec[8] = {b, dp.kb[i], dp.ke[i], bt->context_lens[b] + 1, dp.skip[b], m[am.btoff + b],
                                        dp.off[b + 1] - dp.off[b] == 1, 0};
                at = std::copy(rec, rec + 8, at);
            }
        }
        for (int b = 0; b < B; ++b) cl.decode_keys += bt->context_lens[b] + 1 - dp.skip[b];
    }
    return SLW_OK;
}

CacheLayer cache_layer(const slw_ctx* ctx, int l) {
    const size_t heads = static_cast<size_t>(ctx->kv.num_blocks()) * ctx->cfg.n_kv_heads * l;  // before the layer
    const size_t at = heads * ctx->cfg.head_dim * 16 * (ctx->k_scale ? 1 : 2);
    return {static_cast<char*>(ctx->k_pool) + at, static_cast<char*>(ctx->v_pool) + at,
            ctx->k_scale ? ctx->k_scale + heads : nullptr, ctx->v_scale ? ctx->v_scale + heads : nullptr,
            ctx->cfg.n_kv_heads, ctx->cfg.head_dim};
}

AppendArgs append_args(const slw_ctx* ctx, const AttnMeta& am, const int32_t* dmeta, int l, const void* k,
                       const void* v, int ld) {
    return {cache_layer(ctx, l), k, v, dmeta + am.app, am.n_app, ld};
}

// The attention of one layer: q rows of stride ld (chunk rows, then decodes),
// out [rows][hq * hd], metadata at dmeta, partial sums at ws + P.
struct AttnCall {
    CacheAttnArgs a{};
    bool cache = false;  // the kernels for e4m3 pools or a window
    AttnCall(const slw_ctx* ctx, const AttnMeta& am, const int32_t* dmeta, char* ws, const PartLayout& P, int l,
             const void* q, int ld, void* out) {
        const slw_model_cfg& c = ctx->cfg;
        const int hq = c.n_q_heads, hkv = c.n_kv_heads, hd = c.head_dim;
        const AttnMeta::Class& cl = am.cls[ctx->windowed[l] ? 1 : 0];
        const CacheLayer pool = cache_layer(ctx, l);
        ChunkAttnArgs& ca = a.chunk;
        if (am.C > 0) {
            ca.qkv = q;
            ca.out = out;
            ca.k_pool = pool.k_pool;
            ca.v_pool = pool.v_pool;
            ca.bt = dmeta + am.pre;
            ca.qt_off = dmeta + cl.qtoff;
            ca.part_o = reinterpret_cast<float*>(ws + P.cpart_o);
            ca.part_ml = reinterpret_cast<float*>(ws + P.cpart_ml);
            ca.c = am.C;
            ca.n_qt = am.n_qt;
            ca.qt_row0 = dmeta + am.qt;
            ca.qt_rows = dmeta + am.qt + am.n_qt;
            ca.qt_pos0 = dmeta + am.qt + 2 * am.n_qt;
            ca.qt_bt = dmeta + am.qt + 3 * am.n_qt;
            ca.hq = hq;
            ca.hkv = hkv;
            ca.hd = hd;
            ca.ld_qkv = ld;
            ca.slot_off = dmeta + cl.slot;
            ca.n_items = cl.n_items;
            ca.n_slots = cl.n_slots;
            ca.split = cl.n_items > am.n_qt ? 1 : 0;
            ca.pp = cl.two_phase ? 1 : 0;
        }
        DecodeAttnArgs& da = a.decode;
        if (am.B > 0) {
            da.q = static_cast<const char*>(q) + static_cast<size_t>(am.C) * ld * 2;
            da.out = static_cast<char*>(out) + static_cast<size_t>(am.C) * hq * hd * 2;
            da.k_pool = pool.k_pool;
            da.v_pool = pool.v_pool;
            da.kv_len = dmeta + am.kvlen;
            da.bt_off = dmeta + am.btoff;
            da.bt = dmeta + am.bt;
            da.work_off = dmeta + cl.work_off;
            da.slot_off = dmeta + cl.decode_slot;
            da.n_slots = cl.n_dslots;
            da.part_o = reinterpret_cast<float*>(ws + P.part_o);
            da.part_ml = reinterpret_cast<float*>(ws + P.part_ml);
            da.b = am.B;
            da.n_work = cl.n_work;
            da.hq = hq;
            da.hkv = hkv;
            da.hd = hd;
            da.ld_q = ld;
        }
        cache = ctx->k_scale || ctx->windowed[l];
        if (cache) {
            da.direct = 1;
            a.k_scale = pool.k_scale;
            a.v_scale = pool.v_scale;
            a.chunk_items = dmeta + cl.item;
            a.decode_items = dmeta + cl.work;
            const Window w = ctx->windowed[l] ? ctx->win : Window{};
            a.window = w.window;
            a.sinks = w.window > 0 ? w.sinks : 0;
            a.sink_end = sink_end(w);
            // the decodes' keys and values of all layers against the last-level cache
            const int64_t windowed = std::count_if(ctx->windowed.begin(), ctx->windowed.end(), [](char f) { return f != 0; });
            const int64_t keys = am.cls[0].decode_keys * (c.n_layers - windowed) + am.cls[1].decode_keys * windowed;
            a.once = keys * 2 * hkv * hd * (ctx->k_scale ? 1 : 2) > kLastLevelCache;
        } else {
            ca.item_qt = dmeta + cl.item;
            ca.item_kb = dmeta + cl.item + cl.n_items;
            ca.item_ke = dmeta + cl.item + 2 * cl.n_items;
            ca.slot_items = dmeta + cl.slot_items;
            da.work_b = dmeta + cl.work;
            da.work_kb = dmeta + cl.work + cl.n_work;
            da.work_ke = dmeta + cl.work + 2 * cl.n_work;
        }
    }
    // The parts: chunk and decode in one launch, or each alone.
    void both(hipStream_t s) const {
        if (cache) launch_cache_attention(a, s);
        else launch_attention(a.chunk, a.decode, s);
    }
    void chunk(hipStream_t s) const {
        if (!cache) return launch_chunk_attention(a.chunk, s);
        CacheAttnArgs x = a;
        x.decode = DecodeAttnArgs{};
        launch_cache_attention(x, s);
    }
    void decode(hipStream_t s) const {
        if (!cache) return launch_decode_attention_split(a.decode, s);
        CacheAttnArgs x = a;
        x.chunk = ChunkAttnArgs{};
        launch_cache_attention(x, s);
    }
    void merge(hipStream_t s) const {
        const bool decodes = !a.decode.direct || a.decode.n_work > a.decode.b;
        launch_attention_merge(&a.chunk, decodes ? &a.decode : nullptr, s);
    }
};

// Metadata, upload and kernels of an iteration whose blocks are reserved.
int enqueue_iteration(slw_ctx* ctx, const slw_batch* bt, const void* x_in, void* x_out, void* ws,
                      const Layout& L, const LayerPlans& plans, hipStream_t stream, bool no_alloc) {
    const slw_model_cfg& c = ctx->cfg;
    const int C = bt->C, B = bt->B;
    const std::vector<Prefill>& pre = ctx->prefills;
    int rc = SLW_OK;

    // ---- metadata (host) ----
    const int M = C + B;

    std::vector<int32_t>& m = ctx->meta;
    m.clear();
    m.reserve(meta_ints(*ctx, C, B));
    // slot[M], pos[M]
    std::vector<int32_t>& slots = ctx->slots_build;
    slots.resize(M);
    for (size_t i = 0; i < pre.size(); ++i)
        for (int j = 0; j < pre[i].c; ++j) slots[pre[i].row0 + j] = ctx->batch_seqs[i].first->slot(pre[i].prefix + j, 16);
    for (int b = 0; b < B; ++b) slots[C + b] = ctx->batch_seqs[pre.size() + b].first->slot(bt->context_lens[b], 16);
    m.insert(m.end(), slots.begin(), slots.end());
    for (const Prefill& f : pre)
        for (int j = 0; j < f.c; ++j) m.push_back(f.prefix + j);
    for (int b = 0; b < B; ++b) m.push_back(bt->context_lens[b]);
    AttnMeta am;
    if ((rc = build_attn_meta(ctx, bt, iteration_appends(*ctx), m, am))) return rc;

    if (m.size() > meta_ints(*ctx, C, B)) return fail(SLW_EINVAL, "internal: metadata %zu ints above its region", m.size());

    // ---- upload ----
    const bool timing = !no_alloc && ctx->stage_depth > 0;
    // the first layer's RMSNorm runs in the setup kernel, or, where stages are
    // timed, as a stage of its own
    const void* setup_x = timing ? nullptr : x_in;
    char* wsb = static_cast<char*>(ws);
    int32_t* dmeta = reinterpret_cast<int32_t*>(wsb + L.meta);
    float2* rope = reinterpret_cast<float2*>(wsb + L.rope);
    if (no_alloc) {
        // From the context's host vector, which the next call refills: a copy
        // from pageable memory may still be reading it when hipMemcpyAsync
        // returns, so the stream is synchronised right after it.
        HIP_TRY(hipMemcpyAsync(dmeta, m.data(), m.size() * 4, hipMemcpyHostToDevice, stream));
        HIP_TRY(hipStreamSynchronize(stream));
        launch_iteration_setup(dmeta, nullptr, 0, dmeta + M, rope, M, c.head_dim, static_cast<double>(c.rope_theta),
                               setup_x, ctx->w[0].g1, wsb + L.xn, c.d_model, c.rms_eps, stream);
        HIP_TRY(hipGetLastError());
    } else {
        int32_t* stage = nullptr;
        int slot = 0;
        rc = next_staging(ctx, m.size(), &stage, &slot);
        if (rc) return rc;
        std::memcpy(stage, m.data(), m.size() * 4);
        // metadata copy, RoPE table (positions follow the M slots) and the first RMSNorm in one kernel
        launch_iteration_setup(dmeta, ctx->staging_dev[slot], m.size(), ctx->staging_dev[slot] + M, rope, M,
                               c.head_dim, static_cast<double>(c.rope_theta), setup_x, ctx->w[0].g1, wsb + L.xn,
                               c.d_model, c.rms_eps, stream);
        HIP_TRY(hipGetLastError());
        HIP_TRY(hipEventRecord(ctx->staged[slot], stream));
    }

    const int32_t* d_slot = dmeta;
    void* xn = wsb + L.xn;
    void* qkv = wsb + L.qkv;
    void* attn = wsb + L.attn;
    void* hbuf = wsb + L.h;
    void* act = wsb + L.act;
    void* gpartp = wsb + L.gemm_part;

    const int d = c.d_model, hq = c.n_q_heads, hkv = c.n_kv_heads, hd = c.head_dim, F = c.ffn_dim;
    const int qw = qkv_width(c);

    size_t set_base = 0;
    int set = 0;
    if (timing) {
        set = static_cast<int>(ctx->stage_iter % ctx->stage_depth);
        set_base = static_cast<size_t>(set) * c.n_layers * (kStages + 1);
        ctx->stage_mask[set] = 0;
    }
    auto mark = [&](int l, int stage) -> int {
        if (timing)
            HIP_TRY(hipEventRecord(ctx->stage_ev[set_base + static_cast<size_t>(l) * (kStages + 1) + stage], stream));
        return SLW_OK;
    };

    for (int l = 0; l < c.n_layers; ++l) {
        const slw_layer_weights& wl = ctx->w[l];
        const void* cur = l == 0 ? x_in : x_out;
        const CacheLayer pool = cache_layer(ctx, l);

        if ((rc = mark(l, 0))) return rc;
        if (l > 0 || !setup_x) launch_rmsnorm(cur, false, wl.g1, xn, M, d, c.rms_eps, stream);
        if ((rc = mark(l, 1))) return rc;  // the RoPE table stage is empty: the setup kernel fills the table
        if ((rc = mark(l, 2))) return rc;
        {
            GemmArgs ga{xn, wl.wqkv, qkv, nullptr, M, qw, d, d, qw, EPI_QKV};
            ga.rope_cs = rope;
            ga.slot = d_slot;
            if (!ctx->k_scale) {
                ga.k_pool = pool.k_pool;
                ga.v_pool = pool.v_pool;
            }
            ga.hq = hq;
            ga.hkv = hkv;
            ga.hd = hd;
            launch_gemm(ga, plans.qkv, gpartp, L.gemm_part_bytes, stream);
            if (ctx->k_scale) {  // e4m3 pools take the rows from the projection's output
                const char* k = static_cast<const char*>(qkv) + static_cast<size_t>(hq) * hd * 2;
                launch_cache_append(append_args(ctx, am, dmeta, l, k, k + static_cast<size_t>(hkv) * hd * 2, qw), stream);
            }
        }
        if ((rc = mark(l, 3))) return rc;
        // Both attentions in one launch; per-stage events separate them.
        const AttnCall attention(ctx, am, dmeta, wsb, L.part, l, qkv, qw, attn);
        if (timing) {
            if (C > 0) attention.chunk(stream);
            if ((rc = mark(l, 4))) return rc;
            if (B > 0) attention.decode(stream);
        } else {
            attention.both(stream);
        }
        if ((rc = mark(l, 5))) return rc;
        attention.merge(stream);
        if ((rc = mark(l, 6))) return rc;
        launch_gemm(GemmArgs{attn, wl.wo, hbuf, cur, M, d, hq * hd, hq * hd, d, EPI_RESID_F32OUT}, plans.o, gpartp,
                    L.gemm_part_bytes, stream);
        if ((rc = mark(l, 7))) return rc;
        const bool gu_norm = plans.gu.cfg == kStreamCfg;  // that kernel normalises its rows itself
        if (!gu_norm) launch_rmsnorm(hbuf, true, wl.g2, xn, M, d, c.rms_eps, stream);
        if ((rc = mark(l, 8))) return rc;
        launch_gemm(GemmArgs{gu_norm ? hbuf : xn, wl.wgu, act, nullptr, M, 2 * F, d, d, F, EPI_SWIGLU}, plans.gu,
                    gpartp, L.gemm_part_bytes, stream, {wl.g2, c.rms_eps});
        if ((rc = mark(l, 9))) return rc;
        launch_gemm(GemmArgs{act, wl.wd, x_out, hbuf, M, d, F, F, d, EPI_RESID_F32IN}, plans.d, gpartp,
                    L.gemm_part_bytes, stream);
        if ((rc = mark(l, 10))) return rc;
    }
    HIP_TRY(hipGetLastError());
    if (timing) {
        // the merge stage (5) runs when decodes or split chunk query tiles need it
        bool merge = false;
        for (int l = 0; l < c.n_layers; ++l) {
            const AttnMeta::Class& cl = am.cls[ctx->windowed[l] ? 1 : 0];
            merge |= cl.n_items > am.n_qt || (ctx->k_scale || ctx->windowed[l] ? cl.n_work > B : B > 0);
        }
        ctx->stage_mask[set] = 0x3FFu & ~(C > 0 ? 0u : (1u << 3)) & ~(B > 0 ? 0u : (1u << 4)) &
                               ~(merge ? 0u : (1u << 5));
        ++ctx->stage_iter;
    }
    ctx->last_slots.swap(slots);
    return SLW_OK;
}

}  // namespace

// ---------------------------------------------------------------------------
// C ABI
// ---------------------------------------------------------------------------

extern "C" int slw_create(const slw_model_cfg* cfg, slw_ctx** out) {
    return guarded([&] {
        if (!cfg || !out) return fail(SLW_EINVAL, "null argument");
        *out = nullptr;
        int rc = check_cfg(*cfg);
        if (rc) return rc;
        auto ctx = std::make_unique<slw_ctx>();
        ctx->cfg = *cfg;
        ctx->w.assign(cfg->n_layers, slw_layer_weights{});
        ctx->have_w.assign(cfg->n_layers, 0);
        ctx->windowed.assign(cfg->n_layers, 0);
        *out = ctx.release();
        return SLW_OK;
    });
}

extern "C" int slw_destroy(slw_ctx* ctx) {
    delete ctx;
    return SLW_OK;
}

namespace {

int attention_plan(const slw_model_cfg* cfg, bool cache, int32_t window, int32_t sinks, int32_t B,
                   const int32_t* context_lens, int32_t n_prefill, const int32_t* prefix_lens,
                   const int32_t* chunk_lens, int64_t out[12]) {
    return guarded([&] {
        if (!cfg || !out || (B > 0 && !context_lens) || (n_prefill > 0 && (!prefix_lens || !chunk_lens)))
            return fail(SLW_EINVAL, "null argument");
        int rc = check_cfg(*cfg);
        if (rc) return rc;
        if ((rc = check_window(*cfg, window, sinks))) return rc;
        if (B < 0 || n_prefill < 0 || n_prefill > SLW_MAX_PREFILLS)
            return fail(SLW_EINVAL, "B >= 0 and 0 <= n_prefill <= %d", SLW_MAX_PREFILLS);
        std::vector<Prefill> pre;
        int C = 0;
        for (int i = 0; i < n_prefill; ++i) {
            if (chunk_lens[i] < 1 || prefix_lens[i] < 0 ||
                static_cast<int64_t>(prefix_lens[i]) + chunk_lens[i] > cfg->max_pos)
                return fail(SLW_EINVAL, "prefill %d: chunk >= 1, prefix >= 0, prefix + chunk <= max_pos", i);
            pre.push_back(Prefill{i, prefix_lens[i], chunk_lens[i], C});
            C += chunk_lens[i];
        }
        for (int b = 0; b < B; ++b)
            if (context_lens[b] < 0 || context_lens[b] >= cfg->max_pos)
                return fail(SLW_EINVAL, "decode %d: context in [0, max_pos)", b);
        DecodePlan dp;
        ChunkPlan cp;
        std::vector<int32_t> row0, rows, pos0;
        query_tiles(*cfg, pre, row0, rows, pos0, nullptr, {});
        const Window win{window, sinks};
        if ((rc = plan_chunk(*cfg, win, cache, C, pos0, rows, cp))) return rc;
        if ((rc = plan_decode(*cfg, win, decode_kind(cache, cp), B, context_lens, dp))) return rc;
        const int dslots = static_cast<int>(dp.slot_off.size()) - 1;
        int64_t dmax = 0, dmin = dslots > 0 ? std::numeric_limits<int64_t>::max() : 0;
        for (int sl = 0; sl < dslots; ++sl) {
            int64_t keys = 0;
            for (int i = dp.slot_off[sl]; i < dp.slot_off[sl + 1]; ++i) keys += dp.ke[i] - dp.kb[i];
            dmax = std::max(dmax, keys);
            dmin = std::min(dmin, keys);
        }
        const int cslots = static_cast<int>(cp.slot_off.size()) - 1;
        int64_t cmax = 0, cmin = cslots > 0 ? std::numeric_limits<int64_t>::max() : 0, ctot = 0;
        for (int g = 0; g < cslots; ++g) {
            int64_t tiles = 0;
            for (int k = cp.slot_off[g]; k < cp.slot_off[g + 1]; ++k) {
                const int i = cp.slot_items[k];
                tiles += ceil_div(cp.items[3 * i + 2], 64) - cp.items[3 * i + 1] / 64;
            }
            cmax = std::max(cmax, tiles);
            cmin = std::min(cmin, tiles);
            ctot += tiles;
        }
        const int64_t v[12] = {static_cast<int64_t>(dp.b.size()), dslots, dmax, dmin,
                               static_cast<int64_t>(rows.size()), static_cast<int64_t>(cp.items.size() / 3), cslots,
                               cp.whole ? 1 : 0, cmax, cmin, ctot, cp.two_phase ? 1 : 0};
        for (int i = 0; i < 12; ++i) out[i] = v[i];
        return SLW_OK;
    });
}

}  // namespace

extern "C" int slw_attention_plan(const slw_model_cfg* cfg, int32_t B, const int32_t* context_lens,
                                  int32_t n_prefill, const int32_t* prefix_lens, const int32_t* chunk_lens,
                                  int64_t out[12]) {
    return attention_plan(cfg, false, 0, 0, B, context_lens, n_prefill, prefix_lens, chunk_lens, out);
}

extern "C" int slw_cache_attention_plan(const slw_model_cfg* cfg, int32_t window, int32_t sinks, int32_t B,
                                        const int32_t* context_lens, int32_t n_prefill, const int32_t* prefix_lens,
                                        const int32_t* chunk_lens, int64_t out[12]) {
    return attention_plan(cfg, true, window, sinks, B, context_lens, n_prefill, prefix_lens, chunk_lens, out);
}

extern "C" int slw_gemm_plan(int32_t m, int32_t n, int32_t k, int32_t out[6]) {
    if (!out) return fail(SLW_EINVAL, "null argument");
    if (m < 1 || n < 128 || n % 128 || k < 64 || k % 64)
        return fail(SLW_EINVAL, "m >= 1, n a multiple of 128 and k of 64 (got %d, %d, %d)", m, n, k);
    const GemmPlan p = plan_gemm(m, n, k, true), q = plan_gemm(m, n, k, false);
    const int32_t v[6] = {p.cfg, p.bm, p.bn, p.splits, q.cfg, q.splits};
    for (int i = 0; i < 6; ++i) out[i] = v[i];
    return SLW_OK;
}

extern "C" int slw_set_layer_weights(slw_ctx* ctx, int32_t layer, const slw_layer_weights* w) {
    if (!ctx || !w) return fail(SLW_EINVAL, "null argument");
    if (layer < 0 || layer >= ctx->cfg.n_layers) return fail(SLW_ERANGE, "layer %d out of range", layer);
    if (!w->wqkv || !w->wo || !w->wgu || !w->wd || !w->g1 || !w->g2)
        return fail(SLW_EINVAL, "null weight pointer");
    const void* ptrs[6] = {w->wqkv, w->wo, w->wgu, w->wd, w->g1, w->g2};
    for (const void* p : ptrs)
        if (reinterpret_cast<uintptr_t>(p) % 16) return fail(SLW_EINVAL, "weights must be 16-byte aligned");
    ctx->w[layer] = *w;
    ctx->have_w[layer] = 1;
    return SLW_OK;
}

namespace {

std::atomic<uint64_t> g_kv_ids{0};

int attach_pools(slw_ctx* ctx, void* k_pool, void* v_pool, void* k_scale, void* v_scale, int32_t num_blocks) {
    if (num_blocks < 1) return fail(SLW_EINVAL, "num_blocks must be >= 1");
    if (reinterpret_cast<uintptr_t>(k_pool) % 16 || reinterpret_cast<uintptr_t>(v_pool) % 16)
        return fail(SLW_EINVAL, "pools must be 16-byte aligned");
    ctx->kv_ready = false;
    ctx->kv.reset(num_blocks, 16);
    ctx->k_pool = k_pool;
    ctx->v_pool = v_pool;
    ctx->k_scale = static_cast<float*>(k_scale);
    ctx->v_scale = static_cast<float*>(v_scale);
    ctx->kv_id = ++g_kv_ids;
    ctx->kv_ready = true;
    return SLW_OK;
}

}  // namespace

extern "C" int slw_kv_init(slw_ctx* ctx, void* k_pool, void* v_pool, int32_t num_blocks) {
    return guarded([&] {
        if (!ctx || !k_pool || !v_pool) return fail(SLW_EINVAL, "null argument");
        return attach_pools(ctx, k_pool, v_pool, nullptr, nullptr, num_blocks);
    });
}

extern "C" int slw_kv_init_8bit(slw_ctx* ctx, void* k_pool, void* v_pool, void* k_scale, void* v_scale,
                                int32_t num_blocks) {
    return guarded([&] {
        if (!ctx || !k_pool || !v_pool || !k_scale || !v_scale) return fail(SLW_EINVAL, "null argument");
        if (reinterpret_cast<uintptr_t>(k_scale) % 4 || reinterpret_cast<uintptr_t>(v_scale) % 4)
            return fail(SLW_EINVAL, "scales must be 4-byte aligned");
        return attach_pools(ctx, k_pool, v_pool, k_scale, v_scale, num_blocks);
    });
}

extern "C" int slw_set_window(slw_ctx* ctx, int32_t window, int32_t sinks, const uint8_t* layers) {
    return guarded([&] {
        if (!ctx) return fail(SLW_EINVAL, "null context");
        int rc = check_window(ctx->cfg, window, sinks);
        if (rc) return rc;
        ctx->win = Window{window, sinks};
        ctx->any_windowed = ctx->any_full = false;
        for (int l = 0; l < ctx->cfg.n_layers; ++l) {
            ctx->windowed[l] = window > 0 && (!layers || layers[l]);
            (ctx->windowed[l] ? ctx->any_windowed : ctx->any_full) = true;
        }
        return SLW_OK;
    });
}

// ---------------------------------------------------------------------------
// The cache operators on their own: a batch handed over once, then appends and
// attention per layer.
// ---------------------------------------------------------------------------

struct slw_attn {
    uint64_t kv_id;               // of the pools it was made for
    Window win;                   // and the windows
    std::vector<char> windowed;
    std::vector<Prefill> prompts; // of the batch, in row order
    AttnMeta am;
    PartLayout part;
    char* ws;
};

namespace {

struct AttnLayout {
    size_t meta_bytes;
    PartLayout part;
};
AttnLayout attn_layout(const slw_ctx& ctx, int C, int B) {
    const size_t meta = align_up(attn_meta_ints(ctx, C, B, true) * 4);
    return {meta, part_layout(ctx.cfg, C, B, meta)};
}

int check_attn(const slw_ctx* ctx, const slw_attn* plan, int32_t layer) {
    if (!ctx || !plan) return fail(SLW_EINVAL, "null argument");
    if (!ctx->kv_ready || plan->kv_id != ctx->kv_id)
        return fail(SLW_EINVAL, "the batch was handed over for other KV pools");
    if (plan->windowed != ctx->windowed || plan->win.window != ctx->win.window || plan->win.sinks != ctx->win.sinks)
        return fail(SLW_EINVAL, "the window changed after the batch was handed over");
    if (layer < 0 || layer >= ctx->cfg.n_layers) return fail(SLW_ERANGE, "layer %d out of range", layer);
    return SLW_OK;
}

// Rows that the kernels read or write in 16-byte pieces.
int check_rows(const void* p, int64_t ld, int64_t width, const char* what) {
    if (!p) return fail(SLW_EINVAL, "null %s", what);
    if (reinterpret_cast<uintptr_t>(p) % 16 || ld % 8 || ld < width || ld > INT32_MAX)
        return fail(SLW_EINVAL, "%s rows: 16-byte aligned, stride a multiple of 8 and at least %lld (got %lld)", what,
                    (long long)width, (long long)ld);
    return SLW_OK;
}

}  // namespace

extern "C" int slw_attn_workspace_size(slw_ctx* ctx, int32_t max_C, int32_t max_B, size_t* bytes) {
    return guarded([&] {
        if (!ctx || !bytes) return fail(SLW_EINVAL, "null argument");
        if (max_C < 0 || max_B < 0) return fail(SLW_EINVAL, "negative size");
        *bytes = attn_layout(*ctx, max_C, max_B).part.end;
        return SLW_OK;
    });
}

extern "C" int slw_attn_begin(slw_ctx* ctx, const slw_batch* batch, void* ws, size_t ws_bytes, void* stream,
                              slw_attn** out) {
    return guarded([&] {
        if (!ctx || !batch || !out) return fail(SLW_EINVAL, "null argument");
        *out = nullptr;
        const int C = batch->C, B = batch->B;
        if (C < 0 || B < 0) return fail(SLW_EINVAL, "negative C or B");
        if (!ctx->kv_ready) return fail(SLW_EINVAL, "KV pools not attached");
        hipStream_t s = static_cast<hipStream_t>(stream);
        auto plan = std::make_unique<slw_attn>();
        plan->kv_id = ctx->kv_id;
        plan->win = ctx->win;
        plan->windowed = ctx->windowed;
        plan->ws = static_cast<char*>(ws);
        if (C == 0 && B == 0) {
            *out = plan.release();
            return SLW_OK;
        }
        int rc = check_batch(ctx, batch);
        if (rc) return rc;
        const AttnLayout L = attn_layout(*ctx, C, B);
        if (!ws) return fail(SLW_EINVAL, "null workspace");
        if (reinterpret_cast<uintptr_t>(ws) % 16) return fail(SLW_EINVAL, "the workspace must be 16-byte aligned");
        if (ws_bytes < L.part.end)
            return fail(SLW_ENOMEM, "the workspace holds %zu bytes, this batch needs %zu", ws_bytes, L.part.end);
        if (s) {
            hipStreamCaptureStatus st = hipStreamCaptureStatusNone;
            HIP_TRY(hipStreamIsCapturing(s, &st));
            if (st != hipStreamCaptureStatusNone)
                return fail(SLW_EINVAL, "a batch is handed over outside a capture: its metadata is uploaded once");
        }
        if ((rc = ensure_hip(ctx))) return rc;
        KvManager::Reservation room(ctx->kv);
        if ((rc = room.reserve(ctx->batch_seqs))) return rc;
        plan->part = L.part;
        plan->prompts = ctx->prefills;
        std::vector<int32_t>& m = ctx->meta;
        m.clear();
        if ((rc = build_attn_meta(ctx, batch, true, m, plan->am))) return rc;
        if (m.size() * 4 > L.meta_bytes) return fail(SLW_EINVAL, "internal: metadata %zu ints above its region", m.size());
        int32_t* stage = nullptr;
        int slot = 0;
        if ((rc = next_staging(ctx, m.size(), &stage, &slot))) return rc;
        std::memcpy(stage, m.data(), m.size() * 4);
        launch_iteration_setup(ws, ctx->staging_dev[slot], m.size(), nullptr, nullptr, 0, ctx->cfg.head_dim, 1.0, nullptr,
                               nullptr, nullptr, 0, 0.f, s);
        HIP_TRY(hipGetLastError());
        HIP_TRY(hipEventRecord(ctx->staged[slot], s));
        room.keep();
        *out = plan.release();
        return SLW_OK;
    });
}

extern "C" int slw_attn_append(slw_ctx* ctx, const slw_attn* plan, int32_t layer, const void* k, const void* v,
                               int64_t ld, void* stream) {
    return guarded([&] {
        int rc = check_attn(ctx, plan, layer);
        if (rc) return rc;
        if (plan->am.n_app == 0) return SLW_OK;
        const int64_t width = static_cast<int64_t>(ctx->cfg.n_kv_heads) * ctx->cfg.head_dim;
        if ((rc = check_rows(k, ld, width, "k")) || (rc = check_rows(v, ld, width, "v"))) return rc;
        launch_cache_append(append_args(ctx, plan->am, reinterpret_cast<const int32_t*>(plan->ws), layer, k, v,
                                        static_cast<int>(ld)), static_cast<hipStream_t>(stream));
        HIP_TRY(hipGetLastError());
        return SLW_OK;
    });
}

extern "C" int slw_attn_attend(slw_ctx* ctx, const slw_attn* plan, int32_t layer, const void* q, int64_t ld,
                               void* out, void* stream) {
    return guarded([&] {
        int rc = check_attn(ctx, plan, layer);
        if (rc) return rc;
        if (plan->am.C + plan->am.B == 0) return SLW_OK;
        const int64_t width = static_cast<int64_t>(ctx->cfg.n_q_heads) * ctx->cfg.head_dim;
        if ((rc = check_rows(q, ld, width, "q")) || (rc = check_rows(out, width, width, "out"))) return rc;
        hipStream_t s = static_cast<hipStream_t>(stream);
        const AttnCall attention(ctx, plan->am, reinterpret_cast<const int32_t*>(plan->ws), plan->ws, plan->part, layer,
                                 q, static_cast<int>(ld), out);
        attention.both(s);
        attention.merge(s);
        HIP_TRY(hipGetLastError());
        return SLW_OK;
    });
}

namespace {

int rope_args(const slw_model_cfg& c, const slw_rope& r, RopeArgs* out) {
    if (r.rot_dim < 16 || r.rot_dim % 16 || r.rot_dim > c.head_dim)
        return fail(SLW_EUNSUPPORTED, "rot_dim must be a multiple of 16 in [16, head_dim = %d] (got %d)", c.head_dim, r.rot_dim);
    if (r.interleaved != 0 && r.interleaved != 1) return fail(SLW_EINVAL, "interleaved must be 0 or 1");
    if (!std::isfinite(r.mscale)) return fail(SLW_EINVAL, "mscale must be finite");
    auto positive = [](double x) { return x > 0.0 && std::isfinite(x); };
    RopeArgs a{};
    a.mscale = r.mscale;
    a.rot = r.rot_dim;
    a.interleaved = r.interleaved != 0;
    a.first = 1.0;
    double theta = r.theta;
    if (r.scaling != SLW_ROPE_TABLE && !positive(theta)) return fail(SLW_EINVAL, "theta must be positive and finite");
    if (r.scaling == SLW_ROPE_LINEAR || r.scaling == SLW_ROPE_NTK || r.scaling == SLW_ROPE_BY_PARTS)
        if (!positive(r.factor)) return fail(SLW_EINVAL, "factor must be positive and finite");
    switch (r.scaling) {
        case SLW_ROPE_NONE: break;
        case SLW_ROPE_LINEAR: a.first = 1.0 / r.factor; break;
        case SLW_ROPE_NTK: theta *= std::pow(r.factor, r.rot_dim / (r.rot_dim - 2.0)); break;
        case SLW_ROPE_BY_PARTS:
            if (!std::isfinite(r.low) || !std::isfinite(r.high) || !(r.low < r.high))
                return fail(SLW_EINVAL, "low and high must be finite, low below high");
            if (r.original_len < 1) return fail(SLW_EINVAL, "original_len must be >= 1");
            a.by_parts = true;
            a.turns_in_original = r.original_len / 6.283185307179586477;
            a.low = r.low;
            a.inv_width = 1.0 / (r.high - r.low);
            a.inv_factor = 1.0 / r.factor;
            break;
        case SLW_ROPE_TABLE:
            if (!r.freq || reinterpret_cast<uintptr_t>(r.freq) % 8) return fail(SLW_EINVAL, "freq: 8-byte aligned device memory");
            a.freq = r.freq;
            break;
        default: return fail(SLW_EINVAL, "unknown scaling %d", r.scaling);
    }
    if (!a.freq) {
        a.step = -2.0 * std::log2(theta) / r.rot_dim;
        if (!positive(theta) || !std::isfinite(a.first) || !std::isfinite(a.inv_factor) || (a.by_parts && a.inv_width == 0.0))
            return fail(SLW_EINVAL, "theta, factor, low and high make frequencies that are not finite");
    }
    *out = a;
    return SLW_OK;
}

}  // namespace

extern "C" int slw_attn_rotate(slw_ctx* ctx, const slw_attn* plan, const slw_rope* rope, const void* q, const void* k,
                               int64_t ld, void* q_out, void* k_out, int64_t ld_out, void* stream) {
    return guarded([&] {
        int rc = check_attn(ctx, plan, 0);
        if (rc) return rc;
        if (!rope) return fail(SLW_EINVAL, "null argument");
        const slw_model_cfg& c = ctx->cfg;
        RopeArgs ra;
        if ((rc = rope_args(c, *rope, &ra))) return rc;
        if (!q && !k) return fail(SLW_EINVAL, "neither q nor k rows");
        if (!q != !q_out || !k != !k_out) return fail(SLW_EINVAL, "rows without their outputs, or outputs without rows");
        const int64_t qw = static_cast<int64_t>(c.n_q_heads) * c.head_dim, kw = static_cast<int64_t>(c.n_kv_heads) * c.head_dim;
        if (q && ((rc = check_rows(q, ld, qw, "q")) || (rc = check_rows(q_out, ld_out, qw, "q output")))) return rc;
        if (k && ((rc = check_rows(k, ld, kw, "k")) || (rc = check_rows(k_out, ld_out, kw, "k output")))) return rc;
        if (plan->am.C + plan->am.B == 0) return SLW_OK;
        RotateRows a{};
        a.q = q;
        a.k = k;
        a.q_out = q_out;
        a.k_out = k_out;
        a.kv_len = reinterpret_cast<const int32_t*>(plan->ws) + plan->am.kvlen;
        a.ld = ld;
        a.ld_out = ld_out;
        a.rows = plan->am.C + plan->am.B;
        a.chunk = plan->am.C;
        a.hq = c.n_q_heads;
        a.hkv = c.n_kv_heads;
        a.hd = c.head_dim;
        for (const Prefill& f : plan->prompts) {
            a.row_end[a.n_prompts] = f.row0 + f.c;
            a.shift[a.n_prompts++] = f.prefix - f.row0;
        }
        a.in_place = ld == ld_out && q == q_out && k == k_out;
        launch_rotate(a, ra, static_cast<hipStream_t>(stream));
        HIP_TRY(hipGetLastError());
        return SLW_OK;
    });
}

extern "C" int slw_attn_end(slw_attn* plan) {
    delete plan;
    return SLW_OK;
}

extern "C" int slw_kv_free_blocks(slw_ctx* ctx, int32_t* n_free) {
    if (!ctx || !n_free) return fail(SLW_EINVAL, "null argument");
    if (!ctx->kv_ready) return fail(SLW_EINVAL, "KV pools not attached");
    *n_free = ctx->kv.free_count();
    return SLW_OK;
}

extern "C" int slw_seq_create(slw_ctx* ctx, int64_t id) {
    return guarded([&] {
        if (!ctx) return fail(SLW_EINVAL, "null context");
        if (!ctx->kv_ready) return fail(SLW_EINVAL, "KV pools not attached");
        return ctx->kv.create(id);
    });
}

extern "C" int slw_seq_free(slw_ctx* ctx, int64_t id) {
    return guarded([&] {
        if (!ctx) return fail(SLW_EINVAL, "null context");
        if (!ctx->kv_ready) return fail(SLW_EINVAL, "KV pools not attached");
        return ctx->kv.release(id);
    });
}

extern "C" int slw_seq_reserve(slw_ctx* ctx, int64_t id, int32_t new_len) {
    return guarded([&] {
        if (!ctx) return fail(SLW_EINVAL, "null context");
        if (!ctx->kv_ready) return fail(SLW_EINVAL, "KV pools not attached");
        if (new_len > ctx->cfg.max_pos) return fail(SLW_ERANGE, "length %d above max_pos", new_len);
        return ctx->kv.reserve_all({{id, new_len}});
    });
}

extern "C" int slw_seq_block_table(slw_ctx* ctx, int64_t id, int32_t* out, int32_t cap, int32_t* n) {
    return guarded([&] {
        if (!ctx || !n) return fail(SLW_EINVAL, "null argument");
        if (!ctx->kv_ready || !ctx->kv.exists(id)) return fail(SLW_EINVAL, "sequence %lld unknown", (long long)id);
        const auto& t = ctx->kv.table(id);
        *n = static_cast<int32_t>(t.size());
        if (out) {
            if (cap < *n) return fail(SLW_ERANGE, "table has %d entries, cap %d", *n, cap);
            std::copy(t.begin(), t.end(), out);
        }
        return SLW_OK;
    });
}

extern "C" int slw_workspace_size(slw_ctx* ctx, int32_t max_C, int32_t max_B, size_t* bytes) {
    return guarded([&] {
        if (!ctx || !bytes) return fail(SLW_EINVAL, "null argument");
        if (max_C < 0 || max_B < 0) return fail(SLW_EINVAL, "negative size");
        size_t gp = 0;
        // plans are the same for all row counts of a block of 32 (past the
        // narrow kernel's, which has no partials), and partials grow with the rows
        const int rows = max_C + max_B;
        for (int m = 32; m < rows + 32; m += 32) gp = std::max(gp, plan_layer(ctx->cfg, std::min(m, rows)).partial_bytes());
        *bytes = layout(*ctx, max_C, max_B).end_fixed + gp;
        return SLW_OK;
    });
}

extern "C" int slw_workspace_view(slw_ctx* ctx, int32_t which, int32_t C, int32_t B, size_t* offset,
                                  size_t* bytes) {
    if (!ctx || !offset || !bytes) return fail(SLW_EINVAL, "null argument");
    if (C < 0 || B < 0) return fail(SLW_EINVAL, "negative size");
    const slw_model_cfg& c = ctx->cfg;
    const Layout L = layout(*ctx, C, B);
    const size_t M = static_cast<size_t>(C) + B;
    switch (which) {
        case SLW_VIEW_QKV: *offset = L.qkv; *bytes = M * qkv_width(c) * 2; break;
        case SLW_VIEW_ATTN: *offset = L.attn; *bytes = M * c.n_q_heads * c.head_dim * 2; break;
        case SLW_VIEW_H: *offset = L.h; *bytes = M * c.d_model * 4; break;
        case SLW_VIEW_ACT: *offset = L.act; *bytes = M * c.ffn_dim * 2; break;
        default: return fail(SLW_EINVAL, "unknown view %d", which);
    }
    return SLW_OK;
}

extern "C" int slw_mixed_iteration(slw_ctx* ctx, const slw_batch* batch, const void* x_in, void* x_out,
                                   void* ws, size_t ws_bytes, void* stream) {
    return guarded([&] {
        if (!ctx) return fail(SLW_EINVAL, "null context");
        return mixed_iteration_impl(ctx, batch, x_in, x_out, ws, ws_bytes, static_cast<hipStream_t>(stream));
    });
}

// ---------------------------------------------------------------------------
// The allocation-free variant: the workspace is a file-scope device array of
// SLW_STATIC_WS_BYTES, one copy per GPU, held until the process ends.  Its
// address on each device is taken once, with that device current, through
// hipGetSymbolAddress; host code uses only that address (the array's name
// is a host-side stand-in).  No value in it needs to start at zero: every
// word a kernel reads was written earlier in the same call.  Calls that
// overlap on one GPU share the array and race.
// ---------------------------------------------------------------------------

namespace {

constexpr size_t kStaticWsBytes = SLW_STATIC_WS_BYTES;
static __device__ __attribute__((aligned(256))) unsigned char scratch[kStaticWsBytes];

constexpr int kMaxDevices = 64;
std::mutex g_scratch_mu;
void* g_scratch_ptr[kMaxDevices] = {};

int static_workspace(void** out) {
    int dev = 0;
    HIP_TRY(hipGetDevice(&dev));
    if (dev < 0 || dev >= kMaxDevices) return fail(SLW_ERANGE, "device %d above %d", dev, kMaxDevices - 1);
    std::lock_guard<std::mutex> lock(g_scratch_mu);
    if (!g_scratch_ptr[dev]) {
        void* p = nullptr;
        HIP_TRY(hipGetSymbolAddress(&p, HIP_SYMBOL(scratch)));
        if (!p) return fail(SLW_EHIP, "hipGetSymbolAddress gave a null address");
        g_scratch_ptr[dev] = p;
    }
    *out = g_scratch_ptr[dev];
    return SLW_OK;
}

}  // namespace

extern "C" int slw_mixed_iteration_static(slw_ctx* ctx, const slw_batch* batch, const void* x_in, void* x_out,
                                          void* stream) {
    return guarded([&] {
        if (!ctx) return fail(SLW_EINVAL, "null context");
        void* ws = nullptr;
        int rc = static_workspace(&ws);
        if (rc) return rc;
        return mixed_iteration_impl(ctx, batch, x_in, x_out, ws, kStaticWsBytes, static_cast<hipStream_t>(stream),
                                    true);
    });
}

extern "C" int slw_fill_normal(void* dst, size_t n, uint64_t seed, float mean, float std, void* stream) {
    return guarded([&] {
        if (!dst && n) return fail(SLW_EINVAL, "null buffer");
        if (reinterpret_cast<uintptr_t>(dst) % 2) return fail(SLW_EINVAL, "buffer must be 2-byte aligned");
        if (n / 4 >= (static_cast<size_t>(1) << 62)) return fail(SLW_ERANGE, "too many elements");
        launch_fill_normal(dst, n, seed, mean, std, static_cast<hipStream_t>(stream));
        HIP_TRY(hipGetLastError());
        return SLW_OK;
    });
}

extern "C" int slw_flush_cache(void* buf, size_t bytes, void* stream) {
    return guarded([&] {
        if (!buf && bytes) return fail(SLW_EINVAL, "null buffer");
        if (reinterpret_cast<uintptr_t>(buf) % 16) return fail(SLW_EINVAL, "buffer must be 16-byte aligned");
        launch_cache_sweep(buf, bytes, 0x9e3779b9u, static_cast<hipStream_t>(stream));
        HIP_TRY(hipGetLastError());
        return SLW_OK;
    });
}

extern "C" int slw_set_stage_timing(slw_ctx* ctx, int32_t depth) {
    return guarded([&] {
        if (!ctx) return fail(SLW_EINVAL, "null context");
        if (depth < 0 || depth > 4096) return fail(SLW_ERANGE, "depth must be in [0, 4096]");
        ctx->stage_depth = depth;
        ctx->stage_mask.assign(depth, 0u);
        ctx->stage_iter = 0;
        return SLW_OK;
    });
}

extern "C" int slw_stage_times(slw_ctx* ctx, int32_t ago, float* ms, int32_t cap, int32_t* n) {
    if (!ctx || !ms || !n) return fail(SLW_EINVAL, "null argument");
    if (ctx->stage_depth <= 0) return fail(SLW_EINVAL, "stage timing is off");
    if (ago < 0 || ago >= ctx->stage_depth || ago >= ctx->stage_iter)
        return fail(SLW_ERANGE, "iteration %d ago is not recorded", ago);
    if (cap < kStages) return fail(SLW_ERANGE, "need room for %d stages", kStages);
    const int set = static_cast<int>((ctx->stage_iter - 1 - ago) % ctx->stage_depth);
    const uint32_t mask = ctx->stage_mask[set];
    const size_t base0 = static_cast<size_t>(set) * ctx->cfg.n_layers * (kStages + 1);
    if (mask) HIP_TRY(hipEventSynchronize(ctx->stage_ev[base0 + static_cast<size_t>(ctx->cfg.n_layers) * (kStages + 1) - 1]));
    for (int s = 0; s < kStages; ++s) {
        float tot = 0.f;
        if (mask & (1u << s)) {
            for (int l = 0; l < ctx->cfg.n_layers; ++l) {
                float t = 0.f;
                const size_t base = base0 + static_cast<size_t>(l) * (kStages + 1);
                HIP_TRY(hipEventElapsedTime(&t, ctx->stage_ev[base + s], ctx->stage_ev[base + s + 1]));
                tot += t;
            }
        }
        ms[s] = tot;
    }
    *n = kStages;
    return SLW_OK;
}

extern "C" int slw_last_slots(slw_ctx* ctx, int32_t* out, int32_t cap, int32_t* n) {
    if (!ctx || !n) return fail(SLW_EINVAL, "null argument");
    *n = static_cast<int32_t>(ctx->last_slots.size());
    if (out) {
        if (cap < *n) return fail(SLW_ERANGE, "%d slots, cap %d", *n, cap);
        std::copy(ctx->last_slots.begin(), ctx->last_slots.end(), out);
    }
    return SLW_OK;
}

// ---------------------------------------------------------------------------
// Profiler (Sec. 5.1): time the mixed iteration over a (decode batch, chunk)
// grid, keep every sample, then P50/P99 and a running maximum along chunks.
// ---------------------------------------------------------------------------

namespace {

// Profile planes of the table: for each prefix in p_grid (or the single
// prefix opts->prefix_len when p_grid is null) time the iteration over every
// (b, c) of b_grid x c_grid.
int build_table_core(slw_ctx* ctx, const int32_t* c_grid, int32_t nc, const int32_t* b_grid, int32_t nb,
                     const int32_t* p_grid, int32_t np, const slw_profile_opts* o, slw_cost_table** out) {
    if (!ctx || !o || !out || !c_grid || !b_grid) return fail(SLW_EINVAL, "null argument");
    *out = nullptr;
    if (!ctx->kv_ready) return fail(SLW_EINVAL, "KV pools not attached");
    if (nc < 1 || nb < 1 || (p_grid && np < 1)) return fail(SLW_EINVAL, "empty grid");
    if (o->repeats < 1 || o->warmup < 0) return fail(SLW_EINVAL, "repeats must be >= 1, warmup >= 0");
    if (o->prefix_len < 0 || o->ctx_lo < 0 || o->ctx_hi < o->ctx_lo)
        return fail(SLW_EINVAL, "bad prefix or context range");
    auto t = std::make_unique<slw_cost_table>();
    t->c_grid.assign(c_grid, c_grid + nc);
    t->b_grid.assign(b_grid, b_grid + nb);
    if (p_grid) {
        t->p_grid.assign(p_grid, p_grid + np);
        t->has_ctx = true;
    } else {
        t->p_grid.assign(1, o->prefix_len);
    }
    t->repeats = o->repeats;
    // validate grids before reserving anything (finish_table repeats the check)
    t->samples.assign(static_cast<size_t>(t->np()) * nb * nc * o->repeats, 0);
    int rc = finish_table(t.get());
    if (rc) return rc;
    const int c_last = c_grid[nc - 1], b_last = b_grid[nb - 1];
    const int p_last = t->p_grid.back();

    const int64_t base = INT64_MIN + 1;  // profiler-reserved ids
    const int64_t pre_id = base;
    std::vector<int64_t> dec(b_last);
    std::vector<int32_t> ctxl(b_last);
    std::mt19937_64 rng(o->seed);
    std::uniform_int_distribution<int32_t> dist(o->ctx_lo, o->ctx_hi);
    for (int i = 0; i < b_last; ++i) {
        dec[i] = base + 1 + i;
        ctxl[i] = dist(rng);
    }
    std::vector<int64_t> made;
    auto cleanup = [&] {
        for (int64_t id : made) (void)ctx->kv.release(id);
    };
    rc = ctx->kv.create(pre_id);
    if (rc) return rc;
    made.push_back(pre_id);
    for (int i = 0; i < b_last; ++i) {
        rc = ctx->kv.create(dec[i]);
        if (rc) { cleanup(); return rc; }
        made.push_back(dec[i]);
    }
    std::vector<std::pair<int64_t, int32_t>> req;
    req.emplace_back(pre_id, p_last + c_last);
    for (int i = 0; i < b_last; ++i) req.emplace_back(dec[i], ctxl[i] + 1);
    rc = ctx->kv.reserve_all(req);
    if (rc) { cleanup(); return rc; }

    hipStream_t s = static_cast<hipStream_t>(o->stream);
    auto run = [&](int prefix, int b, int cc) {
        slw_batch batch{cc, pre_id, prefix, b, dec.data(), ctxl.data()};
        return mixed_iteration_impl(ctx, &batch, o->x_in, o->x_out, o->ws, o->ws_bytes, s);
    };
    auto sync = [&]() -> int {
        hipError_t e = hipStreamSynchronize(s);
        if (e != hipSuccess) return fail(SLW_EHIP, "hipStreamSynchronize: %s", hipGetErrorString(e));
        return SLW_OK;
    };
    for (int k = 0; k < t->np() && !rc; ++k)
        for (int i = 0; i < nb && !rc; ++i)
            for (int j = 0; j < nc && !rc; ++j) {
                const int prefix = t->p_grid[k];
                for (int r = 0; r < o->warmup && !rc; ++r) rc = run(prefix, b_grid[i], c_grid[j]);
                if (!rc) rc = sync();
                for (int r = 0; r < o->repeats && !rc; ++r) {
                    if (o->flush_buf && o->flush_bytes) {
                        launch_cache_sweep(o->flush_buf, o->flush_bytes, 0x9e3779b9u + static_cast<uint32_t>(r), s);
                        rc = sync();
                        if (rc) break;
                    }
                    auto t0 = std::chrono::steady_clock::now();
                    rc = run(prefix, b_grid[i], c_grid[j]);
                    if (!rc) rc = sync();
                    auto t1 = std::chrono::steady_clock::now();
                    t->samples[((static_cast<size_t>(k) * nb + i) * nc + j) * o->repeats + r] =
                        std::chrono::duration_cast<std::chrono::nanoseconds>(t1 - t0).count();
                }
            }
    cleanup();
    if (rc) return rc;
    if (!p_grid) t->p_grid.assign(1, 0);  // one plane serves every prefix
    rc = finish_table(t.get());
    if (rc) return rc;
    *out = t.release();
    return SLW_OK;
}

}  // namespace

extern "C" int slw_build_cost_table(slw_ctx* ctx, const int32_t* c_grid, int32_t nc, const int32_t* b_grid,
                                    int32_t nb, const slw_profile_opts* o, slw_cost_table** out) {
    return guarded([&]() -> int { return build_table_core(ctx, c_grid, nc, b_grid, nb, nullptr, 0, o, out); });
}

extern "C" int slw_build_cost_table_ctx(slw_ctx* ctx, const int32_t* c_grid, int32_t nc, const int32_t* b_grid,
                                        int32_t nb, const int32_t* p_grid, int32_t np, const slw_profile_opts* o,
                                        slw_cost_table** out) {
    return guarded([&]() -> int {
        if (!p_grid) return fail(SLW_EINVAL, "null context grid");
        return build_table_core(ctx, c_grid, nc, b_grid, nb, p_grid, np, o, out);
    });
}
