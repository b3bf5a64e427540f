// Attention over the paged cache in e4m3 or bf16, causal, with an optional
// sliding window and sink tokens, on gfx950 matrix cores.
//
// A row at position p sees key t if t <= p and, with a window W > 0, t > p - W
// or t < sinks.  Work lists count in virtual keys (attn_plan.h): the 64-key
// tiles between the sinks and the window, which no row of a query tile (or
// decode) sees, are left out of them, so a windowed layer takes time in
// proportion to the window.
//
// As in the bf16 attention beside this file, scores are transposed,
// S^T = K Q^T with 16 keys as the A operand, softmax is online in fp32 with
// base-2 exponentials, and P in bf16 is the A operand of P V.  Every e4m3
// value is a bf16 value and so is every value times a power of two, so e4m3
// pages are widened exactly (v_cvt_scalef32_pk_bf16_fp8 applies the scale in
// the same instruction) and the products run on the bf16 matrix cores: q and
// P keep their precision, which an e4m3 product would cut to three bits.
#include <math.h>

#include "attn_device.h"
#include "kernels.h"

namespace slw {
namespace {

typedef const float __attribute__((address_space(4))) const_f32;
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr float kSlack = 8.0f;  // lazy rescaling threshold (log2 units), as in the bf16 kernels

// Four e4m3 codes times a power of two, in bf16 (exact; NaN stays NaN).
__device__ __forceinline__ void widen4(uint32_t c, float scale, bf16x8& out, int at) {
    const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, scale, false);
    const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, scale, true);
    out[at] = lo[0];
    out[at + 1] = lo[1];
    out[at + 2] = hi[0];
    out[at + 3] = hi[1];
}
__device__ __forceinline__ bf16x8 widen8(uint32_t c0, uint32_t c1, float scale) {
    bf16x8 r;
    widen4(c0, scale, r, 0);
    widen4(c1, scale, r, 4);
    return r;
}

// Bits i of [0, n) for n in [0, 32].
__device__ __forceinline__ uint32_t low_bits(int n) { return n >= 32 ? 0xFFFFFFFFu : (1u << n) - 1u; }

// ---------------------------------------------------------------------------
// Decode attention, split over the key axis: one wave per (slot, kv head),
// the q heads of the group as the columns of Q^T, as in the bf16 kernel.
//
// A step takes 4 KPL keys: lane group g holds the scores of keys
// KPL g .. KPL g + KPL - 1 (row 4 g + e of score tile tau is key
// KPL g + 4 tau + e), which makes them its operand of P V.  KPL is 16 for
// e4m3, so that a lane's V operand is the 16 bytes of one dimension's page
// row (two MFMAs' worth) and every load takes 16 bytes, and 8 for bf16.  The
// K scale of the lane group's page multiplies its scores, the V scale is
// applied where the codes are widened.
//
// Bound by HBM.
// ---------------------------------------------------------------------------
template <bool Q8, int HD>
struct CacheStep {
    static constexpr int TAU = Q8 ? 4 : 2;                // score tiles
    static constexpr int KL = Q8 ? HD / 64 : HD / 32;     // 16-byte pieces of a key row per lane
    static constexpr int VL = HD / 16;
    u32x4 k[TAU][KL];
    u32x4 v[VL];
    float ks, vs;  // e4m3: scales of the lane group's page
};

template <bool Q8, int HD>
__device__ __forceinline__ void cache_load(CacheStep<Q8, HD>& st, const CacheAttnArgs& a, const const_i32* bt_s, int k0,
                                           int last_pg, int kvh, int col, int grp) {
    constexpr int PAGES = Q8 ? 4 : 2, PB = HD * 16 * (Q8 ? 1 : 2);  // pages of a step, bytes of a page
    const int pg0 = k0 >> 4;
    int b[PAGES];
#pragma unroll
    for (int p = 0; p < PAGES; ++p) b[p] = bt_s[min(pg0 + p, last_pg)];
    auto pick = [&](int i) {
        int r = b[0];
#pragma unroll
        for (int p = 1; p < PAGES; ++p) r = i == p ? b[p] : r;
        return r;
    };
    const uint8_t* kpool = static_cast<const uint8_t*>(a.decode.k_pool);
    const uint8_t* vpool = static_cast<const uint8_t*>(a.decode.v_pool);
    const int hkv = a.decode.hkv;
    // K row `col` of score tile tau: key KPL (col / 4) + 4 tau + col % 4 of the step
    const int kpl = Q8 ? 16 : 8;
    const uint8_t* kpage = kpool + (static_cast<size_t>(pick(Q8 ? col >> 2 : col >> 3)) * hkv + kvh) * PB;
#pragma unroll
    for (int tau = 0; tau < CacheStep<Q8, HD>::TAU; ++tau) {
        const int tok = (kpl * (col >> 2) + 4 * tau + (col & 3)) & 15;
#pragma unroll
        for (int s = 0; s < CacheStep<Q8, HD>::KL; ++s)
            st.k[tau][s] = *reinterpret_cast<const u32x4*>(kpage + s * 1024 + tok * 64 + grp * 16);
    }
    const size_t vbh = static_cast<size_t>(pick(Q8 ? grp : grp >> 1)) * hkv + kvh;
    const uint8_t* vpage = vpool + vbh * PB;
#pragma unroll
    for (int nt = 0; nt < CacheStep<Q8, HD>::VL; ++nt)
        st.v[nt] = *reinterpret_cast<const u32x4*>(vpage + (nt * 16 + col) * (Q8 ? 16 : 32) + (Q8 ? 0 : 16 * (grp & 1)));
    if constexpr (Q8) {
        st.ks = a.k_scale[vbh];
        st.vs = a.v_scale[vbh];
    }
}

template <bool Q8, int HD>
__device__ __forceinline__ void cache_decode_wave(const CacheAttnArgs& a, int slot, int kvh, int lane) {
    using Step = CacheStep<Q8, HD>;
    constexpr int TAU = Step::TAU, KL = Step::KL, NT = HD / 16, KPL = 4 * TAU, KEYS = 4 * KPL;
    const DecodeAttnArgs& d = a.decode;
    const int grp = lane >> 4, col = lane & 15;
    const int group = d.hq / d.hkv;
    const float sl2 = kLog2e / sqrtf(static_cast<float>(HD));

    const int i0 = d.slot_off[slot], i1 = d.slot_off[slot + 1];
    for (int w = i0; w < i1; ++w) {
        const int b = d.work_b[w], v0 = d.work_kb[w], v1 = d.work_ke[w];
        const int len = d.kv_len[b], skip = a.skip[b];
        const int last_pg = (len - 1) >> 4;
        // keys below w_lo are seen only if they are sinks
        const int w_lo = a.window > 0 ? max(len - a.window, 0) : 0;
        const const_i32* bt_s = (const const_i32*)(d.bt + d.bt_off[b]);
        auto key_of = [&](int v) { return v < a.sink_end ? v : v + skip; };

        // Q^T operand: the dims that a lane's K pieces hold
        bf16x8 qf[HD / 32];
        {
            const bf16* q = static_cast<const bf16*>(d.q) + static_cast<size_t>(b) * d.ld_q;
            const int h = kvh * group + col;
#pragma unroll
            for (int kk = 0; kk < HD / 32; ++kk) {
                const int dim = Q8 ? 64 * (kk >> 1) + 16 * grp + 8 * (kk & 1) : 32 * kk + 8 * grp;
                qf[kk] = col < group ? *reinterpret_cast<const bf16x8*>(q + h * HD + dim) : bf16x8{};
            }
        }

        f32x4 o[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) o[nt] = f32x4{};
        float m_run = -INFINITY, l_run = 0.f;

        // Masked keys (past the item's end, where stand-in pages and unwritten
        // slots lie, or outside the window) get score -inf and V 0 without
        // branches, which would make the waits on the prefetch conservative.
        auto compute = [&](Step& st, int c0) {
            const int k0 = key_of(c0) + KPL * grp;
            const int nv = min(max(v1 - (c0 + KPL * grp), 0), KPL);
            const int ns = min(max(a.sinks - k0, 0), KPL), nw = min(max(w_lo - k0, 0), KPL);
            const uint32_t seen = low_bits(nv) & (low_bits(ns) | ~low_bits(nw));
            u32x4 vmask;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (Q8) {  // word j: tokens 4 j .. 4 j + 3
                    const uint32_t n = (seen >> (4 * j)) & 0xFu;
                    vmask[j] = ((n * 0x00204081u) & 0x01010101u) * 0xFFu;
                } else {             // word j: tokens 2 j, 2 j + 1
                    vmask[j] = ((seen >> (2 * j)) & 1u ? 0x0000FFFFu : 0u) | ((seen >> (2 * j)) & 2u ? 0xFFFF0000u : 0u);
                }
            }
            f32x4 s[TAU];
#pragma unroll
            for (int tau = 0; tau < TAU; ++tau) {
                s[tau] = f32x4{};
#pragma unroll
                for (int i = 0; i < KL; ++i) {
                    const u32x4 x = st.k[tau][i];
                    if constexpr (Q8) {
                        s[tau] = mfma16(widen8(x[0], x[1], 1.0f), qf[2 * i], s[tau]);
                        s[tau] = mfma16(widen8(x[2], x[3], 1.0f), qf[2 * i + 1], s[tau]);
                    } else {
                        s[tau] = mfma16(__builtin_bit_cast(bf16x8, x), qf[i], s[tau]);
                    }
                }
            }
            const float scale = Q8 ? sl2 * st.ks : sl2;
            float mx = -INFINITY;
#pragma unroll
            for (int tau = 0; tau < TAU; ++tau)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x = (seen >> (4 * tau + e)) & 1u ? s[tau][e] : -INFINITY;
                    s[tau][e] = x;
                    mx = fmaxf(mx, x);
                }
            mx = rows4_max(mx * scale);
            if (__any(mx > m_run + kSlack)) {
                const float m_new = fmaxf(m_run, mx);
                const float alpha = m_new == -INFINITY ? 1.f : fast_exp2(m_run - m_new);
                l_run *= alpha;
                m_run = m_new;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float ae = __shfl(alpha, grp * 4 + e, 64);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) o[nt][e] *= ae;
                }
            }
            const float m_use = m_run == -INFINITY ? 0.f : m_run;
            float ls = 0.f;
#pragma unroll
            for (int tau = 0; tau < TAU; ++tau)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float v = fast_exp2(fmaf(s[tau][e], scale, -m_use));
                    s[tau][e] = v;
                    ls += v;
                }
            l_run += ls;
#pragma unroll
            for (int j = 0; j < TAU / 2; ++j) {
                const bf16x8 pf = to_bf16x8(s[2 * j], s[2 * j + 1]);  // the lane group's keys 8 j .. 8 j + 7
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const u32x4 x = st.v[nt] & vmask;
                    if constexpr (Q8) o[nt] = mfma16(pf, widen8(x[2 * j], x[2 * j + 1], st.vs), o[nt]);
                    else o[nt] = mfma16(pf, __builtin_bit_cast(bf16x8, x), o[nt]);
                }
            }
        };

        // Loads one step ahead, also past the item's end (they re-read a page
        // of the sequence), so that no branch skips a load.
        Step sa, sb;
        cache_load<Q8, HD>(sa, a, bt_s, key_of(v0), last_pg, kvh, col, grp);
        for (int c0 = v0;; c0 += 2 * KEYS) {
            cache_load<Q8, HD>(sb, a, bt_s, key_of(c0 + KEYS), last_pg, kvh, col, grp);
            compute(sa, c0);
            if (c0 + KEYS >= v1) break;
            cache_load<Q8, HD>(sa, a, bt_s, key_of(c0 + 2 * KEYS), last_pg, kvh, col, grp);
            compute(sb, c0 + KEYS);
            if (c0 + 2 * KEYS >= v1) break;
        }

        const float l = rows4_sum(l_run);
        // a maximum of -inf marks a part that saw no key: where every score
        // seen was NaN, the sum says so instead
        const float m = m_run == -INFINITY && l != l ? 0.f : m_run;
        const size_t hbase = static_cast<size_t>(w) * d.hq + kvh * group;
        if (grp == 0 && col < group) {
            d.part_ml[(hbase + col) * 2 + 0] = m;
            d.part_ml[(hbase + col) * 2 + 1] = l;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int h = grp * 4 + e;
            if (h < group) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) d.part_o[(hbase + h) * HD + nt * 16 + col] = o[nt][e];
            }
        }
    }
}

template <bool Q8, int HD>
__global__ __launch_bounds__(64, 2) void cache_decode_kernel(CacheAttnArgs a) {
    cache_decode_wave<Q8, HD>(a, blockIdx.x, blockIdx.y, threadIdx.x);
}

// ---------------------------------------------------------------------------
// Chunk attention: the rows of a query tile (256 / GROUP positions of one
// prompt, GROUP q heads of one kv head) against its keys, 64 at a time, as in
// the bf16 kernel: eight waves of 32 rows, K and V tiles in bf16 in LDS.
//
// Tiles go through registers on their way to LDS, since e4m3 pages are widened
// there, once per work-group instead of once per wave: the next tile's loads
// are in flight while the current one is multiplied, and are widened and
// written to the other of two buffers after it.
//
// A key that some rows of a wave see and others do not stays out of the
// others' products through a zero probability, unless its V row is not
// finite (0 times it would be NaN).  The waves say for each tile on an edge of
// the mask whether they wrote such a value; a tile that has one takes a path
// that multiplies the finite values alone, and adds what rows that see the
// others get from them, counted with products of visibility and class.
// ---------------------------------------------------------------------------
template <bool Q8, int HD, int GROUP>
__global__ __launch_bounds__(512) void cache_chunk_kernel(CacheAttnArgs a) {
    const ChunkAttnArgs& c = a.chunk;
    {   // decode waves behind the chunk work-groups, as in the bf16 kernel
        const int n_chunk = c.n_slots * c.hkv;
        if (static_cast<int>(blockIdx.x) >= n_chunk) {
            const int v = (static_cast<int>(blockIdx.x) - n_chunk) * 8 +
                          __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
            if (v < a.decode.n_slots * a.decode.hkv)
                cache_decode_wave<Q8, HD>(a, v % a.decode.n_slots, v / a.decode.n_slots, threadIdx.x & 63);
            return;
        }
    }
    constexpr int KK = HD / 32, NT = HD / 16, PAGE = HD * 16;
    constexpr int PB = PAGE * (Q8 ? 1 : 2);     // bytes of a page
    constexpr int HALF = 4 * PB / 16;           // 16-byte pieces of the K (or V) pages of a tile
    constexpr int PT = 2 * HALF / 512;          // pieces a thread moves
    constexpr int PP = PB / 16;                 // pieces of a page
    static_assert(PT >= 1 && PP % 64 == 0, "a wave's pieces lie in one page");
    constexpr int CT = 2, PW = 32 / GROUP;
    __shared__ __attribute__((aligned(16))) bf16 Ks[2][4 * PAGE];
    __shared__ __attribute__((aligned(16))) bf16 Vs[2][4 * PAGE];
    __shared__ int odd[2][8];  // wave w wrote a V value that is not finite (edge tiles only)

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int grp = lane >> 4, col = lane & 15;
    const int pos = xcd_order(blockIdx.x, c.n_slots * c.hkv);
    const int kvh = pos / c.n_slots, slot = pos % c.n_slots;
    const float sl2 = kLog2e / sqrtf(static_cast<float>(HD));
    bf16x8 ones;
#pragma unroll
    for (int e = 0; e < 8; ++e) ones[e] = bf16(1.0f);

    // Piece i of a thread: piece j = 512 i + tid of the tile, K pages first.
    auto piece = [&](int i, bool& is_v, int& page, int& at) {
        const int j = 512 * i + wave * 64;  // wave-uniform part
        is_v = j >= HALF;
        const int jj = is_v ? j - HALF : j;
        page = jj / PP;
        at = jj % PP + lane;
    };

    const int i0 = c.slot_off[slot], i1 = c.slot_off[slot + 1];
    for (int k = i0; k < i1; ++k) {
        const int item = c.slot_items[k];
        const int qt = c.item_qt[item], v0 = c.item_kb[item], v1 = c.item_ke[item];
        const int row0 = c.qt_row0[qt], nrows = c.qt_rows[qt], pos0 = c.qt_pos0[qt], skip = a.qt_skip[qt];
        const const_i32* bt_s = (const const_i32*)(c.bt + c.qt_bt[qt]);
        const int key_end = pos0 + nrows, last_page = (key_end - 1) >> 4;
        const int j0 = wave * PW;
        const int n_tiles = (v1 - v0 + 63) / 64;
        const int lo = pos0 + j0, hi = pos0 + j0 + PW - 1;  // the wave's positions
        const bool wave_live = j0 < nrows;
        const bool whole = c.qt_off[qt + 1] - c.qt_off[qt] == 1;
        // rows at position p see sinks and keys past p - window
        const int window = a.window > 0 ? a.window : 0x7FFFFFFF, sinks = a.sinks;
        auto key0_of = [&](int t) {
            const int v = v0 + 64 * t;
            return v < a.sink_end ? v : v + skip;
        };
        // a key tile that some row from position p0 to p1 does not see whole
        auto edge = [&](int key0, int p0, int p1) { return key0 + 63 > p0 || (p1 - window >= key0 && key0 + 63 >= sinks); };

        bf16x8 qf[CT][KK];
        const bf16* qkv = static_cast<const bf16*>(c.qkv);
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            const int r = ct * 16 + col, j = j0 + r / GROUP, h = kvh * GROUP + r % GROUP;
#pragma unroll
            for (int kk = 0; kk < KK; ++kk)
                qf[ct][kk] = j < nrows ? *reinterpret_cast<const bf16x8*>(
                                             qkv + static_cast<size_t>(row0 + j) * c.ld_qkv + h * HD + kk * 32 + grp * 8)
                                       : bf16x8{};
        }

        u32x4 raw[PT];
        float rscale[PT];
        auto load = [&](int t) {
            const int pg0 = key0_of(t) >> 4;
#pragma unroll
            for (int i = 0; i < PT; ++i) {
                bool is_v;
                int page, at;
                piece(i, is_v, page, at);
                const size_t bh = static_cast<size_t>(bt_s[min(pg0 + page, last_page)]) * c.hkv + kvh;
                raw[i] = *reinterpret_cast<const u32x4*>(static_cast<const uint8_t*>(is_v ? c.v_pool : c.k_pool) + bh * PB + at * 16);
                if constexpr (Q8) rscale[i] = ((const const_f32*)(is_v ? a.v_scale : a.k_scale))[bh];
            }
        };
        // Widen and write a tile.  V values of keys past the sequence's end
        // (unwritten slots, stand-in pages) become 0; their scores are masked.
        auto store = [&](int t) {
            const int key0 = key0_of(t), buf = t & 1;
            bool bad = false;
#pragma unroll
            for (int i = 0; i < PT; ++i) {
                bool is_v;
                int page, at;
                piece(i, is_v, page, at);
                u32x4 x = raw[i];
                if (is_v && key0 + 63 >= key_end) {
                    const int first = key0 + 16 * page + (Q8 ? 0 : 8 * (at & 1));
                    const uint32_t live = low_bits(min(max(key_end - first, 0), 16));
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        if constexpr (Q8) x[w] &= ((((live >> (4 * w)) & 0xFu) * 0x00204081u) & 0x01010101u) * 0xFFu;
                        else x[w] &= ((live >> (2 * w)) & 1u ? 0xFFFFu : 0u) | ((live >> (2 * w)) & 2u ? 0xFFFF0000u : 0u);
                    }
                }
                if (is_v) {
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        if constexpr (Q8) {
                            bad |= (((x[w] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) != 0u;
                        } else {
                            bad |= (x[w] & 0x7F80u) == 0x7F80u || (x[w] & 0x7F800000u) == 0x7F800000u;
                        }
                    }
                }
                bf16* base = &(is_v ? Vs : Ks)[buf][page * PAGE];
                if constexpr (Q8) {
                    const bf16x8 y0 = widen8(x[0], x[1], rscale[i]), y1 = widen8(x[2], x[3], rscale[i]);
                    if (is_v) {
                        *reinterpret_cast<bf16x8*>(base + at * 16 + vswz(at, 0) * 8) = y0;
                        *reinterpret_cast<bf16x8*>(base + at * 16 + vswz(at, 1) * 8) = y1;
                    } else {  // 16 dims of token tok: two of the four 8-dim pieces of a 32-dim slab
                        const int tok = (at & 63) >> 2, q4 = at & 3;
                        bf16* row = base + (2 * (at >> 6) + (q4 >> 1)) * 512 + tok * 32;
                        *reinterpret_cast<bf16x8*>(row + kswz(tok, 2 * (q4 & 1)) * 8) = y0;
                        *reinterpret_cast<bf16x8*>(row + kswz(tok, 2 * (q4 & 1) + 1) * 8) = y1;
                    }
                } else if (is_v) {
                    const int d = at >> 1;
                    *reinterpret_cast<u32x4*>(base + d * 16 + vswz(d, at & 1) * 8) = x;
                } else {
                    const int tok = (at & 63) >> 2;
                    *reinterpret_cast<u32x4*>(base + (at >> 6) * 512 + tok * 32 + kswz(tok, at & 3) * 8) = x;
                }
            }
            const int any = __any(bad);
            if (lane == 0) odd[buf][wave] = any;
        };

        f32x4 o[CT][NT], l_acc[CT];
        float m_run[CT];
        int qpos[CT];  // position of row ct * 16 + col
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) o[ct][nt] = f32x4{};
            l_acc[ct] = f32x4{};
            m_run[ct] = -INFINITY;
            qpos[ct] = lo + (ct * 16 + col) / GROUP;
        }
        auto sees = [&](int kpos, int ct) { return kpos <= qpos[ct] && (kpos < sinks || kpos > qpos[ct] - window); };

        load(0);
        store(0);
        wait_lgkmcnt0();
        barrier_only();
        for (int t = 0; t < n_tiles; ++t) {
            const int buf = t & 1, key0 = key0_of(t);
            if (t + 1 < n_tiles) load(t + 1);
            // tiles that lie past the wave's rows, or before all their windows
            const bool skipped = !wave_live || key0 > hi || (lo - window >= key0 + 63 && key0 >= sinks);
            if (!skipped) {
                const bool masked = edge(key0, lo, hi);
                f32x4 sc[4][CT];  // [2 pair + tile][ct]
#pragma unroll
                for (int p = 0; p < 4; ++p) {
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct) sc[p][ct] = f32x4{};
                    const int key = pair_key(col, p & 1), tok = key & 15;
                    const int base = (2 * (p >> 1) + (key >> 4)) * PAGE + tok * 32 + kswz(tok, grp) * 8;
#pragma unroll
                    for (int kk = 0; kk < KK; ++kk) {
                        const bf16x8 kf = *reinterpret_cast<const bf16x8*>(&Ks[buf][base + kk * 512]);
#pragma unroll
                        for (int ct = 0; ct < CT; ++ct) sc[p][ct] = mfma16(kf, qf[ct][kk], sc[p][ct]);
                    }
                }
                if (masked) {
#pragma unroll
                    for (int p = 0; p < 4; ++p)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int kpos = key0 + 32 * (p >> 1) + pair_key(4 * grp + e, p & 1);
#pragma unroll
                            for (int ct = 0; ct < CT; ++ct) sc[p][ct][e] = sees(kpos, ct) ? sc[p][ct][e] : -INFINITY;
                        }
                }
                float mx[CT];
                bool grow = false;
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) {
                    float m = -INFINITY;
#pragma unroll
                    for (int p = 0; p < 4; ++p)
#pragma unroll
                        for (int e = 0; e < 4; ++e) m = fmaxf(m, sc[p][ct][e]);
                    mx[ct] = rows4_max(m) * sl2;
                    grow |= mx[ct] > m_run[ct] + kSlack;
                }
                if (__any(grow)) {
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct) {
                        const float m_new = fmaxf(m_run[ct], mx[ct]);
                        const float alpha = m_new == -INFINITY ? 1.f : fast_exp2(m_run[ct] - m_new);
                        m_run[ct] = m_new;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float ae = __shfl(alpha, grp * 4 + e, 64);
                            l_acc[ct][e] *= ae;
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) o[ct][nt][e] *= ae;
                        }
                    }
                }
                bf16x8 pf[2][CT];
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) {
                    const float m_use = m_run[ct] == -INFINITY ? 0.f : m_run[ct];
#pragma unroll
                    for (int p = 0; p < 4; ++p)
#pragma unroll
                        for (int e = 0; e < 4; ++e) sc[p][ct][e] = fast_exp2(fmaf(sc[p][ct][e], sl2, -m_use));
#pragma unroll
                    for (int j = 0; j < 2; ++j) pf[j][ct] = to_bf16x8(sc[2 * j][ct], sc[2 * j + 1][ct]);
                }
                int any_odd = 0;
                if (masked) {
#pragma unroll
                    for (int w = 0; w < 8; ++w) any_odd |= odd[buf][w];
                    any_odd = __builtin_amdgcn_readfirstlane(any_odd);
                }
#pragma unroll
                for (int j = 0; j < 2; ++j) {
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct) l_acc[ct] = mfma16(pf[j][ct], ones, l_acc[ct]);
                    bf16x8 vis[CT];
                    if (any_odd) {
#pragma unroll
                        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                vis[ct][e] = bf16(sees(key0 + 32 * j + pair_key(4 * grp + (e & 3), e >> 2), ct) ? 1.0f : 0.0f);
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        const int d = nt * 16 + col;
                        bf16x8 vf = *reinterpret_cast<const bf16x8*>(
                            &Vs[buf][(2 * j + (grp >> 1)) * PAGE + d * 16 + vswz(d, grp & 1) * 8]);
                        if (any_odd) {
                            u32x4 bits = __builtin_bit_cast(u32x4, vf), pinf = {}, ninf = {}, nan = {};
#pragma unroll
                            for (int w = 0; w < 4; ++w)
#pragma unroll
                                for (int h = 0; h < 2; ++h) {
                                    const uint32_t x = (bits[w] >> (16 * h)) & 0xFFFFu, one = 0x3F80u << (16 * h);
                                    if ((x & 0x7F80u) != 0x7F80u) continue;
                                    if (x == 0x7F80u) pinf[w] |= one;
                                    else if (x == 0xFF80u) ninf[w] |= one;
                                    else nan[w] |= one;
                                    bits[w] &= ~(0xFFFFu << (16 * h));
                                }
                            vf = __builtin_bit_cast(bf16x8, bits);
#pragma unroll
                            for (int ct = 0; ct < CT; ++ct) {
                                const f32x4 np = mfma16(vis[ct], __builtin_bit_cast(bf16x8, pinf), f32x4{});
                                const f32x4 nn = mfma16(vis[ct], __builtin_bit_cast(bf16x8, ninf), f32x4{});
                                const f32x4 nx = mfma16(vis[ct], __builtin_bit_cast(bf16x8, nan), f32x4{});
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    if (np[e] > 0.f) o[ct][nt][e] += INFINITY;
                                    if (nn[e] > 0.f) o[ct][nt][e] -= INFINITY;
                                    if (nx[e] > 0.f) o[ct][nt][e] = NAN;
                                }
                            }
                        }
#pragma unroll
                        for (int ct = 0; ct < CT; ++ct) o[ct][nt] = mfma16(pf[j][ct], vf, o[ct][nt]);
                    }
                }
            }
            if (t + 1 < n_tiles) store(t + 1);
            wait_lgkmcnt0();
            barrier_only();
        }
        if (!wave_live) continue;

#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            if (!whole) {
                const size_t rbase = (static_cast<size_t>(item) * c.hkv + kvh) * 256 + wave * 32 + ct * 16;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    // the maximum of row 4 grp + e sits in column 4 grp + e
                    float m = __shfl(m_run[ct], grp * 4 + e, 64);
                    const float l = l_acc[ct][e];
                    m = m == -INFINITY && l != l ? 0.f : m;  // as in the decode kernel
                    if (col == 0) {
                        c.part_ml[(rbase + grp * 4 + e) * 2] = m;
                        c.part_ml[(rbase + grp * 4 + e) * 2 + 1] = l;
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
                        c.part_o[(rbase + grp * 4 + e) * HD + nt * 16 + col] = o[ct][nt][e];
                }
            } else {
                bf16* out = static_cast<bf16*>(c.out);
                const int ldo = c.hq * HD;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int r = ct * 16 + grp * 4 + e;
                    const int j = j0 + r / GROUP, h = kvh * GROUP + r % GROUP;
                    const float inv = 1.0f / l_acc[ct][e];
                    if (j < nrows) {
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
                            out[static_cast<size_t>(row0 + j) * ldo + h * HD + nt * 16 + col] = f2bf(o[ct][nt][e] * inv);
                    }
                }
            }
        }
    }
}

template <bool Q8, int HD, int GROUP>
void launch_g(const CacheAttnArgs& a, hipStream_t s) {
    const int blocks = a.chunk.n_slots * a.chunk.hkv + (a.decode.n_slots * a.decode.hkv + 7) / 8;
    cache_chunk_kernel<Q8, HD, GROUP><<<blocks, 512, 0, s>>>(a);
}

template <bool Q8, int HD>
void launch_hd(const CacheAttnArgs& a, hipStream_t s) {
    if (a.chunk.n_items <= 0) {
        if (a.decode.b > 0) cache_decode_kernel<Q8, HD><<<dim3(a.decode.n_slots, a.decode.hkv), 64, 0, s>>>(a);
        return;
    }
    switch (a.chunk.hq / a.chunk.hkv) {
        case 1: launch_g<Q8, HD, 1>(a, s); break;
        case 2: launch_g<Q8, HD, 2>(a, s); break;
        case 4: launch_g<Q8, HD, 4>(a, s); break;
        case 8: launch_g<Q8, HD, 8>(a, s); break;
        default: launch_g<Q8, HD, 16>(a, s); break;
    }
}

}  // namespace

void launch_cache_attention(const CacheAttnArgs& a, hipStream_t s) {
    const int hd = a.chunk.n_items > 0 ? a.chunk.hd : a.decode.hd;
    if (a.k_scale) {
        if (hd == 128) launch_hd<true, 128>(a, s);
        else launch_hd<true, 64>(a, s);
    } else {
        if (hd == 128) launch_hd<false, 128>(a, s);
        else launch_hd<false, 64>(a, s);
    }
}

}  // namespace slw
