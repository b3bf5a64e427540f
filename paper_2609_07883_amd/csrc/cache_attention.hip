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

#include <type_traits>

#include "attn_device.h"
#include "kernels.h"

namespace slw {
namespace {

typedef const float __attribute__((address_space(4))) const_f32;
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Lists through the scalar cache.
__device__ __forceinline__ int of(const int32_t* p, int i) { return ((const const_i32*)p)[i]; }
__device__ __forceinline__ const const_i32* record(const int32_t* p, int i) { return (const const_i32*)p + 8 * i; }

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
// Bound by HBM.  The waves of a slot's kv heads lie next to each other in the
// launch, since the heads' pages of a block do in memory; where the layers'
// pages exceed the 256 MB last-level cache (a.once), they are loaded as data
// that nobody reads again.  256 chat decodes over the 8-bit cache, 505 MB, in
// runs for 2048 waves: 110.6 -> 98.2 us (the first alone 109.5, the second alone
// 99.9); with runs for 768 (attn_plan.cpp) 91.4 us, 5.5 TB/s, where a large copy
// reaches 5.16; beside a chunk of 64 rows 142 -> 132.  Data that
// is still there is read slower so: 32 decodes of 84 MB beside 256 rows 46
// against 38 us.
//
// A decode of one item is written as its rows, the others as partial sums for
// the merge's launch.  Combining those by the last wave to finish instead took
// longer: with release and acquire fences 45 -> 111 us for 64 decodes, with
// partial sums written through and read past the L2s 45 -> 53.
// ---------------------------------------------------------------------------
template <bool ONCE>
__device__ __forceinline__ u32x4 load_page(const uint8_t* p) {
    if constexpr (ONCE) return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
    else return *reinterpret_cast<const u32x4*>(p);
}

template <bool Q8, int HD>
struct CacheStep {
    static constexpr int TAU = Q8 ? 4 : 2;                // score tiles
    static constexpr int KL = Q8 ? HD / 64 : HD / 32;     // 16-byte pieces of a key row per lane
    static constexpr int VL = HD / 16;
    u32x4 k[TAU][KL];
    u32x4 v[VL];
    float ks, vs;  // e4m3: scales of the lane group's page
};

template <bool Q8, int HD, bool ONCE>
__device__ __forceinline__ void cache_load(CacheStep<Q8, HD>& st, const CacheAttnArgs& a, const const_i32* bt_s, int k0,
                                           int last_pg, int kvh, int col, int grp) {
    constexpr int PAGES = Q8 ? 4 : 2, PB = HD * 16 * (Q8 ? 1 : 2);  // pages of a step, bytes of a page
    const int pg0 = k0 >> 4;
    const int b0 = bt_s[min(pg0, last_pg)], b1 = bt_s[min(pg0 + 1, last_pg)];
    const int b2 = PAGES == 4 ? bt_s[min(pg0 + 2, last_pg)] : 0, b3 = PAGES == 4 ? bt_s[min(pg0 + 3, last_pg)] : 0;
    auto pick = [&](int i) {
        const int lo = i & 1 ? b1 : b0, hi = i & 1 ? b3 : b2;
        return PAGES == 4 && (i & 2) ? hi : lo;
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
            st.k[tau][s] = load_page<ONCE>(kpage + s * 1024 + tok * 64 + grp * 16);
    }
    const size_t vbh = static_cast<size_t>(pick(Q8 ? grp : grp >> 1)) * hkv + kvh;
    const uint8_t* vpage = vpool + vbh * PB;
#pragma unroll
    for (int nt = 0; nt < CacheStep<Q8, HD>::VL; ++nt)
        st.v[nt] = load_page<ONCE>(vpage + (nt * 16 + col) * (Q8 ? 16 : 32) + (Q8 ? 0 : 16 * (grp & 1)));
    if constexpr (Q8) {
        st.ks = a.k_scale[vbh];
        st.vs = a.v_scale[vbh];
    }
}

template <bool Q8, int HD, bool ONCE>
__device__ __forceinline__ void cache_decode_items(const CacheAttnArgs& a, int slot, int kvh, int lane) {
    using Step = CacheStep<Q8, HD>;
    constexpr int TAU = Step::TAU, KL = Step::KL, NT = HD / 16, KPL = 4 * TAU, KEYS = 4 * KPL;
    const DecodeAttnArgs& d = a.decode;
    const int grp = lane >> 4, col = lane & 15;
    const int group = d.hq / d.hkv;
    const float sl2 = kLog2e / sqrtf(static_cast<float>(HD));

    // Through the scalar cache an item's lists take 0.3 to 1 us less.  (Asked
    // for an item ahead, under the first keys of the one before, they took 0.5
    // to 1 us longer: most waves have one item or two.)
    const int i0 = of(d.slot_off, slot), i1 = of(d.slot_off, slot + 1);
    for (int w = i0; w < i1; ++w) {
        const const_i32* rec = record(a.decode_items, w);
        const int b = rec[0], v0 = rec[1], v1 = rec[2], len = rec[3], skip = rec[4], at = rec[5];
        const bool whole = rec[6] != 0;  // all of the decode
        const int last_pg = (len - 1) >> 4;
        // keys below w_lo are seen only if they are sinks
        const int w_lo = a.window > 0 ? max(len - a.window, 0) : 0;
        const const_i32* bt_s = (const const_i32*)(d.bt + at);
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
            // A page with no seen key has no part through its scales either: -inf
            // times one that is 0, NaN or negative (a page never written) is not
            // -inf, and a code of 0 times NaN not 0.
            const float scale = Q8 ? (seen ? sl2 * st.ks : 1.f) : sl2;
            const float v_scale = Q8 && seen ? st.vs : 1.f;
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
                // e4m3: P in two bf16 terms, whose sum has 16 bits; the matrix
                // cores have time to spare here (bf16 V can hold infinities,
                // which a second term of 0 or less would turn into NaN)
                bf16x8 pr;
                if constexpr (Q8) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) pr[e] = f2bf(s[2 * j + (e >> 2)][e & 3] - bf2f(pf[e]));
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const u32x4 x = st.v[nt] & vmask;
                    if constexpr (Q8) {
                        const bf16x8 v = widen8(x[2 * j], x[2 * j + 1], v_scale);
                        o[nt] = mfma16(pf, v, mfma16(pr, v, o[nt]));
                    } else {
                        o[nt] = mfma16(pf, __builtin_bit_cast(bf16x8, x), o[nt]);
                    }
                }
            }
        };

        // A step's loads follow the products of the step two before it, so one or
        // two steps are in flight; past the item's end they re-read a page of
        // the sequence, so that no branch skips a load.
        Step sa, sb;
        cache_load<Q8, HD, ONCE>(sa, a, bt_s, key_of(v0), last_pg, kvh, col, grp);
        cache_load<Q8, HD, ONCE>(sb, a, bt_s, key_of(v0 + KEYS), last_pg, kvh, col, grp);
        for (int c0 = v0;; c0 += 2 * KEYS) {
            compute(sa, c0);
            if (c0 + KEYS >= v1) break;
            cache_load<Q8, HD, ONCE>(sa, a, bt_s, key_of(c0 + 2 * KEYS), last_pg, kvh, col, grp);
            compute(sb, c0 + KEYS);
            if (c0 + 2 * KEYS >= v1) break;
            cache_load<Q8, HD, ONCE>(sb, a, bt_s, key_of(c0 + 3 * KEYS), last_pg, kvh, col, grp);
        }

        const float l = rows4_sum(l_run);
        // a maximum of -inf marks a part that saw no key: where every score
        // seen was NaN, the sum says so instead
        const float m = m_run == -INFINITY && l != l ? 0.f : m_run;
        if (whole) {  // its rows
            bf16* out = static_cast<bf16*>(d.out) + (static_cast<size_t>(b) * d.hq + kvh * group) * HD;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int h = grp * 4 + e;
                const float inv = 1.0f / __shfl(l, h, 64);
                if (h < group) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) out[h * HD + nt * 16 + col] = f2bf(o[nt][e] * inv);
                }
            }
            continue;
        }
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
__device__ __forceinline__ void cache_decode_wave(const CacheAttnArgs& a, int slot, int kvh, int lane) {
    if (a.once) cache_decode_items<Q8, HD, true>(a, slot, kvh, lane);
    else cache_decode_items<Q8, HD, false>(a, slot, kvh, lane);
}

template <bool Q8, int HD>
__global__ __launch_bounds__(64, 2) void cache_decode_kernel(CacheAttnArgs a) {
    cache_decode_wave<Q8, HD>(a, blockIdx.y, blockIdx.x, threadIdx.x);
}

// ---------------------------------------------------------------------------
// Chunk attention: the rows of a query tile (256 / GROUP positions of one
// prompt, GROUP q heads of one kv head) against its keys, 64 at a time, as in
// the bf16 kernels: eight waves of 32 rows, K and V tiles in bf16 in LDS.
//
// Tiles go through registers on their way to LDS, since e4m3 pages are widened
// there, once per work-group instead of once per wave.
//
// A key that some rows of a wave see and others do not stays out of the
// others' products through a zero probability, unless its V row is not finite
// (0 times it would be NaN).  The kernels look for such values in the tiles that
// some row does not see whole; an item that met one is computed again by
// exact_item, which keeps them apart.
// ---------------------------------------------------------------------------

// One work item of a work-group, and the wave's share of it.
struct Item {
    const const_i32* bt;
    int item, row0, nrows, pos0, skip, v0, n_tiles;
    int key_end, last_page;
    int j0, lo, hi;         // the wave's first tile position, first and last sequence position
    int window, sinks, sink_end;
    bool live, whole;

    __device__ __forceinline__ Item(const CacheAttnArgs& a, int index, int wave, int pw) {
        const ChunkAttnArgs& c = a.chunk;
        const const_i32* rec = record(a.chunk_items, index);
        whole = rec[0] < 0;
        item = whole ? ~rec[0] : rec[0];
        v0 = rec[1];
        n_tiles = (rec[2] - v0 + 63) / 64;
        row0 = rec[3];
        nrows = rec[4];
        pos0 = rec[5];
        skip = rec[6];
        bt = (const const_i32*)(c.bt + rec[7]);
        key_end = pos0 + nrows;
        last_page = (key_end - 1) >> 4;
        j0 = wave * pw;
        lo = pos0 + j0;
        hi = lo + pw - 1;
        live = j0 < nrows;
        window = a.window > 0 ? a.window : 0x7FFFFFFF;
        sinks = a.sinks;
        sink_end = a.sink_end;
    }
    __device__ __forceinline__ int key0(int t) const {
        const int v = v0 + 64 * t;
        return v < sink_end ? v : v + skip;
    }
    __device__ __forceinline__ int block(int key0, int page) const {
        return bt[__builtin_amdgcn_readfirstlane(min((key0 >> 4) + page, last_page))];
    }
    // some row of the query tile does not see every key of the tile
    __device__ __forceinline__ bool edge(int key0) const {
        return key0 + 63 > pos0 || (key_end - 1 - window >= key0 && key0 + 63 >= sinks);
    }
    // the wave's rows see no key of the tile / not every key of it
    __device__ __forceinline__ bool unseen(int key0) const {
        return key0 > hi || (lo - window >= key0 + 63 && key0 >= sinks);
    }
    __device__ __forceinline__ bool masked(int key0) const {
        return key0 + 63 > lo || (hi - window >= key0 && key0 + 63 >= sinks);
    }
    __device__ __forceinline__ bool sees(int qpos, int kpos) const {
        return kpos <= qpos && (kpos < sinks || kpos > qpos - window);
    }
};

// Where the 16-byte pieces of a tile's pages go.  A tile has 4 PP pieces of K
// and as many of V; those that a wave moves at once lie in one page.
template <bool Q8, int HD>
struct Pieces {
    static constexpr int PAGE = HD * 16, PB = PAGE * (Q8 ? 1 : 2), PP = PB / 16;
    static_assert(PP % 64 == 0, "a wave's pieces lie in one page");

    // `first`: the piece's number among the K (or V) pieces, of the wave's lane 0
    static __device__ __forceinline__ int page(int first) { return first / PP; }
    static __device__ __forceinline__ int offset(int first, int lane) { return first % PP + lane; }

    static __device__ __forceinline__ void put_k(bf16* tile, int first, int lane, u32x4 x, float scale) {
        const int at = offset(first, lane), tok = (at & 63) >> 2;
        bf16* base = tile + page(first) * PAGE + tok * 32;
        if constexpr (Q8) {  // 16 dims of token tok: two of the four 8-dim pieces of a 32-dim slab
            const int q4 = at & 3;
            bf16* row = base + (2 * (at >> 6) + (q4 >> 1)) * 512;
            *reinterpret_cast<bf16x8*>(row + kswz(tok, 2 * (q4 & 1)) * 8) = widen8(x[0], x[1], scale);
            *reinterpret_cast<bf16x8*>(row + kswz(tok, 2 * (q4 & 1) + 1) * 8) = widen8(x[2], x[3], scale);
        } else {
            *reinterpret_cast<u32x4*>(base + (at >> 6) * 512 + kswz(tok, at & 3) * 8) = x;
        }
    }
    // Values of keys from key_end on (unwritten slots, stand-in pages) become
    // 0; their scores are masked.  Nonzero result: a value is not finite, or
    // may not be once widened: 448 times 2^120 and more, which a scale of a page
    // that no row sees can be.
    static __device__ __forceinline__ uint32_t settle_v(int first, int lane, u32x4& x, int key0, int key_end,
                                                        float scale) {
        if (key0 + 63 >= key_end) {
            const int k = key0 + 16 * page(first) + (Q8 ? 0 : 8 * (offset(first, lane) & 1));
            const uint32_t live = low_bits(min(max(key_end - k, 0), 16));
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                if constexpr (Q8) x[w] &= ((((live >> (4 * w)) & 0xFu) * 0x00204081u) & 0x01010101u) * 0xFFu;
                else x[w] &= ((live >> (2 * w)) & 1u ? 0xFFFFu : 0u) | ((live >> (2 * w)) & 2u ? 0xFFFF0000u : 0u);
            }
        }
        uint32_t odd = 0;
#pragma unroll
        for (int w = 0; w < 4; ++w) {  // an all-ones magnitude (exponent) carries into the sign
            if constexpr (Q8) odd |= (x[w] & 0x7F7F7F7Fu) + 0x01010101u;
            else odd |= (x[w] & 0x7F807F80u) + 0x00800080u;
        }
        odd &= Q8 ? 0x80808080u : 0x80008000u;
        if constexpr (Q8) odd |= ((__float_as_uint(scale) >> 23) & 0xFFu) >= 127u + 120u ? 1u : 0u;
        return odd;
    }
    static __device__ __forceinline__ void put_v(bf16* tile, int first, int lane, u32x4 x, float scale) {
        const int at = offset(first, lane);
        bf16* base = tile + page(first) * PAGE;
        if constexpr (Q8) {
            *reinterpret_cast<bf16x8*>(base + at * 16 + vswz(at, 0) * 8) = widen8(x[0], x[1], scale);
            *reinterpret_cast<bf16x8*>(base + at * 16 + vswz(at, 1) * 8) = widen8(x[2], x[3], scale);
        } else {
            const int d = at >> 1;
            *reinterpret_cast<u32x4*>(base + d * 16 + vswz(d, at & 1) * 8) = x;
        }
    }
};

// A tile on its way through a work-group's registers.
template <bool Q8, int HD>
struct Staged {
    using P = Pieces<Q8, HD>;
    static constexpr int HALF = 4 * P::PP, PT = 2 * HALF / 512;  // pieces of K (or V); pieces a thread moves
    u32x4 raw[PT];
    float scale[PT];
    int blk[PT];

    // Block ids of a tile's pages, through the scalar cache, a tile before load() uses them.
    __device__ __forceinline__ void fetch(const Item& it, int wave, int t) {
        const int key0 = it.key0(t);
#pragma unroll
        for (int i = 0; i < PT; ++i) {
            const int j = 512 * i + 64 * wave;
            blk[i] = it.block(key0, P::page(j >= HALF ? j - HALF : j));
        }
    }
    // The scales come as vectors too: a scalar load in flight would make every
    // wait for an LDS read of the tile before a wait for it.
    __device__ __forceinline__ void load(const CacheAttnArgs& a, int kvh, int wave, int lane) {
#pragma unroll
        for (int i = 0; i < PT; ++i) {
            const int j = 512 * i + 64 * wave;
            const bool is_v = j >= HALF;
            const size_t bh = static_cast<size_t>(blk[i]) * a.chunk.hkv + kvh;
            const void* pool = is_v ? a.chunk.v_pool : a.chunk.k_pool;
            raw[i] = *reinterpret_cast<const u32x4*>(static_cast<const uint8_t*>(pool) + bh * P::PB +
                                                     P::offset(is_v ? j - HALF : j, lane) * 16);
            if constexpr (Q8) {
                uint32_t zero = 0;
                asm volatile("" : "+v"(zero));  // an address in vector registers
                scale[i] = (is_v ? a.v_scale : a.k_scale)[bh + zero];
            }
        }
    }
    // nonzero: a V value of a tile on an edge of the mask is not finite
    __device__ __forceinline__ uint32_t store(bf16* ks, bf16* vs, const Item& it, int wave, int lane, int t) {
        const int key0 = it.key0(t);
        uint32_t odd = 0;
        if (it.edge(key0)) {
#pragma unroll
            for (int i = 0; i < PT; ++i) {
                const int j = 512 * i + 64 * wave;
                if (j >= HALF) odd |= P::settle_v(j - HALF, lane, raw[i], key0, it.key_end, Q8 ? scale[i] : 1.f);
            }
        }
#pragma unroll
        for (int i = 0; i < PT; ++i) {
            const int j = 512 * i + 64 * wave;
            if (j >= HALF) P::put_v(vs, j - HALF, lane, raw[i], scale[i]);
            else P::put_k(ks, j, lane, raw[i], scale[i]);
        }
        return odd;
    }
};

// Q^T operand: row r = ct * 16 + col is tile position j0 + r / GROUP, head kvh * GROUP + r % GROUP.
template <int HD, int GROUP>
__device__ __forceinline__ void load_q(bf16x8 (&qf)[2][HD / 32], const ChunkAttnArgs& c, const Item& it, int kvh, int col,
                                       int grp) {
    const bf16* q = static_cast<const bf16*>(c.qkv);
#pragma unroll
    for (int ct = 0; ct < 2; ++ct) {
        const int r = ct * 16 + col, j = it.j0 + r / GROUP, h = kvh * GROUP + r % GROUP;
#pragma unroll
        for (int kk = 0; kk < HD / 32; ++kk)
            qf[ct][kk] = j < it.nrows ? *reinterpret_cast<const bf16x8*>(
                                            q + static_cast<size_t>(it.row0 + j) * c.ld_qkv + h * HD + kk * 32 + grp * 8)
                                      : bf16x8{};
    }
}

// A wave's rows of an item, in registers: running maximum of row ct * 16 + col,
// row sums and outputs of rows ct * 16 + 4 grp + e, NT 16-dim tiles of them.
template <int HD, int NT = HD / 16>
struct Rows {
    f32x4 o[2][NT], l[2];
    float m[2];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int ct = 0; ct < 2; ++ct) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) o[ct][nt] = f32x4{};
            l[ct] = f32x4{};
            m[ct] = -INFINITY;
        }
    }
    // Scores of a tile, masked, to probabilities against the running maximum.
    template <int GROUP>
    __device__ __forceinline__ void softmax(f32x4 (&sc)[4][2], bf16x8 (&pf)[2][2], const Item& it, int key0, float sl2,
                                            int col, int grp) {
        if (it.masked(key0)) {
#pragma unroll
            for (int p = 0; p < 4; ++p)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int kpos = key0 + 32 * (p >> 1) + pair_key(4 * grp + e, p & 1);
#pragma unroll
                    for (int ct = 0; ct < 2; ++ct)
                        sc[p][ct][e] = it.sees(it.lo + (ct * 16 + col) / GROUP, kpos) ? sc[p][ct][e] : -INFINITY;
                }
        }
        float mx[2];
        bool grow = false;
#pragma unroll
        for (int ct = 0; ct < 2; ++ct) {
            float x = -INFINITY;
#pragma unroll
            for (int p = 0; p < 4; ++p)
#pragma unroll
                for (int e = 0; e < 4; ++e) x = fmaxf(x, sc[p][ct][e]);
            mx[ct] = rows4_max(x) * sl2;
            grow |= mx[ct] > m[ct] + kSlack;
        }
        if (__any(grow)) {
#pragma unroll
            for (int ct = 0; ct < 2; ++ct) {
                const float m_new = fmaxf(m[ct], mx[ct]);
                const float alpha = m_new == -INFINITY ? 1.f : fast_exp2(m[ct] - m_new);
                m[ct] = m_new;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float ae = __shfl(alpha, grp * 4 + e, 64);
                    l[ct][e] *= ae;
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) o[ct][nt][e] *= ae;
                }
            }
        }
#pragma unroll
        for (int ct = 0; ct < 2; ++ct) {
            const float m_use = m[ct] == -INFINITY ? 0.f : m[ct];
#pragma unroll
            for (int p = 0; p < 4; ++p)
#pragma unroll
                for (int e = 0; e < 4; ++e) sc[p][ct][e] = fast_exp2(fmaf(sc[p][ct][e], sl2, -m_use));
#pragma unroll
            for (int j = 0; j < 2; ++j) pf[j][ct] = to_bf16x8(sc[2 * j][ct], sc[2 * j + 1][ct]);
        }
    }
    // Normalised rows, or the item's partial sums, from dim d0 on.
    template <int GROUP>
    __device__ __forceinline__ void write(const ChunkAttnArgs& c, const Item& it, int kvh, int wave, int col, int grp,
                                          int d0 = 0) const {
#pragma unroll
        for (int ct = 0; ct < 2; ++ct) {
            if (!it.whole) {
                const size_t rbase = (static_cast<size_t>(it.item) * c.hkv + kvh) * 256 + wave * 32 + ct * 16;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    // the maximum of row 4 grp + e sits in column 4 grp + e
                    const float x = __shfl(m[ct], grp * 4 + e, 64), s = l[ct][e];
                    if (col == 0) {  // a part of NaN scores alone, as in the decode kernel
                        c.part_ml[(rbase + grp * 4 + e) * 2] = x == -INFINITY && s != s ? 0.f : x;
                        c.part_ml[(rbase + grp * 4 + e) * 2 + 1] = s;
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) c.part_o[(rbase + grp * 4 + e) * HD + d0 + nt * 16 + col] = o[ct][nt][e];
                }
            } else {
                bf16* out = static_cast<bf16*>(c.out);
                const int ldo = c.hq * HD;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int r = ct * 16 + grp * 4 + e;
                    const int j = it.j0 + r / GROUP, h = kvh * GROUP + r % GROUP;
                    const float inv = 1.0f / l[ct][e];
                    if (j < it.nrows) {
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
                            out[static_cast<size_t>(it.row0 + j) * ldo + h * HD + d0 + nt * 16 + col] = f2bf(o[ct][nt][e] * inv);
                    }
                }
            }
        }
    }
};

__device__ __forceinline__ bf16x8 ones8() {
    bf16x8 r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = bf16(1.0f);
    return r;
}

// An item whose V holds values that are not finite: the finite ones are
// multiplied alone, and rows that see one of the others get what it makes of
// their sums (counted by products of visibility and class).  Rare, so it is
// built for few registers, beside the loop that it stands in for: 32 output
// dims at a time, scores and all.
template <bool Q8, int HD, int GROUP>
__device__ __forceinline__ void exact_item(const CacheAttnArgs& a, const Item& it, int kvh, bf16* ks, bf16* vs, float sl2) {
    constexpr int KK = HD / 32, NT = 2, PAGE = HD * 16, CT = 2;
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));  // keeps what follows from it out of the loop that this stands in for
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int grp = lane >> 4, col = lane & 15;
    const bf16x8 ones = ones8();
    bf16x8 qf[CT][KK];
    load_q<HD, GROUP>(qf, a.chunk, it, kvh, col, grp);
#pragma unroll 1
    for (int d0 = 0; d0 < HD; d0 += 16 * NT) {
        Rows<HD, NT> rows;
        rows.clear();
#pragma unroll 1
        for (int t = 0; t < it.n_tiles; ++t) {
            const int key0 = it.key0(t);
            barrier_only();
            {
                Staged<Q8, HD> st;
                st.fetch(it, wave, t);
                st.load(a, kvh, wave, lane);
                st.store(ks, vs, it, wave, lane, t);
            }
            wait_lgkmcnt0();
            barrier_only();
            if (!it.live || it.unseen(key0)) continue;
            f32x4 sc[4][CT];
#pragma unroll
            for (int p = 0; p < 4; ++p) {
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) sc[p][ct] = f32x4{};
                const int key = pair_key(col, p & 1), tok = key & 15;
                const int base = (2 * (p >> 1) + (key >> 4)) * PAGE + tok * 32 + kswz(tok, grp) * 8;
#pragma unroll
                for (int kk = 0; kk < KK; ++kk) {
                    const bf16x8 kf = *reinterpret_cast<const bf16x8*>(&ks[base + kk * 512]);
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct) sc[p][ct] = mfma16(kf, qf[ct][kk], sc[p][ct]);
                }
            }
            bf16x8 pf[2][CT];
            rows.template softmax<GROUP>(sc, pf, it, key0, sl2, col, grp);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                bf16x8 vis[CT];
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) {
                    rows.l[ct] = mfma16(pf[j][ct], ones, rows.l[ct]);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        vis[ct][e] = bf16(it.sees(it.lo + (ct * 16 + col) / GROUP,
                                                  key0 + 32 * j + pair_key(4 * grp + (e & 3), e >> 2)) ? 1.0f : 0.0f);
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const int d = d0 + nt * 16 + col;
                    u32x4 bits = *reinterpret_cast<const u32x4*>(&vs[(2 * j + (grp >> 1)) * PAGE + d * 16 + vswz(d, grp & 1) * 8]);
                    u32x4 pinf = {}, ninf = {}, nan = {};
#pragma unroll
                    for (int w = 0; w < 4; ++w)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const uint32_t x = (bits[w] >> (16 * h)) & 0xFFFFu, one = 0x3F80u << (16 * h);
                            const bool odd = (x & 0x7F80u) == 0x7F80u;
                            pinf[w] |= x == 0x7F80u ? one : 0u;
                            ninf[w] |= x == 0xFF80u ? one : 0u;
                            nan[w] |= odd && (x & 0x7Fu) ? one : 0u;
                            bits[w] &= odd ? ~(0xFFFFu << (16 * h)) : 0xFFFFFFFFu;
                        }
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct) {
                        const f32x4 np = mfma16(vis[ct], __builtin_bit_cast(bf16x8, pinf), f32x4{});
                        const f32x4 nn = mfma16(vis[ct], __builtin_bit_cast(bf16x8, ninf), f32x4{});
                        const f32x4 nx = mfma16(vis[ct], __builtin_bit_cast(bf16x8, nan), f32x4{});
                        f32x4& o = rows.o[ct][nt];
                        o = mfma16(pf[j][ct], __builtin_bit_cast(bf16x8, bits), o);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            if (np[e] > 0.f) o[e] += INFINITY;
                            if (nn[e] > 0.f) o[e] -= INFINITY;
                            if (nx[e] > 0.f) o[e] = NAN;
                        }
                    }
                }
            }
        }
        if (it.live) rows.template write<GROUP>(a.chunk, it, kvh, wave, col, grp, d0);
    }
}

// Whether a wave of the work-group met a V value that is not finite: `odd` is
// nonzero in its lanes.  Every wave is past its last tile when this returns.
__device__ __forceinline__ bool any_odd(uint32_t odd, int* flags) {
    const int tid = threadIdx.x;
    const int mine = __any(odd != 0);
    if ((tid & 63) == 0) flags[tid >> 6] = mine;
    wait_lgkmcnt0();
    barrier_only();
    int all = 0;
#pragma unroll
    for (int w = 0; w < 8; ++w) all |= flags[w];
    return __builtin_amdgcn_readfirstlane(all) != 0;
}

// Decode waves behind the chunk work-groups, as in the bf16 kernel; true in a
// work-group of theirs.
template <bool Q8, int HD>
__device__ __forceinline__ bool decode_group(const CacheAttnArgs& a) {
    const int n_chunk = a.chunk.n_slots * a.chunk.hkv;
    if (static_cast<int>(blockIdx.x) < n_chunk) return false;
    const int v = (static_cast<int>(blockIdx.x) - n_chunk) * 8 +
                  __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
    if (v < a.decode.n_slots * a.decode.hkv)
        cache_decode_wave<Q8, HD>(a, v / a.decode.hkv, v % a.decode.hkv, threadIdx.x & 63);
    return true;
}

// Two LDS buffers: the next tile's loads are in flight while the current one
// is multiplied, and are widened and written to the other buffer after it.
template <bool Q8, int HD, int GROUP>
__global__ __launch_bounds__(512) void cache_chunk_kernel(CacheAttnArgs a) {
    const ChunkAttnArgs& c = a.chunk;
    if (decode_group<Q8, HD>(a)) return;
    constexpr int KK = HD / 32, NT = HD / 16, PAGE = HD * 16, CT = 2, PW = 32 / GROUP;
    __shared__ __attribute__((aligned(16))) bf16 Ks[2][4 * PAGE];
    __shared__ __attribute__((aligned(16))) bf16 Vs[2][4 * PAGE];
    __shared__ int flags[8];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int grp = lane >> 4, col = lane & 15;
    const int pos = xcd_order(blockIdx.x, c.n_slots * c.hkv);
    const int kvh = pos / c.n_slots, slot = pos % c.n_slots;
    const float sl2 = kLog2e / sqrtf(static_cast<float>(HD));
    const bf16x8 ones = ones8();

    const int i0 = of(c.slot_off, slot), i1 = of(c.slot_off, slot + 1);
    for (int k = i0; k < i1; ++k) {
        const Item it(a, k, wave, PW);
        bf16x8 qf[CT][KK];
        load_q<HD, GROUP>(qf, c, it, kvh, col, grp);
        Rows<HD> rows;
        rows.clear();
        uint32_t odd = 0;
        Staged<Q8, HD> st;
        st.fetch(it, wave, 0);
        st.load(a, kvh, wave, lane);
        st.fetch(it, wave, 1);
        odd |= st.store(Ks[0], Vs[0], it, wave, lane, 0);
        wait_lgkmcnt0();
        barrier_only();
        for (int t = 0; t < it.n_tiles; ++t) {
            const int buf = t & 1, key0 = it.key0(t);
            if (t + 1 < it.n_tiles) st.load(a, kvh, wave, lane);
            if (it.live && !it.unseen(key0)) {
                f32x4 sc[4][CT];  // [2 pair + tile][ct]
#pragma unroll
                for (int p = 0; p < 4; ++p)
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct) sc[p][ct] = f32x4{};
                // LDS reads one step ahead of the MFMAs, in the order that the
                // scheduling groups hold, as in the bf16 kernel
                bf16x8 kf[2][KK], vf[2][4];
                auto kread = [&](int p, bf16x8(&f)[KK]) {
                    const int key = pair_key(col, p & 1), tok = key & 15;
                    const int base = (2 * (p >> 1) + (key >> 4)) * PAGE + tok * 32 + kswz(tok, grp) * 8;
#pragma unroll
                    for (int kk = 0; kk < KK; ++kk) f[kk] = *reinterpret_cast<const bf16x8*>(&Ks[buf][base + kk * 512]);
                };
                // V group g: page pair g / (NT / 4), output dims 16 n0 .. + 63, n0 = 4 (g % (NT / 4))
                constexpr int VG = 2 * NT / 4;
                auto vread = [&](int g, bf16x8(&f)[4]) {
                    const int j = g / (NT / 4), n0 = (g % (NT / 4)) * 4;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int d = (n0 + i) * 16 + col;
                        f[i] = *reinterpret_cast<const bf16x8*>(
                            &Vs[buf][(2 * j + (grp >> 1)) * PAGE + d * 16 + vswz(d, grp & 1) * 8]);
                    }
                };
                kread(0, kf[0]);
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    if (p + 1 < 4) kread(p + 1, kf[(p + 1) & 1]);
#pragma unroll
                    for (int kk = 0; kk < KK; ++kk)
#pragma unroll
                        for (int ct = 0; ct < CT; ++ct) sc[p][ct] = mfma16(kf[p & 1][kk], qf[ct][kk], sc[p][ct]);
                }
                vread(0, vf[0]);
                __builtin_amdgcn_sched_group_barrier(0x100, KK, 0);  // 0x100: LDS reads
#pragma unroll
                for (int p = 0; p < 3; ++p) {
#pragma unroll
                    for (int r = 0; r < KK; ++r) {
                        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);  // 0x8: MFMA
                        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                    }
                    if constexpr (KK * CT > KK) __builtin_amdgcn_sched_group_barrier(0x8, KK * CT - KK, 0);
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                }
                if constexpr (KK * CT > 4) __builtin_amdgcn_sched_group_barrier(0x8, KK * CT - 4, 0);
                bf16x8 pf[2][CT];
                rows.template softmax<GROUP>(sc, pf, it, key0, sl2, col, grp);
#pragma unroll
                for (int g = 0; g < VG; ++g) {
                    const int j = g / (NT / 4), n0 = (g % (NT / 4)) * 4;
                    if (g + 1 < VG) vread(g + 1, vf[(g + 1) & 1]);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int ct = 0; ct < CT; ++ct)
                            rows.o[ct][n0 + i] = mfma16(pf[j][ct], vf[g & 1][i], rows.o[ct][n0 + i]);
                    if (n0 == 0) {
#pragma unroll
                        for (int ct = 0; ct < CT; ++ct) rows.l[ct] = mfma16(pf[j][ct], ones, rows.l[ct]);
                    }
                }
#pragma unroll
                for (int g = 0; g < VG; ++g) {
                    if (g + 1 < VG) {
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
                            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                        }
                        if (g % (NT / 4) == 0) __builtin_amdgcn_sched_group_barrier(0x8, 5 * CT - 4, 0);
                        else __builtin_amdgcn_sched_group_barrier(0x8, 4 * CT - 4, 0);
                    } else {
                        if (g % (NT / 4) == 0) __builtin_amdgcn_sched_group_barrier(0x8, 5 * CT, 0);
                        else __builtin_amdgcn_sched_group_barrier(0x8, 4 * CT, 0);
                    }
                }
            }
            if (t + 1 < it.n_tiles) odd |= st.store(Ks[buf ^ 1], Vs[buf ^ 1], it, wave, lane, t + 1);
            wait_lgkmcnt0();
            st.fetch(it, wave, t + 2);
            barrier_only();
        }
        if (it.live) rows.template write<GROUP>(c, it, kvh, wave, col, grp);
        if (any_odd(odd, flags)) exact_item<Q8, HD, GROUP>(a, it, kvh, Ks[0], Vs[0], sl2);  // writes its rows anew
        barrier_only();
    }
}

// ---------------------------------------------------------------------------
// Long work items at head dim 128: two wave groups half a tile apart, as in
// the bf16 kernel of that kind.  A tile's work is two phases with a barrier
// after each,
//   P1(t)  mask, running max, exponentials, P in bf16        (VALU)
//   P2(t)  P V of tile t, then the scores of tile t + 1      (matrix cores)
// and waves 4-7 run one phase behind waves 0-3, so that on every SIMD one
// wave's softmax runs under the other's products.  Every wave computes every
// tile; where its rows see no key of one, the scores are masked.
//
// bf16: rings of four 16 KB tiles of K and of V; P2(t) issues the direct loads
// of V(t + 3) and K(t + 4), as there.
// e4m3: rings of three, and rings of three 8 KB tiles of codes, which direct
// loads fill and where each thread finds the pieces it asked for itself.  P2(t)
// takes the codes of V(t + 2) and K(t + 3) from there, widens and writes them,
// and loads those of V(t + 5) and K(t + 6) in their place, each step between
// two groups of products: a tile's loads have three of them to land.  In slots
// (phases of waves 0-3) the writes of P2(t), slots 2t + 2 and 2t + 3, go to the
// buffers of V(t - 1) and K(t), last read in slot 2t + 1, and are first read in
// slot 2t + 5.  (With the codes in registers instead, one tile ahead, the loads
// were late: 2050 us against 1671 for the bf16 cache at 4096 rows at 28 K.)
// ---------------------------------------------------------------------------
template <bool Q8, int GROUP>
__global__ __launch_bounds__(512) void cache_chunk_pp_kernel(CacheAttnArgs a) {
    constexpr int HD = 128, KK = HD / 32, NT = HD / 16, PAGE = HD * 16, CT = 2, PW = 32 / GROUP;
    const ChunkAttnArgs& c = a.chunk;
    if (decode_group<Q8, HD>(a)) return;
    using P = Pieces<Q8, HD>;
    constexpr int LW = 4 * P::PP / 512;  // 16-byte pieces of each of K and V that a thread moves per tile
    constexpr int RING = Q8 ? 3 : 4;
    __shared__ __attribute__((aligned(16))) bf16 Ks[RING][4 * PAGE];
    __shared__ __attribute__((aligned(16))) bf16 Vs[RING][4 * PAGE];
    __shared__ __attribute__((aligned(16))) u32x4 codes[Q8 ? 2 : 1][Q8 ? 3 : 1][Q8 ? 512 : 1];  // [K, V][tile % 3][thread]
    __shared__ int flags[8];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int behind = wave >> 2;  // 1: the group that runs one phase behind
    const int grp = lane >> 4, col = lane & 15;
    const int pos = xcd_order(blockIdx.x, c.n_slots * c.hkv);
    const int kvh = pos / c.n_slots, slot = pos % c.n_slots;
    const float sl2 = kLog2e / sqrtf(static_cast<float>(HD));
    const bf16x8 ones = ones8();

    // bf16: load i of a wave covers 1 KB slab j = wave + 8 i of K and of V, each
    // lane the 16-byte piece that belongs at its swizzled place
    const int l_k = (lane >> 2) * 32 + kswz(lane >> 2, lane & 3) * 8;
    auto page_of = [&](int i) { return Q8 ? P::page(64 * wave) : (wave + 8 * i) / KK; };

    const int i0 = of(c.slot_off, slot), i1 = of(c.slot_off, slot + 1);
    for (int k = i0; k < i1; ++k) {
        const Item it(a, k, wave, PW);
        const int n_tiles = it.n_tiles;
        bf16x8 qf[CT][KK];
        load_q<HD, GROUP>(qf, c, it, kvh, col, grp);
        uint32_t odd = 0;

        // Block ids of the pages a wave's loads read, through the scalar cache:
        // P2(t) loads K of ids[0], tile t + AHEAD, and V of ids[1], the tile
        // before it.  e4m3: the scales that P2(t) widens K(t + 3) and V(t + 2)
        // with are ksc[0] and vsc[0]; those of tile t + 5 come in before it,
        // in time for memory to answer.  Ids and scales are asked for at the
        // start of P1, which reads nothing from LDS before its end: a scalar
        // load in flight makes a wait for LDS a wait for it (asked for at the
        // end of P2, before its wait for the LDS writes, they cost 400 of
        // 2100 cycles).
        constexpr int AHEAD = Q8 ? 6 : 4;
        int ids[2][LW];
        float ksc[3], vsc[4];
        auto heads = [&](int blk) { return static_cast<size_t>(blk) * c.hkv + kvh; };
        auto k_scale = [&](int blk) { return ((const const_f32*)a.k_scale)[heads(blk)]; };
        auto v_scale = [&](int blk) { return ((const const_f32*)a.v_scale)[heads(blk)]; };
        auto shift = [&](int t) {  // the ids move up by a tile; tile t's come in
#pragma unroll
            for (int i = 0; i < LW; ++i) {
                ids[1][i] = ids[0][i];
                ids[0][i] = it.block(it.key0(t), page_of(i));
            }
        };
        auto next = [&](int t) {  // from P2(t - 1)'s to P2(t)'s
            if constexpr (Q8) {
                ksc[0] = ksc[1];
                ksc[1] = ksc[2];
                ksc[2] = k_scale(ids[0][0]);
                vsc[0] = vsc[1];
                vsc[1] = vsc[2];
                vsc[2] = vsc[3];
                vsc[3] = v_scale(ids[0][0]);
            }
            shift(t + AHEAD);
        };
        auto mod3 = [](int x) { return x >= 3 ? x - 3 : x; };
        auto source = [&](bool is_v, int blk) {  // e4m3: the thread's piece of a page
            return static_cast<const uint8_t*>(is_v ? c.v_pool : c.k_pool) + heads(blk) * P::PB + P::offset(64 * wave, lane) * 16;
        };
        // Loads of tile t (r: t % 3, e4m3) from the block(s) `blk`.
        auto load_k = [&](int i, int t, int r, const int (&blk)[LW]) {
            if constexpr (Q8) {
                load_lds16(source(false, blk[0]), &codes[0][r][64 * wave]);
            } else {
                const int slab = (wave + 8 * i) % KK, at = page_of(i) * PAGE + slab * 512;
                load_lds16(static_cast<const bf16*>(c.k_pool) + heads(blk[i]) * PAGE + slab * 512 + l_k, &Ks[t & 3][at]);
            }
        };
        auto load_v = [&](int i, int t, int r, const int (&blk)[LW]) {
            if constexpr (Q8) {
                load_lds16(source(true, blk[0]), &codes[Q8 ? 1 : 0][r][64 * wave]);
            } else {
                const int slab = (wave + 8 * i) % KK, at = page_of(i) * PAGE + slab * 512;
                const int d = slab * 32 + (lane >> 1), h = (lane & 1) ^ ((d >> 2) & 1);
                load_lds16(static_cast<const bf16*>(c.v_pool) + heads(blk[i]) * PAGE + d * 16 + h * 8, &Vs[t & 3][at]);
            }
        };
        // The pieces of V that a lane loaded itself, on an edge of the mask, once
        // they have landed: in the tile, or, e4m3, among the codes (r: t % 3),
        // which are the next to be widened, with vsc[0].
        auto settle = [&](int t, int r) {
            const int key0 = it.key0(t);
            if constexpr (Q8) {
                if (t < n_tiles && it.edge(key0)) {
                    wait_vmcnt<4>();
                    asm volatile("" ::: "memory");
                    u32x4 x = codes[1][r][tid];
                    odd |= P::settle_v(64 * wave, lane, x, key0, it.key_end, vsc[0]);
                    codes[1][r][tid] = x;
                }
            } else {
                if (t < n_tiles && it.edge(key0)) {
#pragma unroll
                    for (int i = 0; i < LW; ++i) {
                        const int slab = (wave + 8 * i) % KK, d = slab * 32 + (lane >> 1);
                        u32x4* piece = reinterpret_cast<u32x4*>(&Vs[t & 3][page_of(i) * PAGE + slab * 512 + lane * 8]);
                        u32x4 x = *piece;
                        // as the pieces number them: tokens 8 h .. of dim d is piece 2 d + h of its page
                        odd |= P::settle_v(page_of(i) * P::PP, 2 * d + ((lane & 1) ^ ((d >> 2) & 1)), x, key0,
                                           it.key_end, 1.f);
                        *piece = x;
                    }
                    wait_lgkmcnt0();
                }
            }
        };

        Rows<HD> rows;
        rows.clear();
        f32x4 sc[4][CT];
        bf16x8 pf[2][CT];
        // P2 as a chain of fragment groups: VG groups of four V fragments, then
        // the K fragments of the four score tiles.  Groups are read two ahead
        // of their MFMAs; the first two are read at the end of P1.
        constexpr int VG = 2 * NT / 4, NG = VG + 4;
        bf16x8 fr[3][4];
        static_assert(KK == 4, "a group is four fragments");
        auto read = [&](int t, int r, int s) {
            bf16x8(&f)[4] = fr[s % 3];
            if (s < VG) {
                const int j = s / (NT / 4), n0 = (s % (NT / 4)) * 4, v_base = (2 * j + (grp >> 1)) * PAGE;
                const int buf = Q8 ? r : t & 3;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int d = (n0 + i) * 16 + col;
                    f[i] = *reinterpret_cast<const bf16x8*>(&Vs[buf][v_base + d * 16 + vswz(d, grp & 1) * 8]);
                }
            } else {
                const int p = s - VG, key = pair_key(col, p & 1), tok = key & 15;
                const int base = (2 * (p >> 1) + (key >> 4)) * PAGE + tok * 32 + kswz(tok, grp) * 8;
#pragma unroll
                for (int kk = 0; kk < KK; ++kk)
                    f[kk] = *reinterpret_cast<const bf16x8*>(&Ks[Q8 ? mod3(r + 1) : (t + 1) & 3][base + kk * 512]);
            }
        };
        auto mma = [&](int s) {
            const bf16x8(&f)[4] = fr[s % 3];
            if (s < VG) {
                const int j = s / (NT / 4), n0 = (s % (NT / 4)) * 4;
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct) rows.o[ct][n0 + i] = mfma16(pf[j][ct], f[i], rows.o[ct][n0 + i]);
                if (n0 == 0) {
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct) rows.l[ct] = mfma16(pf[j][ct], ones, rows.l[ct]);
                }
            } else {
                const int p = s - VG;
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) sc[p][ct] = f32x4{};
#pragma unroll
                for (int kk = 0; kk < KK; ++kk)
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct) sc[p][ct] = mfma16(f[kk], qf[ct][kk], sc[p][ct]);
            }
        };
        // Groups first .. NG - 1, of which two are read, with four steps of
        // moving tiles spread between them (r: t % 3).
        u32x4 kx, vx;
        auto products = [&](int t, int r, auto first) {
            constexpr int S0 = decltype(first)::value, N = NG - S0;
            if constexpr (Q8) {  // the codes of V(t + 2) and K(t + 3) have landed, two tiles' loads are younger
                wait_vmcnt<4>();
                asm volatile("" ::: "memory");
            }
#pragma unroll
            for (int s = S0; s < NG; ++s) {
                if (s + 2 < NG) read(t, r, s + 2);
                mma(s);
                if constexpr (Q8) {
                    if (s == S0) {
                        vx = codes[1][mod3(r + 2)][tid];
                        kx = codes[0][r][tid];
                    }
                    if (N / 4 == s - S0) P::put_v(Vs[mod3(r + 2)], 64 * wave, lane, vx, vsc[0]);
                    if (2 * N / 4 == s - S0) P::put_k(Ks[r], 64 * wave, lane, kx, ksc[0]);
                    if (3 * N / 4 == s - S0) {
                        load_v(0, t + 5, mod3(r + 2), ids[1]);
                        load_k(0, t + 6, r, ids[0]);
                    }
                    if (N / 4 == s - S0 || 2 * N / 4 == s - S0) {  // the widening between the MFMAs, not behind them
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);    // 0x8: MFMA
                            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);  // 0x100: LDS reads
                            __builtin_amdgcn_sched_group_barrier(0x2, 3, 0);    // 0x2: VALU
                        }
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
                            __builtin_amdgcn_sched_group_barrier(0x2, 3, 0);
                        }
                    }
                } else {
#pragma unroll
                    for (int l = 0; l < 2 * LW; ++l)
                        if ((2 * l + 1) * N / (4 * LW) == s - S0) {
                            if (l < LW) load_v(l, t + 3, 0, ids[1]);
                            else load_k(l - LW, t + 4, 0, ids[0]);
                        }
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        // Before the first slot: K(0 .. 2), V(0) and V(1) in LDS, of e4m3 the
        // last of each and the next two as codes.  The previous item's buffers
        // are free, and no load is in flight.
        wait_vmcnt<0>();  // Q: the compiler then has no loads of its own pending
        shift(0);
        if constexpr (Q8) {
            int b[5];
#pragma unroll
            for (int t = 0; t < 5; ++t) {
                b[t] = ids[0][0];
                shift(t + 1);
            }
            const int b1[LW] = {b[1]}, b2[LW] = {b[2]}, b3[LW] = {b[3]}, b4[LW] = {b[4]};
            load_v(0, 1, 1, b1);
            load_k(0, 2, 2, b2);
            load_v(0, 2, 2, b2);
            load_k(0, 3, 0, b3);
            load_v(0, 3, 0, b3);
            load_k(0, 4, 1, b4);
            const u32x4 k0 = *reinterpret_cast<const u32x4*>(source(false, b[0]));
            u32x4 v0 = *reinterpret_cast<const u32x4*>(source(true, b[0]));
            const u32x4 k1 = *reinterpret_cast<const u32x4*>(source(false, b[1]));
#pragma unroll
            for (int x = 0; x < 3; ++x) ksc[x] = k_scale(b[2 + x]);
#pragma unroll
            for (int x = 0; x < 4; ++x) vsc[x] = v_scale(b[1 + x]);
            P::put_k(Ks[0], 64 * wave, lane, k0, k_scale(b[0]));
            const float vs0 = v_scale(b[0]);
            if (it.edge(it.key0(0))) odd |= P::settle_v(64 * wave, lane, v0, it.key0(0), it.key_end, vs0);
            P::put_v(Vs[0], 64 * wave, lane, v0, vs0);
            P::put_k(Ks[1], 64 * wave, lane, k1, k_scale(b[1]));
            wait_lgkmcnt0();
        } else {
#pragma unroll
            for (int i = 0; i < LW; ++i) load_k(i, 0, 0, ids[0]);
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                shift(t + 1);
#pragma unroll
                for (int i = 0; i < LW; ++i) {
                    load_v(i, t, 0, ids[1]);
                    load_k(i, t + 1, 0, ids[0]);
                }
            }
            shift(3);
        }
        wait_vmcnt<0>();
        barrier_only();
        if constexpr (Q8) settle(1, 1);
        if (behind) {  // slot 0 of the group behind
            if constexpr (!Q8) settle(0, 0);
            barrier_only();
        }
        read(-1, 2, VG);
        read(-1, 2, VG + 1);
        products(-1, 2, std::integral_constant<int, VG>{});
        if constexpr (!Q8) {
            if (!behind) settle(0, 0);
        }
        if constexpr (Q8) wait_lgkmcnt0();
        barrier_only();
        for (int t = 0, r = 0; t < n_tiles; ++t, r = mod3(r + 1)) {
            // P1
            next(t);
            if constexpr (Q8) settle(t + 2, mod3(r + 2));
            rows.template softmax<GROUP>(sc, pf, it, it.key0(t), sl2, col, grp);
            // all of it before the barrier: the compiler would put the second
            // half's exponentials off to where they are used
#pragma unroll
            for (int j = 0; j < 2; ++j) asm volatile("" ::"v"(pf[j][0]), "v"(pf[j][1]));
            if constexpr (!Q8) {
                if (behind) {  // V(t + 1) and K(t + 2) have landed; those of the tile after may not have
                    wait_vmcnt<2 * LW>();
                    settle(t + 1, 0);
                }
            }
            read(t, r, 0);
            read(t, r, 1);
            barrier_only();
            // P2, ahead of the other wave's softmax at every issue
            __builtin_amdgcn_s_setprio(1);
            products(t, r, std::integral_constant<int, 0>{});
            __builtin_amdgcn_s_setprio(0);
            if constexpr (!Q8) {
                if (!behind) {  // the same slot; two tiles' loads are younger
                    wait_vmcnt<4 * LW>();
                    settle(t + 1, 0);
                }
            }
            if (t + 1 == n_tiles) wait_vmcnt<0>();  // nothing in flight into the next item's buffers
            if constexpr (Q8) wait_lgkmcnt0();
            barrier_only();
        }
        if (!behind) barrier_only();

        if (it.live) rows.template write<GROUP>(c, it, kvh, wave, col, grp);
        if (any_odd(odd, flags)) exact_item<Q8, HD, GROUP>(a, it, kvh, Ks[0], Vs[0], sl2);  // writes its rows anew
        barrier_only();
    }
}

template <bool Q8, int HD, int GROUP>
void launch_g(const CacheAttnArgs& a, hipStream_t s) {
    const int blocks = a.chunk.n_slots * a.chunk.hkv + (a.decode.n_slots * a.decode.hkv + 7) / 8;
    if constexpr (HD == 128) {
        if (a.chunk.pp) {
            cache_chunk_pp_kernel<Q8, GROUP><<<blocks, 512, 0, s>>>(a);
            return;
        }
    }
    cache_chunk_kernel<Q8, HD, GROUP><<<blocks, 512, 0, s>>>(a);
}

template <bool Q8, int HD>
void launch_hd(const CacheAttnArgs& a, hipStream_t s) {
    if (a.chunk.n_items <= 0) {
        if (a.decode.b > 0) cache_decode_kernel<Q8, HD><<<dim3(a.decode.hkv, a.decode.n_slots), 64, 0, s>>>(a);
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
