// Append of K/V rows to the paged cache, in e4m3 or in bf16.
//
// The e4m3 cache keeps one scale 2^e per (block of 16 tokens, kv head) of K
// and of V.  Powers of two, because a block fills token by token: when a later
// token raises e, the codes of the tokens before it are rounded again, and
// between powers of two that loses nothing but values that become subnormal,
// where a ratio of arbitrary scales would round every code anew each time.
//   e_new = max(-100, least e with max |x| <= 448 2^e over the new finite x)
//   e     = e_new for a block's first token, else max(e_new, the block's e)
//   code  = x 2^-e to nearest even e4m3; NaN where x is not finite
// The products with 2^-e are exact in fp32 (or far below the smallest code), so
// each code is rounded once.  -100 keeps 2^e times every code a normal bf16.
//
// Bound by HBM: a row is read once (2 hkv hd bf16) and its codes are written
// once.  One wave per (block, kv head, K or V): K pages are token-major, so a
// lane takes 16 dims of one token from the row to the page; V pages are
// dim-major, so a lane takes its dims of all 16 tokens, which transposes in
// registers.  8B heads: 4096 rows 6.6 to 7.5 us (25 MB, 3.4 to 3.8 TB/s); one
// token of each of 256 sequences 5.7 us, start and latency, for 5.6 MB.  In bf16
// 4096 rows take 10.8 us (34 MB, 3.1 TB/s; 6.5 at a large copy's rate) and 1500
// rows 5.6 to 6.4 (12.4 MB; 2.4), of which a launch with one token takes 2 to 3.
#include "device.h"
#include "kernels.h"

namespace slw {
namespace {

constexpr int kMinExp = -100, kMaxExp = 120;
constexpr int kAppendWaves = 4;

__device__ __forceinline__ bool not_finite(uint32_t b) { return (b & 0x7F80u) == 0x7F80u; }  // of bf16 bits
__device__ __forceinline__ float pow2(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }

// |x| as bf16 bits, 0 where x is not finite: ordered as the magnitudes are.
__device__ __forceinline__ uint32_t magnitude(uint32_t b) { return not_finite(b) ? 0u : b & 0x7FFFu; }
// Least e >= kMinExp with amax <= 448 2^e (448 = 1.75 * 2^8; mantissa 0x60 is 1.75).
__device__ __forceinline__ int block_exp(uint32_t amax) {
    return max(kMinExp, static_cast<int>(amax >> 7) - 135 + ((amax & 0x7Fu) > 0x60u ? 1 : 0));
}
__device__ __forceinline__ int scale_exp(float s) {
    return min(max(static_cast<int>((__float_as_uint(s) >> 23) & 0xFFu) - 127, kMinExp), kMaxExp);
}

// Codes of two bf16 values (a word's low and high half) in the low half of the
// result, the other half kept from `keep`, or in the high half.  Nothing to
// clamp: |x| 2^-e <= 448.
template <bool HIGH>
__device__ __forceinline__ uint32_t quantise2(uint32_t w, float inv, uint32_t keep) {
    return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(__uint_as_float(w << 16) * inv,
                                                                 __uint_as_float(w & 0xFFFF0000u) * inv,
                                                                 static_cast<int>(keep), HIGH));
}
__device__ __forceinline__ uint32_t quantise4(uint32_t w0, uint32_t w1, float inv) {
    return quantise2<true>(w1, inv, quantise2<false>(w0, inv, 0u));
}
// Any value, where some are not finite or e is kMaxExp: there a code of 256
// would stand for 2^128, which is no finite float, and the largest is 240.
__device__ __forceinline__ uint32_t quantise_any(uint32_t b, float inv, float lim) {
    const float x = fminf(fmaxf(__uint_as_float(b << 16) * inv, -lim), lim);
    const uint32_t c = static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(x, 0.f, 0, false)) & 0xFFu;
    return not_finite(b) ? 0x7Fu : c;
}
__device__ __forceinline__ uint32_t quantise4_any(uint32_t w0, uint32_t w1, float inv, float lim) {
    return quantise_any(w0 & 0xFFFFu, inv, lim) | quantise_any(w0 >> 16, inv, lim) << 8 |
           quantise_any(w1 & 0xFFFFu, inv, lim) << 16 | quantise_any(w1 >> 16, inv, lim) << 24;
}
// Code at a scale 1 / f times as large (f <= 1).
__device__ __forceinline__ uint32_t requantise(uint32_t c, float f) {
    const float x = __builtin_amdgcn_cvt_f32_fp8(static_cast<int>(c), 0) * f;
    const uint32_t r = static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(x, 0.f, 0, false)) & 0xFFu;
    return (c & 0x7Fu) == 0x7Fu ? 0x7Fu : r;
}
__device__ __forceinline__ uint32_t requantise4(uint32_t c, float f) {
    return requantise(c & 0xFFu, f) | requantise((c >> 8) & 0xFFu, f) << 8 | requantise((c >> 16) & 0xFFu, f) << 16 |
           requantise(c >> 24, f) << 24;
}

// Largest value of the wave, in every lane: rotations within the rows of 16
// lanes, then row swaps.
__device__ __forceinline__ uint32_t wave_umax(uint32_t v) {
    v = max(v, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0x128, 0xF, 0xF, false)));  // row_ror:8
    v = max(v, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0x124, 0xF, 0xF, false)));
    v = max(v, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0x122, 0xF, 0xF, false)));
    v = max(v, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0x121, 0xF, 0xF, false)));
    const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = max(a[0], a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return max(b[0], b[1]);
}

// Largest magnitude of the wave's words of two bf16 values.  Magnitudes that
// are not finite lie above all finite ones, so one pass tells whether there
// are any (`odd`), and only then a second one leaves them out.
template <int N>
__device__ __forceinline__ uint32_t block_max(const uint32_t (&w)[N], bool& odd) {
    uint32_t hi = 0, lo = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        hi = max(hi, w[i] & 0x7FFF0000u);
        lo = max(lo, w[i] & 0x7FFFu);
    }
    uint32_t m = wave_umax(max(hi >> 16, lo));
    odd = m >= 0x7F80u;
    if (odd) {
        m = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) m = max(m, max(magnitude(w[i] & 0xFFFFu), magnitude(w[i] >> 16)));
        m = wave_umax(m);
    }
    return m;
}

struct Item {
    int blk, t0, n, row0;
};

template <int HD>
__device__ __forceinline__ void append_k8(const AppendArgs& a, const Item& it, int kvh, int lane) {
    constexpr int S = HD / 64;
    const int t = lane >> 2, c = lane & 3;
    const bool fresh = t >= it.t0 && t < it.t0 + it.n, older = t < it.t0;
    const size_t bh = static_cast<size_t>(it.blk) * a.cache.hkv + kvh;
    uint32_t* page = reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(a.cache.k_pool) + bh * HD * 16);
    const float s_old = a.cache.k_scale[bh];
    alignas(16) uint32_t x[S * 8] = {};
    const uint16_t* row = static_cast<const uint16_t*>(a.k) + static_cast<size_t>(it.row0 + t - it.t0) * a.ld + kvh * HD;
    if (fresh) {
#pragma unroll
        for (int s = 0; s < S; ++s) {
            *reinterpret_cast<u32x4*>(x + 8 * s) = *reinterpret_cast<const u32x4*>(row + 64 * s + 16 * c);
            *reinterpret_cast<u32x4*>(x + 8 * s + 4) = *reinterpret_cast<const u32x4*>(row + 64 * s + 16 * c + 8);
        }
    }
    bool odd;
    int e = block_exp(block_max(x, odd));
    const int e_old = it.t0 > 0 ? scale_exp(s_old) : kMinExp;
    e = max(e, e_old);
    const float inv = pow2(-e);
    if (odd || e >= kMaxExp) {
        const float lim = e >= kMaxExp ? 240.f : 448.f;
        if (fresh) {
#pragma unroll
            for (int s = 0; s < S; ++s) {
                u32x4 out;
#pragma unroll
                for (int w = 0; w < 4; ++w) out[w] = quantise4_any(x[8 * s + 2 * w], x[8 * s + 2 * w + 1], inv, lim);
                *reinterpret_cast<u32x4*>(page + s * 256 + lane * 4) = out;
            }
        }
    } else if (fresh) {
#pragma unroll
        for (int s = 0; s < S; ++s) {
            u32x4 out;
#pragma unroll
            for (int w = 0; w < 4; ++w) out[w] = quantise4(x[8 * s + 2 * w], x[8 * s + 2 * w + 1], inv);
            *reinterpret_cast<u32x4*>(page + s * 256 + lane * 4) = out;
        }
    }
    if (e > e_old && older) {
        const float f = pow2(max(e_old - e, -126));
#pragma unroll
        for (int s = 0; s < S; ++s) {
            u32x4 held = *reinterpret_cast<const u32x4*>(page + s * 256 + lane * 4);
#pragma unroll
            for (int w = 0; w < 4; ++w) held[w] = requantise4(held[w], f);
            *reinterpret_cast<u32x4*>(page + s * 256 + lane * 4) = held;
        }
    }
    if (lane == 0) a.cache.k_scale[bh] = pow2(e);
}

// A lane's dims of an item's rows: w[t / 2 * D + d] holds dim d of tokens t
// (low half) and t + 1, counted from the block's first; 0 where there is no row.
template <int D>
__device__ __forceinline__ void load_dims(uint32_t (&w)[8 * D], const void* rows, const AppendArgs& a, const Item& it,
                                          int kvh, int lane) {
    const uint16_t* first = static_cast<const uint16_t*>(rows) + static_cast<size_t>(it.row0) * a.ld + kvh * (64 * D);
    uint32_t x[16] = {};
#pragma unroll
    for (int t = 0; t < 16; ++t) {
        if (t >= it.t0 && t < it.t0 + it.n) {
            const uint16_t* row = first + static_cast<size_t>(t - it.t0) * a.ld;
            x[t] = D == 2 ? reinterpret_cast<const uint32_t*>(row)[lane] : row[lane];
        }
    }
#pragma unroll
    for (int p = 0; p < 8; ++p) {
        w[p * D] = (x[2 * p] & 0xFFFFu) | x[2 * p + 1] << 16;
        if constexpr (D == 2) w[p * D + 1] = (x[2 * p] >> 16) | (x[2 * p + 1] & 0xFFFF0000u);
    }
}

// Mask of the bytes of word w that are tokens t0 .. t0 + n - 1.
__device__ __forceinline__ uint32_t token_bytes(int w, const Item& it) {
    const uint32_t live = ((1u << (it.t0 + it.n)) - (1u << it.t0)) >> (4 * w) & 0xFu;
    return ((live * 0x00204081u) & 0x01010101u) * 0xFFu;
}

template <int HD>
__device__ __forceinline__ void append_v8(const AppendArgs& a, const Item& it, int kvh, int lane) {
    constexpr int D = HD / 64;  // dims of a lane
    const size_t bh = static_cast<size_t>(it.blk) * a.cache.hkv + kvh;
    u32x4* page = reinterpret_cast<u32x4*>(static_cast<uint8_t*>(a.cache.v_pool) + bh * HD * 16) + lane * D;
    uint32_t zero = 0;
    asm volatile("" : "+v"(zero));  // a vector load, issued here: a scalar one is put off to its use (+0.2 us)
    const float s_old = a.cache.v_scale[bh + zero];
    u32x4 held[D] = {};
    if (it.n < 16) {
#pragma unroll
        for (int d = 0; d < D; ++d) held[d] = page[d];
    }
    uint32_t x[8 * D];
    load_dims<D>(x, a.v, a, it, kvh, lane);
    bool odd;
    int e = block_exp(block_max(x, odd));
    const int e_old = it.t0 > 0 ? scale_exp(s_old) : kMinExp;
    e = max(e, e_old);
    const float inv = pow2(-e);
    u32x4 out[D];
    if (odd || e >= kMaxExp) {
        const float lim = e >= kMaxExp ? 240.f : 448.f;
#pragma unroll
        for (int d = 0; d < D; ++d)
#pragma unroll
            for (int w = 0; w < 4; ++w) out[d][w] = quantise4_any(x[2 * w * D + d], x[(2 * w + 1) * D + d], inv, lim);
    } else {
#pragma unroll
        for (int d = 0; d < D; ++d)
#pragma unroll
            for (int w = 0; w < 4; ++w) out[d][w] = quantise4(x[2 * w * D + d], x[(2 * w + 1) * D + d], inv);
    }
    if (it.n < 16) {
        if (e > e_old && it.t0 > 0) {
            const float f = pow2(max(e_old - e, -126));
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const uint32_t before = token_bytes(w, Item{0, 0, it.t0, 0});
#pragma unroll
                for (int d = 0; d < D; ++d) held[d][w] = (requantise4(held[d][w], f) & before) | (held[d][w] & ~before);
            }
        }
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const uint32_t m = token_bytes(w, it);
#pragma unroll
            for (int d = 0; d < D; ++d) out[d][w] = (out[d][w] & m) | (held[d][w] & ~m);
        }
    }
#pragma unroll
    for (int d = 0; d < D; ++d) page[d] = out[d];
    if (lane == 0) a.cache.v_scale[bh] = pow2(e);
}

template <int HD>
__device__ __forceinline__ void append_k16(const AppendArgs& a, const Item& it, int kvh, int lane) {
    const int t = lane >> 2, c = lane & 3;
    if (t < it.t0 || t >= it.t0 + it.n) return;
    uint16_t* page = static_cast<uint16_t*>(a.cache.k_pool) + (static_cast<size_t>(it.blk) * a.cache.hkv + kvh) * HD * 16;
    const uint16_t* row = static_cast<const uint16_t*>(a.k) + static_cast<size_t>(it.row0 + t - it.t0) * a.ld + kvh * HD;
    u32x4 x[HD / 32];
#pragma unroll
    for (int s = 0; s < HD / 32; ++s) x[s] = *reinterpret_cast<const u32x4*>(row + 32 * s + 8 * c);
#pragma unroll
    for (int s = 0; s < HD / 32; ++s) *reinterpret_cast<u32x4*>(page + s * 512 + lane * 8) = x[s];
}

template <int HD>
__device__ __forceinline__ void append_v16(const AppendArgs& a, const Item& it, int kvh, int lane) {
    constexpr int D = HD / 64;
    uint16_t* page = static_cast<uint16_t*>(a.cache.v_pool) + (static_cast<size_t>(it.blk) * a.cache.hkv + kvh) * HD * 16 +
                     lane * D * 16;
    uint32_t x[8 * D];
    load_dims<D>(x, a.v, a, it, kvh, lane);
#pragma unroll
    for (int d = 0; d < D; ++d) {
        if (it.n == 1) {  // a decode's token
#pragma unroll
            for (int t = 0; t < 16; ++t)
                if (t == it.t0) page[d * 16 + t] = static_cast<uint16_t>(x[t / 2 * D + d] >> (16 * (t & 1)));
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                u32x4* piece = reinterpret_cast<u32x4*>(page + d * 16 + 8 * h);
                u32x4 held = {}, out;
                if (it.n < 16) held = *piece;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const uint32_t live = (((1u << (it.t0 + it.n)) - (1u << it.t0)) >> (8 * h + 2 * w)) & 3u;
                    const uint32_t m = (live & 1u ? 0xFFFFu : 0u) | (live & 2u ? 0xFFFF0000u : 0u);
                    out[w] = (x[(4 * h + w) * D + d] & m) | (held[w] & ~m);
                }
                *piece = out;
            }
        }
    }
}

template <bool Q8, int HD>
__global__ __launch_bounds__(kAppendWaves * kWave) void cache_append_kernel(AppendArgs a) {
    const int w = static_cast<int>(blockIdx.x) * kAppendWaves + __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
    const int lane = threadIdx.x & 63, per = 2 * a.cache.hkv;
    const int i = w / per, r = w % per;
    if (i >= a.n_items) return;
    const Item it{a.items[i], a.items[a.n_items + i], a.items[2 * a.n_items + i], a.items[3 * a.n_items + i]};
    const bool is_v = r >= a.cache.hkv;
    const int kvh = is_v ? r - a.cache.hkv : r;
    if constexpr (Q8) {
        if (is_v) append_v8<HD>(a, it, kvh, lane);
        else append_k8<HD>(a, it, kvh, lane);
    } else {
        if (is_v) append_v16<HD>(a, it, kvh, lane);
        else append_k16<HD>(a, it, kvh, lane);
    }
}

}  // namespace

void launch_cache_append(const AppendArgs& a, hipStream_t s) {
    if (a.n_items <= 0) return;
    const int64_t waves = static_cast<int64_t>(a.n_items) * 2 * a.cache.hkv;
    const unsigned blocks = static_cast<unsigned>((waves + kAppendWaves - 1) / kAppendWaves);
    const bool q8 = a.cache.k_scale != nullptr;
    if (a.cache.hd == 128) {
        if (q8) cache_append_kernel<true, 128><<<blocks, kAppendWaves * kWave, 0, s>>>(a);
        else cache_append_kernel<false, 128><<<blocks, kAppendWaves * kWave, 0, s>>>(a);
    } else {
        if (q8) cache_append_kernel<true, 64><<<blocks, kAppendWaves * kWave, 0, s>>>(a);
        else cache_append_kernel<false, 64><<<blocks, kAppendWaves * kWave, 0, s>>>(a);
    }
}

}  // namespace slw
