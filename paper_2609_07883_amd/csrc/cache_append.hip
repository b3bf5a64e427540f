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
// registers.
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

// Code of one bf16 value.  At e = 120 a code of 256 would stand for 2^128,
// which is no finite float: the largest there is 240.
__device__ __forceinline__ uint32_t quantise(uint32_t b, float inv, float lim) {
    const float x = fminf(fmaxf(__uint_as_float(b << 16) * inv, -lim), lim);
    const uint32_t c = static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(x, 0.f, 0, false)) & 0xFFu;
    return not_finite(b) ? 0x7Fu : c;
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

__device__ __forceinline__ uint32_t wave_umax(uint32_t v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = max(v, static_cast<uint32_t>(__shfl_xor(static_cast<int>(v), o, kWave)));
    return v;
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
    u32x4 x[S][2] = {}, held[S] = {};
    const uint16_t* row = static_cast<const uint16_t*>(a.k) + static_cast<size_t>(it.row0 + t - it.t0) * a.ld + kvh * HD;
#pragma unroll
    for (int s = 0; s < S; ++s) {
        if (fresh) {
            x[s][0] = *reinterpret_cast<const u32x4*>(row + 64 * s + 16 * c);
            x[s][1] = *reinterpret_cast<const u32x4*>(row + 64 * s + 16 * c + 8);
        }
        if (older) held[s] = *reinterpret_cast<const u32x4*>(page + s * 256 + lane * 4);
    }
    uint32_t amax = 0;
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int w = 0; w < 4; ++w)
                amax = max(amax, max(magnitude(x[s][h][w] & 0xFFFFu), magnitude(x[s][h][w] >> 16)));
    int e = block_exp(wave_umax(amax)), e_old = kMinExp;
    if (it.t0 > 0) {
        e_old = scale_exp(a.cache.k_scale[bh]);
        e = max(e, e_old);
    }
    const float inv = pow2(-e), lim = e >= kMaxExp ? 240.f : 448.f, f = pow2(max(e_old - e, -126));
#pragma unroll
    for (int s = 0; s < S; ++s) {
        u32x4 out;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const uint32_t p = x[s][w >> 1][(w & 1) * 2], q = x[s][w >> 1][(w & 1) * 2 + 1];
            out[w] = quantise(p & 0xFFFFu, inv, lim) | quantise(p >> 16, inv, lim) << 8 |
                     quantise(q & 0xFFFFu, inv, lim) << 16 | quantise(q >> 16, inv, lim) << 24;
            if (older) out[w] = requantise4(held[s][w], f);
        }
        if (fresh || (older && e > e_old)) *reinterpret_cast<u32x4*>(page + s * 256 + lane * 4) = out;
    }
    if (lane == 0) a.cache.k_scale[bh] = pow2(e);
}

template <int HD>
__device__ __forceinline__ void append_v8(const AppendArgs& a, const Item& it, int kvh, int lane) {
    constexpr int D = HD / 64;  // dims of a lane
    const size_t bh = static_cast<size_t>(it.blk) * a.cache.hkv + kvh;
    u32x4* page = reinterpret_cast<u32x4*>(static_cast<uint8_t*>(a.cache.v_pool) + bh * HD * 16) + lane * D;
    u32x4 held[D] = {};
    if (it.n < 16) {
#pragma unroll
        for (int d = 0; d < D; ++d) held[d] = page[d];
    }
    uint32_t x[16][D], amax = 0;
#pragma unroll
    for (int t = 0; t < 16; ++t) {
#pragma unroll
        for (int d = 0; d < D; ++d) x[t][d] = 0;
        if (t >= it.t0 && t < it.t0 + it.n) {
            const uint16_t* row = static_cast<const uint16_t*>(a.v) + static_cast<size_t>(it.row0 + t - it.t0) * a.ld + kvh * HD;
            if constexpr (D == 2) {
                const uint32_t b = reinterpret_cast<const uint32_t*>(row)[lane];
                x[t][0] = b & 0xFFFFu;
                x[t][1] = b >> 16;
            } else {
                x[t][0] = row[lane];
            }
        }
    }
#pragma unroll
    for (int t = 0; t < 16; ++t)
#pragma unroll
        for (int d = 0; d < D; ++d) amax = max(amax, magnitude(x[t][d]));
    int e = block_exp(wave_umax(amax)), e_old = kMinExp;
    if (it.t0 > 0) {
        e_old = scale_exp(a.cache.v_scale[bh]);
        e = max(e, e_old);
    }
    const float inv = pow2(-e), lim = e >= kMaxExp ? 240.f : 448.f, f = pow2(max(e_old - e, -126));
#pragma unroll
    for (int d = 0; d < D; ++d) {
        u32x4 out;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            uint32_t word = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int t = 4 * w + i;
                const uint32_t c = (held[d][w] >> (8 * i)) & 0xFFu;
                const uint32_t v = t < it.t0 ? (e > e_old ? requantise(c, f) : c)
                                   : t < it.t0 + it.n ? quantise(x[t][d], inv, lim) : c;
                word |= v << (8 * i);
            }
            out[w] = word;
        }
        page[d] = out;
    }
    if (lane == 0) a.cache.v_scale[bh] = pow2(e);
}

template <int HD>
__device__ __forceinline__ void append_k16(const AppendArgs& a, const Item& it, int kvh, int lane) {
    const int t = lane >> 2, c = lane & 3;
    if (t < it.t0 || t >= it.t0 + it.n) return;
    uint16_t* page = static_cast<uint16_t*>(a.cache.k_pool) + (static_cast<size_t>(it.blk) * a.cache.hkv + kvh) * HD * 16;
    const uint16_t* row = static_cast<const uint16_t*>(a.k) + static_cast<size_t>(it.row0 + t - it.t0) * a.ld + kvh * HD;
#pragma unroll
    for (int s = 0; s < HD / 32; ++s)
        *reinterpret_cast<u32x4*>(page + s * 512 + lane * 8) = *reinterpret_cast<const u32x4*>(row + 32 * s + 8 * c);
}

template <int HD>
__device__ __forceinline__ void append_v16(const AppendArgs& a, const Item& it, int kvh, int lane) {
    uint16_t* page = static_cast<uint16_t*>(a.cache.v_pool) + (static_cast<size_t>(it.blk) * a.cache.hkv + kvh) * HD * 16;
    const uint16_t* v = static_cast<const uint16_t*>(a.v) + static_cast<size_t>(it.row0) * a.ld + kvh * HD;
#pragma unroll
    for (int d = lane; d < HD; d += kWave) {
        if (it.n == 16) {
            u32x4 out[2];
#pragma unroll
            for (int w = 0; w < 8; ++w)
                out[w >> 2][w & 3] = v[static_cast<size_t>(2 * w) * a.ld + d] |
                                     static_cast<uint32_t>(v[static_cast<size_t>(2 * w + 1) * a.ld + d]) << 16;
            *reinterpret_cast<u32x4*>(page + d * 16) = out[0];
            *reinterpret_cast<u32x4*>(page + d * 16 + 8) = out[1];
        } else {
            for (int j = 0; j < it.n; ++j) page[d * 16 + it.t0 + j] = v[static_cast<size_t>(j) * a.ld + d];
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
