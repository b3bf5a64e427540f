// Products with weights held in 4 bits: out = a W^T, W[n][k] in e2m1 codes with
// one power-of-two scale (e8m0) for 32 values of a row.
//
// gfx950 turns two codes and their scale into two bf16 values in one
// instruction, exactly (a code has 2 significant bits; scales past bf16's range
// give infinities or subnormals, 255 gives NaN), so the products run on the bf16
// matrix cores with the weights' exact values and fp32 sums: nothing is rounded
// before the output.
//
// Layout (slw_w4_pack).  W's rows are cut into tiles of 16, k into steps of 128;
// a tile's step is 1024 bytes, 16 for each lane of a wave: lane l holds row
// l % 16, the 32 codes of the group l / 16, in the order of the source.  A lane's
// 16 bytes are the weight operands of four 16x16x32 MFMAs (j = 0..3: values 8 j
// .. 8 j + 7 of every group; the activations are read in the same order) and
// share one scale; the scale bytes of four steps make one word for each lane.
// Gated weights have gate tiles and up tiles in turn, so that a wave holds the
// two members of a pair in the same lane.
#include <math.h>

#include <algorithm>

#include "device.h"
#include "hip_try.h"
#include "kernels.h"

namespace slw {
namespace {

struct W4Args {
    const u32x4* codes;      // [tiles][steps][64]
    const uint32_t* scales;  // [tiles][words][64]
    const bf16* a;
    void* out;
    int64_t lda, ldo;
    int m, n, k;             // n: columns of out
    int tiles, steps, words;
    bool vec;                // four columns of out in one store
};

__device__ __forceinline__ float silu(float g) { return g / (1.0f + expf(-g)); }

// The scale 2^(byte i of w - 127) as a float whose exponent bits are the byte.
__device__ __forceinline__ float step_scale(uint32_t w, int i) {
    return __uint_as_float((w >> (8 * i) & 0xFFu) << 23);
}

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ bf16x8 widen(uint32_t codes, float scale) {
    union {
        bf16x2 h[4];
        bf16x8 v;
    } u;
    u.h[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0);
    u.h[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
    u.h[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2);
    u.h[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
    return u.v;
}

// Four columns n0 .. n0 + 3 of one row.
template <class Out>
__device__ __forceinline__ void store_cols(const W4Args& g, int row, int n0, f32x4 v) {
    Out* p = static_cast<Out*>(g.out) + row * g.ldo + n0;
    if (g.vec && n0 + 4 <= g.n) {
        typedef Out Out4 __attribute__((ext_vector_type(4)));
        Out4 o;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = static_cast<Out>(v[e]);
        *reinterpret_cast<Out4*>(p) = o;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (n0 + e < g.n) p[e] = static_cast<Out>(v[e]);
    }
}

// A work-group: NT tiles of weights and 16 MT rows; its waves share the k steps
// and add their sums through LDS.
template <int MT, int NT, bool GATED, class Out>
__global__ __launch_bounds__(512) void w4_stream_kernel(W4Args g) {
    extern __shared__ f32x4 red[];  // [waves][NT * MT][64]
    const int wave = threadIdx.x / kWave, waves = blockDim.x / kWave, lane = threadIdx.x % kWave;
    const int tile0 = blockIdx.x * NT, row0 = blockIdx.y * 16 * MT;
    const int col = lane & 15, grp = lane >> 4;
    const bf16* a[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) a[i] = g.a + min(row0 + 16 * i + col, g.m - 1) * g.lda + 32 * grp;
    f32x4 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[i][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int b = wave; b < g.words; b += waves) {
        uint32_t sc[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t)
            sc[t] = g.scales[(static_cast<size_t>(min(tile0 + t, g.tiles - 1)) * g.words + b) * 64 + lane];
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4) {
            const int step = 4 * b + i4;
            if (step >= g.steps) break;
            u32x4 c[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t)
                c[t] = g.codes[(static_cast<size_t>(min(tile0 + t, g.tiles - 1)) * g.steps + step) * 64 + lane];
            bf16x8 x[MT][4];
            const bool in_k = step * 128 + 32 * grp < g.k;
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    x[i][j] = in_k ? *reinterpret_cast<const bf16x8*>(a[i] + step * 128 + 8 * j) : bf16x8{};
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const float s = step_scale(sc[t], i4);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const bf16x8 w = widen(c[t][j], s);
#pragma unroll
                    for (int i = 0; i < MT; ++i) acc[i][t] = mfma16(w, x[i][j], acc[i][t]);
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int t = 0; t < NT; ++t) red[(wave * MT * NT + i * NT + t) * 64 + lane] = acc[i][t];
    __syncthreads();
    constexpr int kPer = GATED ? 2 : 1;
    for (int u = wave; u < MT * NT / kPer; u += waves) {
        const int i = u / (NT / kPer), t = u % (NT / kPer) * kPer;
        f32x4 v[kPer];
#pragma unroll
        for (int p = 0; p < kPer; ++p) {
            v[p] = f32x4{0.f, 0.f, 0.f, 0.f};
            for (int w = 0; w < waves; ++w) v[p] += red[(w * MT * NT + i * NT + t + p) * 64 + lane];
        }
        f32x4 o = v[0];
        if (GATED)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = silu(v[0][e]) * v[kPer - 1][e];
        const int row = row0 + 16 * i + col, n0 = (tile0 + t) / kPer * 16 + 4 * grp;
        if (row < g.m) store_cols<Out>(g, row, n0, o);
    }
}

// One thread for each lane of each tile's step: 16 bytes of codes; the first
// step of four also makes the lane's scale word.
__global__ __launch_bounds__(256) void w4_pack_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                      u32x4* __restrict__ to_codes, uint32_t* __restrict__ to_scales,
                                                      int rows, int k, int tiles, int steps, int words, bool gated) {
    const size_t i = blockIdx.x * static_cast<size_t>(256) + threadIdx.x;
    const int lane = i % 64, step = i / 64 % steps;
    const size_t tile = i / 64 / steps;
    if (tile >= static_cast<size_t>(tiles)) return;
    const int r = (gated ? tile / 2 : tile) * 16 + (lane & 15);  // of the gate or up rows, or of all
    const int groups = k / 32;
    const size_t row = gated && tile % 2 ? static_cast<size_t>(rows) + r : r;
    const int group = step * 4 + lane / 16;
    u32x4 c = {0u, 0u, 0u, 0u};
    if (r < rows && group < groups) c = *reinterpret_cast<const u32x4*>(codes + row * (k / 2) + group * 16);
    to_codes[(tile * steps + step) * 64 + lane] = c;
    if (step % 4) return;
    uint32_t w = 0;
    for (int j = 0; j < 4; ++j)
        if (r < rows && group + 4 * j < groups) w |= static_cast<uint32_t>(scales[row * groups + group + 4 * j]) << (8 * j);
    to_scales[(tile * words + step / 4) * 64 + lane] = w;
}

struct W4Shape {
    int tiles, steps, words;
    size_t code_bytes, bytes;
};
W4Shape w4_shape(int n, int k, bool gated) {
    W4Shape s;
    s.tiles = static_cast<int>(gated ? 2 * ceil_div(n / 2, 16) : ceil_div(n, 16));
    s.steps = static_cast<int>(ceil_div(k, 128));
    s.words = static_cast<int>(ceil_div(s.steps, 4));
    s.code_bytes = static_cast<size_t>(s.tiles) * s.steps * 1024;
    s.bytes = s.code_bytes + static_cast<size_t>(s.tiles) * s.words * 256;
    return s;
}

template <int MT, int NT, bool GATED, class Out>
void stream_launch(const W4Args& g, int waves, hipStream_t s) {
    const dim3 grid(static_cast<unsigned>(ceil_div(g.tiles, NT)), static_cast<unsigned>(ceil_div(g.m, 16 * MT)));
    w4_stream_kernel<MT, NT, GATED, Out><<<grid, 64 * waves, static_cast<size_t>(waves) * MT * NT * 1024, s>>>(g);
}

template <bool GATED, class Out>
void stream_by_rows(const W4Args& g, hipStream_t s) {
    const int waves = std::min(8, g.words);
    if (g.m <= 16) stream_launch<1, 2, GATED, Out>(g, waves, s);
    else if (g.m <= 32) stream_launch<2, 2, GATED, Out>(g, waves, s);
    else stream_launch<4, 2, GATED, Out>(g, waves, s);
}

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

int check_w4(int32_t n, int32_t k, int32_t gated) {
    if (gated != 0 && gated != 1) return fail(SLW_EINVAL, "gated must be 0 or 1");
    if (n < 1 || n > SLW_W4_MAX_N || (gated && n % 2))
        return fail(SLW_EUNSUPPORTED, "n must be in [1, %d], and even for gated weights (got %d)", SLW_W4_MAX_N, n);
    if (k < 32 || k % 32 || k > SLW_W4_MAX_K)
        return fail(SLW_EUNSUPPORTED, "k must be a multiple of 32 in [32, %d] (got %d)", SLW_W4_MAX_K, k);
    return SLW_OK;
}

}  // namespace
}  // namespace slw

using namespace slw;

extern "C" int slw_w4_packed_bytes(int32_t n, int32_t k, int32_t gated, size_t* bytes) {
    return guarded([&] {
        if (!bytes) return fail(SLW_EINVAL, "null argument");
        int rc = check_w4(n, k, gated);
        if (rc) return rc;
        *bytes = w4_shape(n, k, gated).bytes;
        return SLW_OK;
    });
}

extern "C" int slw_w4_pack(const void* codes, const void* scales, int32_t n, int32_t k, int32_t gated, void* packed,
                           void* stream) {
    return guarded([&] {
        int rc = check_w4(n, k, gated);
        if (rc) return rc;
        if (!codes || !scales || !packed) return fail(SLW_EINVAL, "null argument");
        if (!aligned16(codes) || !aligned16(packed)) return fail(SLW_EINVAL, "codes and packed weights must be 16-byte aligned");
        const W4Shape w = w4_shape(n, k, gated);
        const size_t threads = w.code_bytes / 16;
        w4_pack_kernel<<<static_cast<unsigned>((threads + 255) / 256), 256, 0, static_cast<hipStream_t>(stream)>>>(
            static_cast<const uint8_t*>(codes), static_cast<const uint8_t*>(scales), static_cast<u32x4*>(packed),
            reinterpret_cast<uint32_t*>(static_cast<char*>(packed) + w.code_bytes), gated ? n / 2 : n, k, w.tiles, w.steps,
            w.words, gated != 0);
        HIP_TRY(hipGetLastError());
        return SLW_OK;
    });
}

extern "C" int slw_w4_workspace_size(int32_t n, int32_t k, int32_t gated, int32_t max_m, size_t* bytes) {
    return guarded([&] {
        if (!bytes) return fail(SLW_EINVAL, "null argument");
        int rc = check_w4(n, k, gated);
        if (rc) return rc;
        if (max_m < 0) return fail(SLW_EINVAL, "negative rows");
        *bytes = 0;
        return SLW_OK;
    });
}

extern "C" int slw_w4_product(const slw_w4* w, const void* a, int64_t lda, int32_t m, void* out, int64_t ldo,
                              int32_t out_f32, void* ws, size_t ws_bytes, void* stream) {
    return guarded([&] {
        if (!w) return fail(SLW_EINVAL, "null argument");
        int rc = check_w4(w->n, w->k, w->gated);
        if (rc) return rc;
        if (m < 0) return fail(SLW_EINVAL, "negative rows");
        if (m > SLW_W4_MAX_M) return fail(SLW_EUNSUPPORTED, "more than %d rows", SLW_W4_MAX_M);
        if (out_f32 != 0 && out_f32 != 1) return fail(SLW_EINVAL, "out_f32 must be 0 or 1");
        if (m == 0) return SLW_OK;
        const int n_out = w->gated ? w->n / 2 : w->n;
        if (!w->packed || !a || !out) return fail(SLW_EINVAL, "null argument");
        if (!aligned16(w->packed) || !aligned16(a) || lda % 8 || lda < w->k)
            return fail(SLW_EINVAL, "packed weights and rows: 16-byte aligned, stride a multiple of 8 and at least %d (got %lld)",
                        w->k, (long long)lda);
        if (ldo < n_out || reinterpret_cast<uintptr_t>(out) % (out_f32 ? 4 : 2))
            return fail(SLW_EINVAL, "out: aligned to its type, stride at least %d (got %lld)", n_out, (long long)ldo);
        const W4Shape sh = w4_shape(w->n, w->k, w->gated);
        W4Args g{};
        g.codes = static_cast<const u32x4*>(w->packed);
        g.scales = reinterpret_cast<const uint32_t*>(static_cast<const char*>(w->packed) + sh.code_bytes);
        g.a = static_cast<const bf16*>(a);
        g.out = out;
        g.lda = lda;
        g.ldo = ldo;
        g.m = m;
        g.n = n_out;
        g.k = w->k;
        g.tiles = sh.tiles;
        g.steps = sh.steps;
        g.words = sh.words;
        g.vec = ldo % 4 == 0 && reinterpret_cast<uintptr_t>(out) % (out_f32 ? 16 : 8) == 0;
        hipStream_t s = static_cast<hipStream_t>(stream);
        if (w->gated) out_f32 ? stream_by_rows<true, float>(g, s) : stream_by_rows<true, bf16>(g, s);
        else out_f32 ? stream_by_rows<false, float>(g, s) : stream_by_rows<false, bf16>(g, s);
        HIP_TRY(hipGetLastError());
        return SLW_OK;
    });
}
