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
// a tile's step is 1024 bytes, 16 for each lane of a wave, the weight operands of
// four 16x16x32 MFMAs: word j of lane l holds row l % 16, values 8 (l / 16) .. + 7
// of the step's group j.  So an MFMA takes one group of 32, whose scale is one
// for the row, and the activations' operands are 64 consecutive bytes of a row.
// The four scale bytes of a row's step make a word, the words of four steps 16
// consecutive bytes.  Gated weights have gate tiles and up tiles in turn, so that a
// wave holds the two members of a pair in the same lane.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "device.h"
#include "hip_try.h"
#include "kernels.h"

namespace slw {
namespace {

constexpr int64_t kMostTileStride = 1 << 22;  // the tile and ring kernels' row offsets are 32 bits
constexpr int kMostSplitRows = 4096;  // k is split for fewer rows only
constexpr int kStep = 128;   // k of a step: a lane's 16 bytes of four groups

struct W4Args {
    const u32x4* codes;      // [tiles][steps][64]
    const uint32_t* scales;  // [tiles][words][16][4]: row, step of four
    const bf16* a;
    void* out;
    int64_t lda, ldo;
    int m, n, k;             // n: columns of out
    int tiles, steps, words;
    bool vec;                // four columns of out in one store
    bool gated, f32;
    float* part;             // tile kernel with its k split: [splits][m][16 tiles] sums
    int splits;
};

__device__ __forceinline__ float silu(float g) { return g / (1.0f + expf(-g)); }

// The scale 2^(byte j of w - 127) as a float whose exponent bits are the byte.
__device__ __forceinline__ float group_scale(uint32_t w, int j) { return __uint_as_float((w >> (8 * j) & 0xFFu) << 23); }

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

// The outputs of one row in the lane of a wave: NB tiles' sums, from tile `tile` on.
template <int NB>
__device__ __forceinline__ void store_row(const W4Args& g, int row, int tile, int grp, const f32x4 (&v)[NB]) {
    if (NB > 1 && g.gated) {
#pragma unroll
        for (int t = 0; t + 1 < NB; t += 2) {
            f32x4 o;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = silu(v[t][e]) * v[t + 1][e];
            const int n0 = (tile + t) / 2 * 16 + 4 * grp;
            if (g.f32) store_cols<float>(g, row, n0, o);
            else store_cols<bf16>(g, row, n0, o);
        }
    } else {
#pragma unroll
        for (int t = 0; t < NB; ++t) {
            const int n0 = (tile + t) * 16 + 4 * grp;
            if (g.f32) store_cols<float>(g, row, n0, v[t]);
            else store_cols<bf16>(g, row, n0, v[t]);
        }
    }
}

// The same, or where k is split over work-groups this one's sums, [split][m][16 tiles].
template <int NB>
__device__ __forceinline__ void store_sums(const W4Args& g, int row, int tile, int grp, const f32x4 (&v)[NB]) {
    if (g.splits == 1) {
        store_row<NB>(g, row, tile, grp, v);
        return;
    }
    float* p = g.part + (static_cast<size_t>(blockIdx.z) * g.m + row) * (16 * static_cast<size_t>(g.tiles)) + 4 * grp;
#pragma unroll
    for (int t = 0; t < NB; ++t)
        if (tile + t < g.tiles) *reinterpret_cast<f32x4*>(p + (tile + t) * 16) = v[t];
}

// Words of N consecutive steps (of four that are loaded together).
template <int N>
struct Words {
    uint32_t w[N];
    __device__ __forceinline__ void load(const uint32_t* p) {
        if constexpr (N == 4) {
            const u32x4 v = *reinterpret_cast<const u32x4*>(p);
            w[0] = v[0], w[1] = v[1], w[2] = v[2], w[3] = v[3];
        } else if constexpr (N == 2) {
            const u32x2 v = *reinterpret_cast<const u32x2*>(p);
            w[0] = v[0], w[1] = v[1];
        } else {
            w[0] = *p;
        }
    }
};

// Stream kernel, for a few rows: a work-group has NT tiles of weights and 16 MT
// rows, its waves share the k steps and add their sums through LDS; k may be
// split over work-groups too.  A wave takes D steps at a time, 4 KB of codes,
// which it loads a turn ahead; the rows' operands come straight from the caches.
// The weights' bytes bound it: 1 row of 4096 -> 28672 (62 MB) takes 15.4 us from HBM, 12.8
// where the last-level cache has them (12.2 at a copy's 5.1 TB/s); of 4096 -> 4096 4.0, which
// is a launch, one load's latency and the join in LDS.
template <int MT, int NT, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void w4_stream_kernel(W4Args g) {
    constexpr int D = 4 / NT;
    extern __shared__ f32x4 red[];  // [waves][NT * MT][64]
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x / kWave));
    const int waves = blockDim.x / kWave;
    const int tile0 = blockIdx.x * NT, row0 = blockIdx.y * 16 * MT;
    const int col = lane & 15, grp = lane >> 4;
    const bf16* a[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) a[i] = g.a + min(row0 + 16 * i + col, g.m - 1) * g.lda + 8 * grp;
    const u32x4* codes[NT];
    const uint32_t* scales[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const size_t tile = min(tile0 + t, g.tiles - 1);
        codes[t] = g.codes + tile * g.steps * 64 + lane;
        scales[t] = g.scales + tile * g.words * 64 + col * 4;
    }
    f32x4 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[i][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    u32x4 c[NT][D];
    Words<D> s[NT];
    auto load = [&](int step, u32x4 (&to)[NT][D], Words<D> (&sc)[NT]) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int d = 0; d < D; ++d) to[t][d] = codes[t][static_cast<size_t>(min(step + d, g.steps - 1)) * 64];
            sc[t].load(scales[t] + step / 4 * 64 + step % 4);
        }
    };
    const int stride = D * waves * gridDim.z, last = g.k % kStep ? g.k % kStep / 32 : 4;  // groups of the last step
    int step = D * (blockIdx.z * waves + wave);
    if (step < g.steps) load(step, c, s);
    for (; step < g.steps; step += stride) {
        bf16x8 x[D][MT][4];
#pragma unroll
        for (int d = 0; d < D; ++d)
            if (step + d < g.steps) {
                const int groups = step + d == g.steps - 1 ? last : 4;
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (j < groups) x[d][i][j] = *reinterpret_cast<const bf16x8*>(a[i] + (step + d) * kStep + 32 * j);
            }
        u32x4 c_next[NT][D];
        Words<D> s_next[NT];
        if (step + stride < g.steps) load(step + stride, c_next, s_next);
#pragma unroll
        for (int d = 0; d < D; ++d)
            if (step + d < g.steps) {
                const int groups = step + d == g.steps - 1 ? last : 4;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (j < groups)
#pragma unroll
                        for (int t = 0; t < NT; ++t) {
                            const bf16x8 w = widen(c[t][d][j], group_scale(s[t].w[d], j));
#pragma unroll
                            for (int i = 0; i < MT; ++i) acc[i][t] = mfma16(w, x[d][i][j], acc[i][t]);
                        }
            }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            s[t] = s_next[t];
#pragma unroll
            for (int d = 0; d < D; ++d) c[t][d] = c_next[t][d];
        }
    }
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int t = 0; t < NT; ++t) red[(wave * MT * NT + i * NT + t) * 64 + lane] = acc[i][t];
    __syncthreads();
    // a wave adds a row tile's pair of column tiles (or its only one)
    constexpr int kPer = NT > 1 ? 2 : 1;
    for (int u = wave; u < MT * NT / kPer; u += waves) {
        const int i = u / (NT / kPer), t = u % (NT / kPer) * kPer, row = row0 + 16 * i + col;
        f32x4 v[kPer];
#pragma unroll
        for (int p = 0; p < kPer; ++p) {
            v[p] = f32x4{0.f, 0.f, 0.f, 0.f};
            for (int w = 0; w < waves; ++w) v[p] += red[(w * MT * NT + i * NT + t + p) * 64 + lane];
        }
        if (row < g.m) store_sums<kPer>(g, row, tile0 + t, grp, v);
    }
}

// Tile kernel: 2 x WN waves compute 32 HA rows times 64 WN columns of W; a wave
// holds HA x 4 tiles.  The rows of a step of k come through LDS (two buffers,
// direct global->LDS loads), chunk c of row r at c ^ (r % 16) so that a read
// serves 16 rows on distinct banks.  The weights never pass through LDS: a
// wave's operands of a step are 4 KB of consecutive codes, loaded a step ahead
// into registers and widened there.  The matrix cores bound it: 2080 rows of 4096 -> 28672
// take 384 us back to back, 1.27 PFLOP/s at the power limit, where a large bf16 library product
// reaches 1.40; of 14336 -> 4096 200, of 4096 -> 4096 70.  A step that waits for its loads in one
// place and branches nowhere is what got it there (395 us with a branch for a last step in
// each, in a session where it took 371).
template <int HA, int WN>
__global__ __launch_bounds__(128 * WN, 2) void w4_tile_kernel(W4Args g, int nt_m, int nt_n, int steps_per_split) {
    constexpr int BM = 32 * HA, NW = 2 * WN, BUF = BM * 256, LOADS = BM / 4 / NW;
    static_assert(BM / 4 % NW == 0, "whole loads for every wave");
    __shared__ __attribute__((aligned(1024))) char smem[2 * BUF];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
    const int wm = wave / WN, wn = wave % WN, col = lane & 15, grp = lane >> 4;
    int tm, tn;
    tile_coords(xcd_order(blockIdx.x, nt_m * nt_n), nt_m, nt_n, tm, tn);
    const int m0 = tm * BM, tile0 = (tn * WN + wn) * 4;
    const int t0 = blockIdx.z * steps_per_split, t1 = min(t0 + steps_per_split, g.steps);
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(reinterpret_cast<uintptr_t>(&smem[0])));

    // loads: piece x of this wave is 4 rows; lane l brings chunk (l % 16) ^ (row % 16) of row l / 16.
    // Rows past m read row m - 1, chunks past k the step's first chunk (no product takes them).
    const char* base = reinterpret_cast<const char*>(g.a + m0 * g.lda);
    const int tail = g.k % kStep / 8;  // chunks of a last step that is not whole
    uint32_t off[LOADS];
#pragma unroll
    for (int x = 0; x < LOADS; ++x) {
        const int row = (x * NW + wave) * 4 + (lane >> 4);
        off[x] = static_cast<uint32_t>(min(row, g.m - 1 - m0)) * static_cast<uint32_t>(g.lda * 2) + (((lane & 15) ^ (row & 15)) << 4);
    }
    auto load_row = [&](int x, int t) {
        const int row = (x * NW + wave) * 4 + (lane >> 4), c = (lane & 15) ^ (row & 15);
        const bool past = tail && t == g.steps - 1 && c >= tail;
        load_lds16(base + static_cast<size_t>(t) * 256, off[x] - (past ? c << 4 : 0), lds0 + (t - t0 & 1) * BUF + (x * NW + wave) * 1024);
    };
    // wave-uniform bases, so that a load takes one lane offset for all tiles
    const char* codes[4];
    const char* scales[4];
#pragma unroll
    for (int b = 0; b < 4; ++b) {
        const size_t tile = min(tile0 + b, g.tiles - 1);
        codes[b] = reinterpret_cast<const char*>(g.codes) + tile * g.steps * 1024;
        scales[b] = reinterpret_cast<const char*>(g.scales) + tile * g.words * 256;
    }
    const uint32_t code_off = lane * 16, scale_off = col * 16;
    u32x4 next[4];
    uint32_t sc[4], sc_next[4];
    auto load_weights = [&](int t) {
        const size_t at = static_cast<size_t>(t) * 1024, word = static_cast<size_t>(t / 4) * 256 + t % 4 * 4;
#pragma unroll
        for (int b = 0; b < 4; ++b) next[b] = *reinterpret_cast<const u32x4*>(codes[b] + at + code_off);
#pragma unroll
        for (int b = 0; b < 4; ++b) sc_next[b] = *reinterpret_cast<const uint32_t*>(scales[b] + word + scale_off);
    };
    const char* frag[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) frag[j] = smem + (wm * 16 * HA + col) * 256 + (((4 * j + grp) ^ col) << 4);
    f32x4 acc[HA][4];
#pragma unroll
    for (int i = 0; i < HA; ++i)
#pragma unroll
        for (int b = 0; b < 4; ++b) acc[i][b] = f32x4{0.f, 0.f, 0.f, 0.f};

    load_weights(t0);
#pragma unroll
    for (int x = 0; x < LOADS; ++x) load_row(x, t0);
    // A step is four groups of two units, a unit the products of half of the wave's
    // rows.  Operands are read a unit ahead, a group's weights widened under the unit
    // before it, the next step's rows asked for in the first units (issued together
    // they held up the MFMAs; with a step's order left to the compiler it read all
    // rows at once and spilled).  The one barrier of a step stands before its last
    // unit, whose operands are in registers by then: the next step's first operands
    // are read, from rows that every wave has waited for, while that unit computes,
    // and the buffer of this step is free.
    constexpr int H0 = (HA + 1) / 2, H1 = HA - H0, UNITS = H1 ? 8 : 4, PER = UNITS / 4, EACH = (LOADS + UNITS / 2 - 1) / (UNITS / 2);
    bf16x8 x[2][H0], w[2][4];
    u32x4 c[4];
    auto read = [&](int u, int at) {  // into x[u % 2]
        const int j = u / PER, h = u % PER;
#pragma unroll
        for (int i = 0; i < (h ? H1 : H0); ++i)
            x[u & 1][i] = *reinterpret_cast<const bf16x8*>(frag[j] + at + (h * H0 + i) * 4096);
    };
    auto widen_group = [&](int j) {
#pragma unroll
        for (int b = 0; b < 4; ++b) w[j & 1][b] = widen(c[b][j], group_scale(sc[b], j));
    };
    auto take_weights = [&] {
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            c[b] = next[b];
            sc[b] = sc_next[b];
        }
        widen_group(0);
    };
    wait_vmcnt<0>();
    barrier_only();
    read(0, 0);
    take_weights();
    // MORE: another step follows, so this one has all four groups.  Within such a step
    // nothing branches: across a branch the compiler waits for every read.
    auto step = [&](auto more_c, int t) {
        constexpr bool MORE = decltype(more_c)::value;
        const int groups = tail && t == g.steps - 1 ? tail / 4 : 4;
        const int at = (t - t0 & 1) * BUF;
        if (MORE) load_weights(t + 1);
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            const int j = u / PER, h = u % PER;
            if (u + 1 < UNITS) {
                read(u + 1, at);
            } else if (MORE) {
                wait_lgkmcnt<0>();
                wait_vmcnt<0>();
                barrier_only();
                read(0, BUF - at);
            }
            if (MORE)
#pragma unroll
                for (int q = u * EACH; q < (u + 1) * EACH && q < LOADS; ++q) load_row(q, t + 1);
            if (h == PER - 1 && j < 3) widen_group(j + 1);
            if (u + 1 == UNITS && MORE) take_weights();
            if (MORE || j < groups)
#pragma unroll
                for (int i = 0; i < (h ? H1 : H0); ++i)
#pragma unroll
                    for (int b = 0; b < 4; ++b) acc[h * H0 + i][b] = mfma16(w[j & 1][b], x[u & 1][i], acc[h * H0 + i][b]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
#pragma unroll 1
    for (int t = t0; t + 1 < t1; ++t) step(std::integral_constant<bool, true>{}, t);
    step(std::integral_constant<bool, false>{}, t1 - 1);
    const int row0 = m0 + wm * 16 * HA + col;
#pragma unroll
    for (int i = 0; i < HA; ++i) {
        const int row = row0 + 16 * i;
        if (row >= g.m) continue;
        store_sums<4>(g, row, tile0, grp, acc[i]);
    }
}

// Direct global->LDS load of 4 bytes per lane, as load_lds16.
__device__ __forceinline__ void load_lds4(const void* base, uint32_t off, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" ::"v"(off), "s"(base), "s"(lds) : "memory");
}

// Ring kernel, for some rows: four waves with two tiles each share 16 MT rows.
// Codes, scale words and rows all come through LDS, a ring of DEPTH steps filled by
// direct loads, so that two work-groups' 140 KB a CU are under way at no cost in
// registers; the rows are read from the caches once for 128 columns, where the
// stream kernel's waves, each with 64 columns, spend most of their loads on rows.
// 32 rows of 14336 -> 4096 take 12 us and 3 for the join of eight splits (33 MB, 6.4 at a
// copy's rate), 23 of 4096 -> 100003 57 (227 MB, 44.5).
// (Four tiles a wave halve that again but leave half the work-groups: slower.)
template <int MT, int DEPTH>
__global__ __launch_bounds__(256, 2) void w4_ring_kernel(W4Args g, int steps_per_split) {
    constexpr int NB = 2, WAVE = NB * 1024 + 256, ROWS = MT * 4096, STAGE = 4 * WAVE + ROWS, EACH = NB + 1 + MT;
    static_assert((DEPTH - 2) * EACH < 64, "vmcnt range");
    __shared__ __attribute__((aligned(1024))) char smem[DEPTH * STAGE];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
    const int col = lane & 15, grp = lane >> 4;
    const int tile0 = (blockIdx.x * 4 + wave) * NB;
    const int t0 = blockIdx.z * steps_per_split, t1 = min(t0 + steps_per_split, g.steps);
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(reinterpret_cast<uintptr_t>(&smem[0])));

    const char* codes[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b)
        codes[b] = reinterpret_cast<const char*>(g.codes) + static_cast<size_t>(min(tile0 + b, g.tiles - 1)) * g.steps * 1024;
    // scale words: lane l brings those of tile l / 16, row l % 16
    const size_t first = min(tile0, g.tiles - 1);
    const char* scales = reinterpret_cast<const char*>(g.scales) + first * g.words * 256;
    const uint32_t scale_off = static_cast<uint32_t>(min(tile0 + min(grp, NB - 1), g.tiles - 1) - first) * g.words * 256 + col * 16;
    // rows as in the tile kernel
    const char* base = reinterpret_cast<const char*>(g.a);
    const int tail = g.k % kStep / 8;
    uint32_t off[MT];
#pragma unroll
    for (int x = 0; x < MT; ++x) {
        const int row = (x * 4 + wave) * 4 + grp;
        off[x] = static_cast<uint32_t>(min(row, g.m - 1)) * static_cast<uint32_t>(g.lda * 2) + ((col ^ (row & 15)) << 4);
    }
    auto ask = [&](int t) {
        const uint32_t stage = lds0 + (t - t0) % DEPTH * STAGE, mine = stage + wave * WAVE;
#pragma unroll
        for (int b = 0; b < NB; ++b) load_lds16(codes[b] + static_cast<size_t>(t) * 1024, lane * 16, mine + b * 1024);
        load_lds4(scales + static_cast<size_t>(t / 4) * 256 + t % 4 * 4, scale_off, mine + NB * 1024);
#pragma unroll
        for (int x = 0; x < MT; ++x) {
            const int c = col ^ (((x * 4 + wave) * 4 + grp) & 15);
            const bool past = tail && t == g.steps - 1 && c >= tail;
            load_lds16(base + static_cast<size_t>(t) * 256, off[x] - (past ? c << 4 : 0), stage + 4 * WAVE + (x * 4 + wave) * 1024);
        }
    };
    uint32_t frag[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) frag[j] = 4 * WAVE + col * 256 + (((4 * j + grp) ^ col) << 4);
    f32x4 acc[MT][NB];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int b = 0; b < NB; ++b) acc[i][b] = f32x4{0.f, 0.f, 0.f, 0.f};

#pragma unroll
    for (int d = 0; d < DEPTH - 1; ++d)
        if (t0 + d < t1) ask(t0 + d);
#pragma unroll 1
    for (int t = t0; t < t1; ++t) {
        // this step's loads have landed, everyone's rows too; the step before it is read out of the ring
        if (t + DEPTH - 1 <= t1) wait_vmcnt<(DEPTH - 2) * EACH>();
        else wait_vmcnt<0>();
        barrier_only();
        if (t + DEPTH - 1 < t1) ask(t + DEPTH - 1);
        const char* stage = smem + (t - t0) % DEPTH * STAGE;
        const char* mine = stage + wave * WAVE;
        u32x4 c[NB];
        uint32_t s[NB];
        bf16x8 x[4][MT];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            c[b] = *reinterpret_cast<const u32x4*>(mine + b * 1024 + lane * 16);
            s[b] = *reinterpret_cast<const uint32_t*>(mine + NB * 1024 + (b * 16 + col) * 4);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < MT; ++i) x[j][i] = *reinterpret_cast<const bf16x8*>(stage + frag[j] + i * 4096);
        const int groups = tail && t == g.steps - 1 ? tail / 4 : 4;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (j >= groups) break;
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const bf16x8 w = widen(c[b][j], group_scale(s[b], j));
#pragma unroll
                for (int i = 0; i < MT; ++i) acc[i][b] = mfma16(w, x[j][i], acc[i][b]);
            }
        }
        wait_lgkmcnt<0>();
    }
#pragma unroll
    for (int i = 0; i < MT; ++i)
        if (16 * i + col < g.m) store_sums<NB>(g, 16 * i + col, tile0, grp, acc[i]);
}

// Adds a split product's sums, four columns (or pairs) of a row a thread, and stores them.
__global__ __launch_bounds__(256) void w4_join_kernel(W4Args g) {
    const int per = g.gated ? 2 : 1, quads = g.tiles / per * 4;
    const int i = blockIdx.x * 256 + threadIdx.x, row = blockIdx.y;
    if (i >= quads) return;
    const int tile = i / 4 * per, grp = i % 4;
    const size_t ld = 16 * static_cast<size_t>(g.tiles);
    f32x4 v[2] = {};
    for (int s = 0; s < g.splits; ++s) {
        const float* p = g.part + (static_cast<size_t>(s) * g.m + row) * ld + tile * 16 + 4 * grp;
        v[0] += *reinterpret_cast<const f32x4*>(p);
        if (g.gated) v[1] += *reinterpret_cast<const f32x4*>(p + 16);
    }
    if (g.gated) {
        store_row<2>(g, row, tile, grp, v);
    } else {
        f32x4 one[1] = {v[0]};
        store_row<1>(g, row, tile, grp, one);
    }
}

// A thread for each lane of each tile's step: four words of codes; the first 16
// lanes of every step make the row's scale word.
constexpr size_t kPackGroups = 1 << 20;  // at most; they go on that far apart
__global__ __launch_bounds__(256) void w4_pack_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                      u32x4* __restrict__ to_codes, uint32_t* __restrict__ to_scales,
                                                      int rows, int k, int tiles, int steps, int words, bool gated) {
    for (size_t i = blockIdx.x * static_cast<size_t>(256) + threadIdx.x; i < static_cast<size_t>(tiles) * words * 256;
         i += gridDim.x * static_cast<size_t>(256)) {
        const int lane = i % 64, step = i / 64 % (4 * words);
        const size_t tile = i / 64 / (4 * words);
        const int r = (gated ? tile / 2 : tile) * 16 + (lane & 15);  // of the gate or up rows, or of all
        const int groups = k / 32;
        const size_t row = gated && tile % 2 ? static_cast<size_t>(rows) + r : r;
        if (step < steps) {
            u32x4 c = {0u, 0u, 0u, 0u};
            for (int j = 0; j < 4; ++j)
                if (r < rows && 4 * step + j < groups)
                    c[j] = *reinterpret_cast<const uint32_t*>(codes + row * (k / 2) + (4 * step + j) * 16 + 4 * (lane / 16));
            to_codes[(tile * steps + step) * 64 + lane] = c;
        }
        if (lane >= 16) continue;
        uint32_t w = 0;
        for (int j = 0; j < 4; ++j)
            if (r < rows && 4 * step + j < groups) w |= static_cast<uint32_t>(scales[row * groups + 4 * step + j]) << (8 * j);
        to_scales[((tile * words + step / 4) * 16 + lane) * 4 + step % 4] = w;
    }
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

constexpr int kMostSplits = 32;  // the join reads them one after the other: 23 rows of 65536 -> 64 take 20 us, with 128 36
// Most waves of a stream work-group.
constexpr int kStreamWaves = 8;

// Which kernel a product runs on.
struct W4Plan {
    int kind;    // 0: stream, 1: tile, 2: ring
    int mt, nt;  // stream: row and column tiles of a work-group; tile: HA, WN; ring: row tiles
    int waves;   // stream
    int splits;
};

W4Plan plan_w4(const W4Shape& s, int m, bool gated) {
    W4Plan p{};
    p.splits = 1;
    // Some rows: the ring, where its 128 columns a work-group, with k split in parts of
    // four steps at least, make some 200 of them.  us with the ring / the stream kernel:
    // 32 rows of 14336 -> 4096 16.0 / 18.5, of 4096 -> 28672 21.7 / 25.1, of 4096 -> 6144 11.7 / 14.2,
    // 23 of 4096 -> 100003 55.5 / 69.2, 16 of them 51.3 / 55.8; but 32 of 4096 -> 4096 11.2 / 10.1
    // and 16 of 4096 -> 28672 18.2 / 17.8.  64 rows against the tile kernel: 27.5 / 31.1, 19.6 /
    // 22.8, 13.7 / 14.1.  Parts of eight steps: 64 rows of 14336 -> 2048 17.8, of seven 16.4.
    // (One work-group a CU with nine steps in its ring rather than four: 12.4 / 10.9, 19.1 / 16.0.)
    if (m <= 64 && (m > 32 || (m > 16 && (s.tiles >= 384 || s.steps >= 64)) || (m > 8 && s.tiles >= 4096))) {
        p.kind = 2;
        p.mt = m <= 16 ? 1 : m <= 32 ? 2 : 4;
        while (ceil_div(s.tiles, 8) * p.splits * 2 <= 256 && p.splits * 2 * 4 <= s.steps && p.splits < kMostSplits) p.splits *= 2;
        p.splits = static_cast<int>(ceil_div(s.steps, ceil_div(s.steps, p.splits)));
        return p;
    }
    if (m <= 32) {
        p.mt = m <= 16 ? 1 : 2;
        // Waves of 64 columns read the rows least, narrow ones give more work-groups: 4096 ->
        // 28672 15.4 / 16.8 (32 columns), 4096 -> 6144 at 1 row 7.6 (64) / 5.9 (32) / 6.3 (16), 4096 ->
        // 4096 7.5 / 5.5 / 5.1.  Beyond 8 rows of a long k the rows cost most, and k is
        // split for the wide waves instead: 16 rows of 14336 -> 4096 14.3 / 19.0, 8 13.3 / 13.4.
        const bool wide = m > 16 || (m > 8 && s.steps >= 64);
        p.nt = wide || s.tiles >= 1024 ? 4 : gated || s.tiles >= 384 ? 2 : 1;
        while (wide && ceil_div(s.tiles, p.nt) * p.splits < 256 && p.splits * 2 * 8 <= s.steps && p.splits < kMostSplits) p.splits *= 2;
        p.waves = std::min(p.nt == 4 && p.splits == 1 ? 4 : kStreamWaves, s.words);
        return p;
    }
    // More rows: rounds of the work-groups that run together (eight waves a CU) times
    // their steps.  us a step, fitted at 512 .. 2080 rows of products of 4096 and 14336:
    // 0.45 + 0.305 HA (2.89 at HA 8, 2.28 at 6, 1.64 at 4; WN 2 1.64 at HA 4, 1.35 at 3),
    // never below 1.05, the wait for a step; work-groups alone on their CU take
    // 0.65 of that.  A split's sums are written and read at 6 TB/s, by one launch
    // more.  (WN 1 as well would win up to 0.05 of the time, on few shapes.)
    p.kind = 1;
    double best = 0;
    for (int wn = 4; wn >= 2; wn /= 2)
        for (int ha = wn / 2; ha <= 2 * wn; ++ha) {
            if (ha == 7) continue;
            const int64_t tiles = ceil_div(m, 32 * ha) * ceil_div(s.tiles, 4 * wn), slots = 256 * 4 / wn;
            for (int sp = 1; sp == 1 || (sp <= 8 && sp * 4 <= s.steps && m <= kMostSplitRows); sp *= 2) {
                const int64_t per = ceil_div(s.steps, sp), groups = tiles * sp;
                double step = std::max(1.05, 0.45 + 0.305 * ha);
                if (wn < 4 && groups <= 256) step *= 0.65;
                const double t = ceil_div(groups, slots) * (per * step + 1.5) +
                                 (sp > 1 ? 2.0 + sp * static_cast<double>(m) * s.tiles * 16 * 4 * 2 / 6e6 : 0.0);
                if (best == 0 || t < best) {
                    best = t;
                    p.mt = ha;
                    p.nt = wn;
                    p.splits = static_cast<int>(ceil_div(s.steps, per));
                }
            }
        }
    return p;
}

size_t w4_partial_bytes(const W4Shape& s, const W4Plan& p, int m) {
    return p.splits > 1 ? static_cast<size_t>(p.splits) * m * s.tiles * 64 : 0;
}

template <int MT, int NT>
void stream_launch(const W4Args& g, int waves, hipStream_t s) {
    const dim3 grid(static_cast<unsigned>(ceil_div(g.tiles, NT)), static_cast<unsigned>(ceil_div(g.m, 16 * MT)),
                    static_cast<unsigned>(g.splits));
    w4_stream_kernel<MT, NT, kStreamWaves><<<grid, 64 * waves, static_cast<size_t>(waves) * MT * NT * 1024, s>>>(g);
}

template <int MT, int DEPTH>
void ring_launch(const W4Args& g, hipStream_t s) {
    w4_ring_kernel<MT, DEPTH><<<dim3(static_cast<unsigned>(ceil_div(g.tiles, 8)), 1, static_cast<unsigned>(g.splits)), 256, 0, s>>>(
        g, static_cast<int>(ceil_div(g.steps, g.splits)));
}

template <int HA, int WN>
void tile_launch(const W4Args& g, hipStream_t s) {
    const int nt_m = static_cast<int>(ceil_div(g.m, 32 * HA)), nt_n = static_cast<int>(ceil_div(g.tiles, 4 * WN));
    const int per = static_cast<int>(ceil_div(g.steps, g.splits));
    w4_tile_kernel<HA, WN><<<dim3(static_cast<unsigned>(nt_m * nt_n), 1, static_cast<unsigned>(g.splits)), 128 * WN, 0, s>>>(
        g, nt_m, nt_n, per);
}

void launch_w4(const W4Args& g, const W4Plan& p, hipStream_t s) {
    if (p.kind == 0) {
        if (p.mt == 2) stream_launch<2, 4>(g, p.waves, s);
        else if (p.nt == 1) stream_launch<1, 1>(g, p.waves, s);
        else if (p.nt == 2) stream_launch<1, 2>(g, p.waves, s);
        else stream_launch<1, 4>(g, p.waves, s);
    } else if (p.kind == 2) {
        if (p.mt == 1) ring_launch<1, 5>(g, s);
        else if (p.mt == 2) ring_launch<2, 4>(g, s);
        else ring_launch<4, 3>(g, s);
    } else switch (p.nt * 16 + p.mt) {
        case 64 + 2: tile_launch<2, 4>(g, s); break;
        case 64 + 3: tile_launch<3, 4>(g, s); break;
        case 64 + 4: tile_launch<4, 4>(g, s); break;
        case 64 + 5: tile_launch<5, 4>(g, s); break;
        case 64 + 6: tile_launch<6, 4>(g, s); break;
        case 64 + 8: tile_launch<8, 4>(g, s); break;
        case 32 + 1: tile_launch<1, 2>(g, s); break;
        case 32 + 2: tile_launch<2, 2>(g, s); break;
        case 32 + 3: tile_launch<3, 2>(g, s); break;
        default: tile_launch<4, 2>(g, s); break;
    }
    if (p.splits > 1) {
        const int quads = g.tiles / (g.gated ? 2 : 1) * 4;
        w4_join_kernel<<<dim3(static_cast<unsigned>(ceil_div(quads, 256)), static_cast<unsigned>(g.m)), 256, 0, s>>>(g);
    }
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
        const size_t groups = std::min(static_cast<size_t>(w.tiles) * w.words, kPackGroups);
        w4_pack_kernel<<<static_cast<unsigned>(groups), 256, 0, static_cast<hipStream_t>(stream)>>>(
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
        const W4Shape s = w4_shape(n, k, gated);
        *bytes = 0;
        for (int m = 1; m <= max_m && m <= kMostSplitRows; ++m)
            *bytes = std::max(*bytes, w4_partial_bytes(s, plan_w4(s, m, gated), m));
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
        g.gated = w->gated != 0;
        g.f32 = out_f32 != 0;
        const W4Plan plan = lda > kMostTileStride ? W4Plan{0, m <= 16 ? 1 : 2, 4, std::min(4, sh.words), 1} : plan_w4(sh, m, g.gated);
        const size_t need = w4_partial_bytes(sh, plan, m);
        if (need) {
            if (!ws || !aligned16(ws)) return fail(SLW_EINVAL, "the workspace must be 16-byte aligned device memory");
            if (ws_bytes < need) return fail(SLW_ENOMEM, "the workspace holds %zu bytes, %d rows need %zu", ws_bytes, m, need);
        }
        g.part = static_cast<float*>(ws);
        g.splits = plan.splits;
        launch_w4(g, plan, static_cast<hipStream_t>(stream));
        HIP_TRY(hipGetLastError());
        return SLW_OK;
    });
}
