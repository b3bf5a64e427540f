// The next token of each row of logits, from a given random number.
//
// w_t = 2^((x_t - M) log2(e) / T), M the largest logit.  The filters keep a head
// of the tokens sorted by (logit descending, index ascending): the first top_k;
// of those, the ones with less than top_p of their mass before them; of those,
// w >= min_p.  So every filter is a cut in that order, (key, index) of the last
// token kept, and no row is ever sorted.  A row is cut into slices, so that a few
// rows fill the chip, and dealt with by two kernels:
//   1. a slice's largest logit and, as the row needs them, the largest of every
//      thread (any filter), the mass of the tokens in bins of 1/16 octave of w (top_p alone),
//      or the mass of sixteenths of the slice (no filter);
//   2. a row's token.  top_k up to the number of threads: the k-th largest of the
//      threads' largest bounds the k-th largest logit from below, and what is not
//      below it, a little more than k tokens, is collected in LDS, from those threads'
//      pieces alone.  top_p: the running sum over bins says in which one the cut is; the
//      tokens down to that bin are collected, or where they are too many those of the
//      bin alone.  A short list is drawn from by ranks.  In a longer one cuts and the draw
//      are one thing, the first value of an order at which a running sum reaches a
//      target, found digit by digit with a histogram: by logit and count for top_k, by
//      logit and mass for top_p, by index and mass for the draw.  Where more tokens are
//      kept than were collected, or all, sums over ranges of the row say in which the
//      running sum passes u Z, then over sixteenths of that range, and so on.
//
// Every mass is held in 64 bits: w from an exponential good to 2^-36, bins and
// lists in fixed point (integer sums: the order of the atomics does not matter),
// all else in doubles summed in a fixed order, of slices whose number depends on the
// batch's rows.  So a cut or a draw is the definition's where its target is further than
// some 2^-36 of the mass from a running sum; and at exact ties of equal logits with
// nothing else in the row, where all of these are whole numbers.  With fp32 sums one draw
// in a few hundred would be another token.
//
// What bounds it (times of calls back to back).  A few rows: latency.  One row of 32768 with
// top_k and top_p takes 15.6 us where the list has up to 256 tokens: 5 for the first kernel, 1
// between the two, 9 for a chain of some 25 steps with a barrier each, which meet their code
// cold and so are loops of few instructions rather than unrolled; 26 us with top_k 650, by digits.
// 256 rows of 131072 bf16 logits (67 MB, 13 us at a copy's rate): greedy 18.2 us; top_k 41 (18 +
// 19 us of kernels); no filter 49 and top_p 90, where the first kernel's instructions take 36 and
// 40 us (23 a token, half of them fp64), and a nucleus beyond the list takes the second kernel 50: a
// pass for the bin's tokens, then sums over its slice and over the slice's sixteenths.
// Slow are rows whose cut is among more tokens of one bin than a list holds: 50 passes of
// bisection by one work-group.  131072 equal logits with top_p 2.4 ms; 262144 of standard deviation 2 at
// T = 2 with top_p 0.9 4.8, 64 such rows 5.0 (fp32 6.4).
#include <math.h>

#include <algorithm>

#include "device.h"
#include "hip_try.h"
#include "kernels.h"

namespace slw {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / kWave;
constexpr int kBins = 896;          // of a slice: 16 for an octave; the last one holds w < 2^-55, 2^-35 in all, and is weighed nowhere
constexpr int kHeld = 4096;         // 16 bytes each of a slice that wait in LDS to be weighed (256 rows top_p 43 us; read again 44)
constexpr int kQueue = 8 * kWave + 64;  // logits a wave has queued: a piece of every lane beside 63 left over
constexpr int kRowBins = kThreads;  // of a row that goes by its own (Row::bin_at)
constexpr int kMost = 4096;         // most groups of threads of a row whose largest logits are kept
constexpr int kMostSlices = 16;     // of a row
constexpr int kList = 4096;         // tokens of a row's list in LDS, in any order

struct SampleArgs {
    const void* logits;
    int64_t ld;
    const float* temperature;
    const int32_t* top_k;
    const float* top_p;
    const float* min_p;
    const float* u;
    int32_t* tokens;
    float* logprob;
    int vocab, rows;
    // workspace; a slice is slices * row + its number
    int slices;
    uint64_t* best;     // [slice]: its largest logit's key, ~ the first index that has it; 0: nothing but -inf
    int32_t* ref;       // [slice]: top_p: sixteenths of an octave from logit 0 that its masses count from
    double* sums;       // [slice][16]
    uint64_t* bins;     // [slice][kBins]
    uint32_t* most;     // [row][kMost]: the largest keys of groups of threads
};

// Ascending with the value; both zeros alike, NaN as -inf.
__device__ __forceinline__ uint32_t key_of(float x) {
    if (!(x == x)) x = -INFINITY;
    const uint32_t b = __float_as_uint(x + 0.0f);
    return b ^ (b & 0x80000000u ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) {
    return __uint_as_float(key ^ (key & 0x80000000u ? 0x80000000u : 0xFFFFFFFFu));
}

// Sixteenths of an octave from logit 0, whole.  Never falls as x grows; near enough to
// 0, single precision moves few x to the next one, past a half by 2^-6 at most.
__device__ __forceinline__ bool near_zero(float x, double c16, double margin = 0.0) {
    return fabs(static_cast<double>(x)) * c16 <= 0x1p17 - margin && c16 <= 0x1p100;
}
__device__ __forceinline__ float sixteenth(float x, float c16) { return rintf(x * c16); }

// How w depends on x.  In a row that has +inf those tokens alone have mass.
struct Row {
    float M;          // the largest logit; 0 where that is +inf
    bool at_inf;
    double c16;       // 16 log2(e) / T: w in sixteenths of an octave
    double min_p;
    int n;            // tokens
    const __attribute__((address_space(3))) double* root;  // LDS: 2^(i / 16), i < 16
    __device__ float fix(float x) const { return x == INFINITY ? 0.f : -INFINITY; }
    // sixteenths of an octave below M, <= 0; NaN and -inf as far down
    __device__ __forceinline__ double depth(float x) const {
        return fmax((static_cast<double>(x) - static_cast<double>(M)) * c16, -17600.0);
    }
    // 2^(t / 16): t = 16 q + i + f, |f| <= 1/2, 2^(f / 16) by a polynomial fitted to
    // 5e-12, 2^(i / 16) from the table, whose 16 entries lie on distinct banks.
    __device__ __forceinline__ double weight(double t, int& n) const { return weight_from(t, 0, n); }
    // 2^((t - ref) / 16), n: t - ref to the nearest whole
    __device__ __forceinline__ double weight_from(double t, int ref, int& n) const {
        const double p = of_sixteenth(t, n);
        n -= ref;
        return ldexp(p * root[n & 15], n >> 4);
    }
    // 2^((t - n) / 16), n the nearest whole number
    static __device__ __forceinline__ double of_sixteenth(double t, int& n) {
        const double whole = rint(t);
        n = static_cast<int>(whole);
        return power(t - whole, 1.0);
    }
    // one - 1 + 2^(f / 16)
    static __device__ __forceinline__ double power(double f, double one) {
        return fma(f, fma(f, fma(f, fma(f, 0x1.3b2c4ac7eb38ap-23, 0x1.c6b3488226c3bp-17), 0x1.ebfbdff6988cep-11),
                          0x1.62e42fee4615cp-5), one);
    }
    // 2^(f / 16) in units of 2^-42: the low bits of a number near 2^10
    static __device__ __forceinline__ uint64_t units(double f) {
        return static_cast<uint64_t>(__double_as_longlong(power(f, 1.0 + 0x1p10)) - __double_as_longlong(0x1p10));
    }
    __device__ __forceinline__ double w(float x) const {
        int n;
        return weight(depth(x), n);
    }
    // The bin, of kRowBins, of what lies d sixteenths below M: 16 octaves of one each, then 128
    // bins for the next 16 octaves, for the 32 after them, and so on, so that a count is cut among
    // few tokens at any temperature; d >= 16384 is beyond them, as no w below 2^-1022 is to be told from 0.
    static __device__ __forceinline__ int bin_at(int d) {
        const int s = max(24 - __clz(d | 1), 0);
        return 128 * s + (d >> s);
    }
    static __device__ __forceinline__ int start_of(int bin) {
        const int s = max(bin / 128 - 1, 0);
        return (bin - 128 * s) << s;
    }
    __device__ __forceinline__ int bin_of(float x) const { return bin_at(-static_cast<int>(rint(depth(x)))); }
};

struct Shared {
    union {
        struct {
            uint64_t list[kList];  // key, index
            double w[kList];
        };
        float queue[kWaves][kQueue];
    };
    uint64_t mass[kRowBins];
    __attribute__((aligned(16))) float ends[16];
    double root[16];
    double red_d[kWaves];
    uint64_t best[kMostSlices];
    int32_t ref[kMostSlices];
    uint64_t goal, sum, before;
    double found_d, above_d;
    int n_list, n_groups, found, digit;
    uint16_t groups[kMost / 2];
};

// Inclusive sums over the lanes of a wave by data-parallel moves: within rows of 16
// lanes, then the last lane of a row onto the next one, then of the first half onto
// the second.  A shuffle goes through LDS, several times as long.
template <int CTRL, int ROWS, class V>
__device__ __forceinline__ V moved(V v) {
    static_assert(sizeof(V) == 4 || sizeof(V) == 8, "one or two registers");
    union {
        V v;
        int w[sizeof(V) / 4];
    } from{v}, to;
#pragma unroll
    for (size_t i = 0; i < sizeof(V) / 4; ++i) to.w[i] = __builtin_amdgcn_update_dpp(0, from.w[i], CTRL, ROWS, 0xf, false);
    return to.v;
}
template <class V>
__device__ __forceinline__ V of_lane(V v, int lane);
__device__ __forceinline__ uint64_t wave_max(uint64_t v) {
    v = max(v, moved<0x111, 0xf>(v));
    v = max(v, moved<0x112, 0xf>(v));
    v = max(v, moved<0x114, 0xf>(v));
    v = max(v, moved<0x118, 0xf>(v));
    v = max(v, moved<0x142, 0xa>(v));
    v = max(v, moved<0x143, 0xc>(v));
    return of_lane(v, kWave - 1);
}
template <class V>
__device__ __forceinline__ V wave_scan(V v) {
    v += moved<0x111, 0xf>(v);  // one lane up
    v += moved<0x112, 0xf>(v);
    v += moved<0x114, 0xf>(v);
    v += moved<0x118, 0xf>(v);
    v += moved<0x142, 0xa>(v);  // lane 15 of a row
    v += moved<0x143, 0xc>(v);  // lane 31
    return v;
}
// A lane's value, on every lane.
template <class V>
__device__ __forceinline__ V of_lane(V v, int lane) {
    union {
        V v;
        int w[sizeof(V) / 4];
    } x{v};
#pragma unroll
    for (size_t i = 0; i < sizeof(V) / 4; ++i) x.w[i] = __builtin_amdgcn_readlane(x.w[i], lane);
    return x.v;
}
// A value that is the same on every lane, in scalar registers.
template <class V>
__device__ __forceinline__ V uniform(V v) { return of_lane(v, 0); }
template <class V>
__device__ __forceinline__ V wave_total(V v) { return of_lane(wave_scan(v), kWave - 1); }

// threadIdx.x, of which the compiler does not know that it is the same each time: what
// the steps of a row compute from it would be kept in registers over all of them, and
// spilled (one row of 32768 with top_k and top_p 15.3 us; with threadIdx.x 16.3).
__device__ __forceinline__ int thread_id() {
    int t = threadIdx.x;
    asm volatile("" : "+v"(t));
    return t;
}

// The same for any value: what is computed from it is not kept over the steps of a row.
template <class V>
__device__ __forceinline__ V anew(V v) {
    asm volatile("" : "+v"(v));
    return v;
}

// LDS accesses of the lanes of one wave keep their order across it.
__device__ __forceinline__ void wave_fence() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

// *at becomes the first thread for which `is` holds, where that is below it; of a
// wave one lane tells, as LDS would take the lanes one after the other.
__device__ __forceinline__ void first_thread(bool is, int* at) {
    const uint64_t mask = __ballot(is);
    if (mask && threadIdx.x % kWave == 0) atomicMin(at, static_cast<int>(threadIdx.x) + __ffsll(static_cast<unsigned long long>(mask)) - 1);
}

// Sum over the work-group, in a fixed order, on every thread.
__device__ __forceinline__ double block_sum(double v, Shared& sh) {
    v = wave_total(v);
    __syncthreads();
    if (threadIdx.x % kWave == 0) sh.red_d[threadIdx.x / kWave] = v;
    __syncthreads();
    v = 0.0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) v += sh.red_d[w];
    return v;
}

// Of the waves' sums in sh.red_d, which follow `before`: the first at which the running
// sum passes u of all (or, once that is known, `target`), else the last with any mass.
struct Part {
    int at;
    double before, total;
};
__device__ __forceinline__ Part find_part(double before, double u, double target, Shared& sh) {
    const int lane = threadIdx.x % kWave;
    const double mine = lane < kWaves ? sh.red_d[lane] : 0.0, upto = before + wave_scan(mine);
    Part p;
    p.total = of_lane(upto, kWave - 1);
    const uint64_t some = __ballot(mine > 0.0), here = __ballot(mine > 0.0 && upto > (u >= 0.0 ? u * p.total : target));
    p.at = here ? __ffsll(static_cast<unsigned long long>(here)) - 1 : max(63 - __clzll(static_cast<long long>(some)), 0);
    p.before = p.at > 0 ? of_lane(upto, p.at - 1) : before;
    return p;
}

// Inclusive sums over the work-group's threads, in thread order.
__device__ __forceinline__ double block_scan(double v, Shared& sh) {
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    v = wave_scan(v);
    __syncthreads();
    if (lane == kWave - 1) sh.red_d[wave] = v;
    __syncthreads();
    double before = 0.0;
#pragma unroll
    for (int w = 0; w < kWaves - 1; ++w) before += w < wave ? sh.red_d[w] : 0.0;
    return before + v;
}

// The row in pieces of 8 tokens, aligned to 16 bytes as far as the row's start
// allows: piece v holds tokens 8 v - shift .. + 7, those outside the row as -inf.
// The first and the last piece, which may have such, wait in LDS.
typedef const __attribute__((address_space(3))) f32x4* LdsVec;
template <class T>
struct Pieces {
    const T* row;
    int n, shift, count;
    LdsVec ends;
    // by every thread, before the work-group's next barrier
    __device__ __forceinline__ Pieces(const T* r, int n_, float (&lds)[16]) : row(r), n(n_) {
        shift = static_cast<int>(reinterpret_cast<uintptr_t>(r) % 16 / sizeof(T));
        count = (n + shift + 7) / 8;
        ends = (LdsVec)lds;
        if (threadIdx.x < 16) {
            const int i = 8 * (threadIdx.x < 8 ? 0 : count - 1) - shift + static_cast<int>(threadIdx.x % 8);
            lds[threadIdx.x] = i >= 0 && i < n ? static_cast<float>(row[i]) : -INFINITY;
        }
    }
    struct Raw {
        f32x4 w[sizeof(T) / 2];
    };
    // A piece inside the row (or the nearest such), for `spread`: nothing waits for it yet.
    __device__ __forceinline__ Raw ask(int v) const {
        Raw r;
        const f32x4* at = reinterpret_cast<const f32x4*>(row + (8 * min(max(v, 1), count - 2) - shift));
        if (count >= 3)
#pragma unroll
            for (size_t i = 0; i < sizeof(T) / 2; ++i) r.w[i] = at[i];
        return r;
    }
    __device__ __forceinline__ void spread(const Raw& r, int v, float (&x)[8]) const {
        if (v == 0 || v == count - 1) {
            const f32x4 a = ends[v == 0 ? 0 : 2], b = ends[v == 0 ? 1 : 3];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[e] = a[e];
                x[4 + e] = b[e];
            }
            return;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t w = __float_as_uint(r.w[sizeof(T) == 2 ? 0 : e / 4][sizeof(T) == 2 ? e / 2 : e % 4]);
            x[e] = __uint_as_float(sizeof(T) == 4 ? w : e % 2 ? w & 0xFFFF0000u : w << 16);
        }
    }
    __device__ __forceinline__ void load(int v, float (&x)[8]) const { spread(ask(v), v, x); }
};

// Pieces v, v + stride, ... below `end`, f(x, v).  N are asked for at a time, and
// where that is one, it is asked for while f looks at the one before it.
template <int N, class T, class F>
__device__ __forceinline__ void each_piece(const Pieces<T>& p, int v, int end, int stride, F&& f) {
    typename Pieces<T>::Raw raw[N];
    if (N == 1) raw[0] = p.ask(v);
#pragma unroll 1
    for (; v < end; v += N * stride) {
        float x[8];
        if (N == 1) {
            p.spread(raw[0], v, x);
            raw[0] = p.ask(v + stride);
            f(x, v);
            continue;
        }
#pragma unroll
        for (int q = 0; q < N; ++q) raw[q] = p.ask(v + q * stride);
#pragma unroll
        for (int q = 0; q < N; ++q)
            if (v + q * stride < end) {
                p.spread(raw[q], v + q * stride, x);
                f(x, v + q * stride);
            }
    }
}

__device__ __forceinline__ float largest(const float (&x)[8]) {
    return fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
}

// Every token of the row, f(x, index); a row with +inf as Row::fix has it.  One at a
// time: for what few rows come to.
template <class T, class F>
__device__ __forceinline__ void each(const Pieces<T>& p, const Row& r, F&& f) {
#pragma unroll 1
    for (int i = threadIdx.x; i < p.n; i += kThreads) {
        const float x = static_cast<float>(p.row[i]);
        f(r.at_inf ? r.fix(x) : x, i);
    }
}

// A head of the sorted tokens: those with a larger key than `key`, and those with
// it up to index `last`.
struct Cut {
    uint32_t key;
    int last;
    __device__ bool keeps(uint32_t k, int i) const { return k > key || (k == key && i <= last); }
};

// The head of tokens within `in` that ends with the token at which the count
// (by_mass: the mass) reaches the target, by bisection on the key and, among
// equals, on the index: where the other ways have no room.
template <class T>
__device__ __forceinline__ Cut bisect(const Pieces<T>& p, const Row& r, const Cut& in, bool by_mass, double target, Shared& sh) {
    auto sum = [&](const Cut& c) {
        double s = 0.0;
        each(p, r, [&](float x, int i) {
            const uint32_t k = key_of(x);
            if (in.keeps(k, i) && c.keeps(k, i)) s += by_mass ? r.w(x) : 1.0;
        });
        return block_sum(s, sh);
    };
    // the largest key for which everything from it up reaches the target
    uint32_t lo = in.key, hi = key_of(r.M);
#pragma unroll 1
    while (lo < hi) {
        const uint32_t mid = hi - (hi - lo) / 2;  // lo < mid <= hi
        if (sum(Cut{mid, p.n}) >= target) lo = mid;
        else hi = mid - 1;
    }
    int a = 0, b = lo == in.key ? min(in.last, p.n - 1) : p.n - 1;
#pragma unroll 1
    while (a < b) {
        const int mid = a + (b - a) / 2;
        if (sum(Cut{lo, mid}) >= target) b = mid;
        else a = mid + 1;
    }
    return Cut{lo, a};
}

// Pieces of slice s of a row, a whole number for every thread (the last ones may have fewer, or none).
__device__ __forceinline__ int slice_pieces(int count, int slices) {
    return ((count + slices - 1) / slices + kThreads - 1) / kThreads * kThreads;
}

// Threads of a slice whose largest logit is kept together.
__device__ __forceinline__ int group_size(int slices) { return max(1, slices * kThreads / kMost); }

// Tokens of `in` from `lo` up and below `hi` (none: +inf), in LDS (in any order); how many there are, of
// which the first kList are there, or any number above kList.  Where at most half of the groups of threads have
// such a token, only their pieces are read.
template <class T>
__device__ __forceinline__ int collect(const Pieces<T>& p, const Row& r, float lo, float hi, const Cut& in,
                                       const uint32_t (&most)[kMost / kThreads], int slices, Shared& sh) {
    const int tid = threadIdx.x;
    __syncthreads();
    if (tid == 0) sh.n_list = sh.n_groups = 0;
    __syncthreads();
    // in a row with +inf, where they count as 0 and all else as -inf, only they can be meant
    const float from = r.at_inf ? INFINITY : lo, below = r.at_inf ? NAN : hi;
    const uint32_t least = key_of(from);
#pragma unroll
    for (int s = 0; s < kMost / kThreads; ++s)
        if (most[s] >= least) {
            const int at = atomicAdd(&sh.n_groups, 1);
            if (at < kMost / 2) sh.groups[at] = static_cast<uint16_t>(s * kThreads + tid);
        }
    auto look = [&](const float (&x)[8], int v) {
        uint32_t keeps = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) keeps |= x[e] >= from && !(x[e] >= below) ? 1u << e : 0u;
        if (in.key != 0) {  // few rows come with a cut
#pragma unroll 1
            for (int e = 0; e < 8; ++e) {
                float y = x[0];
#pragma unroll
                for (int j = 1; j < 8; ++j) y = e == j ? x[j] : y;
                if (!in.keeps(key_of(r.at_inf ? r.fix(y) : y), 8 * v - p.shift + e)) keeps &= ~(1u << e);
            }
        }
        if (!keeps) return;
        int at = atomicAdd(&sh.n_list, __popc(keeps));
#pragma unroll 1
        for (; keeps; keeps &= keeps - 1, ++at) {
            const int e = __ffs(keeps) - 1;
            float y = x[0];
#pragma unroll
            for (int j = 1; j < 8; ++j) y = e == j ? x[j] : y;
            if (at < kList)
                sh.list[at] = static_cast<uint64_t>(key_of(r.at_inf ? r.fix(y) : y)) << 32 | static_cast<uint32_t>(8 * v - p.shift + e);
        }
    };
    __syncthreads();
    const int groups = uniform(sh.n_groups), size = group_size(slices), in_slice = kThreads / size;
    if (2 * groups <= slices * in_slice) {
        const int per = slice_pieces(p.count, slices), rounds = per / kThreads;
#pragma unroll 1
        for (int j = tid; j < groups * rounds * size; j += kThreads) {
            const int group = sh.groups[j / (rounds * size)], i = j % (rounds * size);
            const int slice = group / in_slice, v = slice * per + group % in_slice * size + i % size + i / size * kThreads;
            if (v >= p.count) continue;
            float x[8];
            p.load(v, x);
            look(x, v);
        }
    } else {
        // first which pieces have any, 32 of a thread at a time; a wave has one in most of its
        // rounds, and would go through all of `look` in each
#pragma unroll 1
        for (int v0 = tid; v0 < p.count; v0 += 32 * kThreads) {
            uint32_t pending = 0;
            each_piece<4>(p, v0, min(v0 + 32 * kThreads, p.count), kThreads, [&](const float (&x)[8], int v) {
                bool any = false;
#pragma unroll
                for (int e = 0; e < 8; ++e) any |= x[e] >= from && !(x[e] >= below);
                pending |= any ? 1u << (v - v0) / kThreads : 0u;
            });
#pragma unroll 1
            for (; pending && *static_cast<volatile int*>(&sh.n_list) <= kList; pending &= pending - 1) {
                const int v = v0 + (__ffs(pending) - 1) * kThreads;
                float x[8];
                p.load(v, x);
                look(x, v);
            }
        }
    }
    __syncthreads();
    const int n = sh.n_list;
    __syncthreads();
    return n;
}

// The smallest key whose value `holds`, as every larger one does, M's too:
// every wave tries 64 keys at a time.
template <class F>
__device__ __forceinline__ uint32_t edge(const Row& r, F&& holds) {
    uint32_t lo = 0x00800000u, hi = key_of(r.M);  // lo: the lowest finite key; hi holds
    const uint32_t lane = thread_id() % kWave;
#pragma unroll 1
    while (lo < hi) {
        const uint32_t step = max((hi - lo) / kWave, 1u), key = lo + lane * step;
        const uint64_t in = __ballot(key < hi && holds(value_of(key)));
        // keys below the first that is in are not; it is not below the one before it
        const uint32_t first = in ? static_cast<uint32_t>(__ffsll(static_cast<unsigned long long>(in)) - 1) : kWave;
        if (in) hi = lo + first * step;
        if (first > 0) {
            const uint32_t out = lo + (first - 1) * step;  // the last key tried that is not in
            lo = min(out, hi - 1) + 1;
        }
    }
    return hi;
}

constexpr int kDigit = 9;

// By wave 0: the first of 512 amounts up to which they add up to the goal (with
// what lies before them; 512: none), and what lies before that one.
__device__ __forceinline__ void find_digit(uint64_t before, uint64_t goal, uint64_t sum8, Shared& sh) {
    const int lane = thread_id();
    const uint64_t upto = before + wave_scan(sum8);
    const uint64_t reach = __ballot(upto >= goal);
    const int l = reach ? __ffsll(static_cast<unsigned long long>(reach)) - 1 : kWave - 1;
    const uint64_t one = lane < 8 ? sh.mass[8 * l + lane] : 0, run = of_lane(upto - sum8, l) + wave_scan(one);
    const uint64_t hit = __ballot(lane < 8 && run >= goal);
    if (lane == (hit ? __ffsll(static_cast<unsigned long long>(hit)) - 1 : 7)) {
        sh.digit = reach ? 8 * l + lane : 512;
        sh.before = run - one;
    }
}
// The lane's eight amounts of those.
__device__ __forceinline__ uint64_t eight(const Shared& sh) {
    const int tid = thread_id();
    uint64_t s = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) s += sh.mass[8 * tid + i];
    return s;
}

// The collected tokens: cut to a count (count > 0), then to a mass (mass > 0, as it
// is or as a share of theirs), each by key and among equals by index; then, if the
// rest is all that the row keeps, the token is drawn.  Returns the last cut made.
// No key is below `least`.
struct Targets {
    double count, mass;
    bool share, draw;
};
// w in units of 2^-50: the low bits of w + 4.  In a draw tokens without any mass are left out and the
// others have a unit at least: u = 0 draws the first that has any, however little.
__device__ __forceinline__ uint64_t amount_of(double w) {
    return static_cast<uint64_t>(__double_as_longlong(w + 4.0) - __double_as_longlong(4.0));
}
// The running sum that a mass to keep, and the one that a draw, has to reach.
__device__ __forceinline__ uint64_t goal_of(double t, uint64_t sum) { return min(t >= 1.0 ? static_cast<uint64_t>(ceil(t)) : 1, sum); }
// u sum exactly, as a sum may have more bits than a double: u = 1/2 of a row of two like halves draws from the second.
__device__ __forceinline__ uint64_t goal_of_draw(double u, uint64_t sum) {
    return min(static_cast<uint64_t>(static_cast<unsigned __int128>(static_cast<uint64_t>(u * 0x1p64)) * sum >> 64) + 1, sum);
}

// The draw from a few tokens: four threads compare each with a quarter of all, which
// gives their ranks; their amounts, put in that order, are summed up over a wave's lanes.
// 3.2 us for 20 tokens and 5 for 120, where digits take some eight rounds of 1.1.
constexpr int kFew = 256;
constexpr int kFewParts = kThreads / kFew, kPlaces = kFew / kWave;
// How many of others[n] come above this thread's (nothing, 0, is above none), to rank[].
template <class V, class F>
__device__ __forceinline__ void rank_of(V mine, int n, int* rank, F&& other) {
    const int tid = thread_id(), part = tid / kFew, per = (n + kFewParts - 1) / kFewParts;
    int above = 0;
#pragma unroll 4
    for (int i = part * per; i < min((part + 1) * per, n); ++i) above += other(i) > mine;
    if (mine && above) atomicAdd(rank + tid % kFew, above);
    __syncthreads();
}
struct Few {
    uint64_t upto[kPlaces], total;  // of this lane's places, of all
    // by one or more whole waves alike: the first n places
    __device__ __forceinline__ Few(const uint64_t* place, int n) {
        const int at = kPlaces * (thread_id() % kWave);
        uint64_t mine = 0;
#pragma unroll
        for (int e = 0; e < kPlaces; ++e) upto[e] = mine += at + e < n ? place[at + e] : 0;
        const uint64_t before = wave_scan(mine) - mine;
#pragma unroll
        for (int e = 0; e < kPlaces; ++e) upto[e] += before;
        total = of_lane(upto[kPlaces - 1], kWave - 1);
    }
    // the first place where they reach the goal, which is not above the total
    __device__ __forceinline__ int reach(uint64_t goal) const {
        int short_of = 0;
#pragma unroll
        for (int e = 0; e < kPlaces; ++e) short_of += __popcll(__ballot(upto[e] < goal));
        return short_of;
    }
};
__device__ __forceinline__ void draw_of_few(const Row& r, int n, const Targets& to, double u, int32_t* token, float* logprob, Shared& sh) {
    const int tid = thread_id(), at = tid % kFew;
    int* rank = reinterpret_cast<int*>(sh.mass);              // [2][kFew]: by logit, by index
    uint64_t* place = reinterpret_cast<uint64_t*>(sh.w);      // [2][kFew]
    uint32_t* index = reinterpret_cast<uint32_t*>(place + 2 * kFew);  // [kFew] of the kept, ~: larger is earlier
    if (tid < 2 * kFew) {
        rank[tid] = 0;
        place[tid] = 0;
    }
    // larger keys first, then smaller indices
    const uint64_t order = at < n ? sh.list[at] ^ 0xFFFFFFFFu : 0;
    const bool mine = tid < kFew && at < n;
    const double w = mine ? r.w(value_of(static_cast<uint32_t>(order >> 32))) : 0.0;
    const uint64_t amount = amount_of(w);
    __syncthreads();
    rank_of(order, n, rank, [&](int i) { return sh.list[i] ^ 0xFFFFFFFFu; });
    if (mine) place[rank[at]] = amount;
    __syncthreads();
    if (tid < kFew) {
        int keeps = to.count > 0.0 ? min(n, static_cast<int>(to.count)) : n;
        if (to.mass > 0.0) {
            const Few f(place, keeps);
            keeps = min(keeps, f.reach(goal_of(to.mass * (to.share ? static_cast<double>(f.total) : 0x1p50), f.total)) + 1);
        }
        index[tid] = mine && rank[at] < keeps && w >= r.min_p && w > 0.0 ? static_cast<uint32_t>(order) : 0;
    }
    __syncthreads();
    rank_of(index[at], n, rank + kFew, [&](int i) { return index[i]; });
    if (mine && index[at]) place[kFew + rank[kFew + at]] = max(amount, uint64_t{1});
    __syncthreads();
    if (tid >= kFew) return;
    const Few f(place + kFew, kFew);
    const int drawn = f.reach(goal_of_draw(u, f.total));
    if (mine && index[at] && rank[kFew + at] == drawn) {
        *token = static_cast<int32_t>(~index[at]);
        if (logprob) *logprob = static_cast<float>(log(w * 0x1p50 / static_cast<double>(f.total)));
    }
}

// Of bf16 logits the keys' upper 16 bits say which (low_bits 16).
__device__ __forceinline__ Cut cut_list(const Row& r, int n, uint32_t least, int low_bits, const Targets& to, double u,
                                        int32_t* token, float* logprob, Shared& sh) {
    constexpr uint32_t kDigits = 1u << kDigit;
    const int tid = thread_id();
    Cut cut{0, r.n};
    if (to.draw && n <= kFew) {
        draw_of_few(r, n, to, u, token, logprob, sh);
        return cut;
    }
#pragma unroll 1
    for (int i = tid; i < n; i += kThreads) sh.w[i] = r.w(value_of(static_cast<uint32_t>(sh.list[i] >> 32)));
    const uint32_t top = key_of(r.M) >> low_bits, depth = top - (least >> low_bits);
    uint64_t rest = 0;  // of the goal, for the ones that equal the last by key
    // 0, 1: count by key, by index; 2, 3: mass; 4: the draw
#pragma unroll 1
    for (int step = 0; step < 5; ++step) {
        if (step < 2 ? !(to.count > 0.0) : step < 4 ? !(to.mass > 0.0) : !to.draw) continue;
        const bool by_key = step == 0 || step == 2, draw = step == 4;
        const int bits = by_key ? 32 - __clz(depth | 1) : 32 - __clz(r.n), shift0 = (bits - 1) / kDigit * kDigit;
        uint32_t value = 0;
        uint64_t goal = 0, before = 0, sum = 0;
#pragma unroll 1
        for (int shift = shift0; shift >= 0; shift -= kDigit) {
            __syncthreads();
#pragma unroll 1
            for (int b = tid; b < static_cast<int>(kDigits); b += kThreads) sh.mass[b] = 0;
            __syncthreads();
#pragma unroll 1
            for (int i = tid; i < n; i += kThreads) {
                const uint64_t t = sh.list[i];
                const uint32_t key = static_cast<uint32_t>(t >> 32), idx = static_cast<uint32_t>(t), v = by_key ? top - (key >> low_bits) : idx;
                const double w = sh.w[i];
                bool in = cut.keeps(key, static_cast<int>(idx)) && (shift == shift0 || v >> (shift + kDigit) == value);
                if (!by_key) in = in && (draw ? w >= r.min_p && w > 0.0 : key >> low_bits == cut.key >> low_bits);
                uint64_t amount = step < 2 ? 1 : amount_of(w);
                if (draw) amount = max(amount, uint64_t{1});
                if (in) atomicAdd(reinterpret_cast<unsigned long long*>(&sh.mass[v >> shift & (kDigits - 1)]), static_cast<unsigned long long>(amount));
            }
            __syncthreads();
            if (tid < kWave) {
                const uint64_t mine = eight(sh);
                if (shift == shift0) {  // the goal, as of the sum
                    sum = wave_total(mine);
                    const double t = step == 0 ? to.count : to.share ? to.mass * static_cast<double>(sum) : to.mass * 0x1p50;
                    goal = by_key ? goal_of(t, sum) : draw ? goal_of_draw(u, sum) : min(rest, sum);
                    if (tid == 0) {
                        sh.goal = goal;
                        sh.sum = sum;
                    }
                }
                find_digit(before, goal, mine, sh);
            }
            __syncthreads();
            goal = sh.goal;
            sum = sh.sum;
            before = sh.before;
            value = value << kDigit | static_cast<uint32_t>(sh.digit);
        }
        if (by_key) {
            const uint32_t k = (top - value) << low_bits;  // a negative bf16 number's key ends in ones
            cut = Cut{low_bits && !(k >> 31) ? k | 0xFFFFu : k, r.n};
            rest = goal - before;
        } else if (!draw) {
            if (goal < sum) cut.last = static_cast<int>(value);  // else all of the equal ones
        } else {
#pragma unroll 1
            for (int i = tid; i < n; i += kThreads)
                if (static_cast<uint32_t>(sh.list[i]) == value) {
                    *token = static_cast<int32_t>(value);
                    if (logprob) *logprob = static_cast<float>(log(sh.w[i] * 0x1p50 / static_cast<double>(sum)));
                }
        }
    }
    return cut;
}

// The tokens of `in` weighed (or counted) in bins: where the running sum reaches
// `target` (of them, or of all of their mass), what lies above that bin, and
// their mass and the number of tokens down to it.
struct Found {
    int bin;  // kThreads: fewer tokens than the target have any mass
    double above, z, about;
};
template <class T>
__device__ __forceinline__ Found find_bin(const Pieces<T>& p, const Row& r, const Cut& in, bool by_mass, double target, Shared& sh) {
    const int tid = thread_id();
    __syncthreads();
    sh.mass[tid] = 0;
    __syncthreads();
    Found f;
    f.z = 0.0;
    each(p, r, [&](float x, int i) {
        if (!in.keeps(key_of(x), i)) return;
        int n;
        const double w = r.weight(r.depth(x), n);
        f.z += w;
        // w in units of 2^-42 of the bin's octave: the low bits of such a number + 2^10
        const int b = Row::bin_at(-n);
        if (b < kRowBins)
            atomicAdd(reinterpret_cast<unsigned long long*>(&sh.mass[b]),
                      static_cast<unsigned long long>(by_mass ? __double_as_longlong(ldexp(w, Row::start_of(b) >> 4) + 0x1p10) -
                                                                __double_as_longlong(0x1p10) : 1));
    });
    f.z = block_sum(f.z, sh);
    const double amount = static_cast<double>(sh.mass[thread_id()]);
    const int start = Row::start_of(thread_id());
    const double mine = by_mass ? ldexp(amount, -42 - (start >> 4)) : amount, upto = block_scan(mine, sh);
    if (tid == 0) sh.found = kThreads;
    if (tid == kThreads - 1) sh.found_d = upto;
    __syncthreads();
    const double aim = by_mass ? target * sh.found_d : target;
    first_thread(upto >= aim, &sh.found);
    __syncthreads();
    f.bin = sh.found;
    if (tid == f.bin) sh.above_d = upto - mine;
    // a bin's mass says how many tokens it has, to 2.2% either way down to 16 octaves
    f.about = block_sum(tid <= f.bin ? by_mass ? amount * 0x1p-42 * r.root[start & 15] : amount : 0.0, sh);
    f.above = sh.above_d;
    return f;
}

// What a row asks for.
struct Wants {
    double c16, min_p, prob, u;
    int k;
    bool greedy;
    __device__ Wants(const SampleArgs& a, int row) {
        const float t0 = a.temperature ? a.temperature[row] : 1.f, low0 = a.min_p ? a.min_p[row] : 0.f;
        const float p0 = a.top_p ? a.top_p[row] : 1.f, x0 = a.u[row];
        const int32_t k0 = a.top_k ? a.top_k[row] : 0;
        const float t = uniform(t0), low = uniform(low0), p = uniform(p0), x = uniform(x0);
        const int32_t top_k = uniform(k0);
        greedy = !(t > 0.f);
        c16 = uniform(16.0 * 1.4426950408889634074 / static_cast<double>(t));
        min_p = uniform(low > 0.f ? fmin(static_cast<double>(low), 1.0) : 0.0);
        k = top_k > 0 && top_k < a.vocab ? top_k : 0;
        prob = uniform(p < 1.f ? fmax(static_cast<double>(p), 0.0) : 1.0);
        u = uniform(x > 0.f ? fmin(static_cast<double>(x), 0x1.fffffffffffffp-1) : 0.0);
    }
    __device__ bool free() const { return !greedy && k == 0 && prob >= 1.0 && min_p == 0.0; }
    __device__ bool by_mass() const { return !greedy && k == 0 && prob < 1.0; }
    __device__ bool by_count() const { return !greedy && k > 0 && k <= kThreads; }
};

// 1. What is known of a slice.
template <class T>
__global__ __launch_bounds__(kThreads, 8) void sample_slices_kernel(SampleArgs a) {
    __shared__ double root[16];
    __shared__ __attribute__((aligned(16))) float ends[16];
    __shared__ uint64_t bins[kBins];
    __shared__ f32x4 held[kHeld];
    __shared__ uint64_t red_u[kWaves];
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    const size_t slice = blockIdx.x;
    const int row = static_cast<int>(slice / a.slices);
    // the first pieces, which wait in LDS to be weighed, are asked for before all else
    constexpr int kRegs = sizeof(T) / 2, kWait = kHeld / kRegs, kFirst = kWait / kThreads;
    const Pieces<T> p(static_cast<const T*>(a.logits) + row * a.ld, a.vocab, ends);
    const int per = slice_pieces(p.count, a.slices), from = static_cast<int>(slice % a.slices) * per, to = min(from + per, p.count);
    typename Pieces<T>::Raw first[kFirst];
#pragma unroll
    for (int q = 0; q < kFirst; ++q) first[q] = p.ask(from + tid + q * kThreads);
    const Wants want(a, row);
    if (tid < 16) root[tid] = exp2(tid / 16.0);
    for (int b = tid; b < kBins; b += kThreads) bins[b] = 0;
    __syncthreads();

    // the thread's largest logit and the first piece that has it (NaN is below everything)
    float mine = -INFINITY;
    int at = -1;
    auto look = [&](const float (&x)[8], int v) {
        const float m = largest(x);
        if (m > mine) {
            mine = m;
            at = v;
        }
    };
#pragma unroll
    for (int q = 0; q < kFirst; ++q) {
        const int v = from + tid + q * kThreads;
#pragma unroll
        for (int i = 0; i < kRegs; ++i) held[i * kWait + v - from] = first[q].w[i];
        float x[8];
        p.spread(first[q], v, x);
        if (v < to) look(x, v);
    }
    each_piece<4>(p, from + tid + kWait, to, kThreads, look);
    // a piece once more
    auto again = [&](int v, float (&x)[8]) {
        typename Pieces<T>::Raw raw;
        if (v - from < kWait) {
#pragma unroll
            for (int i = 0; i < kRegs; ++i) raw.w[i] = held[i * kWait + v - from];
        } else {
            raw = p.ask(v);
        }
        p.spread(raw, v, x);
    };
    uint64_t best = 0;
    if (at >= 0) {
        float x[8];
        again(at, x);
        int i = 0;
#pragma unroll
        for (int e = 7; e >= 0; --e)
            if (x[e] == mine) i = 8 * at - p.shift + e;
        best = static_cast<uint64_t>(key_of(mine)) << 32 | (0xFFFFFFFFu - static_cast<uint32_t>(i));
    }
    best = wave_max(best);
    if (lane == 0) red_u[wave] = best;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) best = max(best, red_u[w]);
    if (tid == 0) a.best[slice] = best;
    if (!want.greedy && !want.free()) {  // of four threads together from sixteen slices on, of two from eight on
        const int group = group_size(a.slices);
        if (group >= 2) mine = fmaxf(mine, __shfl_xor(mine, 1, kWave));
        if (group >= 4) mine = fmaxf(mine, __shfl_xor(mine, 2, kWave));
        if (tid % group == 0)
            a.most[static_cast<size_t>(row) * kMost + (slice % a.slices) * (kThreads / group) + tid / group] = key_of(mine);
    }
    const float m = value_of(static_cast<uint32_t>(best >> 32));
    const bool by_mass = want.by_mass() && best != 0 && m != INFINITY;
    if (!by_mass && !want.free()) return;

    double s = 0.0;
    if (by_mass) {
        // By bins of whole sixteenths of an octave, which all slices share; in units of
        // 2^-42 of the bin's w.  Far from logit 0 single precision knows no sixteenths: such a
        // slice has no bins.
        const bool near = near_zero(m, want.c16);
        const float c = static_cast<float>(want.c16), first = near ? sixteenth(m, c) : -0x1p30f, floor = first - kBins;
        const int ref = uniform(static_cast<int>(first));
        if (tid == 0) a.ref[slice] = ref;
        if (!near) return;
#pragma unroll 1
        for (int v = from + tid; v < to; v += kThreads) {
            float x[8];
            again(v, x);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                // Nothing that has a mass lies above the slice's largest, and what has none (-inf, NaN, places beside
                // the row) comes to -inf or NaN in sixteenths, also where c is 0: `floor`, which is in no bin.
                const float whole = fmaxf(sixteenth(x[e], c), floor);
                const double f = fma(static_cast<double>(x[e]), want.c16, -static_cast<double>(whole));
                const int n = static_cast<int>(whole);
                if (ref - n < kBins - 1)
                    atomicAdd(reinterpret_cast<unsigned long long*>(&bins[ref - n]), static_cast<unsigned long long>(Row::units(f)));
            }
        }
        __syncthreads();
        for (int b = tid; b < kBins; b += kThreads) a.bins[slice * kBins + b] = bins[b];
        return;
    }
    // of a sixteenth of the slice each wave, from the slice's largest logit
    Row r;
    r.at_inf = m == INFINITY;
    r.M = r.at_inf || best == 0 ? 0.f : m;
    r.c16 = want.c16;
    r.root = (const __attribute__((address_space(3))) double*)root;
    const int each_wave = per / kWaves, v1 = min(from + (wave + 1) * each_wave, to);
#pragma unroll 1
    for (int v = from + wave * each_wave + lane; v < v1; v += kWave) {
        float x[8];
        again(v, x);
        if (r.at_inf)
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = r.fix(x[e]);
        double w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = r.w(x[e]);
        s += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
    }
    s = wave_total(s);
    if (lane == 0) a.sums[slice * kWaves + wave] = best ? s : 0.0;
}

// The bin of the slices' masses where the running sum reaches prob of all of it; masses
// as of M = 1, bins counted from `ref` down.
__device__ __forceinline__ Found find_bin_of_slices(const SampleArgs& a, int row, const Row& r, double prob, int ref, Shared& sh) {
    const int tid = threadIdx.x;
    const size_t s0 = static_cast<size_t>(row) * a.slices;
    const bool has = tid < kBins - 1;
    uint64_t mass = 0;
#pragma unroll 8
    for (int s = 0; s < a.slices; ++s) {
        const int b = tid - (ref - sh.ref[s]);  // the slice's bin that is this thread's
        mass += has && b >= 0 && sh.best[s] ? a.bins[(s0 + s) * kBins + b] : 0;
    }
    int n;
    const double tokens = static_cast<double>(mass) * 0x1p-42;  // nearly
    double mine = tokens * r.weight_from(ref - tid - static_cast<double>(anew(r.M)) * r.c16, 0, n);
    if (tid == 0) {
        // In M's bin by what one M adds to it, so that M weighs 1 here as in the lists.  Only among equal
        // logits does prob of the mass end with a token exactly; m of them come to m, where the factor
        // above, the product of two approximations, makes it m (1 + 1e-14) and one token more.
        const uint64_t one = Row::units(fma(static_cast<double>(anew(r.M)), r.c16, -static_cast<double>(ref)));
        const double inv = 1.0 / static_cast<double>(one), whole = rint(static_cast<double>(mass) * inv);
        mine = whole + static_cast<double>(static_cast<int64_t>(mass - static_cast<uint64_t>(whole) * one)) * inv;
    }
    const double upto = block_scan(mine, sh);
    if (tid == 0) sh.found = kThreads;
    if (tid == kBins - 2) sh.found_d = upto;
    __syncthreads();
    Found f;
    f.z = sh.found_d;
    first_thread(has && upto >= prob * f.z, &sh.found);
    __syncthreads();
    f.bin = sh.found;
    if (tid == f.bin) sh.above_d = upto - mine;
    f.about = block_sum(has && tid <= f.bin ? tokens : 0.0, sh);
    f.above = sh.above_d;
    return f;
}

// 2. The token of a row.
template <class T>
__global__ __launch_bounds__(kThreads) void sample_rows_kernel(SampleArgs a) {
    __shared__ Shared sh;
    const int row = blockIdx.x, tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    // what only some rows need is asked for before it is known which: all of it is a microsecond away
    const size_t slice0 = static_cast<size_t>(row) * a.slices;
    double range_sum = tid < a.slices * kWaves ? a.sums[slice0 * kWaves + tid] : 0.0;
    uint32_t most[kMost / kThreads];
#pragma unroll
    for (int s = 0; s < kMost / kThreads; ++s) most[s] = s < a.slices ? a.most[static_cast<size_t>(row) * kMost + s * kThreads + tid] : 0;
    const Wants want(a, row);
    if (tid < a.slices) {
        const uint64_t key = a.best[slice0 + tid];
        const int32_t ref = a.ref[slice0 + tid];
        sh.best[tid] = key;
        sh.ref[tid] = key ? ref : 0;  // a slice of nothing has none
    }
    const Pieces<T> p(static_cast<const T*>(a.logits) + row * a.ld, a.vocab, sh.ends);
    if (tid < 16) sh.root[tid] = exp2(tid / 16.0);
    if (tid == 0) {
        sh.found = kThreads;
        sh.digit = 0;
    }
    __syncthreads();
    uint64_t best = 0;
#pragma unroll 1
    for (int s = 0; s < a.slices; ++s) best = max(best, sh.best[s]);
    best = uniform(best);
    int32_t* token = a.tokens + row;
    float* logprob = a.logprob ? a.logprob + row : nullptr;
    if (best == 0 || want.greedy) {
        if (tid == 0) {
            *token = best == 0 ? -1 : static_cast<int32_t>(0xFFFFFFFFu - static_cast<uint32_t>(best));
            if (logprob) *logprob = best == 0 ? -INFINITY : 0.f;
        }
        return;
    }
    Row r;
    r.M = value_of(static_cast<uint32_t>(best >> 32));
    r.at_inf = r.M == INFINITY;
    if (r.at_inf) r.M = 0.f;
    r.c16 = want.c16;
    r.min_p = want.min_p;
    r.n = a.vocab;
    r.root = (const __attribute__((address_space(3))) double*)sh.root;
    const int k = want.k;
    const double prob = want.prob;
    double z = 0.0, before = 0.0, target = 0.0;
    int from = 0, to = p.count;
    bool summed = false;
    Cut cut{0, a.vocab};

    if (want.free()) {
        // the slices' sixteenths count from the slice's own largest
        double mine = range_sum;
        if (tid < a.slices * kWaves) {
            const int s = tid / kWaves;
            const float m = value_of(static_cast<uint32_t>(sh.best[s] >> 32));
            mine *= !sh.best[s] ? 0.0 : r.at_inf ? (m == INFINITY ? 1.0 : 0.0) : r.w(m);
            // A sixteenth to draw from needs a token whose own w is not 0: of its 2^16 tokens at most
            // one has 2^-1066 then.
            if (mine < 0x1p-1050) mine = 0.0;
        }
        const double upto = block_scan(mine, sh);
        if (tid == kThreads - 1) sh.found_d = upto;
        __syncthreads();
        z = uniform(sh.found_d);
        target = want.u * z;
        first_thread(mine > 0.0 && upto > target, &sh.found);
        const uint64_t any = __ballot(mine > 0.0);  // the last with any mass, where rounding leaves none
        if (any && lane == 0) atomicMax(&sh.digit, tid + 63 - __clzll(static_cast<long long>(any)));
        __syncthreads();
        const int range = uniform(sh.found < kThreads ? sh.found : sh.digit), width = slice_pieces(p.count, a.slices) / kWaves;
        if (tid == range) sh.above_d = upto - mine;
        __syncthreads();
        before = uniform(sh.above_d);
        from = range * width;
        to = min(from + width, p.count);
        summed = true;
    }

    // the slices' bins count, where sixteenths from 0 on are as good as from M on
    // (slices that have none, as they are further from it, are 2^-64 of M at most then)
    const bool slices = want.by_mass() && !r.at_inf && near_zero(r.M, r.c16, 1024.0);
    const float c16 = static_cast<float>(r.c16);
    const int ref = slices ? static_cast<int>(sixteenth(r.M, c16)) : 0;
    auto bin_of = [&](float x) {  // a whole number; far down beyond any int
        return slices ? static_cast<float>(ref) - sixteenth(x, c16) : static_cast<float>(r.bin_of(x));
    };
    int bin = -1, listed = 0;  // the bin of the cut, whose kept tokens are among those in LDS

    // 0: top_k by the threads' largest; 1: top_k by bins, where that is no help; 2: top_p; 3: min_p alone
#pragma unroll 1
    for (int way = 0; way < 4; ++way) {
        if (way == 0 ? !want.by_count() : way == 1 ? k == 0 : way == 2 ? prob >= 1.0 : r.min_p == 0.0) continue;
        uint32_t lo;
        float hi = INFINITY;
        double mass = 0.0;
        Targets goal{};
        if (way == 0) {
            // a bound of the k-th largest of the threads' largest: counts by the distance of
            // their keys' upper 16 bits from M's, in steps of 1, 16, 256, ...
            const uint32_t top = key_of(r.M) >> 16;
            uint32_t down = 0;
#pragma unroll 1
            for (int step = 0; step < 16; step += 4) {
                __syncthreads();
                if (tid < 512) sh.mass[tid] = 0;
                __syncthreads();
#pragma unroll
                for (int s = 0; s < kMost / kThreads; ++s) {
                    uint32_t key = most[s];
                    if (r.at_inf) key = key_of(r.fix(value_of(key)));
                    const uint32_t far = (top - (key >> 16)) >> step;
                    if (far < 512) atomicAdd(reinterpret_cast<unsigned int*>(&sh.mass[far]), 1u);
                }
                __syncthreads();
                if (tid < kWave) find_digit(0, k, eight(sh), sh);
                __syncthreads();
                down = ((static_cast<uint32_t>(sh.digit) + 1) << step) - 1;
                if (sh.digit < 512) break;
            }
            // as far as -inf, fewer threads than k have any: all tokens, where LDS holds them (256
            // rows of 1000 with top_k and top_p 35 us, by bins 47)
            const bool none = down >= top - (0x007FFFFFu >> 16);
            if (none && r.n > kList) continue;
            lo = none ? 0x00800000u : (top - down) << 16;
            goal = Targets{static_cast<double>(k), prob < 1.0 ? fmax(prob, 0x1p-1000) : 0.0, true, true};
        } else {
            const bool by_mass = way == 2, low = way == 3;
            if (!low) {
                const Found f = by_mass && slices ? find_bin_of_slices(a, row, r, prob, ref, sh)
                                                  : find_bin(p, r, cut, by_mass, by_mass ? prob : k, sh);
                if (f.bin == kThreads) continue;
                bin = f.bin;
                mass = f.z;
                // the tokens down to the bin where LDS holds them, else the bin's alone
                const bool all = by_mass && f.about < 0.97 * kList;
                if (by_mass) goal = Targets{0.0, fmax(prob * mass - (all ? 0.0 : f.above), 0x1p-1000), false, all};
                else goal = Targets{k - f.above, 0.0, false, false};
            } else {
                goal.draw = true;
            }
            // the edges of the tokens to collect
            lo = 0;
#pragma unroll 1
            for (int i = 0; i < (goal.draw || bin == 0 ? 1 : 2); ++i) {
                const uint32_t e = edge(r, [&](float x) { return low ? r.w(x) >= r.min_p : bin_of(x) <= bin - i; });
                if (i == 0) lo = e;
                else hi = value_of(e);
            }
            if (low && lo <= cut.key) continue;  // the cut is above it
        }
        const int n = collect(p, r, value_of(lo), hi, cut, most, a.slices, sh);
        listed = n <= kList ? n : -1;
        if (n <= kList) {
            const Cut c = cut_list(r, n, lo, sizeof(T) == 2 ? 16 : 0, goal, want.u, token, logprob, sh);
            if (goal.draw) return;
            cut = c;
        } else if (way == 3) {
            cut = Cut{lo, a.vocab};
        } else if (way > 0) {
            cut = bisect(p, r, cut, way == 2, way == 2 ? fmax(prob * mass, 0x1p-1000) : k, sh);
        }
    }

    if (slices && !summed && listed >= 0) {
        // A slice's kept mass: its bins above the cut's, and the kept tokens of that bin.  A wave a slice.
        double s = 0.0;
        uint64_t listed_mass = 0;  // whole units, as the list's order is any
        if (wave < a.slices && sh.best[wave]) {
            const int down = ref - sh.ref[wave], width = slice_pieces(p.count, a.slices);
            // bins 64 apart are four octaves apart
            const uint64_t* bins = a.bins + (slice0 + wave) * kBins;
#pragma unroll 4
            for (int b = (min(bin - down, kBins - 1) - 1 - lane) / kWave * kWave + lane; b >= 0; b -= kWave)
                s = s * 0x1p-4 + (b < bin - down ? static_cast<double>(bins[b]) : 0.0);
            int n;
            s *= 0x1p-42 * r.weight_from(ref - down - lane - static_cast<double>(anew(r.M)) * r.c16, 0, n);
#pragma unroll 1
            for (int i = lane; i < listed; i += kWave) {
                const uint64_t t = sh.list[i];
                const int idx = static_cast<int>(static_cast<uint32_t>(t));
                if (idx + p.shift - 8 * width * wave >= 0 && idx + p.shift - 8 * width * (wave + 1) < 0 && cut.keeps(static_cast<uint32_t>(t >> 32), idx))
                    listed_mass += amount_of(r.w(value_of(static_cast<uint32_t>(t >> 32))));
            }
        }
        s = wave_total(s) + static_cast<double>(wave_total(listed_mass)) * 0x1p-50;
        __syncthreads();
        if (lane == 0) sh.red_d[wave] = s;
        __syncthreads();
        const Part part = find_part(0.0, want.u, 0.0, sh);
        z = part.total;
        target = want.u * z;
        before = part.before;
        from = part.at * slice_pieces(p.count, a.slices);
        to = min(from + slice_pieces(p.count, a.slices), p.count);
        summed = true;
    }

    // The kept tokens' mass in sixteenths of the range, a wave each.  Under a cut most
    // tokens are out: a wave queues those that are in, in any order, and weighs 64 at a time.
    const float cut_x = cut.key == 0 ? -INFINITY : value_of(cut.key);
    float* queue = sh.queue[wave];
    auto kept = [&](float x, int i) { return x > cut_x || (x == cut_x && i <= cut.last); };
    __syncthreads();
#pragma unroll 1
    while (!summed || to - from > kWave) {
        const int per = ((to - from + kWaves - 1) / kWaves + kWave - 1) / kWave * kWave;
        const int v1 = min(from + (wave + 1) * per, to);
        double s = 0.0;
        int n = 0;
        auto weigh = [&](int least) {  // 64 at a time, while there are that many
#pragma unroll 1
            while (n >= least) {
                const int m = min(n, kWave);
                n -= m;
                const double w = lane < m ? r.w(queue[n + lane]) : 0.0;
                s += w >= r.min_p ? w : 0.0;
            }
            wave_fence();
        };
        // whole waves: pieces past the range count as -inf
        each_piece<1>(p, from + wave * per + lane, (v1 - (from + wave * per) + kWave - 1) / kWave * kWave + from + wave * per, kWave,
                   [&](const float (&x)[8], int v) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float y = r.at_inf ? r.fix(x[e]) : x[e];
                const bool in = v < v1 && kept(y, 8 * v - p.shift + e) && y > -INFINITY;
                const uint64_t mask = __ballot(in);
                const int at = n + __builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(mask >> 32),
                                                             __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(mask), 0));
                if (in) queue[at] = y;
                n += __popcll(mask);
            }
            wave_fence();
            weigh(kWave);
        });
        weigh(1);
        s = wave_total(s);
        __syncthreads();
        if (lane == 0) sh.red_d[wave] = s;
        __syncthreads();
        const Part part = find_part(before, summed ? -1.0 : want.u, target, sh);
        if (!summed) {
            z = part.total;
            target = want.u * z;
            summed = true;
        }
        before = part.before;
        from += part.at * per;
        to = min(from + per, to);
    }
    if (wave > 0) return;
    // one wave: 64 pieces, whose lanes' eight weights go through LDS
    {
        float x[8];
        p.load(from + lane, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) queue[8 * lane + e] = from + lane >= to ? -INFINITY : r.at_inf ? r.fix(x[e]) : x[e];
    }
    wave_fence();
    const int i0 = 8 * (from + lane) - p.shift;
    auto weigh = [&](int e) {
        const float x = queue[8 * lane + e];
        const double w = kept(x, i0 + e) ? r.w(x) : 0.0;
        return w >= r.min_p ? w : 0.0;
    };
    double sum = 0.0;
#pragma unroll 1
    for (int e = 0; e < 8; ++e) sum += weigh(e);
    const double upto = before + wave_scan(sum);
    const uint64_t here = __ballot(upto > target && sum > 0.0), some = __ballot(sum > 0.0);
    const int l = here ? __ffsll(static_cast<unsigned long long>(here)) - 1 : 63 - __clzll(static_cast<long long>(some));
    if (lane != l) return;
    double run = upto - sum, wb = 0.0;
    int chosen = -1;
#pragma unroll 1
    for (int e = 0; e < 8 && !(chosen >= 0 && run > target); ++e) {
        const double w = weigh(e);
        if (w <= 0.0) continue;
        run += w;
        chosen = i0 + e;
        wb = w;
    }
    *token = chosen;
    if (logprob) *logprob = static_cast<float>(log(wb / z));
}

// Slices of a row, a power of two: a work-group for every CU, of a piece a thread at
// least, and of four at most.  us with slices of 8192 / 16384 / 32768 / 65536 tokens: 64
// rows of 131072 with top_p 72 / 65 / 62 / -, with no filter 33 / 28 / 26 / -; 256 rows - / - / 91 / 99;
// 256 rows of 32768 62 / 57 / 53 and with top_k 36 / 31 / 36; 8 rows with no filter 18 / 21.
constexpr int kLongSlice = 4 * 8 * kThreads;
int sample_slices(int64_t rows, int vocab) {
    int slices = 1;
    while (slices < kMostSlices && slices * 8 * kThreads < vocab && (slices * rows < 256 || slices * kLongSlice < vocab) &&
           2 * slices * rows < 1 << 22)  // what a grid can have of 1024 threads
        slices *= 2;
    return slices;
}

// Places of a call's workspace; the most slices of any call of up to `rows` rows.
struct SampleLayout {
    size_t best, ref, sums, bins, most, end;
};
SampleLayout sample_layout(size_t slices, size_t rows) {
    SampleLayout l{};
    size_t off = 0;
    auto take = [&](size_t bytes) {
        const size_t at = off;
        off += (bytes + 255) / 256 * 256;
        return at;
    };
    l.best = take(slices * 8);
    l.ref = take(slices * 4);
    l.sums = take(slices * kWaves * 8);
    l.bins = take(slices * kBins * 8);
    l.most = take(rows * kMost * 4);
    l.end = off;
    return l;
}

template <class T>
void launch_sample(const SampleArgs& a, hipStream_t s) {
    const unsigned rows = static_cast<unsigned>(a.rows), slices = rows * static_cast<unsigned>(a.slices);
    sample_slices_kernel<T><<<slices, kThreads, 0, s>>>(a);
    sample_rows_kernel<T><<<rows, kThreads, 0, s>>>(a);
}

}  // namespace
}  // namespace slw

using namespace slw;

extern "C" int slw_sample_workspace_size(int32_t max_rows, int32_t vocab, size_t* bytes) {
    return guarded([&] {
        if (!bytes) return fail(SLW_EINVAL, "null argument");
        if (max_rows < 0) return fail(SLW_EINVAL, "negative rows");
        if (max_rows > SLW_SAMPLE_MAX_ROWS) return fail(SLW_EUNSUPPORTED, "more than %d rows", SLW_SAMPLE_MAX_ROWS);
        if (vocab < 1 || vocab > SLW_SAMPLE_MAX_VOCAB)
            return fail(SLW_EUNSUPPORTED, "vocab must be in [1, %d] (got %d)", SLW_SAMPLE_MAX_VOCAB, vocab);
        // the slices of a call are fewer than twice 256, or those that the vocabulary asks for, and those of one row each at most
        const size_t rows = static_cast<size_t>(max_rows), of_any = sample_slices(1, vocab), of_many = sample_slices(256, vocab);
        *bytes = rows ? sample_layout(std::min(std::max<size_t>(rows * of_many, 511), rows * of_any), rows).end : 0;
        return SLW_OK;
    });
}

extern "C" int slw_sample(const slw_sample_args* a, void* ws, size_t ws_bytes, void* stream) {
    return guarded([&] {
        if (!a) return fail(SLW_EINVAL, "null argument");
        if (a->rows < 0) return fail(SLW_EINVAL, "negative rows");
        if (a->rows > SLW_SAMPLE_MAX_ROWS) return fail(SLW_EUNSUPPORTED, "more than %d rows", SLW_SAMPLE_MAX_ROWS);
        if (a->vocab < 1 || a->vocab > SLW_SAMPLE_MAX_VOCAB)
            return fail(SLW_EUNSUPPORTED, "vocab must be in [1, %d] (got %d)", SLW_SAMPLE_MAX_VOCAB, a->vocab);
        if (a->logits_f32 != 0 && a->logits_f32 != 1) return fail(SLW_EINVAL, "logits_f32 must be 0 or 1");
        if (a->rows == 0) return SLW_OK;
        if (!a->logits || !a->u || !a->tokens) return fail(SLW_EINVAL, "null argument");
        const size_t one = a->logits_f32 ? 4 : 2;
        if (reinterpret_cast<uintptr_t>(a->logits) % one || a->ld < a->vocab)
            return fail(SLW_EINVAL, "logits: aligned to their type, stride at least %d (got %lld)", a->vocab, (long long)a->ld);
        const void* words[] = {a->temperature, a->top_k, a->top_p, a->min_p, a->u, a->tokens, a->logprob};
        for (const void* p : words)
            if (reinterpret_cast<uintptr_t>(p) % 4) return fail(SLW_EINVAL, "parameters, tokens and logprob must be 4-byte aligned");
        SampleArgs g{};
        g.slices = sample_slices(a->rows, a->vocab);
        const size_t slices = static_cast<size_t>(a->rows) * g.slices;
        const SampleLayout l = sample_layout(slices, a->rows);
        if (!ws || reinterpret_cast<uintptr_t>(ws) % 16) return fail(SLW_EINVAL, "the workspace must be 16-byte aligned device memory");
        if (ws_bytes < l.end) return fail(SLW_ENOMEM, "the workspace holds %zu bytes, %d rows need %zu", ws_bytes, a->rows, l.end);
        g.logits = a->logits;
        g.ld = a->ld;
        g.temperature = a->temperature;
        g.top_k = a->top_k;
        g.top_p = a->top_p;
        g.min_p = a->min_p;
        g.u = a->u;
        g.tokens = a->tokens;
        g.logprob = a->logprob;
        g.vocab = a->vocab;
        g.rows = a->rows;
        char* w = static_cast<char*>(ws);
        g.best = reinterpret_cast<uint64_t*>(w + l.best);
        g.ref = reinterpret_cast<int32_t*>(w + l.ref);
        g.sums = reinterpret_cast<double*>(w + l.sums);
        g.bins = reinterpret_cast<uint64_t*>(w + l.bins);
        g.most = reinterpret_cast<uint32_t*>(w + l.most);
        hipStream_t s = static_cast<hipStream_t>(stream);
        if (a->logits_f32) launch_sample<float>(g, s);
        else launch_sample<bf16>(g, s);
        HIP_TRY(hipGetLastError());
        return SLW_OK;
    });
}
