// The next token of each row of logits, from a given random number.
//
// w_t = 2^((x_t - M) log2(e) / T), M the largest logit.  The filters keep a head
// of the tokens sorted by (logit descending, index ascending): the first top_k;
// of those, the ones with less than top_p of their mass before them; of those,
// w >= min_p.  So every filter is a cut in that order, (key, index) of the last
// token kept, and no row is ever sorted whole.  One work-group a row:
//   1. a pass finds M, and each thread's largest logit;
//   2. top_k up to the number of threads: the k-th largest of the threads' largest
//      bounds the k-th largest logit from below, and a pass collects what is not
//      below it, a little more than k tokens, in LDS; they are sorted, cut, sorted
//      by index, and the token is drawn;
//   3. top_p: a pass weighs the tokens in bins of 1/16 octave of w; the running sum
//      over bins says in which one the cut is.  The tokens down to that bin are
//      collected as above, or where they are too many those of the bin alone, which
//      gives the cut;
//   4. with no filter, or a cut of more tokens than LDS holds, the token is found by
//      sums of the kept w over sixteenths of the row, then of that sixteenth, ...
//
// Every mass is held in 64 bits: w from an exponential good to 2^-37, bins in
// fixed point (integer sums: the order of the atomics does not matter), all else
// in doubles summed in a fixed order.  With fp32 sums one draw in a few hundred
// would be another token; a result depends on the row alone.
#include <math.h>

#include <algorithm>

#include "device.h"
#include "hip_try.h"
#include "kernels.h"

namespace slw {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / kWave;
constexpr int kBins = 768;          // 16 for an octave; the last one holds w < 2^-47 and is weighed nowhere
constexpr int kQueue = 8 * kWave + 64;  // logits a wave has queued: a piece of every lane beside 63 left over
constexpr int kList = 4096;         // tokens sorted in LDS

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
    int vocab;
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
    __device__ __forceinline__ double weight(double t, int& n) const {
        const double whole = rint(t), f = t - whole;
        n = static_cast<int>(whole);
        const double p = fma(f, fma(f, fma(f, fma(f, 0x1.3b2c4ac7eb38ap-23, 0x1.c6b3488226c3bp-17), 0x1.ebfbdff6988cep-11),
                                    0x1.62e42fee4615cp-5), 1.0);
        return ldexp(p * root[n & 15], n >> 4);
    }
    __device__ __forceinline__ double w(float x) const {
        int n;
        return weight(depth(x), n);
    }
    __device__ __forceinline__ int bin_of(float x) const { return min(-static_cast<int>(rint(depth(x))), kBins - 1); }
};

struct Shared {
    union {
        uint64_t list[kList];
        float queue[kWaves][kQueue];
    };
    uint64_t mass[kBins];
    double root[16];
    double red_d[kWaves];
    uint64_t red_u[kWaves];
    int n_list, found, digit;
    uint64_t before;
    double found_d, above_d;
};

__device__ __forceinline__ double wave_sum_d(double v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
    return v;
}

// LDS accesses of the lanes of one wave keep their order across it.
__device__ __forceinline__ void wave_fence() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

// Threads that deal with a list together: the work-group, or one wave of it alone,
// which needs no barriers.
struct Group {
    bool solo;
    __device__ __forceinline__ int size() const { return solo ? kWave : kThreads; }
    __device__ __forceinline__ void sync() const {
        wave_fence();
        if (!solo) __syncthreads();
    }
    __device__ __forceinline__ uint64_t sum(uint64_t v, Shared& sh) const {
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
        if (solo) return v;
        __syncthreads();
        if (threadIdx.x % kWave == 0) sh.red_u[threadIdx.x / kWave] = v;
        __syncthreads();
        v = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) v += sh.red_u[w];
        return v;
    }
};

// Sum over the work-group, in a fixed order, on every thread.
__device__ __forceinline__ double block_sum(double v, Shared& sh) {
    v = wave_sum_d(v);
    __syncthreads();
    if (threadIdx.x % kWave == 0) sh.red_d[threadIdx.x / kWave] = v;
    __syncthreads();
    v = 0.0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) v += sh.red_d[w];
    return v;
}

// Inclusive sums over the work-group's threads, in thread order.
__device__ __forceinline__ double block_scan(double v, Shared& sh) {
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const double p = __shfl_up(v, o, kWave);
        if (lane >= o) v += p;
    }
    __syncthreads();
    if (lane == kWave - 1) sh.red_d[wave] = v;
    __syncthreads();
    double before = 0.0;
#pragma unroll
    for (int w = 0; w < kWaves - 1; ++w) before += w < wave ? sh.red_d[w] : 0.0;
    return before + v;
}

__device__ __forceinline__ uint64_t block_max(uint64_t v, Shared& sh) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        const uint64_t p = __shfl_xor(v, o, kWave);
        v = p > v ? p : v;
    }
    __syncthreads();
    if (threadIdx.x % kWave == 0) sh.red_u[threadIdx.x / kWave] = v;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) v = sh.red_u[w] > v ? sh.red_u[w] : v;
    return v;
}

// The row in pieces of 8 tokens, aligned to 16 bytes as far as the row's start
// allows: piece v holds tokens 8 v - shift .. + 7, those outside the row as -inf.
template <class T>
struct Pieces {
    const T* row;
    int n, shift, count;
    __device__ Pieces(const T* r, int n_) : row(r), n(n_) {
        shift = static_cast<int>(reinterpret_cast<uintptr_t>(r) % 16 / sizeof(T));
        count = (n + shift + 7) / 8;
    }
    __device__ void load(int v, float (&x)[8]) const {
        const int at = 8 * v - shift;
        if (at >= 0 && at + 8 <= n) {
            if (sizeof(T) == 2) {
                const bf16x8 t = *reinterpret_cast<const bf16x8*>(row + at);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = static_cast<float>(t[e]);
            } else {
                const f32x4 a = *reinterpret_cast<const f32x4*>(row + at), b = *reinterpret_cast<const f32x4*>(row + at + 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[e] = a[e];
                    x[4 + e] = b[e];
                }
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = at + e >= 0 && at + e < n ? static_cast<float>(row[at + e]) : -INFINITY;
        }
    }
};

// Every token of the row, f(x, index); a row with +inf as Row::fix has it.  Up to 14
// places outside the row come too, as -inf.
template <class T, class F>
__device__ __forceinline__ void each(const Pieces<T>& p, const Row& r, F&& f) {
#pragma unroll 1
    for (int v = threadIdx.x; v < p.count; v += kThreads) {
        float x[8];
        p.load(v, x);
        if (r.at_inf)
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = r.fix(x[e]);
#pragma unroll
        for (int e = 0; e < 8; ++e) f(x[e], 8 * v - p.shift + e);
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
            if (i >= 0 && i < p.n && in.keeps(k, i) && c.keeps(k, i)) s += by_mass ? r.w(x) : 1.0;
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

// Tokens of `in` with lo <= key < hi, in LDS (in any order); how many there are, of which the first kList are there.
template <class T>
__device__ __forceinline__ int collect(const Pieces<T>& p, const Row& r, uint32_t lo, uint32_t hi, const Cut& in, Shared& sh) {
    __syncthreads();
    if (threadIdx.x == 0) sh.n_list = 0;
    __syncthreads();
#pragma unroll 1
    for (int v = threadIdx.x; v < p.count; v += kThreads) {
        float x[8];
        p.load(v, x);
        if (r.at_inf)
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = r.fix(x[e]);
        uint32_t keeps = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t k = key_of(x[e]);
            keeps |= k >= lo && k < hi && in.keeps(k, 8 * v - p.shift + e) ? 1u << e : 0u;
        }
        if (keeps) {
            int at = atomicAdd(&sh.n_list, __popc(keeps));
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (keeps >> e & 1) {
                    if (at < kList) sh.list[at] = static_cast<uint64_t>(key_of(x[e])) << 32 | static_cast<uint32_t>(8 * v - p.shift + e);
                    ++at;
                }
        }
    }
    __syncthreads();
    const int n = sh.n_list;
    __syncthreads();
    return n;
}

// The smallest key whose token falls into bin `bin` or one before it: every wave
// tries 64 keys at a time.
__device__ __forceinline__ uint32_t bin_edge(const Row& r, int bin) {
    uint32_t lo = 0x00800000u, hi = key_of(r.M);  // lo: the lowest finite key; hi is in the bin or before it
    const uint32_t lane = threadIdx.x % kWave;
#pragma unroll 1
    while (lo < hi) {
        const uint32_t step = max((hi - lo) / kWave, 1u), key = lo + lane * step;
        const uint64_t in = __ballot(key < hi && r.bin_of(value_of(key)) <= bin);
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

constexpr int kSolo = 256;  // tokens that one wave deals with alone
constexpr int kDigit = 9;

// w in units of 2^-50: the low bits of w + 4.
__device__ __forceinline__ uint64_t fixed(double w) {
    return static_cast<uint64_t>(__double_as_longlong(w + 4.0) - __double_as_longlong(4.0));
}

// The least value v[] (of `bits` bits) of the tokens that are `in` up to which their
// amounts add up to the target, 0 < target <= their sum, and what lies before it:
// nine bits at a time, by sums over the values of the next nine.
__device__ __forceinline__ uint32_t select(const Group& g, const uint32_t (&v)[4], const uint64_t (&amount)[4],
                                           const bool (&in)[4], int bits, uint64_t target, uint64_t& before, Shared& sh) {
    constexpr uint32_t kMask = (1u << kDigit) - 1;
    const int tid = threadIdx.x;
    uint32_t prefix = 0;
    before = 0;
#pragma unroll 1
    for (int shift = (bits - 1) / kDigit * kDigit; shift >= 0; shift -= kDigit) {
        g.sync();
        for (int b = tid; b <= static_cast<int>(kMask); b += g.size()) sh.mass[b] = 0;
        g.sync();
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (in[e] && (shift + kDigit >= 32 || v[e] >> (shift + kDigit) == prefix))
                atomicAdd(reinterpret_cast<unsigned long long*>(&sh.mass[v[e] >> shift & kMask]), static_cast<unsigned long long>(amount[e]));
        g.sync();
        if (tid < kWave) {  // eight digits a lane
            uint64_t m[8], sum = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                m[i] = sh.mass[8 * tid + i];
                sum += m[i];
            }
            uint64_t upto = sum;
#pragma unroll
            for (int o = 1; o < kWave; o <<= 1) {
                const uint64_t q = __shfl_up(upto, o, kWave);
                if (tid >= o) upto += q;
            }
            const uint64_t reach = __ballot(before + upto >= target);
            if (reach && tid == __ffsll(static_cast<unsigned long long>(reach)) - 1) {
                uint64_t run = before + upto - sum;
                int d = 0;
#pragma unroll
                for (int i = 0; i < 7; ++i)
                    if (d == i && run + m[i] < target) {
                        run += m[i];
                        d = i + 1;
                    }
                sh.digit = 8 * tid + d;
                sh.before = run;
            }
        }
        g.sync();
        prefix = prefix << kDigit | static_cast<uint32_t>(sh.digit);
        before = sh.before;
    }
    return prefix;
}

// The collected tokens, four a thread: cut to a count (count > 0), then to a mass
// (mass > 0, as it is or as a share of theirs), each by key and among equals by
// index; then, if the rest is all that the row keeps, the token is drawn.  Returns
// the last cut made.
struct Targets {
    double count, mass;
    bool share, draw;
};
__device__ __forceinline__ Cut cut_list(const Row& r, int n, const Targets& to, double u, int32_t* token, float* logprob,
                                        Shared& sh) {
    const Group g{to.draw && n <= kSolo};
    Cut cut{0, r.n};
    if (g.solo && threadIdx.x >= kWave) return cut;
    uint32_t key[4], idx[4];
    double w[4];
    bool in[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int i = threadIdx.x + e * g.size();
        in[e] = i < n;
        const uint64_t t = in[e] ? sh.list[i] : 0;
        key[e] = static_cast<uint32_t>(t >> 32);
        idx[e] = static_cast<uint32_t>(t);
        w[e] = in[e] ? r.w(value_of(key[e])) : 0.0;
    }
    const uint32_t top = key_of(r.M);
    const int index_bits = 32 - __clz(r.n);
    uint64_t target = 0, before = 0, all = 0;
    uint32_t found = 0;
    bool ties = false;
    // 0, 1: count by key, by index; 2, 3: mass; 4: the draw
#pragma unroll 1
    for (int step = 0; step < 5; ++step) {
        if ((step < 2 && !(to.count > 0.0)) || (step >= 2 && step < 4 && !(to.mass > 0.0)) || (step == 4 && !to.draw)) continue;
        const bool by_key = step == 0 || step == 2;
        if ((step == 1 || step == 3) && !ties) continue;
        uint32_t v[4];
        uint64_t amount[4], sum = 0;
        bool some[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (step == 4) in[e] = in[e] && w[e] >= r.min_p;
            v[e] = by_key ? top - key[e] : idx[e];
            amount[e] = step < 2 ? 1 : fixed(w[e]);
            some[e] = in[e] && (step == 4 || by_key || key[e] == found);
            sum += some[e] ? amount[e] : 0;
        }
        sum = g.sum(sum, sh);
        if (by_key) {
            const double t = step == 0 ? to.count : to.share ? to.mass * static_cast<double>(sum) : to.mass * 0x1p50;
            target = min(t >= 1.0 ? static_cast<uint64_t>(ceil(t)) : 1, sum);
        } else if (step < 4) {
            target -= before;
            if (sum <= target) continue;  // all of the equal ones
        } else {
            all = sum;
            target = min(static_cast<uint64_t>(u * static_cast<double>(sum)) + 1, sum);
        }
        const uint32_t got = select(g, v, amount, some, by_key ? 32 : index_bits, target, before, sh);
        if (by_key) {
            found = top - got;
            ties = true;
            cut = Cut{found, r.n};
        } else {
            cut.last = static_cast<int>(got);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (step < 4) in[e] = in[e] && (key[e] > cut.key || (key[e] == cut.key && static_cast<int>(idx[e]) <= cut.last));
            else if (in[e] && idx[e] == got) {
                *token = static_cast<int32_t>(got);
                if (logprob) *logprob = static_cast<float>(log(w[e] * 0x1p50 / static_cast<double>(all)));
            }
        }
    }
    return cut;
}

// The tokens of `in` weighed (or counted) in bins: where the running sum reaches
// `target` (of them, or of all of their mass), what lies above that bin, and
// their mass and the number of tokens down to it.
struct Found {
    int bin;  // kBins: beyond the weighed tokens, whose rest has no mass
    double above, z, about;
};
template <class T>
__device__ __forceinline__ Found find_bin(const Pieces<T>& p, const Row& r, const Cut& in, bool by_mass, double target, Shared& sh) {
    const int tid = threadIdx.x;
    __syncthreads();
    for (int b = tid; b < kBins; b += kThreads) sh.mass[b] = 0;
    __syncthreads();
    Found f;
    f.z = 0.0;
    each(p, r, [&](float x, int i) {
        if (!in.keeps(key_of(x), i)) return;
        int n;
        const double w = r.weight(r.depth(x), n);
        f.z += w;
        // w in units of 2^-42: the low bits of w + 2^10
        if (n > 1 - kBins)
            atomicAdd(reinterpret_cast<unsigned long long*>(&sh.mass[-n]),
                      static_cast<unsigned long long>(by_mass ? __double_as_longlong(w + 0x1p10) - __double_as_longlong(0x1p10) : 1));
    });
    f.z = block_sum(f.z, sh);
    // a bin's mass says how many tokens it has to 2.2% either way
    const bool has = tid < kBins - 1;
    const double mine = has ? static_cast<double>(sh.mass[tid]) : 0.0, upto = block_scan(mine, sh);
    if (tid == 0) sh.found = kBins;
    if (tid == kBins - 2) sh.found_d = upto;
    __syncthreads();
    const double aim = by_mass ? target * sh.found_d : target;
    if (has && upto >= aim) atomicMin(&sh.found, tid);
    __syncthreads();
    f.bin = sh.found;
    if (tid == f.bin) sh.above_d = upto - mine;
    f.about = block_sum(has && tid <= f.bin ? by_mass ? mine * 0x1p-42 * exp2(tid * (1 / 16.0)) : mine : 0.0, sh);
    f.above = by_mass ? sh.above_d * 0x1p-42 : sh.above_d;
    return f;
}

// The token of a row whose kept tokens are those of `cut` with w >= min_p: the
// pieces are cut into sixteen ranges, one a wave, the first is taken in which the
// running sum passes u Z, and so on down to 64 pieces, one a lane.
template <class T>
__device__ __forceinline__ void draw_from_row(const Pieces<T>& p, const Row& r, const Cut& cut, double u, int32_t* token, float* logprob,
                              Shared& sh) {
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const bool all = cut.key == 0, low = r.min_p > 0.0;
    // in logits: equal values have one key, and -inf has no mass either way
    const float cut_x = all ? -INFINITY : value_of(cut.key);
    auto piece = [&](int v, double (&w)[8]) {
        float x[8];
        p.load(v, x);
        if (r.at_inf)
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = r.fix(x[e]);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            w[e] = r.w(x[e]);  // 0 outside the row, where x is -inf
            if (!(x[e] > cut_x || (x[e] == cut_x && 8 * v - p.shift + e <= cut.last))) w[e] = 0.0;
            if (low && w[e] < r.min_p) w[e] = 0.0;
        }
    };
    // Under a cut most tokens are out: a wave queues those that are in, in any order,
    // and weighs 64 at a time.
    float* queue = sh.queue[wave];
    // well below what min_p keeps
    const double low_t = low ? 16.0 * log2(r.min_p) - 0.01 : 0.0;
    const double low_d = low ? static_cast<double>(r.M) + low_t / r.c16 : -INFINITY;
    const float low_x = static_cast<float>(low_d - fabs(low_d) * 0x1p-20);
    int a = 0, b = p.count;
    double z = 0.0, before = 0.0, target = 0.0;
    bool first = true;
    __syncthreads();
#pragma unroll 1
    while (first || b - a > kWave) {
        const int per = ((b - a + kWaves - 1) / kWaves + kWave - 1) / kWave * kWave;
        const int from = a + wave * per, to = min(from + per, b);
        double s = 0.0;
        if (all && !low) {
#pragma unroll 1
            for (int v = from + lane; v < to; v += kWave) {
                double w[8];
                piece(v, w);
                s += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
            }
        } else {
            int n = 0;
#pragma unroll 1
            for (int v0 = from; v0 < to; v0 += kWave) {
                float x[8];
                const int v = v0 + lane;
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = -INFINITY;
                if (v < to) {
                    p.load(v, x);
                    if (r.at_inf)
#pragma unroll
                        for (int e = 0; e < 8; ++e) x[e] = r.fix(x[e]);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const bool in = (x[e] > cut_x || (x[e] == cut_x && 8 * v - p.shift + e <= cut.last)) && x[e] >= low_x;
                    const uint64_t mask = __ballot(in);
                    const int at = n + __builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(mask >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(mask), 0));
                    if (in) queue[at] = x[e];
                    n += __popcll(mask);
                }
                wave_fence();
                while (n >= kWave) {
                    n -= kWave;
                    const double w = r.w(queue[n + lane]);
                    s += w >= r.min_p ? w : 0.0;
                }
                wave_fence();
            }
            if (lane < n) {
                const double w = r.w(queue[lane]);
                s += w >= r.min_p ? w : 0.0;
            }
        }
        s = wave_sum_d(s);
        __syncthreads();
        if (lane == 0) sh.red_d[wave] = s;
        __syncthreads();
        if (first) {
            for (int i = 0; i < kWaves; ++i) z += sh.red_d[i];
            target = u * z;
            first = false;
        }
        // the first range that passes the target; the last with any mass where rounding leaves none
        int at = 0;
        double run = before, at_before = before;
#pragma unroll 1
        for (int i = 0; i < kWaves; ++i) {
            if (sh.red_d[i] <= 0.0) continue;
            at = i;
            at_before = run;
            run += sh.red_d[i];
            if (run > target) break;
        }
        before = at_before;
        a += at * per;
        b = min(a + per, b);
    }
    if (wave > 0) return;
    double w[8] = {}, sum = 0.0;
    if (a + lane < b) piece(a + lane, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum += w[e];
    double upto = sum;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const double q = __shfl_up(upto, o, kWave);
        if (lane >= o) upto += q;
    }
    const uint64_t here = __ballot(before + upto > target && sum > 0.0), some = __ballot(sum > 0.0);
    const int l = here ? __ffsll(static_cast<unsigned long long>(here)) - 1 : 63 - __clzll(static_cast<long long>(some));
    if (lane == l) {
        double run = before + upto - sum, wb = 0.0;
        int best = -1;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (w[e] <= 0.0 || (best >= 0 && run > target)) continue;
            run += w[e];
            best = 8 * (a + lane) - p.shift + e;
            wb = w[e];
        }
        *token = best;
        if (logprob) *logprob = static_cast<float>(log(wb / z));
    }
}

template <class T>
__global__ __launch_bounds__(kThreads) void sample_kernel(SampleArgs a) {
    __shared__ Shared sh;
    const int row = blockIdx.x, tid = threadIdx.x;
    const Pieces<T> p(static_cast<const T*>(a.logits) + row * a.ld, a.vocab);
    int32_t* token = a.tokens + row;
    float* logprob = a.logprob ? a.logprob + row : nullptr;
    if (tid < 16) sh.root[tid] = exp2(tid / 16.0);
    // asked for before the row, so that they are there after it
    const float temperature = a.temperature ? a.temperature[row] : 1.f, min_p = a.min_p ? a.min_p[row] : 0.f;
    const float top_p = a.top_p ? a.top_p[row] : 1.f, u_in = a.u[row];
    const int32_t top_k = a.top_k ? a.top_k[row] : 0;

    // the thread's largest logit and the first piece that has it (NaN is below everything)
    float mine = -INFINITY;
    int at = -1;
#pragma unroll 2
    for (int v = tid; v < p.count; v += kThreads) {
        float x[8];
        p.load(v, x);
        const float m = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
        if (m > mine) {
            mine = m;
            at = v;
        }
    }
    uint64_t best = 0;
    if (at >= 0) {
        float x[8];
        p.load(at, x);
        int i = 0;
#pragma unroll
        for (int e = 7; e >= 0; --e)
            if (x[e] == mine) i = 8 * at - p.shift + e;
        best = static_cast<uint64_t>(key_of(mine)) << 32 | (0xFFFFFFFFu - static_cast<uint32_t>(i));
    }
    best = block_max(best, sh);
    if (best == 0 || !(temperature > 0.f)) {
        if (tid == 0) {
            *token = best == 0 ? -1 : static_cast<int32_t>(0xFFFFFFFFu - static_cast<uint32_t>(best));
            if (logprob) *logprob = best == 0 ? -INFINITY : 0.f;
        }
        return;
    }
    Row r;
    r.M = value_of(static_cast<uint32_t>(best >> 32));
    r.at_inf = r.M == INFINITY;
    if (r.at_inf) {
        r.M = 0.f;
        mine = r.fix(mine);
    }
    r.c16 = 16.0 * 1.4426950408889634074 / static_cast<double>(temperature);
    r.root = (const __attribute__((address_space(3))) double*)sh.root;
    r.n = a.vocab;
    r.min_p = min_p > 0.f ? fmin(static_cast<double>(min_p), 1.0) : 0.0;
    const int k = top_k > 0 && top_k < a.vocab ? top_k : 0;
    const double prob = top_p < 1.f ? fmax(static_cast<double>(top_p), 0.0) : 1.0;
    const double u = u_in > 0.f ? fmin(static_cast<double>(u_in), 0x1.fffffffffffffp-1) : 0.0;

    // 0: top_k by the threads' largest; 1: top_k by bins, where that is no help; 2: top_p
    Cut cut{0, a.vocab};
#pragma unroll 1
    for (int way = 0; way < 3; ++way) {
        if (way == 0 ? k == 0 || k > kThreads : way == 1 ? k == 0 : prob >= 1.0) continue;
        uint32_t lo, hi = 0xFFFFFFFFu;
        double z = 0.0;
        Targets to{};
        if (way == 0) {
            // the k-th largest of the threads' largest, in its upper 16 bits: wave 0 counts them all
            uint32_t* keys = reinterpret_cast<uint32_t*>(sh.list);
            keys[tid] = key_of(mine);
            __syncthreads();
            if (tid < kWave) {
                uint32_t mine16[kWaves];
#pragma unroll
                for (int w = 0; w < kWaves; ++w) mine16[w] = keys[w * kWave + tid] >> 16;
                uint32_t least = 0, most = key_of(r.M) >> 16;
#pragma unroll 1
                while (least < most) {
                    const uint32_t mid = most - (most - least) / 2;
                    int count = 0;
#pragma unroll
                    for (int w = 0; w < kWaves; ++w) count += __popcll(__ballot(mine16[w] >= mid));
                    if (count >= k) least = mid;
                    else most = mid - 1;
                }
                if (tid == 0) sh.found = static_cast<int>(least);
            }
            __syncthreads();
            lo = static_cast<uint32_t>(sh.found) << 16;
            if (lo <= 0x007FFFFFu) continue;  // -inf
            to = Targets{static_cast<double>(k), prob < 1.0 ? fmax(prob, 0x1p-1000) : 0.0, true, true};
        } else {
            const bool by_mass = way == 2;
            const Found f = find_bin(p, r, cut, by_mass, by_mass ? prob : k, sh);
            if (f.bin == kBins) continue;
            z = f.z;
            lo = bin_edge(r, f.bin);
            // the tokens down to the bin where LDS holds them, else the bin's alone
            const bool all = by_mass && f.about < 0.97 * kList;
            if (!all && f.bin > 0) hi = bin_edge(r, f.bin - 1);
            if (by_mass) to = Targets{0.0, fmax(prob * z - (all ? 0.0 : f.above), 0x1p-1000), false, all};
            else to = Targets{k - f.above, 0.0, false, false};
        }
        const int n = collect(p, r, lo, hi, cut, sh);
        if (n <= kList) {
            const Cut c = cut_list(r, n, to, u, token, logprob, sh);
            if (to.draw) return;
            cut = c;
            if (way == 1) continue;
            break;
        }
        if (way > 0) cut = bisect(p, r, cut, way == 2, way == 2 ? fmax(prob * z, 0x1p-1000) : k, sh);
    }
    draw_from_row(p, r, cut, u, token, logprob, sh);
}

}  // namespace
}  // namespace slw

using namespace slw;

extern "C" int slw_sample_workspace_size(int32_t max_rows, int32_t vocab, size_t* bytes) {
    return guarded([&] {
        if (!bytes) return fail(SLW_EINVAL, "null argument");
        if (max_rows < 0) return fail(SLW_EINVAL, "negative rows");
        if (vocab < 1 || vocab > SLW_SAMPLE_MAX_VOCAB)
            return fail(SLW_EUNSUPPORTED, "vocab must be in [1, %d] (got %d)", SLW_SAMPLE_MAX_VOCAB, vocab);
        *bytes = 0;
        return SLW_OK;
    });
}

extern "C" int slw_sample(const slw_sample_args* a, void* ws, size_t ws_bytes, void* stream) {
    return guarded([&] {
        if (!a) return fail(SLW_EINVAL, "null argument");
        if (a->rows < 0) return fail(SLW_EINVAL, "negative rows");
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
        const SampleArgs g{a->logits, a->ld, a->temperature, a->top_k, a->top_p, a->min_p, a->u, a->tokens, a->logprob, a->vocab};
        hipStream_t s = static_cast<hipStream_t>(stream);
        if (a->logits_f32) sample_kernel<float><<<a->rows, kThreads, 0, s>>>(g);
        else sample_kernel<bf16><<<a->rows, kThreads, 0, s>>>(g);
        HIP_TRY(hipGetLastError());
        return SLW_OK;
    });
}
