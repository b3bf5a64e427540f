// The next token of each row of logits, from a given random number.
//
// w_t = 2^((x_t - M) log2(e) / T), M the largest logit.  The filters keep a head
// of the tokens sorted by (logit descending, index ascending): the first top_k;
// of those, the ones with less than top_p of their mass before them; of those,
// w >= min_p.  So every filter is a cut in that order, (key, index) of the last
// token kept, and no row is ever sorted whole:
//   1. a pass finds M;
//   2. a pass counts (top_k) or weighs (top_p) the tokens by their distance to
//      M, in bins of 1/16 octave of w; the running sum over bins says in which
//      one the cut is;
//   3. a pass collects the tokens down to that bin, a few hundred as a rule, in
//      LDS; they are sorted, cut, sorted by index, and the token is drawn.
// Where more than kList tokens are kept (or no filter is set) the cut is found by
// bisection on key and index, and the token from sums of 512 tokens at a time.
//
// Every mass is held in 64 bits: w from an exponential good to 2^-46, bins in
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
constexpr int kList = 4096;         // tokens sorted in LDS
constexpr int kSums = SLW_SAMPLE_MAX_VOCAB / 512 + 1;
constexpr double kFixed = 0x1p42;   // fixed point of the bins' masses: 2^20 tokens of w = 1 make 2^62

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

// 2^y for y <= 0 (y = -inf: 0).
__device__ __forceinline__ double weight_of(double y) { return y < -1000.0 ? 0.0 : exp2(y); }

struct Row {
    float M;
    double c;   // log2(e) / T
    float bin;  // 16 c
    double min_p;
    int n;
    // x as a distance below M; finite or +inf
    __device__ float below(float x) const { return x == M ? 0.f : x == x ? M - x : INFINITY; }
    __device__ double y(float x) const {
        return x == M ? 0.0 : below(x) == INFINITY ? -INFINITY : (static_cast<double>(x) - static_cast<double>(M)) * c;
    }
    __device__ double w(float x) const { return weight_of(y(x)); }
    __device__ int bin_of(float x) const { return static_cast<int>(fminf(below(x) * bin, static_cast<float>(kBins - 1))); }
};

struct Shared {
    union {
        uint64_t list[kList];
        double sums[kSums];
    };
    uint64_t mass[kBins];
    uint32_t count[kBins];
    double red_d[kWaves];
    uint64_t red_u[kWaves];
    int n_list, found;
    double found_d;
};

__device__ __forceinline__ double wave_sum_d(double v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
    return v;
}

// Sum over the work-group, in a fixed order, on every thread.
__device__ double block_sum(double v, Shared& sh) {
    v = wave_sum_d(v);
    __syncthreads();
    if (threadIdx.x % kWave == 0) sh.red_d[threadIdx.x / kWave] = v;
    __syncthreads();
    v = 0.0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) v += sh.red_d[w];
    return v;
}

__device__ uint64_t block_max(uint64_t v, Shared& sh) {
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

// Inclusive sums over the work-group's threads, in thread order.
__device__ double block_scan(double v, Shared& sh) {
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
    for (int w = 0; w < wave; ++w) before += sh.red_d[w];
    return before + v;
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
    __device__ bool real(int v, int e) const { return 8 * v - shift + e >= 0 && 8 * v - shift + e < n; }
};

template <class T, class F>
__device__ __forceinline__ void each(const Pieces<T>& p, F&& f) {
    for (int v = threadIdx.x; v < p.count; v += kThreads) {
        float x[8];
        p.load(v, x);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (p.real(v, e)) f(x[e], 8 * v - p.shift + e);
    }
}

// list[0 .. n) ascending, n a power of two.
__device__ void sort_list(Shared& sh, int n) {
    for (int k = 2; k <= n; k <<= 1)
        for (int j = k >> 1; j > 0; j >>= 1) {
            __syncthreads();
            for (int i = threadIdx.x; i < n / 2; i += kThreads) {
                const int a = (i & ~(j - 1)) << 1 | (i & (j - 1)), b = a + j;
                const uint64_t x = sh.list[a], y = sh.list[b];
                if ((x > y) == ((a & k) == 0)) {
                    sh.list[a] = y;
                    sh.list[b] = x;
                }
            }
        }
    __syncthreads();
}

// A head of the sorted tokens: those with a larger key than `key`, and those with
// it up to index `last`.
struct Cut {
    uint32_t key;
    int last;
    __device__ bool keeps(uint32_t k, int i) const { return k > key || (k == key && i <= last); }
};

// The head of tokens within `in` that ends with the token at which the count
// (by_mass: the mass before it is still less than) target is reached, by
// bisection on the key and, among equals, on the index.
template <class T>
__device__ Cut bisect(const Pieces<T>& p, const Row& r, const Cut& in, bool by_mass, double target, Shared& sh) {
    // sum of what lies above: tokens that `c` keeps
    auto sum = [&](const Cut& c) {
        double s = 0.0;
        each(p, [&](float x, int i) {
            const uint32_t k = key_of(x);
            if (in.keeps(k, i) && c.keeps(k, i)) s += by_mass ? r.w(x) : 1.0;
        });
        return block_sum(s, sh);
    };
    // the largest key for which everything from it up reaches the target; `in`'s own
    // last key where nothing does
    uint32_t lo = in.key, hi = key_of(r.M);
    while (lo < hi) {
        const uint32_t mid = hi - (hi - lo) / 2;  // lo < mid <= hi
        if (sum(Cut{mid, p.n}) >= target) lo = mid;
        else hi = mid - 1;
    }
    int a = 0, b = p.n - 1;
    while (a < b) {
        const int mid = a + (b - a) / 2;
        if (sum(Cut{lo, mid}) >= target) b = mid;
        else a = mid + 1;
    }
    return Cut{lo, lo == in.key && a > in.last ? in.last : a};
}

// The token of a row whose kept tokens are those of `cut` with w >= min_p.
template <class T>
__device__ void draw_from_row(const Pieces<T>& p, const Row& r, const Cut& cut, double u, int32_t* token, float* logprob,
                              Shared& sh) {
    const int lane = threadIdx.x % kWave;
    auto weight = [&](float x, int i) {
        if (!cut.keeps(key_of(x), i)) return 0.0;
        const double w = r.w(x);
        return w >= r.min_p ? w : 0.0;
    };
    const int groups = (p.count + kWave - 1) / kWave;
    __syncthreads();
    for (int g = threadIdx.x / kWave; g < groups; g += kWaves) {
        const int v = g * kWave + lane;
        double s = 0.0;
        if (v < p.count) {
            float x[8];
            p.load(v, x);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (p.real(v, e)) s += weight(x[e], 8 * v - p.shift + e);
        }
        s = wave_sum_d(s);
        if (lane == 0) sh.sums[g] = s;
    }
    __syncthreads();
    if (threadIdx.x >= kWave) return;
    // one wave: the group in which the running sum passes u Z, then the token
    const int per = (groups + kWave - 1) / kWave;
    double mine = 0.0;
    for (int i = 0; i < per; ++i)
        if (lane * per + i < groups) mine += sh.sums[lane * per + i];
    double upto = mine;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const double q = __shfl_up(upto, o, kWave);
        if (lane >= o) upto += q;
    }
    const double z = __shfl(upto, kWave - 1, kWave), target = u * z;
    // the first lane whose sum passes the target (the last that has any, where rounding leaves none)
    const uint64_t passes = __ballot(upto > target && mine > 0.0), any = __ballot(mine > 0.0);
    const int at = passes ? __ffsll(static_cast<unsigned long long>(passes)) - 1 : 63 - __clzll(static_cast<long long>(any));
    double before = __shfl(upto - mine, at, kWave);
    int g = -1;
    for (int i = at * per; i < min((at + 1) * per, groups); ++i) {
        const double s = sh.sums[i];
        if (s <= 0.0) continue;
        if (g >= 0) before += sh.sums[g];
        g = i;
        if (before + s > target) break;
    }
    const int v = g * kWave + lane;
    double w[8], sum = 0.0;
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = 0.0;
    if (v < p.count) {
        float x[8];
        p.load(v, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (p.real(v, e)) w[e] = weight(x[e], 8 * v - p.shift + e);
            sum += w[e];
        }
    }
    double to = sum;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const double q = __shfl_up(to, o, kWave);
        if (lane >= o) to += q;
    }
    const uint64_t here = __ballot(before + to > target && sum > 0.0), some = __ballot(sum > 0.0);
    const int l = here ? __ffsll(static_cast<unsigned long long>(here)) - 1 : 63 - __clzll(static_cast<long long>(some));
    if (lane == l) {
        double run = before + to - sum;
        int best = -1;
        double wb = 0.0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (w[e] <= 0.0 || (best >= 0 && run > target)) continue;
            run += w[e];
            best = 8 * v - p.shift + e;
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

    // the largest logit, and the first token that has it
    uint64_t best = 0;
    each(p, [&](float x, int i) {
        const uint64_t k = static_cast<uint64_t>(key_of(x)) << 32 | (0xFFFFFFFFu - static_cast<uint32_t>(i));
        best = k > best ? k : best;
    });
    best = block_max(best, sh);
    Row r;
    r.M = value_of(static_cast<uint32_t>(best >> 32));
    r.n = a.vocab;
    const float temperature = a.temperature ? a.temperature[row] : 1.f;
    if (r.M == -INFINITY || !(temperature > 0.f)) {
        if (tid == 0) {
            *token = r.M == -INFINITY ? -1 : static_cast<int32_t>(0xFFFFFFFFu - static_cast<uint32_t>(best));
            if (logprob) *logprob = r.M == -INFINITY ? -INFINITY : 0.f;
        }
        return;
    }
    r.c = 1.4426950408889634074 / static_cast<double>(temperature);
    r.bin = fminf(static_cast<float>(16.0 * r.c), 3.0e38f);
    const float min_p = a.min_p ? a.min_p[row] : 0.f;
    r.min_p = min_p > 0.f ? fmin(static_cast<double>(min_p), 1.0) : 0.0;
    const int32_t top_k = a.top_k ? a.top_k[row] : 0;
    int k = top_k > 0 && top_k < a.vocab ? top_k : 0;
    const float top_p = a.top_p ? a.top_p[row] : 1.f;
    const double prob = top_p < 1.f ? fmax(static_cast<double>(top_p), 0.0) : 1.0;
    const float u_in = a.u[row];
    const double u = u_in > 0.f ? fmin(static_cast<double>(u_in), 0x1.fffffffffffffp-1) : 0.0;

    Cut cut{0, a.vocab};
    if (k == 0 && prob >= 1.0) {
        draw_from_row(p, r, cut, u, token, logprob, sh);
        return;
    }

    // counts, and masses where the cut goes by them
    for (int b = tid; b < kBins; b += kThreads) {
        sh.count[b] = 0;
        sh.mass[b] = 0;
    }
    __syncthreads();
    const bool weigh = k == 0;
    double z_all = 0.0;
    each(p, [&](float x, int) {
        const double w = weigh ? r.w(x) : 0.0;
        z_all += w;
        const int b = r.bin_of(x);
        if (b == kBins - 1) return;
        atomicAdd(&sh.count[b], 1u);
        if (weigh) atomicAdd(reinterpret_cast<unsigned long long*>(&sh.mass[b]), static_cast<unsigned long long>(rint(w * kFixed)));
    });
    z_all = block_sum(z_all, sh);
    // inclusive sums over the bins; the first bin that reaches the target
    const bool has = tid < kBins - 1;
    const double n_upto = block_scan(has ? sh.count[tid] : 0.0, sh);
    const double m_upto = weigh ? block_scan(has ? static_cast<double>(sh.mass[tid]) : 0.0, sh) : 0.0;
    if (tid == 0) sh.found = kBins;
    if (tid == kBins - 2) sh.found_d = m_upto;
    __syncthreads();
    const double target = weigh ? prob * sh.found_d : k;
    if (has && (weigh ? m_upto : n_upto) >= target) atomicMin(&sh.found, tid);
    __syncthreads();
    const int last_bin = sh.found;
    __syncthreads();
    if (tid == min(last_bin, kBins - 2)) sh.n_list = static_cast<int>(n_upto);
    __syncthreads();
    const int n = sh.n_list;  // tokens in the bins up to that one

    if (n > kList) {
        if (k > 0) cut = bisect(p, r, cut, false, k, sh);
        if (prob < 1.0) {
            double z = 0.0;
            each(p, [&](float x, int i) { z += cut.keeps(key_of(x), i) ? r.w(x) : 0.0; });
            z = block_sum(z, sh);
            cut = bisect(p, r, cut, true, fmax(prob * z, 0x1p-1000), sh);
        }
        draw_from_row(p, r, cut, u, token, logprob, sh);
        return;
    }

    __syncthreads();
    if (tid == 0) sh.n_list = 0;
    __syncthreads();
    each(p, [&](float x, int i) {
        const int b = r.bin_of(x);
        if (b <= last_bin && b < kBins - 1)
            sh.list[atomicAdd(&sh.n_list, 1)] = static_cast<uint64_t>(~key_of(x)) << 32 | static_cast<uint32_t>(i);
    });
    __syncthreads();
    int size = 64;
    while (size < n) size <<= 1;
    for (int i = n + tid; i < size; i += kThreads) sh.list[i] = ~0ull;
    sort_list(sh, size);

    // masses in sorted order, four neighbours a thread
    int kept = k > 0 ? min(k, n) : n;
    auto weights = [&](double (&w)[4], int count) {
        double s = 0.0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = 4 * tid + e;
            w[e] = i < count ? r.w(value_of(~static_cast<uint32_t>(sh.list[i] >> 32))) : 0.0;
            s += w[e];
        }
        return s;
    };
    double w[4];
    double s = weights(w, kept);
    double upto = block_scan(s, sh);
    {
        const double z = k > 0 ? block_sum(s, sh) : z_all;
        const double limit = prob * z;
        double before = upto - s;
        double in = 0.0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = 4 * tid + e;
            if (i < kept && (i == 0 || ((prob >= 1.0 || before < limit) && w[e] >= r.min_p))) in += 1.0;
            before += w[e];
        }
        kept = static_cast<int>(block_sum(in, sh));
    }
    // by index: the kept ones are a head of the sorted list
    size = 64;
    while (size < kept) size <<= 1;
    __syncthreads();
    for (int i = tid; i < size; i += kThreads) {
        const uint64_t t = sh.list[i];
        sh.list[i] = i < kept ? t << 32 | static_cast<uint32_t>(~(t >> 32)) : ~0ull;
    }
    sort_list(sh, size);
    s = 0.0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int i = 4 * tid + e;
        w[e] = i < kept ? r.w(value_of(static_cast<uint32_t>(sh.list[i]))) : 0.0;
        s += w[e];
    }
    upto = block_scan(s, sh);
    const double z = block_sum(s, sh), aim = u * z;
    if (tid == 0) sh.found = kept - 1;
    __syncthreads();
    double run = upto - s;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        run += w[e];
        if (4 * tid + e < kept && run > aim && w[e] > 0.0) {
            atomicMin(&sh.found, 4 * tid + e);
            break;
        }
    }
    __syncthreads();
    if (tid == 0) {
        const uint64_t t = sh.list[sh.found];
        *token = static_cast<int32_t>(t >> 32);
        if (logprob) *logprob = static_cast<float>(log(r.w(value_of(static_cast<uint32_t>(t))) / z));
    }
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
