// What stands between the cache operators and the projections of a decoder
// block: the residual stream's update with the norms on both sides of it, and
// the rotary positions of a batch's query and key rows.  Both read every value
// once and write it once, so the memory's rate bounds them, or for a few rows
// the launch.
#include <math.h>

#include <cmath>

#include "device.h"
#include "hip_try.h"
#include "kernels.h"

namespace slw {
namespace {

struct F8 {
    float v[8];
};

__device__ __forceinline__ F8 load8(const bf16* p) {
    const bf16x8 x = *reinterpret_cast<const bf16x8*>(p);
    F8 r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r.v[e] = bf2f(x[e]);
    return r;
}
__device__ __forceinline__ F8 load8(const float* p) {
    const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
    return F8{{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}};
}
__device__ __forceinline__ void store8(bf16* p, const F8& x) {
    bf16x8 o;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = f2bf(x.v[e]);
    *reinterpret_cast<bf16x8*>(p) = o;
}
__device__ __forceinline__ void store8(float* p, const F8& x) {
    *reinterpret_cast<f32x4*>(p) = f32x4{x.v[0], x.v[1], x.v[2], x.v[3]};
    *reinterpret_cast<f32x4*>(p + 4) = f32x4{x.v[4], x.v[5], x.v[6], x.v[7]};
}

// Past the caches, for what is read a whole block later.
__device__ __forceinline__ void stream8(bf16* p, const F8& x) {
    bf16x8 o;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = f2bf(x.v[e]);
    __builtin_nontemporal_store(o, reinterpret_cast<bf16x8*>(p));
}
__device__ __forceinline__ void stream8(float* p, const F8& x) {
    __builtin_nontemporal_store(f32x4{x.v[0], x.v[1], x.v[2], x.v[3]}, reinterpret_cast<f32x4*>(p));
    __builtin_nontemporal_store(f32x4{x.v[4], x.v[5], x.v[6], x.v[7]}, reinterpret_cast<f32x4*>(p + 4));
}

// Sum over the threads of a row: a wave, or the W waves of the work-group.
template <int W>
__device__ __forceinline__ float row_sum(float v, float* red) {
    v = wave_sum(v);
    if (W == 1) return v;
    if ((threadIdx.x & (kWave - 1)) == 0) red[threadIdx.x / kWave] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) v += red[w];
    return v;
}

// r' = r + scale * gate * P(o), y = r' / sqrt(mean(r'^2) + eps) * gain, all in
// fp32 between the loads and the one rounding of each output; y is taken of r'
// before that rounding.  A row stays in the registers of W waves, NV vectors of
// 8 values a thread, between the loads, the one or two sums and the stores: one
// pass, whose bytes bound it.  One vector a thread up to 8192 values, as the sums
// then wait for one load: 1 row of 4096 2.4 us, with two 3.1.  4104 rows of 4096 (fp32
// stream, post-norm and gate, 202 MB) take 43 us, 4.7 TB/s, where a copy reaches 5.1; with
// two vectors 47.  r' goes past the caches, as the next block's end reads it: 2080 rows of
// a bf16 stream 11.7 us, 13.5 through them.
template <int W, int NV, class R>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void residual_norm_kernel(NormRows a) {
    constexpr int kThreads = 64 * W;
    __shared__ float red[2][W];
    const int row = W == 1 ? blockIdx.x * 4 + threadIdx.x / 64 : blockIdx.x;
    const int t = W == 1 ? threadIdx.x % 64 : threadIdx.x;
    if (row >= a.rows) return;  // W == 1 only, where a wave goes its own way
    const int nvec = a.d / 8;
    const R* r_in = static_cast<const R*>(a.resid) + static_cast<size_t>(row) * a.ld_resid;
    F8 r[NV], o[NV];
    float ss = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int i = t + j * kThreads;
        if (i < nvec) {
            r[j] = load8(r_in + 8 * i);
            if (a.block) o[j] = load8(static_cast<const bf16*>(a.block) + static_cast<size_t>(row) * a.ld_block + 8 * i);
        }
    }
    if (a.block) {
        float inv = 1.f;
        if (a.post_gain) {
#pragma unroll
            for (int j = 0; j < NV; ++j)
                if (t + j * kThreads < nvec)
#pragma unroll
                    for (int e = 0; e < 8; ++e) ss += o[j].v[e] * o[j].v[e];
            inv = 1.0f / sqrtf(row_sum<W>(ss, red[0]) / static_cast<float>(a.d) + a.eps);
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int i = t + j * kThreads;
            if (i >= nvec) continue;
            if (a.post_gain) {
                const F8 g = load8(static_cast<const bf16*>(a.post_gain) + 8 * i);
#pragma unroll
                for (int e = 0; e < 8; ++e) o[j].v[e] *= inv * g.v[e];
            }
            if (a.gate) {
                const F8 g = load8(static_cast<const bf16*>(a.gate) + static_cast<size_t>(row) * a.ld_gate + 8 * i);
#pragma unroll
                for (int e = 0; e < 8; ++e) o[j].v[e] *= g.v[e];
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) r[j].v[e] += a.scale * o[j].v[e];
        }
    }
    ss = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int i = t + j * kThreads;
        if (i >= nvec) continue;
        if (a.resid_out) stream8(static_cast<R*>(a.resid_out) + static_cast<size_t>(row) * a.ld_resid_out + 8 * i, r[j]);
#pragma unroll
        for (int e = 0; e < 8; ++e) ss += r[j].v[e] * r[j].v[e];
    }
    if (!a.out) return;
    const float inv = 1.0f / sqrtf(row_sum<W>(ss, red[1]) / static_cast<float>(a.d) + a.eps);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int i = t + j * kThreads;
        if (i >= nvec) continue;
        const F8 g = load8(static_cast<const bf16*>(a.gain) + 8 * i);
#pragma unroll
        for (int e = 0; e < 8; ++e) r[j].v[e] *= inv * g.v[e];
        store8(static_cast<bf16*>(a.out) + static_cast<size_t>(row) * a.ld_out + 8 * i, r[j]);
    }
}

template <class R>
void residual_norm_by_width(const NormRows& a, hipStream_t s) {
    const unsigned rows = static_cast<unsigned>(a.rows);
    if (a.d <= 512) residual_norm_kernel<1, 1, R><<<(rows + 3) / 4, 256, 0, s>>>(a);
    else if (a.d <= 2048) residual_norm_kernel<4, 1, R><<<rows, 256, 0, s>>>(a);
    else if (a.d <= 4096) residual_norm_kernel<8, 1, R><<<rows, 512, 0, s>>>(a);
    else if (a.d <= 8192) residual_norm_kernel<16, 1, R><<<rows, 1024, 0, s>>>(a);
    else residual_norm_kernel<16, 4, R><<<rows, 1024, 0, s>>>(a);
}

// Turns of pair i at position 1 (f_i / 2 pi), in fp64: at position p the angle is
// p times as large, and its fraction of a turn keeps 2^-53 p f_i.
__device__ __forceinline__ double rope_turns(const RopeArgs& r, int i) {
    double f = r.freq ? r.freq[i] : exp2(i * r.step) * r.first;
    if (r.by_parts) {
        const double g = fmin(1.0, fmax(0.0, (f * r.turns_in_original - r.low) * r.inv_width));
        f *= (1.0 - g) * r.inv_factor + g;
    }
    return f * 0.15915494309189533577;
}

// LDS accesses of the lanes of one wave keep their order across it.
__device__ __forceinline__ void wave_fence() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

// One wave a row (it takes rows a grid apart): lane i forms the cos and sin of
// pair i, all lanes share them through LDS, and each takes the same 16 values of
// a head for every head that falls to it: the values (8 u .. 8 u + 7) and their
// partners rot / 2 further, or 16 u .. 16 u + 15 interleaved; units past rot
// are copied.  Waves do not wait for each other.  The bytes bound it: 4104 rows of
// 32 + 8 heads of 128 (84 MB) take 17.6 us, 4.8 TB/s; 18.7 with a head's values asked
// for when it is their turn.  fp64 keeps an angle's fraction of a turn at any position
// (fp32 would be 0.01 off at 131072), and costs one lane a pair.
template <int HD, bool INTERLEAVED>
__global__ __launch_bounds__(256) void rotate_kernel(RotateRows a, RopeArgs rope) {
    constexpr int kUnits = HD / 16, kHeadLanes = kWave / kUnits;
    __shared__ float cs[4][2][HD / 2];
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const int u = lane % kUnits, h0 = lane / kUnits;
    const int turning = rope.rot / 16, half = rope.rot / 2;
    const int lo = u >= turning || INTERLEAVED ? 16 * u : 8 * u;
    const int hi = u >= turning || INTERLEAVED ? lo + 8 : lo + half;
    const double turns = lane < half ? rope_turns(rope, lane) : 0.0;
    const int heads = a.hq + a.hkv, first = a.q ? 0 : a.hq, last = a.k ? heads : a.hq;
    const bool copies = u >= turning && a.in_place;  // nothing to do
    for (int row = blockIdx.x * 4 + wave; row < a.rows; row += gridDim.x * 4) {
        // a head's values are asked for before those of the head before it are dealt with, the first before the angles
        F8 x, y;
        auto place = [&](int h, int64_t ld) {
            return static_cast<size_t>(row) * ld + static_cast<size_t>(h < a.hq ? h : h - a.hq) * HD;
        };
        auto ask = [&](int h, F8& p, F8& q) {
            const bf16* in = static_cast<const bf16*>(h < a.hq ? a.q : a.k) + place(h, a.ld);
            p = load8(in + lo);
            q = load8(in + hi);
        };
        if (!copies && first + h0 < last) ask(first + h0, x, y);
        int pos;
        if (row < a.chunk) {
            int i = 0;
            while (i + 1 < a.n_prompts && row >= a.row_end[i]) ++i;
            pos = row + a.shift[i];
        } else {
            pos = a.kv_len[row - a.chunk] - 1;
        }
        if (lane < half) {
            const double at = turns * pos;
            float s, c;
            sincospif(static_cast<float>(2.0 * (at - rint(at))), &s, &c);
            cs[wave][0][lane] = c * rope.mscale;
            cs[wave][1][lane] = s * rope.mscale;
        }
        wave_fence();
        F8 c, s;
        if (u < turning) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                c.v[e] = cs[wave][0][8 * u + e];
                s.v[e] = cs[wave][1][8 * u + e];
            }
        }
        wave_fence();  // the next row's values come after these reads
        if (copies) continue;
        for (int h = first + h0; h < last; h += kHeadLanes) {
            F8 p = x, q = y, x_next, y_next;
            if (h + kHeadLanes < last) ask(h + kHeadLanes, x_next, y_next);
            if (u < turning) {
                if (INTERLEAVED) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        p.v[2 * e] = x.v[2 * e] * c.v[e] - x.v[2 * e + 1] * s.v[e];
                        p.v[2 * e + 1] = x.v[2 * e + 1] * c.v[e] + x.v[2 * e] * s.v[e];
                        q.v[2 * e] = y.v[2 * e] * c.v[4 + e] - y.v[2 * e + 1] * s.v[4 + e];
                        q.v[2 * e + 1] = y.v[2 * e + 1] * c.v[4 + e] + y.v[2 * e] * s.v[4 + e];
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        p.v[e] = x.v[e] * c.v[e] - y.v[e] * s.v[e];
                        q.v[e] = y.v[e] * c.v[e] + x.v[e] * s.v[e];
                    }
                }
            }
            bf16* out = static_cast<bf16*>(h < a.hq ? a.q_out : a.k_out) + place(h, a.ld_out);
            store8(out + lo, p);
            store8(out + hi, q);
            x = x_next;
            y = y_next;
        }
    }
}

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

}  // namespace

void launch_residual_norm(const NormRows& a, hipStream_t s) {
    if (a.resid_f32) residual_norm_by_width<float>(a, s);
    else residual_norm_by_width<bf16>(a, s);
}

void launch_rotate(const RotateRows& a, const RopeArgs& rope, hipStream_t s) {
    const unsigned groups = static_cast<unsigned>((a.rows + 3) / 4);
    if (a.hd == 128) {
        if (rope.interleaved) rotate_kernel<128, true><<<groups, 256, 0, s>>>(a, rope);
        else rotate_kernel<128, false><<<groups, 256, 0, s>>>(a, rope);
    } else {
        if (rope.interleaved) rotate_kernel<64, true><<<groups, 256, 0, s>>>(a, rope);
        else rotate_kernel<64, false><<<groups, 256, 0, s>>>(a, rope);
    }
}

}  // namespace slw

using namespace slw;

namespace {

int check_norm_rows(const void* p, int64_t ld, int32_t d, const char* what) {
    if (!aligned16(p) || ld % 8 || ld < d)
        return fail(SLW_EINVAL, "%s rows: 16-byte aligned, stride a multiple of 8 and at least %d (got %lld)", what, d,
                    (long long)ld);
    return SLW_OK;
}

}  // namespace

extern "C" int slw_residual_norm(const slw_norm_args* a, void* stream) {
    return guarded([&] {
        if (!a) return fail(SLW_EINVAL, "null argument");
        if (a->rows < 0) return fail(SLW_EINVAL, "negative rows");
        if (a->rows > SLW_NORM_MAX_ROWS) return fail(SLW_EUNSUPPORTED, "more than %d rows", SLW_NORM_MAX_ROWS);
        if (a->d < 8 || a->d % 8 || a->d > SLW_NORM_MAX_D)
            return fail(SLW_EUNSUPPORTED, "d must be a multiple of 8 in [8, %d] (got %d)", SLW_NORM_MAX_D, a->d);
        if (!(a->eps >= 0.f) || !std::isfinite(a->eps) || !std::isfinite(a->scale))
            return fail(SLW_EINVAL, "eps must be finite and not negative, scale finite");
        if (!a->resid) return fail(SLW_EINVAL, "null residual");
        if (!a->resid_out && !a->out) return fail(SLW_EINVAL, "nothing to write");
        if (a->out && !a->gain) return fail(SLW_EINVAL, "null gain");
        if (!a->block && (a->post_gain || a->gate)) return fail(SLW_EINVAL, "a post-norm or gate without a block's output");
        int rc = check_norm_rows(a->resid, a->ld_resid, a->d, "residual");
        if (!rc && a->block) rc = check_norm_rows(a->block, a->ld_block, a->d, "block");
        if (!rc && a->gate) rc = check_norm_rows(a->gate, a->ld_gate ? a->ld_gate : a->d, a->d, "gate");
        if (!rc && a->resid_out) rc = check_norm_rows(a->resid_out, a->ld_resid_out, a->d, "residual output");
        if (!rc && a->out) rc = check_norm_rows(a->out, a->ld_out, a->d, "output");
        if (rc) return rc;
        if (!aligned16(a->gain) || !aligned16(a->post_gain)) return fail(SLW_EINVAL, "gains must be 16-byte aligned");
        if (a->rows == 0) return SLW_OK;
        launch_residual_norm({a->resid, a->block, a->post_gain, a->gate, a->gain, a->resid_out, a->out, a->ld_resid,
                              a->ld_block, a->ld_gate, a->ld_resid_out, a->ld_out, a->rows, a->d, a->resid_f32 != 0,
                              a->scale, a->eps}, static_cast<hipStream_t>(stream));
        HIP_TRY(hipGetLastError());
        return SLW_OK;
    });
}
