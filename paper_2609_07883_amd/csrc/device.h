// Device-side types and helpers shared by the gfx950 kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace slw {

typedef __bf16 bf16;
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kWave = 64;

__device__ __forceinline__ float bf2f(bf16 v) { return static_cast<float>(v); }
__device__ __forceinline__ bf16 f2bf(float v) { return static_cast<bf16>(v); }  // RNE

// 16x16x32 bf16 MFMA, fp32 accumulate.  Lane l supplies row (A) / column (B)
// l % 16 and the eight k values of group l / 16; the result holds, in lane l,
// element i: row 4 * (l / 16) + i, column l % 16.
__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Work-groups of a launch are dispatched round-robin to the 8 XCDs (linear id
// % 8), each with its own L2.  Position in a work order of linear block id
// `pid` out of `total` such that every XCD takes a contiguous range of the
// order: work that shares operands, placed next to each other in the order,
// then runs on one XCD and shares its L2.
__device__ __forceinline__ int xcd_order(int pid, int total) {
    constexpr int kXcd = 8;
    const int q = total / kXcd, r = total % kXcd;
    const int xcd = pid % kXcd, local = pid / kXcd;
    return xcd < r ? xcd * (q + 1) + local : r * (q + 1) + (xcd - r) * q + local;
}

// Tile (tm, tn) at position t of the grouped tile order: group_m tile rows
// at a time, column by column within a group, so that tiles that run
// together share A rows and B columns.  With at most 16 tile rows a group
// spans them all: each weight panel is then streamed into an L2 once for
// every row tile.
__device__ __forceinline__ void tile_coords(int t, int nt_m, int nt_n, int& tm, int& tn) {
    const int GROUP_M = nt_m <= 16 ? nt_m : 8;
    const int per_group = GROUP_M * nt_n;
    const int first_m = (t / per_group) * GROUP_M;
    const int gsize = min(nt_m - first_m, GROUP_M);
    const int in_group = t % per_group;
    tm = first_m + in_group % gsize;
    tn = in_group / gsize;
}

// Wait until at most n vector-memory operations of this wave are
// outstanding (gfx9 s_waitcnt encoding, other counters left alone).
template <int N>
__device__ __forceinline__ void wait_vmcnt() {
    static_assert(N >= 0 && N < 64, "vmcnt range");
    __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (0x7 << 4) | (0xF << 8));
}

// Wait until at most N LDS operations of this wave are outstanding.
template <int N>
__device__ __forceinline__ void wait_lgkmcnt() {
    static_assert(N >= 0 && N < 16, "lgkmcnt range");
    __builtin_amdgcn_s_waitcnt(0xC07F | (N << 8));
}

// Direct global->LDS load of 16 bytes per lane from base + off (base is
// wave-uniform): lane l's bytes land at lds + 16 l (lds is wave-uniform).
// Issued as assembly so that the compiler, which cannot tell which LDS buffer
// such a load writes, does not make every later LDS read wait for all of
// them; the main loop waits for them itself.  M0 is a reserved register that
// the compiler sets right before each instruction that reads it; no
// compiler-generated code in these kernels uses it, so the value left there
// is never relied on.
__device__ __forceinline__ void load_lds16(const void* base, uint32_t off, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "s"(lds) : "memory");
}

// Workgroup barrier with no memory fence: the asm statement's memory clobber
// keeps the compiler from moving LDS or global accesses across it, and the
// waits it needs are issued explicitly before it.
__device__ __forceinline__ void barrier_only() { asm volatile("s_barrier" ::: "memory"); }

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
    return v;
}

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, kWave));
    return v;
}

}  // namespace slw
