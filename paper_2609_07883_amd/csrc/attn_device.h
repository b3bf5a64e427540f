// Device helpers shared by the attention kernels.
#pragma once

#include "device.h"

namespace slw {

constexpr float kLog2e = 1.4426950408889634f;

// 2^x straight on the transcendental unit (v_exp_f32).  Results below
// 2^-126 may flush to zero, which softmax weights taken relative to a running
// maximum can afford; the library exp2f adds range scaling around the same
// instruction, five more VALU operations per call.
__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// Block tables read through the scalar cache: a wave-uniform index into
// constant-address-space memory.
typedef const int32_t __attribute__((address_space(4))) const_i32;

// Max and sum over lanes l, l ^ 16, l ^ 32 and l ^ 48 (the four 16-lane rows
// of a wave), with the gfx950 row-swap instructions instead of LDS permutes:
// a swap of a register with itself leaves, in every lane, its own value in
// one result and its partner's in the other.
__device__ __forceinline__ float rows4_max(float x) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float rows4_sum(float x) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

__device__ __forceinline__ bf16x8 to_bf16x8(f32x4 lo, f32x4 hi) {
    bf16x8 r;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        r[e] = f2bf(lo[e]);
        r[4 + e] = f2bf(hi[e]);
    }
    return r;
}

// Keys of the two score tiles of a pair of pages (32 keys): row r of tile
// tau holds key 16 (r / 8) + 8 ((r / 4) % 2) + 4 tau + r % 4, so that lane
// group g (rows 4 g .. 4 g + 3 of both tiles) ends up with keys 8 g .. 8 g + 7:
// the eight consecutive tokens of one page that the P V product's k slice g
// covers, and one 16-byte chunk of a dim-major V page.
__device__ __forceinline__ int pair_key(int r, int tau) { return 16 * (r >> 3) + 8 * ((r >> 2) & 1) + 4 * tau + (r & 3); }

// LDS swizzles of 16-byte chunks: K rows (64 B = four chunks of 8 dims) and
// V rows (32 B = two chunks of 8 tokens).  An operand read serves eight lanes
// per pass: for K the rows of tokens {0..3, 8..11} or {4..7, 12..15} of a
// page, for V eight consecutive dims; both swizzles put those on distinct
// banks.
__device__ __forceinline__ int kswz(int t, int sub) { return sub ^ (((t >> 1) & 1) | (((t >> 3) & 1) << 1)); }
__device__ __forceinline__ int vswz(int d, int h) { return h ^ ((d >> 2) & 1); }

// Direct global->LDS load of 16 bytes per lane: lane l's bytes land at
// lds + 16 l (lds is wave-uniform).  Issued as assembly so that the compiler,
// which cannot tell which LDS buffer such a load writes, does not make every
// later LDS read wait for all of them; the kernel waits for them itself.
// M0 is a reserved register that the compiler sets right before each
// instruction that reads it; no compiler-generated code in these kernels
// uses it, so the value left there is never relied on.
__device__ __forceinline__ void load_lds16(const void* src, void* lds) {
    const uint32_t dst = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(reinterpret_cast<uintptr_t>(lds)));
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(src), "s"(dst) : "memory");
}

// Wait until at most N vector-memory operations of this wave are outstanding.
template <int N>
__device__ __forceinline__ void wait_vmcnt() {
    static_assert(N >= 0 && N < 64, "vmcnt range");
    __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (0x7 << 4) | (0xF << 8));
}

// Wait until this wave's LDS operations are complete (vector memory
// operations may stay outstanding).
__device__ __forceinline__ void wait_lgkmcnt0() { __builtin_amdgcn_s_waitcnt(0xC07F); }

// Workgroup barrier with no memory fence (the memory clobber keeps the
// compiler from moving LDS or global accesses across it).
__device__ __forceinline__ void barrier_only() { asm volatile("s_barrier" ::: "memory"); }

}  // namespace slw
