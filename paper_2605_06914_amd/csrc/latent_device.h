// Pieces that the latent-cache kernels share.
#pragma once
#include "latent_kernels.h"

namespace taper {
namespace latent {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

#define DEV __device__ __forceinline__

// 16x16x32: lane l supplies A[l%16][8*(l/16)..+7] and B[8*(l/16)..+7][l%16] and receives C[4*(l/16)..+3][l%16].
DEV f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
DEV float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
DEV bf16x8 cat(bf16x4 a, bf16x4 b) { return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7); }

// (maximum, not maxnum: it takes its values as they are, where maxnum first quiets each; a NaN makes its row NaN.)
DEV float max2(float a, float b) { return __builtin_elementwise_maximum(a, b); }
DEV float max4(f32x4 v) { return max2(max2(v[0], v[1]), max2(v[2], v[3])); }

// A row of scores lives in lanes n, n + 16, n + 32, n + 48: these bring its four parts together by lane swaps.
DEV float max_lane_groups(float v) {
    unsigned u = __float_as_uint(v);
    auto p = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    u = __float_as_uint(max2(__uint_as_float(p[0]), __uint_as_float(p[1])));
    p = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    return max2(__uint_as_float(p[0]), __uint_as_float(p[1]));
}
DEV float sum_lane_groups(float v) {
    unsigned u = __float_as_uint(v);
    auto p = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    u = __float_as_uint(__uint_as_float(p[0]) + __uint_as_float(p[1]));
    p = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}

// The power of two that brings the largest magnitude `most` into [0.5, 1) when divided by it; 2^e and 2^-e are normal numbers.
DEV int exponent_of(float most) {
    const int e = (int)((__float_as_uint(most) >> 23) & 0xff) - 126;
    return e < -126 ? -126 : (e > 126 ? 126 : e);
}

DEV unsigned lds_address(const void* p) { return (unsigned)(uintptr_t)(__attribute__((address_space(3))) const char*)p; }
// 64 lanes x 16 bytes: lane l's from base + off (per lane) to LDS address `lds` + 16 l.  The statement itself keeps the wait
// states between a vector instruction's write of the base and the load (the compiler does not look inside).
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
DEV void load_to_lds(const char* base, unsigned off, unsigned lds) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "s"(lds) : "m0", "memory");
}
// 64 lanes x 4 bytes likewise: what matters is that their lines are in the L2 afterwards.
DEV void word_to_lds(const char* base, unsigned off, unsigned lds) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 4\n\tglobal_load_lds_dword %0, %1" ::"v"(off), "s"(base), "s"(lds) : "m0", "memory");
}
#pragma clang diagnostic pop
// All but this wave's N youngest loads have landed, its LDS accesses are done, and every wave of the workgroup is here.
template <int N>
DEV void wait_loads_and_meet() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}
// LDS accesses are done and every wave is here; loads stay in flight.
DEV void meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// A per-lane value the compiler must not reason about: what is derived from it is computed where it is used, and not kept in registers
// from earlier on.
DEV int opaque(int v) {
    asm volatile("" : "+v"(v));
    return v;
}

// Integers of a plan, which no kernel writes: read by scalar loads.
typedef const __attribute__((address_space(4))) int32_t* scalar_row;

DEV int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

}  // namespace latent
}  // namespace taper
