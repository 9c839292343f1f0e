// Device code shared by the kernels of 4-bit caches: what a strip of 16 tokens holds (include/sim_kv.h) as 16-bit floats.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "sim_kv_internal.h"

namespace simgb {

namespace {

// N 32-bit words that lie N words apart from the neighbours', so aligned as far as N allows.
template <int N>
__device__ __forceinline__ void words(const void *from, uint32_t *w) {
    if constexpr (N % 4 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const uint4 v = static_cast<const uint4 *>(from)[i / 4];
            w[i] = v.x, w[i + 1] = v.y, w[i + 2] = v.z, w[i + 3] = v.w;
        }
    } else if constexpr (N % 2 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            const uint2 v = static_cast<const uint2 *>(from)[i / 2];
            w[i] = v.x, w[i + 1] = v.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = static_cast<const uint32_t *>(from)[i];
    }
}

template <bool BF>
__device__ __forceinline__ uint32_t fma16(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t d;
    if (BF) asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    else asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}
template <bool BF>
__device__ __forceinline__ uint32_t add16(uint32_t a, uint32_t b) {
    uint32_t d;
    if (BF) asm("add.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    else asm("add.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}

// (a & b) | c, in one instruction.
__device__ __forceinline__ uint32_t and_or(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t d;
    asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}

// Codes at bits 4 I and 16 + 4 I of w, as the values that they stand for: a code is put under the exponent whose unit it is
// (128 + code, 1024 + code), which is then taken away, exactly; lo + code step is rounded once.  (Whole numbers made floats by an exponent beside
// them, for quantised weights: Kim, Henry, Fahim and Hassan Awadalla, arXiv 2211.10017.)
template <bool BF, int I>
__device__ __forceinline__ uint32_t values(uint32_t w, uint32_t step, uint32_t lo) {
    // float16 has room for a code four bits further up, as 1024 + 16 code: two of the three shifts are not needed
    constexpr bool kUp = !BF && I % 2 == 1;
    const uint32_t code = and_or(I < (BF ? 1 : 2) ? w : w >> (BF ? 4 * I : 8), kUp ? 0x00f000f0u : 0x000f000fu, BF ? 0x43004300u : 0x64006400u);
    return fma16<BF>(kUp ? fma16<BF>(code, 0x2c002c00u, 0xd400d400u) : add16<BF>(code, BF ? 0xc300c300u : 0xe400e400u), step, lo);
}
template <bool BF>
__device__ __forceinline__ void values4(uint32_t w, uint32_t step, uint32_t lo, uint32_t *x) {
    x[0] = values<BF, 0>(w, step, lo);
    x[1] = values<BF, 1>(w, step, lo);
    x[2] = values<BF, 2>(w, step, lo);
    x[3] = values<BF, 3>(w, step, lo);
}
// The lower, the upper half twice: as moves, which the instruction that takes them can do by itself (as permutations: 168 instead of
// 161 us for 384 sequences of up to 2600 keys).
__device__ __forceinline__ uint32_t low_twice(uint32_t x) {
    uint32_t d;
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tmov.b32 %0, {l, l};\n\t}" : "=r"(d) : "r"(x));
    return d;
}
__device__ __forceinline__ uint32_t high_twice(uint32_t x) {
    uint32_t d;
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tmov.b32 %0, {h, h};\n\t}" : "=r"(d) : "r"(x));
    return d;
}

}  // namespace

}  // namespace simgb
