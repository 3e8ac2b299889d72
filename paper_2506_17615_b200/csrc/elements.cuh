// Element types, and what several kernels do with a few elements in registers.
#pragma once
#include <cuda_fp16.h>

#include <cstdint>
#include <cstring>

namespace equarx {
namespace ff {

enum DType { kBf16 = 0, kFp16 = 1, kFp32 = 2 };

// ---------------------------------------------------------------- element types
__device__ __forceinline__ uint32_t pack2(float lo, float hi, int dtype) {
    uint32_t r;
    if (dtype == kBf16)
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float2 unpack2(uint32_t w, int dtype) {
    if (dtype == kBf16) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
    __half2 h;
    memcpy(&h, &w, 4);
    return __half22float2(h);
}
__device__ __forceinline__ void store1(void* p, size_t i, float v, int dtype) {
    if (dtype == kFp32)
        static_cast<float*>(p)[i] = v;
    else
        static_cast<uint16_t*>(p)[i] = uint16_t(pack2(v, v, dtype));
}

// ---------------------------------------------------------------- 8-bit scales
__device__ __forceinline__ uint32_t to_e4m3(float v) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(0.0f), "f"(v));
    return r & 0xFF;
}
__device__ __forceinline__ float from_e4m3(uint32_t b) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(uint16_t(b)));
    return unpack2(h, kFp16).x;
}
// 2^(byte - 127); 255 is NaN
__device__ __forceinline__ float from_e8m0(uint32_t b) {
    if (b == 255) return __uint_as_float(0x7FFFFFFFu);
    return b ? __uint_as_float(b << 23) : __uint_as_float(0x00400000u);
}

constexpr uint32_t kInfBits = 0x7F800000u;

// two products with one instruction, each rounded as a single one is
__device__ __forceinline__ void mul2(float& a, float& b, float c) {
    uint64_t v, w;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b));
    asm("mov.b64 %0, {%1, %1};" : "=l"(w) : "f"(c));
    asm("mul.rn.f32x2 %0, %0, %1;" : "+l"(v) : "l"(w));
    asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v));
}
// the four scale bytes of 4 neighbouring blocks as one word; a block is PER lanes
template <int PER>
__device__ __forceinline__ uint32_t gather_scales(uint32_t byte) {
    uint32_t word = byte << (8 * (threadIdx.x / PER % 4));
    word |= __shfl_xor_sync(0xFFFFFFFFu, word, PER);
    word |= __shfl_xor_sync(0xFFFFFFFFu, word, 2 * PER);
    return word;
}

// ---------------------------------------------------------------- wide accesses
// 256-bit accesses (sm_100): what is read once, or written and not read again here
__device__ __forceinline__ void load_256(const void* p, uint32_t* w) {
    asm volatile("ld.global.L1::no_allocate.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                 : "l"(p)
                 : "memory");
}
__device__ __forceinline__ void store_256(void* p, const uint32_t* w) {
    asm volatile("st.global.L1::no_allocate.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]),
                 "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                 : "memory");
}

}  // namespace ff
}  // namespace equarx
