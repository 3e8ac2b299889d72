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
// pairs of fp32 with one instruction, each rounded as a single one is.  (A product that feeds an addition may be contracted.)
__device__ __forceinline__ uint64_t pair_bits(float2 a) {
    uint64_t v;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a.x), "f"(a.y));
    return v;
}
__device__ __forceinline__ float2 pair_of(uint64_t v) {
    float2 a;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(a.x), "=f"(a.y) : "l"(v));
    return a;
}
__device__ __forceinline__ float2 add_pair(float2 a, float2 b) {
    uint64_t v;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(v) : "l"(pair_bits(a)), "l"(pair_bits(b)));
    return pair_of(v);
}
__device__ __forceinline__ float2 mul_pair(float2 a, float2 b) {
    uint64_t v;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(v) : "l"(pair_bits(a)), "l"(pair_bits(b)));
    return pair_of(v);
}
__device__ __forceinline__ float2 fma_pair(float2 a, float2 b, float2 c) {
    uint64_t v;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(v) : "l"(pair_bits(a)), "l"(pair_bits(b)), "l"(pair_bits(c)));
    return pair_of(v);
}
__device__ __forceinline__ float2 twice(float a) { return make_float2(a, a); }
// the largest magnitude of three; NaN wins
__device__ __forceinline__ float max_abs(float a, float b, float c) {
    float m;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(a), "f"(b), "f"(c));
    return m;
}
// the four scale bytes of 4 neighbouring blocks as one word; a block is PER lanes
template <int PER>
__device__ __forceinline__ uint32_t gather_scales(uint32_t byte) {
    uint32_t word = byte << (8 * (threadIdx.x / PER % 4));
    word |= __shfl_xor_sync(0xFFFFFFFFu, word, PER);
    word |= __shfl_xor_sync(0xFFFFFFFFu, word, 2 * PER);
    return word;
}

// ---------------------------------------------------------------- microscaled 8-bit floating point
// 32 neighbouring elements of a row share e = max(floor(log2 amax) - 8, -127), the power of two that brings the largest
// into [256, 512); code = e4m3_rn(v / 2^e), above 448 it saturates.  Every step but the rounding is exact.  An element
// that is not finite makes its block's scale NaN.  Scales lie as in 4 bits: the one of row r and block b at byte
// (r % 32) * 16 + (r % 128 / 32) * 4 + b % 4 of the 512-byte tile (r / 128, b / 4), which is one 128-byte stage of codes.
__host__ __device__ inline size_t fp8_stages(size_t cols) { return (cols + 127) / 128; }
__host__ __device__ inline size_t fp8_stride(size_t cols) { return (cols + 31) / 32 * 32; }
__host__ __device__ inline size_t fp8_scale_offset(size_t row, size_t block, size_t stages) {
    return (row / 128 * stages + block / 4) * 512 + (row % 32) * 16 + (row % 128 / 32) * 4 + block % 4;
}
// a block's scale and what its elements are multiplied by, from its largest magnitude as fp32 bits
__device__ __forceinline__ void fp8_block_scale(uint32_t amax, uint32_t& byte, float& inv) {
    const int e = max(int(amax >> 23) - 8, 0);             // the stored byte: exponent + 127
    byte = amax >= kInfBits ? 255u : uint32_t(e);
    inv = amax >= kInfBits ? 0.0f : __uint_as_float(uint32_t(254 - e) << 23);
}
// two codes, the first in the low byte
__device__ __forceinline__ uint32_t encode_e4m3(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float2 decode_e4m3(uint32_t codes) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(uint16_t(codes)));
    return unpack2(h, kFp16);
}
__device__ __forceinline__ uint4 encode_e4m3(float (&v)[16], float inv) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 16; i += 2) mul2(v[i], v[i + 1], inv);
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = encode_e4m3(v[4 * i], v[4 * i + 1]) | encode_e4m3(v[4 * i + 2], v[4 * i + 3]) << 16;
    return make_uint4(w[0], w[1], w[2], w[3]);
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
