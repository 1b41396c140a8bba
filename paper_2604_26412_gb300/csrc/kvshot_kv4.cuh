// kvshot_kv4.cuh -- the 4-bit target cache's format on the device: where a slot's bytes are, and the conversions between
// e2m1 codes with e4m3 block scales and f16 / fp32.  The format itself is defined in kvshot.h.
#pragma once

#include <cuda_fp16.h>
#include <stdint.h>

#include "kvshot.h"

namespace kvshot {

// Division by a number that the host knows: n / d for 0 <= n < 2^31.
struct Div {
  uint32_t mul, shift, d;
  static Div by(uint32_t d) {
    uint32_t l = 0;
    while ((1ull << l) < d) ++l;
    return Div{static_cast<uint32_t>(((1ull << 32) * ((1ull << l) - d)) / d + 1), l, d};
  }
  __device__ __forceinline__ int operator()(int n) const {
    return static_cast<int>((__umulhi(static_cast<uint32_t>(n), mul) + static_cast<uint32_t>(n)) >> shift);
  }
};

namespace kv4 {

constexpr int kKv4Tokens = KVSHOT_KV4_GROUP_TOKENS;
constexpr int kKv4Bytes = KVSHOT_KV4_GROUP_BYTES;
constexpr int kBlockDims = 16;               // dims that share a scale
constexpr int kChunkBytes = 16;              // codes of 32 dims of one token
constexpr int kChunkStride = 256;            // from a token's chunk to its next one
constexpr int kVCodes = 1024;                // V codes of a group
constexpr int kScales = 2048;                // K scales, then V scales (128 bytes each)
constexpr int kScaleBytes = 128;
static_assert(kScales + 2 * kScaleBytes == kKv4Bytes, "a group's parts");

namespace {  // internal linkage: every translation unit gets its own copy

// Eight e2m1 codes (low nibble of the lowest byte first) -> four f16x2 words; exact.
__device__ __forceinline__ void e2m1x8_to_f16(uint32_t codes, uint32_t (&o)[4]) {
  asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\tmov.b32 {b0, b1, b2, b3}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, b0;\n\tcvt.rn.f16x2.e2m1x2 %1, b1;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, b2;\n\tcvt.rn.f16x2.e2m1x2 %3, b3;\n\t}"
      : "=r"(o[0]), "=r"(o[1]), "=r"(o[2]), "=r"(o[3])
      : "r"(codes));
}

// Two e4m3 numbers (low byte first) -> f16x2; exact.
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint32_t two) {
  uint32_t r;
  asm("{\n\t.reg .b16 h;\n\tcvt.u16.u32 h, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, h;\n\t}" : "=r"(r) : "r"(two));
  return r;
}

__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
  const __half2 r = __hmul2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}

// e4m3 number nearest to x >= 2^-9, at most 448 (or NaN).
__device__ __forceinline__ uint32_t f32_to_e4m3(float x) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(0.f), "f"(x));
  return r & 0xffu;
}

// e2m1 codes nearest to lo (low nibble) and hi.
__device__ __forceinline__ uint32_t f32x2_to_e2m1(float lo, float hi) {
  uint32_t r;
  asm("{\n\t.reg .b8 b;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %1, %2;\n\tmov.b32 %0, {b, 0, 0, 0};\n\t}"
      : "=r"(r)
      : "f"(hi), "f"(lo));
  return r;
}

}  // namespace
}  // namespace kv4
}  // namespace kvshot
