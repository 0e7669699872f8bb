// The 8-bit cache: its blocks of 16 tokens, and e4m3 codes as numbers.
#pragma once

#include "cache.cuh"

namespace conduit {

constexpr int kBlockTokens = 16;
constexpr int kLeastExp = -40, kMostExp = 119;  // of a scale
constexpr float kMostCode = 448.f;

__host__ __device__ __forceinline__ constexpr int fp8_block_bytes(int d) { return 2 * kBlockTokens * d + 16; }

// Block of tokens `slot` .. (slot a multiple of 16) of page `id`, layer l, head g.
__device__ __forceinline__ uint8_t* fp8_block(const PackedDev& kv, int l, int g, int id, int slot) {
  return kv.page(l, g, id) + int64_t((slot & ((1 << kv.page_shift) - 1)) >> 4) * fp8_block_bytes(kv.d);
}

// 2^e for e in [-126, 127].
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float(uint32_t(e + 127) << 23); }
// e of a scale 2^e as it is stored (what is no such scale: the nearest end of the range).
__device__ __forceinline__ int exponent_of(float scale) {
  return min(max(int(__float_as_uint(scale) >> 23) - 127, kLeastExp), kMostExp);
}
// Least e with top <= 448 2^e = 1.75 x 2^(e + 8): the exponent of top less 8, or less 7 past 1.75.
__device__ __forceinline__ int exponent_for(float top) {
  return min(max(int((__float_as_uint(top) + 0x1FFFFFu) >> 23) - 127 - 8, kLeastExp), kMostExp);
}

// Codes of x (low byte) and y (high byte), half to even, +-448 for what lies beyond, NaN for NaN.
__device__ __forceinline__ uint32_t fp8_pair(float x, float y) {
  uint16_t w;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %2, %1;" : "=h"(w) : "f"(x), "f"(y));
  return w;
}
// The numbers of the codes in the low and in the high half of w, exactly.
__device__ __forceinline__ uint32_t halves_lo(uint32_t w) {
  uint32_t y;
  asm("{ .reg .b16 a, b; mov.b32 {a, b}, %1; cvt.rn.f16x2.e4m3x2 %0, a; }" : "=r"(y) : "r"(w));
  return y;
}
__device__ __forceinline__ uint32_t halves_hi(uint32_t w) {
  uint32_t y;
  asm("{ .reg .b16 a, b; mov.b32 {a, b}, %1; cvt.rn.f16x2.e4m3x2 %0, b; }" : "=r"(y) : "r"(w));
  return y;
}
__device__ __forceinline__ float2 floats_lo(uint32_t w) {
  const uint32_t h = halves_lo(w);
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}
__device__ __forceinline__ float2 floats_hi(uint32_t w) {
  const uint32_t h = halves_hi(w);
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

cudaError_t launch_fp8_append(const PackedDev& kv, const SeqsDev& s, const RopeDev& rope, int dtype,
                              const RowsDev& k, const RowsDev& v, const RowsDev& q, const RowsDev& q_out,
                              int32_t* status, cudaStream_t stream);
cudaError_t launch_fp8_read(const PackedDev& kv, const int32_t* first, const KvDev& dst, const BatchDev& b,
                            int max_tokens, int32_t* status, cudaStream_t stream);

}  // namespace conduit
