// Eight neighbouring dims of a row: loads, and their rotation in fp32 (both quantised caches' appends).
#pragma once

#include "rotate.cuh"
#include "tc_common.cuh"

namespace conduit {

// a + b of products that were rounded before. A packed multiply followed by a packed
// add comes out as one fused operation; two scalar additions do not merge with it.
__device__ __forceinline__ float2 add_rounded(float2 a, float2 b) {
  return make_float2(__fadd_rn(a.x, b.x), __fadd_rn(a.y, b.y));
}

// 8 elements as they lie in memory, and as fp32.
template <typename T>
struct Raw8 {
  uint4 w[sizeof(T) / 2];
};
template <typename T>
__device__ __forceinline__ Raw8<T> load8(const T* p, bool wide) {
  Raw8<T> r;
  if (wide) {
#pragma unroll
    for (int c = 0; c < int(sizeof(T) / 2); ++c) r.w[c] = reinterpret_cast<const uint4*>(p)[c];
  } else {
    T e8[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) e8[e] = p[e];
#pragma unroll
    for (int c = 0; c < int(sizeof(T) / 2); ++c) r.w[c] = reinterpret_cast<const uint4*>(e8)[c];
  }
  return r;
}
template <typename T>
__device__ __forceinline__ void to_floats(const Raw8<T>& r, float (&x)[8]) {
  const T* e8 = reinterpret_cast<const T*>(r.w);
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = to_float(e8[e]);
}

// How the pairs of a chunk of 8 dims lie: none, in the matching chunk of the other half
// (half a multiple of 8), as neighbours inside the chunk, or anywhere.
enum { kNoTurn = 0, kChunks = 1, kNeighbours = 2, kAnywhere = 3 };

__host__ __device__ __forceinline__ int pairing(const RopeDev& rope) {
  if (rope.rot == 0) return kNoTurn;
  if (rope.layout == CONDUIT_ROPE_PAIRS) return rope.rot % 8 == 0 ? kNeighbours : kAnywhere;
  return rope.half % 8 == 0 ? kChunks : kAnywhere;
}

// Cosine and signed sine of each dim of the chunk at i0: y = x cos + partner sin.
template <int kPairing>
__device__ __forceinline__ void load_turn8(const RopeDev& rope, const int (&pos)[CONDUIT_MAX_AXES], int i0,
                                           float2 (&cs)[8]) {
  if (kPairing == kNoTurn || i0 >= rope.rot) return;
  if (kPairing == kChunks) {
    const bool first = i0 < rope.half;
    load_turn<8>(rope, pos, first ? i0 : i0 - rope.half, cs);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (first) cs[e].y = -cs[e].y;
  } else if (kPairing == kNeighbours) {
    float2 pair[4];
    load_turn<4>(rope, pos, i0 / 2, pair);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      cs[2 * e] = make_float2(pair[e].x, -pair[e].y);
      cs[2 * e + 1] = pair[e];
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int i = i0 + e;
      if (i >= rope.rot) continue;
      const bool halves = rope.layout == CONDUIT_ROPE_HALVES, first = halves ? i < rope.half : !(i & 1);
      float2 one[1];
      load_turn<1>(rope, pos, halves ? (first ? i : i - rope.half) : i >> 1, one);
      cs[e] = make_float2(one[0].x, first ? -one[0].y : one[0].y);
    }
  }
}

// The chunk's dims after rotation; `far`: the matching chunk of the other half (kChunks). The
// products are rounded before they are added.
template <int kPairing, typename T>
__device__ __forceinline__ void turn8(const RopeDev& rope, const T* row, int i0, const Raw8<T>& far,
                                      const float2 (&cs)[8], float (&x)[8]) {
  if (kPairing == kNoTurn || i0 >= rope.rot) return;
  float other[8];
  if (kPairing == kChunks) {
    to_floats(far, other);
  } else if (kPairing == kNeighbours) {
#pragma unroll
    for (int e = 0; e < 8; ++e) other[e] = x[e ^ 1];
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int i = i0 + e;
      const int j = rope.layout == CONDUIT_ROPE_PAIRS ? i ^ 1 : i < rope.half ? i + rope.half : i - rope.half;
      other[e] = i < rope.rot ? to_float(row[j]) : 0.f;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (i0 + e < rope.rot) x[e] = __fadd_rn(__fmul_rn(x[e], cs[e].x), __fmul_rn(other[e], cs[e].y));
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    const float2 own = tc::fmul2(make_float2(x[e], x[e + 1]), make_float2(cs[e].x, cs[e + 1].x));
    const float2 add = tc::fmul2(make_float2(other[e], other[e + 1]), make_float2(cs[e].y, cs[e + 1].y));
    const float2 y = add_rounded(own, add);
    x[e] = y.x;
    x[e + 1] = y.y;
  }
}

}  // namespace conduit
