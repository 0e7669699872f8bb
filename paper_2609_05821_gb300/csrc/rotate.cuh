// One thread's share of a rotated row: VEC pairs, that is two chunks of VEC
// elements, or one chunk that does not rotate.
#pragma once

#include "cache.cuh"

namespace conduit {

template <typename T, int VEC>
struct alignas(sizeof(T) * VEC) Chunk {
  T v[VEC];
};

// A chunk that is read or written once in a long pass (16-byte chunks go past the caches'
// reuse order: 5 % on query rows of 16 384 tokens).
template <typename T, int VEC>
__device__ __forceinline__ Chunk<T, VEC> load_once(const T* p) {
  if constexpr (sizeof(T) * VEC == 16) {
    const uint4 w = __ldcs(reinterpret_cast<const uint4*>(p));
    return *reinterpret_cast<const Chunk<T, VEC>*>(&w);
  } else {
    return *reinterpret_cast<const Chunk<T, VEC>*>(p);
  }
}
template <typename T, int VEC>
__device__ __forceinline__ void store_once(T* p, const Chunk<T, VEC>& c) {
  if constexpr (sizeof(T) * VEC == 16)
    __stcs(reinterpret_cast<uint4*>(p), *reinterpret_cast<const uint4*>(&c));
  else
    *reinterpret_cast<Chunk<T, VEC>*>(p) = c;
}

// Unit u of a row: two chunks of VEC elements at `a` and `b` that rotate, or that pass
// (the last of those may be one chunk: b < 0).
struct Unit {
  int a, b;
  bool turns;
};

template <int VEC>
__device__ __forceinline__ Unit unit_of(const RopeDev& rope, int d, int u) {
  const int nr = rope.half / VEC;
  if (u >= nr) {
    const int at = rope.rot + (u - nr) * 2 * VEC;
    return Unit{at, at + VEC < d ? at + VEC : -1, false};
  }
  if (rope.layout == CONDUIT_ROPE_HALVES) return Unit{u * VEC, rope.half + u * VEC, true};
  return Unit{2 * u * VEC, 2 * u * VEC + VEC, true};
}

template <int VEC>
__host__ __device__ __forceinline__ int units_per_row(const RopeDev& rope, int d) {
  return rope.half / VEC + ((d - rope.rot) / VEC + 1) / 2;
}

// The positions of row t on the axes; false if one lies outside of the table.
__device__ __forceinline__ bool load_positions(const RopeDev& rope, int64_t t, int (&pos)[CONDUIT_MAX_AXES]) {
  bool ok = true;
#pragma unroll
  for (int a = 0; a < CONDUIT_MAX_AXES; ++a) pos[a] = a < rope.axes ? rope.pos[int64_t(a) * rope.T + t] : 0;
#pragma unroll
  for (int a = 0; a < CONDUIT_MAX_AXES; ++a) ok &= pos[a] >= 0 && (pos[a] < rope.len || a >= rope.axes);
  return ok;
}

// Cosines and (signed) sines of pairs p0 .. p0 + VEC - 1 at positions inside the table.
template <int VEC>
__device__ __forceinline__ void load_turn(const RopeDev& rope, const int (&pos)[CONDUIT_MAX_AXES], int p0,
                                          float2 (&cs)[VEC]) {
  auto row_of = [&](int p) {
    const int a = (rope.axis[p >> 4] >> (2 * (p & 15))) & 3;
    return int64_t(a == 0 ? pos[0] : a == 1 ? pos[1] : a == 2 ? pos[2] : pos[3]) * rope.half;
  };
  if constexpr (VEC % 4 == 0) {
    // pairs of one axis (p0 is a multiple of VEC, so they share a word of `axis`) lie side by side in the table
    const uint32_t axes = (rope.axis[p0 >> 4] >> (2 * (p0 & 15))) & ((1u << (2 * VEC)) - 1);
    if (axes == (axes & 3) * (0x5555u & ((1u << (2 * VEC)) - 1)) && (rope.half & 1) == 0) {
      const float4* row = reinterpret_cast<const float4*>(rope.table + row_of(p0) + p0);
#pragma unroll
      for (int e = 0; e < VEC / 2; ++e) {
        const float4 x = row[e];
        cs[2 * e] = make_float2(x.x, x.y * rope.sign);
        cs[2 * e + 1] = make_float2(x.z, x.w * rope.sign);
      }
      return;
    }
  }
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    cs[e] = rope.table[row_of(p0 + e) + p0 + e];
    cs[e].y *= rope.sign;
  }
}

// The products are rounded before they are added: the value of the formula's own
// operations in fp32, whatever the compiler would contract.
template <typename T, int VEC>
__device__ __forceinline__ void turn_chunks(const RopeDev& rope, const float2 (&cs)[VEC], Chunk<T, VEC>& a,
                                            Chunk<T, VEC>& b) {
  if (rope.layout == CONDUIT_ROPE_HALVES || VEC == 1) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const float x = to_float(a.v[e]), y = to_float(b.v[e]);
      a.v[e] = from_float<T>(__fsub_rn(__fmul_rn(x, cs[e].x), __fmul_rn(y, cs[e].y)));
      b.v[e] = from_float<T>(__fadd_rn(__fmul_rn(y, cs[e].x), __fmul_rn(x, cs[e].y)));
    }
  } else {
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      T* c = e < VEC / 2 ? a.v : b.v;
      const int i = 2 * e % VEC;
      const float x = to_float(c[i]), y = to_float(c[i + 1]);
      c[i] = from_float<T>(__fsub_rn(__fmul_rn(x, cs[e].x), __fmul_rn(y, cs[e].y)));
      c[i + 1] = from_float<T>(__fadd_rn(__fmul_rn(y, cs[e].x), __fmul_rn(x, cs[e].y)));
    }
  }
}

// Whether rows can be moved in chunks of 16 bytes: pairs and passing dims come in
// whole chunks, and every row starts on a 16-byte boundary.
inline bool rows_aligned(const RowsDev& r, int vec) {
  return (reinterpret_cast<uintptr_t>(r.p) & 15u) == 0 && r.ls % vec == 0 && r.rs % vec == 0 && r.hs % vec == 0;
}
inline bool dims_in_chunks(const RopeDev& rope, int d, int vec) {
  return rope.half % vec == 0 && (d - rope.rot) % vec == 0;
}

}  // namespace conduit
