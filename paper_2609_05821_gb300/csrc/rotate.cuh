// One thread's share of a rotated row: VEC pairs, that is two chunks of VEC
// elements, or one chunk that does not rotate.
#pragma once

#include "cache.cuh"

namespace conduit {

template <typename T, int VEC>
struct alignas(sizeof(T) * VEC) Chunk {
  T v[VEC];
};

// Unit u of a row: u < half / VEC are rotating units with their chunks at `a` and
// `b`; the others copy the chunk at `a`.
struct Unit {
  int a, b;
  bool turns;
};

template <int VEC>
__device__ __forceinline__ Unit unit_of(const RopeDev& rope, int u) {
  const int nr = rope.half / VEC;
  if (u >= nr) return Unit{rope.rot + (u - nr) * VEC, 0, false};
  if (rope.layout == CONDUIT_ROPE_HALVES) return Unit{u * VEC, rope.half + u * VEC, true};
  return Unit{2 * u * VEC, 2 * u * VEC + VEC, true};
}

template <int VEC>
__host__ __device__ __forceinline__ int units_per_row(const RopeDev& rope, int d) {
  return rope.half / VEC + (d - rope.rot) / VEC;
}

// Cosines and (signed) sines of pairs p0 .. p0 + VEC - 1 for row t; false if one of
// the positions lies outside of the table.
template <int VEC>
__device__ __forceinline__ bool load_turn(const RopeDev& rope, int64_t t, int p0, float2 (&cs)[VEC]) {
  int pos[CONDUIT_MAX_AXES];
  bool ok = true;
#pragma unroll
  for (int a = 0; a < CONDUIT_MAX_AXES; ++a) {
    pos[a] = a < rope.axes ? rope.pos[int64_t(a) * rope.T + t] : 0;
    ok &= pos[a] >= 0 && pos[a] < rope.len;
  }
  if (!ok) return false;
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    const int p = p0 + e;
    const int a = (rope.axis[p >> 4] >> (2 * (p & 15))) & 3;
    const int at = a == 0 ? pos[0] : a == 1 ? pos[1] : a == 2 ? pos[2] : pos[3];
    cs[e] = rope.table[int64_t(at) * rope.half + p];
    cs[e].y *= rope.sign;
  }
  return true;
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
