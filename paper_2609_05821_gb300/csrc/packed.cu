// The 4-bit cache: append with rotation and packing, and the read back into a
// plain cache.
//
// Mathematics: groups of 32 dims, s = fp16((hi - lo)/15), m = fp16(lo + 8 s),
// c = clamp(rint((x - m)/s), -8, 7); a value stands for m + s c. Every operation is
// a separately rounded fp32 one, so that a plain program finds the same codes.
// Bound: the rows once, and d + d/4 bytes per token and KV head of the cache.
#include "rotate.cuh"

namespace conduit {
namespace {

constexpr int kThreads = 256;
constexpr float kClip = 61440.f;  // m +- 8 s stays inside fp16

// The 8 dims of a chunk as fp32.
template <typename T>
__device__ __forceinline__ void load8(const T* p, bool wide, float (&x)[8]) {
  if (wide) {
    constexpr int N = 16 / sizeof(T);
#pragma unroll
    for (int c = 0; c < 8 / N; ++c) {
      const Chunk<T, N> w = *reinterpret_cast<const Chunk<T, N>*>(p + c * N);
#pragma unroll
      for (int e = 0; e < N; ++e) x[c * N + e] = to_float(w.v[e]);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = to_float(p[e]);
  }
}

// The chunk's dims after rotation. Pairs may straddle chunks (rot_dim of any even
// size), so each dim finds its own pair.
template <typename T>
__device__ __forceinline__ void rotate8(const RopeDev& rope, const T* row, const int (&pos)[CONDUIT_MAX_AXES], int i0,
                                        bool wide, float (&x)[8]) {
  if (i0 >= rope.rot) return;
  const bool halves = rope.layout == CONDUIT_ROPE_HALVES;
  float other[8];
  if (halves && rope.half % 8 == 0 && i0 + 8 <= rope.rot) {
    load8(row + (i0 < rope.half ? i0 + rope.half : i0 - rope.half), wide, other);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int i = i0 + e;
      const int j = !halves ? i ^ 1 : i < rope.half ? i + rope.half : i - rope.half;
      other[e] = i < rope.rot ? to_float(row[j]) : 0.f;
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int i = i0 + e;
    if (i >= rope.rot) continue;
    const bool first = halves ? i < rope.half : !(i & 1);
    const int p = halves ? (first ? i : i - rope.half) : i >> 1;
    const int a = (rope.axis[p >> 4] >> (2 * (p & 15))) & 3;
    const int at = a == 0 ? pos[0] : a == 1 ? pos[1] : a == 2 ? pos[2] : pos[3];
    const float2 cs = rope.table[int64_t(at) * rope.half + p];
    const float s = first ? -cs.y : cs.y;
    x[e] = __fadd_rn(__fmul_rn(x[e], cs.x), __fmul_rn(other[e], s));
  }
}

// Four neighbouring lanes hold a group of 32 dims; returns this lane's eight codes
// (0..15) as nibbles of a word, and the group's (s, m).
__device__ __forceinline__ uint32_t pack8(const float (&in)[8], __half2* param, bool* nonfinite) {
  float x[8], lo = INFINITY, hi = -INFINITY;
  bool nan = false, bad = false;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    nan |= in[e] != in[e];
    bad |= !(fabsf(in[e]) < INFINITY);
    x[e] = fminf(fmaxf(in[e], -kClip), kClip);
    lo = fminf(lo, x[e]);
    hi = fmaxf(hi, x[e]);
  }
  int any = nan;
#pragma unroll
  for (int o = 1; o < 4; o <<= 1) {
    lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    any |= __shfl_xor_sync(0xffffffffu, any, o);
  }
  const __half s = __float2half_rn(__fmul_rn(__fsub_rn(hi, lo), 1.f / 15.f));
  const __half m = __float2half_rn(__fadd_rn(lo, 8.f * __half2float(s)));
  const float sf = __half2float(s), mf = __half2float(m);
  const float inv = sf > 0.f ? 1.f / sf : 0.f;
  uint32_t w = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float c = fminf(fmaxf(rintf(__fmul_rn(__fsub_rn(x[e], mf), inv)), -8.f), 7.f);
    w |= uint32_t(int(c) + 8) << (4 * e);
  }
  *param = any ? __halves2half2(__float2half_rn(0.f), __float2half_rn(NAN)) : __halves2half2(s, m);
  *nonfinite = bad;
  return w;
}

// Blocks below kv_blocks pack keys and values: a thread owns 8 dims of a row, four
// threads a group. The blocks after them rotate queries, a pair unit per thread.
template <typename T, int VEC>
__global__ void __launch_bounds__(kThreads)
    packed_append_kernel(PackedDev kv, SeqsDev s, RopeDev rope, int kv_blocks, bool wide, RowsDev k, RowsDev v,
                         RowsDev q, RowsDev q_out, int32_t* status) {
  const int r = blockIdx.y, l = blockIdx.z;
  const int t0 = s.row_off[r], n = s.row_off[r + 1] - t0;
  const bool pack = int(blockIdx.x) < kv_blocks;
  const uint32_t lin = (pack ? blockIdx.x : blockIdx.x - kv_blocks) * uint32_t(kThreads) + threadIdx.x;
  const uint32_t per = pack ? kv.d / 8 : units_per_row<VEC>(rope, kv.d), heads = pack ? 2 * kv.Hkv : kv.Hq;
  const int u = int(lin % per), h = int(lin / per % heads);
  const int64_t i64 = lin / per / heads;
  const int i = int(i64);
  bool live = i < n;
  const int64_t t = int64_t(t0) + i;
  const int slot = live ? s.len[r] - n + i : 0;
  bool ok = live && slot >= 0 && slot < s.max_len && slot < kv.capacity();
  int page = 0;
  if (ok) {
    page = kv.page_table[int64_t(r) * kv.max_pages + (slot >> kv.page_shift)];
    ok = page >= 0 && page < kv.P;
  }
  int pos[CONDUIT_MAX_AXES] = {0, 0, 0, 0};
  if (ok && rope.rot) {
#pragma unroll
    for (int a = 0; a < CONDUIT_MAX_AXES; ++a)
      if (a < rope.axes) {
        pos[a] = rope.pos[int64_t(a) * rope.T + t];
        ok &= pos[a] >= 0 && pos[a] < rope.len;
      }
  }
  if (live && !ok && u == 0 && h == 0) flag_status(status, CONDUIT_FLAG_INDEX);
  if (!pack) {
    if (!ok) return;
    using C = Chunk<T, VEC>;
    const Unit un = unit_of<VEC>(rope, u);
    const T* src = static_cast<const T*>(q.p) + l * q.ls + t * q.rs + h * q.hs;
    T* dst = static_cast<T*>(q_out.p) + l * q_out.ls + t * q_out.rs + h * q_out.hs;
    C a = *reinterpret_cast<const C*>(src + un.a);
    if (un.turns) {
      float2 cs[VEC];
      load_turn<VEC>(rope, t, u * VEC, cs);
      C b = *reinterpret_cast<const C*>(src + un.b);
      turn_chunks<T, VEC>(rope, cs, a, b);
      *reinterpret_cast<C*>(dst + un.b) = b;
    }
    *reinterpret_cast<C*>(dst + un.a) = a;
    return;
  }
  const int is_v = h >= kv.Hkv, g = is_v ? h - kv.Hkv : h;
  float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  if (ok) {
    const RowsDev& from = is_v ? v : k;
    const T* row = static_cast<const T*>(from.p) + l * from.ls + t * from.rs + g * from.hs;
    load8(row + 8 * u, wide, x);
    if (!is_v) rotate8(rope, row, pos, 8 * u, wide, x);
  }
  __half2 param;
  bool bad;
  const uint32_t w = pack8(x, &param, &bad);  // whole warps: four lanes of a group share `ok`
  if (!ok) return;
  if (bad) flag_status(status, CONDUIT_FLAG_NONFINITE);
  uint8_t* at = kv.page(l, g, page);
  const int row = slot & ((1 << kv.page_shift) - 1), groups = kv.d / 32, grp = u / 4, c = u % 4;
  uint8_t* codes = at + kv.codes(is_v, row);
  if (is_v) {
    uint16_t* half_words = reinterpret_cast<uint16_t*>(codes);
    half_words[(2 * c) * groups + grp] = uint16_t(w);
    half_words[(2 * c + 1) * groups + grp] = uint16_t(w >> 16);
  } else {
    reinterpret_cast<uint32_t*>(codes)[c * groups + grp] = w;
  }
  if (c == 0) reinterpret_cast<__half2*>(at + kv.params(is_v, row))[grp] = param;
}

// A thread turns 8 dims of a token's K and of its V into values.
template <typename T>
__global__ void __launch_bounds__(kThreads)
    packed_read_kernel(PackedDev kv, const int32_t* first, KvDev dst, BatchDev b, int32_t* status) {
  const int r = blockIdx.y, l = blockIdx.z;
  const int t0 = b.tok_off[r], n = b.tok_off[r + 1] - t0;
  const uint32_t per = kv.d / 8, lin = blockIdx.x * uint32_t(kThreads) + threadIdx.x;
  const int u = int(lin % per), g = int(lin / per % kv.Hkv), t = int(lin / per / kv.Hkv);
  if (t >= n) return;
  const int64_t from = int64_t(first ? first[r] : 0) + t;
  bool ok = from >= 0 && from < kv.capacity();
  int page = 0;
  if (ok) {
    page = kv.page_table[int64_t(r) * kv.max_pages + (from >> kv.page_shift)];
    ok = page >= 0 && page < kv.P;
  }
  if (ok && dst.page_size) {
    const int to = dst.page_table[int64_t(r) * dst.max_pages + t / dst.page_size];
    ok = to >= 0 && to < dst.num_pages;
  }
  if (!ok) {
    if (u == 0 && g == 0) flag_status(status, CONDUIT_FLAG_INDEX);
    return;
  }
  const uint8_t* at = kv.page(l, g, page);
  const int row = int(from) & ((1 << kv.page_shift) - 1), groups = kv.d / 32, grp = u / 4, c = u % 4;
  const int64_t out = dst.row(l, g, r, int64_t(t0) + t, t) + 8 * u;
#pragma unroll
  for (int is_v = 0; is_v < 2; ++is_v) {
    const uint8_t* codes = at + kv.codes(is_v, row);
    uint32_t w;
    if (is_v) {
      const uint16_t* half_words = reinterpret_cast<const uint16_t*>(codes);
      w = half_words[(2 * c) * groups + grp] | uint32_t(half_words[(2 * c + 1) * groups + grp]) << 16;
    } else {
      w = reinterpret_cast<const uint32_t*>(codes)[c * groups + grp];
    }
    const float2 sm = __half22float2(reinterpret_cast<const __half2*>(at + kv.params(is_v, row))[grp]);
    constexpr int N = 16 / sizeof(T);
    T* to = static_cast<T*>(is_v ? dst.v : dst.k) + out;
#pragma unroll
    for (int p = 0; p < 8 / N; ++p) {
      Chunk<T, N> y;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const int code = int((w >> (4 * (p * N + e))) & 15u) - 8;
        y.v[e] = from_float<T>(fmaf(sm.x, float(code), sm.y));  // s c is exact in fp32
      }
      *reinterpret_cast<Chunk<T, N>*>(to + p * N) = y;
    }
  }
}

template <typename T, int VEC>
cudaError_t append(const PackedDev& kv, const SeqsDev& s, const RopeDev& rope, bool wide, const RowsDev& k,
                   const RowsDev& v, const RowsDev& q, const RowsDev& q_out, int32_t* status, cudaStream_t stream) {
  auto blocks = [&](int64_t threads) { return int((threads + kThreads - 1) / kThreads); };
  const int kv_blocks = blocks(int64_t(s.max_rows) * 2 * kv.Hkv * (kv.d / 8));
  const int q_blocks = q.p ? blocks(int64_t(s.max_rows) * kv.Hq * units_per_row<VEC>(rope, kv.d)) : 0;
  packed_append_kernel<T, VEC><<<dim3(kv_blocks + q_blocks, s.R, kv.L), kThreads, 0, stream>>>(
      kv, s, rope, kv_blocks, wide, k, v, q, q_out, status);
  count_launches(1);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_packed_append(const PackedDev& kv, const SeqsDev& s, const RopeDev& rope, int dtype,
                                 const RowsDev& k, const RowsDev& v, const RowsDev& q, const RowsDev& q_out,
                                 int32_t* status, cudaStream_t stream) {
  const int vec = dtype == CONDUIT_BF16 ? 8 : 4;
  const bool wide = rows_aligned(k, vec) && rows_aligned(v, vec);
  const bool wide_q = q.p && dims_in_chunks(rope, kv.d, vec) && rows_aligned(q, vec) && rows_aligned(q_out, vec);
  if (dtype == CONDUIT_BF16)
    return wide_q ? append<__nv_bfloat16, 8>(kv, s, rope, wide, k, v, q, q_out, status, stream)
                  : append<__nv_bfloat16, 1>(kv, s, rope, wide, k, v, q, q_out, status, stream);
  return wide_q ? append<float, 4>(kv, s, rope, wide, k, v, q, q_out, status, stream)
                : append<float, 1>(kv, s, rope, wide, k, v, q, q_out, status, stream);
}

cudaError_t launch_packed_read(const PackedDev& kv, const int32_t* first, const KvDev& dst, const BatchDev& b,
                               int max_tokens, int32_t* status, cudaStream_t stream) {
  const int64_t threads = int64_t(max_tokens) * kv.Hkv * (kv.d / 8);
  const dim3 grid(unsigned((threads + kThreads - 1) / kThreads), b.R, kv.L);
  if (dst.dtype == CONDUIT_BF16)
    packed_read_kernel<__nv_bfloat16><<<grid, kThreads, 0, stream>>>(kv, first, dst, b, status);
  else
    packed_read_kernel<float><<<grid, kThreads, 0, stream>>>(kv, first, dst, b, status);
  count_launches(1);
  return cudaGetLastError();
}

}  // namespace conduit
