// The 4-bit cache: append with rotation and packing, and the read back into a
// plain cache.
//
// Mathematics: groups of 32 dims, s = fp16((hi - lo)/15), m = fp16(lo + 8 s),
// c = clamp(rint((x - m)/s), -8, 7); a value stands for m + s c. Every operation is
// a separately rounded fp32 one, so that a plain program finds the same codes.
// Bound: the rows once, and d + d/4 bytes per token and KV head of the cache; the append
// beside it by its issue slots (78 % busy: rotation, range, codes and their places, and at 72 registers
// a thread spills of 64 bytes in bf16 and 152 in fp32, read once each). Measured, 28
// layers of 8 192 tokens, 4 heads of 128 in bf16: append 176 us (3.5 TB/s), read 119 us (5.2 TB/s).
#include <algorithm>

#include "rotate.cuh"
#include "tc_common.cuh"

namespace conduit {
namespace {

constexpr int kThreads = 128;
constexpr float kClip = 61440.f;  // m +- 8 s stays inside fp16

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

// Least and largest of eight values; true if one of them is not finite.
__device__ __forceinline__ bool range8(const float (&x)[8], float* lo, float* hi) {
  *lo = fminf(x[0], x[1]);
  *hi = fmaxf(x[0], x[1]);
  float2 zero = make_float2(0.f, 0.f);
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    if (e) {
      *lo = tc::fmin3(*lo, x[e], x[e + 1]);
      *hi = tc::fmax3(*hi, x[e], x[e + 1]);
    }
    zero = tc::ffma2(make_float2(x[e], x[e + 1]), make_float2(0.f, 0.f), zero);  // NaN from NaN and infinities
  }
  return !(zero.x + zero.y == 0.f);
}

// Codes c + 8 of eight values as nibbles: c = rint((x - m) inv), clamped where `clamp`.
__device__ __forceinline__ uint32_t codes8(const float (&x)[8], float m, float inv, bool clamp) {
  uint32_t w = 0;
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    float2 c = tc::fmul2(tc::fadd2(make_float2(x[e], x[e + 1]), make_float2(-m, -m)), make_float2(inv, inv));
    if (clamp) c = make_float2(fminf(fmaxf(c.x, -8.f), 7.f), fminf(fmaxf(c.y, -8.f), 7.f));
    // 1.5 x 2^23 + 8 + c, rounded to an integer: bits 0x4B400000 + 8 + c, whose upper part is taken off the sum below
    c = add_rounded(c, make_float2(12582920.f, 12582920.f));
    w += __float_as_uint(c.x) << (4 * e);
    w += __float_as_uint(c.y) << (4 * e + 4);
  }
  constexpr uint32_t kUpper = 0x4B400000u * 0x11111111u;
  return w - kUpper;
}

// Four neighbouring lanes hold a group of 32 dims of a key (x) and of a value (y).
// Returns this lane's eight codes of each and the groups' (s, m); true if one of this
// lane's values is not finite. Called by whole warps. The lower two lanes of a group
// work out the key's s and m, the upper two the value's.
__device__ __forceinline__ bool pack8(float (&x)[8], float (&y)[8], int c, uint32_t* kw, uint32_t* vw, __half2* kp,
                                      __half2* vp) {
  constexpr unsigned kAll = 0xffffffffu;
  float lo[2], hi[2];
  const bool bad_x = range8(x, &lo[0], &hi[0]), bad_y = range8(y, &lo[1], &hi[1]);
  const bool bad = bad_x || bad_y;
  int nan = 0;
  const bool wild = bad || fmaxf(hi[0], hi[1]) > kClip || fminf(lo[0], lo[1]) < -kClip;
  if (__any_sync(kAll, wild)) {  // clip and look for NaN only where a group of the warp needs it
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      float(&z)[8] = b ? y : x;
      lo[b] = INFINITY;
      hi[b] = -INFINITY;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        nan |= int(z[e] != z[e]) << b;
        z[e] = fminf(fmaxf(z[e], -kClip), kClip);
        lo[b] = fminf(lo[b], z[e]);
        hi[b] = fmaxf(hi[b], z[e]);
      }
    }
    nan |= __shfl_xor_sync(kAll, nan, 1);
    nan |= __shfl_xor_sync(kAll, nan, 2);
  }
  // one lane of each pair carries the key's range on, the other the value's
  const bool is_v = c & 2;
  float l = is_v ? lo[1] : lo[0], h = is_v ? hi[1] : hi[0];
  l = fminf(l, __shfl_xor_sync(kAll, is_v ? lo[0] : lo[1], 2));
  h = fmaxf(h, __shfl_xor_sync(kAll, is_v ? hi[0] : hi[1], 2));
  l = fminf(l, __shfl_xor_sync(kAll, l, 1));
  h = fmaxf(h, __shfl_xor_sync(kAll, h, 1));
  const __half s = __float2half_rn(__fmul_rn(__fsub_rn(h, l), 1.f / 15.f));
  const __half m = __float2half_rn(__fadd_rn(l, 8.f * __half2float(s)));
  const float sf = __half2float(s), mf = __half2float(m);
  const float inv = sf > 0.f ? __frcp_rn(sf) : 0.f;
  // codes leave -8 .. 7 only where the rounding of m is coarse next to s
  const bool clamp = __any_sync(kAll, !(__fmul_rn(__fsub_rn(l, mf), inv) > -8.5f && __fmul_rn(__fsub_rn(h, mf), inv) < 7.5f));
  __half2 own = __halves2half2(s, m);
  uint32_t other = __shfl_xor_sync(kAll, *reinterpret_cast<uint32_t*>(&own), 2);
  const float inv2 = __shfl_xor_sync(kAll, inv, 2);
  const __half2 theirs = *reinterpret_cast<__half2*>(&other);
  *kp = is_v ? theirs : own;
  *vp = is_v ? own : theirs;
  *kw = codes8(x, __high2float(*kp), is_v ? inv2 : inv, clamp);
  *vw = codes8(y, __high2float(*vp), is_v ? inv : inv2, clamp);
  const __half2 none = __halves2half2(__float2half_rn(0.f), __float2half_rn(NAN));
  if (nan & 1) *kp = none;
  if (nan & 2) *vp = none;
  return bad;
}

// Blocks below kv_blocks pack keys and values: a thread owns 8 dims of a row's heads hg,
// hg + HG, ... (four threads a group). The blocks after them rotate queries, a unit of
// pairs per thread. Either walks over layers blockIdx.z, + gridDim.z, ...: a row's place,
// positions and cosines are worked out once for all of them.
template <typename T, int VEC, int kPairing>
__global__ void __launch_bounds__(kThreads, 7)
    packed_append_kernel(PackedDev kv, SeqsDev s, RopeDev rope, int kv_blocks, int HG, bool wide, RowsDev k, RowsDev v,
                         RowsDev q, RowsDev q_out, int32_t* status) {
  const int r = blockIdx.y;
  const int t0 = s.row_off[r], n = s.row_off[r + 1] - t0, len = s.len[r];
  if (n == 0) return;
  const bool pack = int(blockIdx.x) < kv_blocks;
  const uint32_t lin = (pack ? blockIdx.x : blockIdx.x - kv_blocks) * uint32_t(kThreads) + threadIdx.x;
  const uint32_t per = pack ? kv.d / 8 : units_per_row<VEC>(rope, kv.d), heads = pack ? HG : kv.Hq;
  const uint32_t rest = lin / per;
  const int u = int(lin - rest * per), i = int(rest / heads), h0 = int(rest - uint32_t(i) * heads);
  const bool live = i < n;
  const int64_t t = int64_t(t0) + (live ? i : 0);
  const int slot = len - n + i;
  bool ok = live && slot >= 0 && slot < s.max_len && slot < kv.capacity();
  const int page = kv.page_table[int64_t(r) * kv.max_pages + (ok ? slot >> kv.page_shift : 0)];
  ok &= page >= 0 && page < kv.P;
  int pos[CONDUIT_MAX_AXES];
  if (rope.rot) ok &= load_positions(rope, t, pos);
  if (live && !ok && u == 0 && h0 == 0) flag_status(status, CONDUIT_FLAG_INDEX);
  if (!pack) {
    if (!ok) return;
    using C = Chunk<T, VEC>;
    const Unit un = unit_of<VEC>(rope, kv.d, u);
    float2 cs[VEC];
    if (un.turns) load_turn<VEC>(rope, pos, u * VEC, cs);
    for (int l = blockIdx.z; l < kv.L; l += gridDim.z) {
      const T* src = static_cast<const T*>(q.p) + l * q.ls + t * q.rs + h0 * q.hs;
      T* dst = static_cast<T*>(q_out.p) + l * q_out.ls + t * q_out.rs + h0 * q_out.hs;
      C a = *reinterpret_cast<const C*>(src + un.a), b;
      if (un.b >= 0) b = *reinterpret_cast<const C*>(src + un.b);
      if (un.turns) turn_chunks<T, VEC>(rope, cs, a, b);
      *reinterpret_cast<C*>(dst + un.a) = a;
      if (un.b >= 0) *reinterpret_cast<C*>(dst + un.b) = b;
    }
    return;
  }
  float2 cs[8];
  if (ok) load_turn8<kPairing>(rope, pos, 8 * u, cs);
  const int row = slot & ((1 << kv.page_shift) - 1), groups = kv.d / 32, grp = u / 4, c = u % 4;
  bool bad = false;
  // Layer by layer and head by head, the next rows under way while one is packed. A thread without
  // a row reads row 0's; the count of heads is the same for every thread of a warp, past the last
  // one it is read again.
  const int i0 = 8 * u, far0 = i0 >= rope.rot ? i0 : i0 < rope.half ? i0 + rope.half : i0 - rope.half;
  const int steps = (kv.Hkv + HG - 1) / HG;
  const T *kr = nullptr, *vr = nullptr;
  Raw8<T> k_raw, far_raw, v_raw;
  auto fetch = [&](int l, int step) {
    const int g = min(h0 + step * HG, kv.Hkv - 1);
    kr = static_cast<const T*>(k.p) + l * k.ls + t * k.rs + g * k.hs;
    vr = static_cast<const T*>(v.p) + l * v.ls + t * v.rs + g * v.hs;
    k_raw = load8(kr + i0, wide);
    if (kPairing == kChunks) far_raw = load8(kr + far0, wide);
    v_raw = load8(vr + i0, wide);
  };
  int l = blockIdx.z;
  if (l < kv.L) fetch(l, 0);
  while (l < kv.L) {
    // the first head's places; a head is a page record further
    uint8_t* at = kv.page(l, h0, ok ? page : 0);
    uint32_t* key_word = reinterpret_cast<uint32_t*>(at + kv.codes(0, row)) + c * groups + grp;
    uint16_t* value_words = reinterpret_cast<uint16_t*>(at + kv.codes(1, row)) + 2 * c * groups + grp;
    __half2* params = reinterpret_cast<__half2*>(at + kv.params(c >> 1, row)) + grp;
    const int next_l = l + gridDim.z;
    for (int step = 0; step < steps; ++step) {
      float x[8], y[8];
      to_floats(k_raw, x);
      to_floats(v_raw, y);
      if (ok) turn8<kPairing>(rope, kr, i0, far_raw, cs, x);
      if (step + 1 < steps)
        fetch(l, step + 1);
      else if (next_l < kv.L)
        fetch(next_l, 0);
      uint32_t kw, vw;
      __half2 kp, vp;
      const bool wild = pack8(x, y, c, &kw, &vw, &kp, &vp);
      if (ok && h0 + step * HG < kv.Hkv) {
        bad |= wild;
        *key_word = kw;
        value_words[0] = uint16_t(vw);
        value_words[groups] = uint16_t(vw >> 16);
        if ((c & 1) == 0) *params = c ? vp : kp;
      }
      key_word += HG * kv.page_bytes / 4;
      value_words += HG * kv.page_bytes / 2;
      params += HG * kv.page_bytes / 4;
    }
    l = next_l;
  }
  if (bad) flag_status(status, CONDUIT_FLAG_NONFINITE);
}

// The eight codes of a word as values m + s c, in order; s c is exact in fp32.
template <typename T>
__device__ __forceinline__ void store_values(T* to, uint32_t w, __half2 param) {
  const float2 sm = __half22float2(param);
  constexpr int N = 16 / sizeof(T);
#pragma unroll
  for (int p = 0; p < 8 / N; ++p) {
    Chunk<T, N> y;
#pragma unroll
    for (int e = 0; e < N; e += 2) {
      const int at = 4 * (p * N + e);  // the nibbles under the exponent of 2^23 are 2^23 + u
      float2 u = make_float2(__uint_as_float(((w >> at) & 15u) | 0x4B000000u),
                             __uint_as_float(((w >> (at + 4)) & 15u) | 0x4B000000u));
      u = tc::ffma2(make_float2(sm.x, sm.x), tc::fadd2(u, make_float2(-8388616.f, -8388616.f)), make_float2(sm.y, sm.y));
      y.v[e] = from_float<T>(u.x);
      y.v[e + 1] = from_float<T>(u.y);
    }
    store_once<T, N>(to + p * N, y);
  }
}

// A thread turns 8 dims of a token's K and V into values, for heads hg, hg + HG, ...
template <typename T>
__global__ void __launch_bounds__(kThreads, 10)
    packed_read_kernel(PackedDev kv, const int32_t* first, KvDev dst, BatchDev b, int HG, int32_t* status) {
  const int r = blockIdx.y;
  const int t0 = b.tok_off[r], n = b.tok_off[r + 1] - t0;
  const uint32_t per = kv.d / 8, lin = blockIdx.x * uint32_t(kThreads) + threadIdx.x;
  const uint32_t rest = lin / per;
  const int u = int(lin - rest * per), t = int(rest / uint32_t(HG)), hg = int(rest - uint32_t(t) * HG);
  if (t >= n) return;
  const int64_t from = int64_t(first ? first[r] : 0) + t;
  bool ok = from >= 0 && from < kv.capacity();
  const int page = kv.page_table[int64_t(r) * kv.max_pages + (ok ? from >> kv.page_shift : 0)];
  ok &= page >= 0 && page < kv.P;
  if (ok && dst.page_size) {
    const int to = dst.page_table[int64_t(r) * dst.max_pages + t / dst.page_size];
    ok = to >= 0 && to < dst.num_pages;
  }
  if (!ok) {
    if (u == 0 && hg == 0) flag_status(status, CONDUIT_FLAG_INDEX);
    return;
  }
  const int row = int(from) & ((1 << kv.page_shift) - 1), groups = kv.d / 32, grp = u / 4, c = u % 4;
  const int64_t step = (dst.page_size ? int64_t(dst.page_size) : dst.n_tot) * dst.d;  // a head of dst
  for (int l = blockIdx.z; l < kv.L; l += gridDim.z) {
    const uint8_t* at = kv.page(l, 0, page);
    const int64_t out = dst.row(l, 0, r, int64_t(t0) + t, t) + 8 * u;
#pragma unroll 2
    for (int g = hg; g < kv.Hkv; g += HG) {
      const uint8_t* p = at + g * kv.page_bytes;
      const uint32_t kw = reinterpret_cast<const uint32_t*>(p + kv.codes(0, row))[c * groups + grp];
      const uint16_t* half_words = reinterpret_cast<const uint16_t*>(p + kv.codes(1, row));
      const uint32_t v0 = half_words[(2 * c) * groups + grp], v1 = half_words[(2 * c + 1) * groups + grp];
      const __half2 kp = reinterpret_cast<const __half2*>(p + kv.params(0, row))[grp];
      const __half2 vp = reinterpret_cast<const __half2*>(p + kv.params(1, row))[grp];
      store_values(static_cast<T*>(dst.k) + out + g * step, kw, kp);
      store_values(static_cast<T*>(dst.v) + out + g * step, v0 | v1 << 16, vp);
    }
  }
}

// How many heads and layers a thread takes: one while the launch does not fill the SMs twice,
// then up to four heads, then up to eight layers (8 192 tokens of 28 layers, 4 heads of 128
// dims, append: one layer a thread 241 us, eight 203; one head and one layer 400).
struct Share {
  int head_groups, layer_groups;
};
Share share_of(int64_t rows, int heads, int layers) {
  const int64_t full = 2 * 152 * 1024, threads = rows * heads * layers;
  const int per_head = int(std::min<int64_t>(4, std::max<int64_t>(1, threads / full)));
  const int groups = (heads + per_head - 1) / per_head;
  const int per_layer = int(std::min<int64_t>(8, std::max<int64_t>(1, rows * groups * layers / full)));
  return Share{groups, (layers + per_layer - 1) / per_layer};
}

template <typename T, int VEC, int kPairing>
cudaError_t append_with(const PackedDev& kv, const SeqsDev& s, const RopeDev& rope, bool wide, const RowsDev& k,
                        const RowsDev& v, const RowsDev& q, const RowsDev& q_out, int32_t* status,
                        cudaStream_t stream) {
  auto blocks = [&](int64_t threads) { return int((threads + kThreads - 1) / kThreads); };
  const int64_t rows = int64_t(s.max_rows) * (kv.d / 8);
  const Share share = share_of(rows * s.R, kv.Hkv, kv.L);
  const int HG = share.head_groups;
  const int kv_blocks = blocks(rows * HG);
  const int q_blocks = q.p ? blocks(int64_t(s.max_rows) * kv.Hq * units_per_row<VEC>(rope, kv.d)) : 0;
  packed_append_kernel<T, VEC, kPairing><<<dim3(kv_blocks + q_blocks, s.R, share.layer_groups), kThreads, 0, stream>>>(
      kv, s, rope, kv_blocks, HG, wide, k, v, q, q_out, status);
  count_launches(1);
  return cudaGetLastError();
}

template <typename T, int VEC>
cudaError_t append(const PackedDev& kv, const SeqsDev& s, const RopeDev& rope, bool wide, const RowsDev& k,
                   const RowsDev& v, const RowsDev& q, const RowsDev& q_out, int32_t* status, cudaStream_t stream) {
  switch (pairing(rope)) {
    case kNoTurn: return append_with<T, VEC, kNoTurn>(kv, s, rope, wide, k, v, q, q_out, status, stream);
    case kChunks: return append_with<T, VEC, kChunks>(kv, s, rope, wide, k, v, q, q_out, status, stream);
    case kNeighbours: return append_with<T, VEC, kNeighbours>(kv, s, rope, wide, k, v, q, q_out, status, stream);
    default: return append_with<T, VEC, kAnywhere>(kv, s, rope, wide, k, v, q, q_out, status, stream);
  }
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
  const int64_t rows = int64_t(max_tokens) * (kv.d / 8);
  const Share share = share_of(rows * b.R, kv.Hkv, kv.L);
  const int HG = share.head_groups;
  const int64_t threads = rows * HG;
  const dim3 grid(unsigned((threads + kThreads - 1) / kThreads), b.R, share.layer_groups);
  if (dst.dtype == CONDUIT_BF16)
    packed_read_kernel<__nv_bfloat16><<<grid, kThreads, 0, stream>>>(kv, first, dst, b, HG, status);
  else
    packed_read_kernel<float><<<grid, kThreads, 0, stream>>>(kv, first, dst, b, HG, status);
  count_launches(1);
  return cudaGetLastError();
}

}  // namespace conduit
