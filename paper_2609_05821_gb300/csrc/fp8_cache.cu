// The 8-bit cache: append with rotation and the scales of blocks, and the read back into a plain cache.
//
// Mathematics: a block of 16 tokens of a head shares e, the least with max |x| <= 448 2^e;
// code = e4m3(x 2^-e), a value stands for code 2^e. Powers of two scale exactly, so a value is
// rounded once, and the rotation's fp32 operations are rounded one by one: a plain program finds the same codes.
//
// Shape: a warp owns a block of one head (two heads of 64 dims, four of 32), keys first, then
// values: both have to be seen whole before the first code. Lane 16 c + u has dims 8 u .. 8 u + 7
// (and, past 128 dims, 8 (u + 16) ..) of the tokens of parity c, so a row is read in one piece by
// 16 lanes; the codes of a value column meet in pairs of lanes that swap half of their dims. A CTA stays with a
// block of tokens over its heads and layers: cosines and signed sines of the block's tokens lie in shared memory, dim by dim.
// Rows pass through shared memory too, each of a warp's two buffers filled again as soon as it has been read: the values of
// a unit are on their way while its keys are packed, the next unit's keys meanwhile (in registers: 316 us for append and read of
// 28 layers of 8 192 tokens, 281 so).
// Bound: the rows once and 2 d + 1 bytes a token and head of the cache. Measured, 28 layers of 8 192 tokens, 4 heads of 128 in
// bf16: append 159 us (4.4 TB/s; the load/store unit is 66 % busy, nearly half of it the keys' reads from shared memory, and 168
// registers leave 12 warps an SM), read 102 us (6.9 TB/s, at the copy rate). One token of 64 requests: append 10 us, read 6.
#include <algorithm>
#include <type_traits>

#include "fp8.cuh"
#include "rotate.cuh"
#include "tc_common.cuh"
#include "turn8.cuh"

namespace conduit {
namespace {

constexpr int kThreads = 128;

// Lanes of a head's row, and heads that share a warp.
__host__ __device__ constexpr int heads_per_warp(int d) { return d <= 32 ? 4 : d <= 64 ? 2 : 1; }

// Where this lane stands: head of the warp's, chunk of 8 dims, parity of its tokens.
struct Place {
  int head, u, c;
  bool on;
};
__device__ __forceinline__ Place place_in_warp(int d, int lane) {
  const int per = 16 / heads_per_warp(d), in = lane & 15;
  return Place{in / per, in % per, lane >> 4, in % per < d / 8};
}
// The largest over the lanes of a head.
__device__ __forceinline__ float head_max(float x, int d) {
  constexpr unsigned kAll = 0xffffffffu;
  x = fmaxf(x, __shfl_xor_sync(kAll, x, 16));
#pragma unroll
  for (int s = 1; s < 16; s <<= 1) {
    const float y = __shfl_xor_sync(kAll, x, s);
    if (s < 16 / heads_per_warp(d)) x = fmaxf(x, y);
  }
  return x;
}

// Largest |x| of eight numbers into top; wild becomes NaN where one is not finite.
__device__ __forceinline__ void look_at(const float (&x)[8], float* top, float2* wild) {
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    *top = tc::fmax3(*top, fabsf(x[e]), fabsf(x[e + 1]));
    *wild = tc::ffma2(make_float2(x[e], x[e + 1]), make_float2(0.f, 0.f), *wild);
  }
}
// NaN and infinities of a lane's numbers become NaN and leave the largest alone.
template <int NC>
__device__ __forceinline__ void mend(float (&x)[NC][8][8], float* top) {
  *top = 0.f;
#pragma unroll
  for (int m = 0; m < NC; ++m)
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (fabsf(x[m][i][e]) < INFINITY)
          *top = fmaxf(*top, fabsf(x[m][i][e]));
        else
          x[m][i][e] = NAN;
      }
}

// Word of four codes, rescaled by 2^n (n <= 0): exact products, one rounding.
__device__ __forceinline__ uint32_t rescaled(uint32_t w, float by) {
  const float2 a = floats_lo(w), b = floats_hi(w);
  return fp8_pair(a.x * by, a.y * by) | fp8_pair(b.x * by, b.y * by) << 16;
}

// A whole block's codes. K: each lane has its chunk of eight tokens of parity c, x[i] of token 2 i + c.
template <int NC>
__device__ __forceinline__ void put_keys(uint8_t* block, const Place& p, int d, int e, const float (&x)[NC][8][8]) {
  const float down = power_of_two(-e);
#pragma unroll
  for (int n = 0; n < NC; ++n) {
    const int u = p.u + 16 * n;
    if (!p.on || u >= d / 8) continue;
    uint8_t* at = block + (u >> 1) * 128 + (u & 1) * 8;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int t = 2 * i + p.c;
      float y[8];
#pragma unroll
      for (int k = 0; k < 8; k += 2) {
        const float2 z = tc::fmul2(make_float2(x[n][i][k], x[n][i][k + 1]), make_float2(down, down));
        y[k] = z.x, y[k + 1] = z.y;
      }
      *reinterpret_cast<uint2*>(at + (t >> 3) * 8 * d + (t & 7) * 16) =
          make_uint2(fp8_pair(y[0], y[1]) | fp8_pair(y[2], y[3]) << 16, fp8_pair(y[4], y[5]) | fp8_pair(y[6], y[7]) << 16);
    }
  }
}

// The same of the values, whose rows are dims: byte 4 a + 2 b + c of a row is token 8 b + 2 a + c, so a
// lane's codes of tokens 2 a + c and 2 a + 8 + c are the halfword (a, c) and its partner's the other.
template <int NC>
__device__ __forceinline__ void put_values(uint8_t* block, const Place& p, int d, int e, const float (&x)[NC][8][8]) {
  constexpr unsigned kAll = 0xffffffffu;
  const float down = power_of_two(-e);
#pragma unroll
  for (int n = 0; n < NC; ++n) {
    const int u = p.u + 16 * n;
    uint32_t w[8][2];  // dim k: halfwords a = 0, 1 and a = 2, 3
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      uint32_t h[4];
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        const float2 y = tc::fmul2(make_float2(x[n][a][k], x[n][a + 4][k]), make_float2(down, down));
        h[a] = fp8_pair(y.x, y.y);
      }
      w[k][0] = h[0] | h[1] << 16;
      w[k][1] = h[2] | h[3] << 16;
    }
    uint4* rows = reinterpret_cast<uint4*>(block + 16 * d + (8 * u + 4 * p.c) * 16);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      // parity 0 keeps dims 0-3 and hands on 4-7, parity 1 the other way round
      uint32_t own[2], got[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        own[j] = p.c ? w[k + 4][j] : w[k][j];
        got[j] = __shfl_xor_sync(kAll, p.c ? w[k][j] : w[k + 4][j], 16);
      }
      const uint32_t even[2] = {p.c ? got[0] : own[0], p.c ? got[1] : own[1]};
      const uint32_t odd[2] = {p.c ? own[0] : got[0], p.c ? own[1] : got[1]};
      // even: tokens (2 a, 2 a + 8), odd: (2 a + 1, 2 a + 9)
      if (p.on && u < d / 8)
        rows[k] = make_uint4(__byte_perm(even[0], odd[0], 0x5140), __byte_perm(even[0], odd[0], 0x7362),
                             __byte_perm(even[1], odd[1], 0x5140), __byte_perm(even[1], odd[1], 0x7362));
    }
  }
}

// CTAs below kv_grid: a block of the call's tokens, its heads and layers dealt out over the warps of grid.z. Those after
// them rotate queries, a unit of pairs per thread, and walk over the layers.
template <typename T, bool kWide, int kPairing, int NC>
__global__ void __launch_bounds__(kThreads, NC == 1 ? 3 : 2)
    fp8_append_kernel(PackedDev kv, SeqsDev s, RopeDev rope, int kv_grid, RowsDev k, RowsDev v, RowsDev q, RowsDev q_out,
                      int32_t* status) {
  constexpr int VEC = kWide ? 16 / int(sizeof(T)) : 1;
  const int r = blockIdx.y;
  const int t0 = s.row_off[r], n = s.row_off[r + 1] - t0, len = s.len[r];
  if (n == 0) return;
  const int64_t begin = int64_t(len) - n;  // slot of the call's first row
  if (int(blockIdx.x) >= kv_grid) {
    const uint32_t lin = (blockIdx.x - kv_grid) * uint32_t(kThreads) + threadIdx.x;
    const uint32_t per = units_per_row<VEC>(rope, kv.d), rest = lin / per;
    const int u = int(lin - rest * per), i = int(rest / uint32_t(kv.Hq)), h = int(rest - uint32_t(i) * kv.Hq);
    if (i >= n) return;
    const int64_t t = int64_t(t0) + i;
    const int64_t slot = begin + i;
    bool ok = slot >= 0 && slot < s.max_len && slot < kv.capacity();
    const int page = kv.page_table[int64_t(r) * kv.max_pages + (ok ? int(slot) >> kv.page_shift : 0)];
    ok &= page >= 0 && page < kv.P;
    int pos[CONDUIT_MAX_AXES];
    if (rope.rot) ok &= load_positions(rope, t, pos);
    if (!ok) return;  // flagged beside the row's key
    using C = Chunk<T, VEC>;
    const Unit un = unit_of<VEC>(rope, kv.d, u);
    float2 cs[VEC];
    if (un.turns) load_turn<VEC>(rope, pos, u * VEC, cs);
    for (int l = blockIdx.z; l < kv.L; l += gridDim.z) {
      const T* src = static_cast<const T*>(q.p) + l * q.ls + t * q.rs + h * q.hs;
      T* dst = static_cast<T*>(q_out.p) + l * q_out.ls + t * q_out.rs + h * q_out.hs;
      C a = *reinterpret_cast<const C*>(src + un.a), b;
      if (un.b >= 0) b = *reinterpret_cast<const C*>(src + un.b);
      if (un.turns) turn_chunks<T, VEC>(rope, cs, a, b);
      *reinterpret_cast<C*>(dst + un.a) = a;
      if (un.b >= 0) *reinterpret_cast<C*>(dst + un.b) = b;
    }
    return;
  }
  // slots count from the block of the first row (rows before slot 0 lie in blocks of their own)
  const int64_t first = (begin >> 4) * 16 + 16 * int64_t(blockIdx.x);
  if (first >= len) return;
  const int lane = threadIdx.x % 32, hp = heads_per_warp(kv.d), groups = (kv.Hkv + hp - 1) / hp;
  const Place p = place_in_warp(kv.d, lane);

  // Which of the block's tokens belong to the call. Their rows, page, positions and cosines go out together: a decoding
  // step is a chain of loads, and none of these waits for another but the cosines for the positions.
  const int64_t own_slot = first + (lane & 15);  // lane t looks at token t
  const bool called = own_slot >= begin && own_slot < len;
  const uint32_t asked = __ballot_sync(0xffffffffu, called) & 0xFFFFu, my_asked = (asked >> p.c) & 0x5555u;  // bit 2 i: token 2 i + c
  const int64_t row0 = int64_t(t0) + (first - begin);  // row of the call of the block's token 0
  const int units = groups * kv.L, step = gridDim.z * (kThreads / 32), first_unit = blockIdx.z * (kThreads / 32) + threadIdx.x / 32;
  // [16][2][d / 8][4] cosines, then signed sines: dims 8 u + 4 h .. of a token at [h][u], so that the lanes of a row read side by side
  extern __shared__ __align__(16) float turns[];
  float *cosines = turns, *sines = turns + kBlockTokens * kv.d;
  // this warp's rows: 16 tokens of a unit's keys, and of its values
  const int row_bytes = hp * kv.d * int(sizeof(T));
  uint8_t* rows_at = reinterpret_cast<uint8_t*>(turns) + (kPairing == kNoTurn ? 0 : 2 * kBlockTokens * kv.d * int(sizeof(float))) +
                     threadIdx.x / 32 * 2 * kBlockTokens * row_bytes;
  auto head_of = [&](int n) { return n % groups * hp + p.head; };
  // dim i0 of this lane's token 2 i + c and head (a lane without a chunk is at the first one; what it reads is left out)
  auto row_at = [&](int which, int i, int i0) {
    return reinterpret_cast<T*>(rows_at + (which * kBlockTokens + 2 * i + p.c) * row_bytes) + p.head * kv.d + i0;
  };
  auto copy_rows = [&](auto all, const RowsDev& x, int which, int n) {
    const int head = head_of(n), l = n / groups;
    if (n < units && p.on && head < kv.Hkv) {
      const T* row = static_cast<const T*>(x.p) + l * x.ls + head * x.hs + (row0 + p.c) * x.rs + 8 * p.u;
#pragma unroll
      for (int i = 0; i < 8; ++i, row += 2 * x.rs) {
        if (!decltype(all)::value && !(my_asked >> (2 * i) & 1u)) continue;
#pragma unroll
        for (int m = 0; m < NC; ++m) {
          if (NC > 1 && p.u + 16 * m >= kv.d / 8) continue;
          T* to = row_at(which, i, 8 * (p.u + 16 * m));
          if (kWide) {
#pragma unroll
            for (int c = 0; c < int(sizeof(T) / 2); ++c)
              asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(tc::smem_u32(to) + 16 * c),
                           "l"(row + 128 * m + 16 / sizeof(T) * c)
                           : "memory");
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) to[e] = row[128 * m + e];
          }
        }
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  copy_rows(std::false_type{}, k, 0, first_unit);
  copy_rows(std::false_type{}, v, 1, first_unit);

  const int most = min(s.max_len, kv.capacity());
  bool in_range = first >= 0 && first < most;
  const int page = kv.page_table[int64_t(r) * kv.max_pages + (in_range ? int(first) >> kv.page_shift : 0)];
  bool fine = called;
  if (called && rope.rot) {
    int pos[CONDUIT_MAX_AXES];
    fine = load_positions(rope, int64_t(t0) + (own_slot - begin), pos);
  }
  if (kPairing != kNoTurn) {
    const int chunks = kv.d / 8;
    for (int e = threadIdx.x; e < kBlockTokens * chunks; e += kThreads) {
      const int t = e / chunks, i0 = e % chunks * 8;
      if (!(asked >> t & 1u)) continue;
      int pos[CONDUIT_MAX_AXES];
      if (!load_positions(rope, row0 + t, pos)) continue;
      float2 cs[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) cs[k] = make_float2(1.f, 0.f);
      load_turn8<kPairing>(rope, pos, i0, cs);
#pragma unroll
      for (int k = 0; k < 8; k += 4) {
        const int at = t * kv.d + (k * kv.d + 4 * i0) / 8;
        *reinterpret_cast<float4*>(cosines + at) = make_float4(cs[k].x, cs[k + 1].x, cs[k + 2].x, cs[k + 3].x);
        *reinterpret_cast<float4*>(sines + at) = make_float4(cs[k].y, cs[k + 1].y, cs[k + 2].y, cs[k + 3].y);
      }
    }
  }
  in_range &= page >= 0 && page < kv.P;
  const uint32_t now = __ballot_sync(0xffffffffu, fine && in_range && own_slot < most) & 0xFFFFu;  // the tokens that are written
  if (now != asked && threadIdx.x == 0 && blockIdx.z == 0) flag_status(status, CONDUIT_FLAG_INDEX);
  if (now == 0) {
    asm volatile("cp.async.wait_all;" ::: "memory");
    return;
  }
  const int before = int(min(max(begin - first, int64_t(0)), int64_t(16)));
  const uint32_t older = (1u << before) - 1u, mine = (now >> p.c) & 0x5555u;
  if (kPairing != kNoTurn) __syncthreads();

  auto rows_here = [&] {  // all but the last rows that this warp has asked for
    asm volatile("cp.async.wait_group 1;" ::: "memory");
    __syncwarp();
  };
  // A lane's eight numbers of token 2 i + c from dim i0 on, keys turned.
  auto numbers = [&](int which, int i, int i0, float (&y)[8]) {
    to_floats(load8(row_at(which, i, i0), true), y);
    if (which || kPairing == kNoTurn || i0 >= rope.rot) return;
    const int t = 2 * i + p.c;
    float other[8];
    if (kPairing == kChunks) {
      to_floats(load8(row_at(0, i, i0 < rope.half ? i0 + rope.half : i0 - rope.half), true), other);
    } else if (kPairing == kNeighbours) {
#pragma unroll
      for (int e = 0; e < 8; ++e) other[e] = y[e ^ 1];
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int at = i0 + e;
        const int j = rope.layout == CONDUIT_ROPE_PAIRS ? at ^ 1 : at < rope.half ? at + rope.half : at - rope.half;
        other[e] = at < rope.rot ? to_float(*row_at(0, i, j)) : 0.f;
      }
    }
    const float *c8 = cosines + t * kv.d + i0 / 2, *s8 = sines + t * kv.d + i0 / 2;
#pragma unroll
    for (int e = 0; e < 8; e += 4) {
      const float4 c = *reinterpret_cast<const float4*>(c8 + e * kv.d / 8), s = *reinterpret_cast<const float4*>(s8 + e * kv.d / 8);
      // the products are rounded before they are added; a dim past rot has cosine 1 and sine 0
      const float2 a0 = tc::fmul2(make_float2(y[e], y[e + 1]), make_float2(c.x, c.y));
      const float2 b0 = tc::fmul2(make_float2(other[e], other[e + 1]), make_float2(s.x, s.y));
      const float2 a1 = tc::fmul2(make_float2(y[e + 2], y[e + 3]), make_float2(c.z, c.w));
      const float2 b1 = tc::fmul2(make_float2(other[e + 2], other[e + 3]), make_float2(s.z, s.w));
      const float2 y0 = add_rounded(a0, b0), y1 = add_rounded(a1, b1);
      y[e] = y0.x, y[e + 1] = y0.y, y[e + 2] = y1.x, y[e + 3] = y1.y;
    }
  };
  bool bad = false;
  if (now == 0xFFFFu) {  // whole blocks: everything in registers between one reading and one writing
#pragma unroll 1
    for (int unit = first_unit; unit < units; unit += step) {
      const int head = head_of(unit);
      const bool on = p.on && head < kv.Hkv;
      const Place here{p.head, p.u, p.c, on};
      uint8_t* block = fp8_block(kv, unit / groups, on ? head : 0, page, int(first));
      float* scales = reinterpret_cast<float*>(block + 32 * kv.d);
      float x[NC][8][8];
      auto gather = [&](auto which, float* top) {
        float2 wild = make_float2(0.f, 0.f);
        *top = 0.f;
        rows_here();
#pragma unroll
        for (int m = 0; m < NC; ++m)
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int i0 = p.on ? 8 * (p.u + 16 * m) : 0;
            if (NC == 1 || i0 < kv.d) {
              numbers(decltype(which)::value, i, i0, x[m][i]);
            } else {
#pragma unroll
              for (int e = 0; e < 8; ++e) x[m][i][e] = 0.f;
            }
            look_at(x[m][i], top, &wild);
          }
        __syncwarp();
        copy_rows(std::true_type{}, decltype(which)::value ? v : k, decltype(which)::value, unit + step);
        if (!(wild.x + wild.y == 0.f)) bad |= on, mend(x, top);
        if (!on) *top = 0.f;
      };
      float top;
      gather(std::integral_constant<int, 0>{}, &top);
      int e = exponent_for(head_max(top, kv.d));
      put_keys<NC>(block, here, kv.d, e, x);
      if (on && p.u == 0 && p.c == 0) scales[0] = power_of_two(e);
      gather(std::integral_constant<int, 1>{}, &top);
      e = exponent_for(head_max(top, kv.d));
      put_values<NC>(block, here, kv.d, e, x);
      if (on && p.u == 0 && p.c == 0) scales[1] = power_of_two(e);
    }
  } else {
    // Part filled blocks, token by token and read twice (largest number, codes): a decoding step fetches this
    // code once a call, and its length is what the call takes (with all tokens' steps laid out 19 us for a step of 64 requests).
#pragma unroll 1
    for (int unit = first_unit; unit < units; unit += step) {
      const int head = head_of(unit);
      const bool on = p.on && head < kv.Hkv;
      uint8_t* block = fp8_block(kv, unit / groups, on ? head : 0, page, int(first));
      float* scales = reinterpret_cast<float*>(block + 32 * kv.d);
      float2 was2 = make_float2(0.f, 0.f);
      if (older) was2 = *reinterpret_cast<const float2*>(scales);
#pragma unroll 1
      for (int which = 0; which < 2; ++which) {
        rows_here();
        const int was = older ? exponent_of(which ? was2.y : was2.x) : kLeastExp;
        int e = was;
        float down = 0.f;
#pragma unroll 1
        for (int pass = 0; pass < 2; ++pass) {
          float top = 0.f;
#pragma unroll 1
          for (int i = 0; i < 8; i += 2) {  // two tokens of each parity side by side; what the call has none of is read and dropped
            if (!(now >> (2 * i) & 15u)) continue;
#pragma unroll 1
            for (int u = p.u; u < kv.d / 8; u += 16) {
              if (!on) continue;
              float y[2][8];
#pragma unroll
              for (int j = 0; j < 2; ++j) numbers(which, i + j, 8 * u, y[j]);
#pragma unroll
              for (int j = 0; j < 2; ++j) {
                const bool live = mine >> (2 * (i + j)) & 1u;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                  const bool finite = fabsf(y[j][k]) < INFINITY;
                  bad |= live && !finite;
                  y[j][k] = finite ? y[j][k] : NAN;
                  top = fmaxf(top, live ? fabsf(y[j][k]) : 0.f);
                }
              }
              if (pass == 0) continue;
#pragma unroll
              for (int j = 0; j < 2; ++j) {
                if (!(mine >> (2 * (i + j)) & 1u)) continue;
                const int t = 2 * (i + j) + p.c;
                uint32_t w[2];
#pragma unroll
                for (int k = 0; k < 2; ++k)
                  w[k] = fp8_pair(y[j][4 * k] * down, y[j][4 * k + 1] * down) | fp8_pair(y[j][4 * k + 2] * down, y[j][4 * k + 3] * down) << 16;
                if (which == 0) {
                  *reinterpret_cast<uint2*>(block + (t >> 3) * 8 * kv.d + (u >> 1) * 128 + (t & 7) * 16 + (u & 1) * 8) = make_uint2(w[0], w[1]);
                } else {
                  uint8_t* to = block + 16 * kv.d + 8 * u * 16 + (t & 7) / 2 * 4 + (t >> 3) * 2 + (t & 1);
#pragma unroll
                  for (int k = 0; k < 8; ++k) to[16 * k] = uint8_t(w[k / 4] >> (8 * (k % 4)));
                }
              }
            }
          }
          if (pass == 1) break;
          e = max(exponent_for(head_max(top, kv.d)), was);
          down = power_of_two(-e);
          if (__any_sync(0xffffffffu, on && older && was < e)) {  // (every lane of a head alike)
            const float by = power_of_two(max(was - e, -126));
            if (on && was < e) {
#pragma unroll 1
              for (int u = p.u; u < kv.d / 8; u += 16) {
                if (which == 0) {
#pragma unroll 1
                  for (int t = p.c; t < before; t += 2) {
                    uint2* at = reinterpret_cast<uint2*>(block + (t >> 3) * 8 * kv.d + (u >> 1) * 128 + (t & 7) * 16 + (u & 1) * 8);
                    const uint2 w = *at;
                    *at = make_uint2(rescaled(w.x, by), rescaled(w.y, by));
                  }
                } else {
#pragma unroll 1
                  for (int k = 0; k < 16; ++k) {  // words of dims 8 u + 4 c .. of four tokens each
                    const int a = k & 3;
                    uint32_t past = 0;
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                      if (8 * (j >> 1) + 2 * a + (j & 1) < before) past |= 0xFFu << (8 * j);
                    uint32_t* at = reinterpret_cast<uint32_t*>(block + 16 * kv.d + (8 * u + 4 * p.c + (k >> 2)) * 16) + a;
                    const uint32_t w = *at;
                    *at = (rescaled(w, by) & past) | (w & ~past);
                  }
                }
              }
            }
            __syncwarp();  // before other lanes write bytes of the same words
          }
        }
        __syncwarp();
        copy_rows(std::false_type{}, which ? v : k, which, unit + step);
        if (on && p.u == 0 && p.c == 0) scales[which] = power_of_two(e);
      }
    }
  }
  if (bad) flag_status(status, CONDUIT_FLAG_NONFINITE);
}

// Eight numbers as a row's elements.
template <typename T>
__device__ __forceinline__ void store8(T* to, const float (&x)[8]) {
  constexpr int N = 16 / sizeof(T);
#pragma unroll
  for (int p = 0; p < 8 / N; ++p) {
    Chunk<T, N> y;
#pragma unroll
    for (int e = 0; e < N; ++e) y.v[e] = from_float<T>(x[p * N + e]);
    store_once<T, N>(to + p * N, y);
  }
}

// A warp turns a block of one head (or of the heads that share a warp) into rows: the mapping of the append.
template <typename T>
__global__ void __launch_bounds__(kThreads)
    fp8_read_kernel(PackedDev kv, const int32_t* first, KvDev dst, BatchDev b, int32_t* status) {
  constexpr unsigned kAll = 0xffffffffu;
  const int r = blockIdx.y, l = blockIdx.z, lane = threadIdx.x % 32;
  const int t0 = b.tok_off[r], n = b.tok_off[r + 1] - t0;
  const int64_t from = first ? first[r] : 0;
  const int hp = heads_per_warp(kv.d), groups = (kv.Hkv + hp - 1) / hp;
  const uint32_t unit = blockIdx.x * uint32_t(kThreads / 32) + threadIdx.x / 32;
  const int64_t slot = (from >> 4) * 16 + 16 * int64_t(unit / uint32_t(groups));
  if (slot >= from + n) return;
  const int head0 = int(unit % uint32_t(groups)) * hp;
  const Place p = place_in_warp(kv.d, lane);
  const int head = head0 + p.head;
  const bool on = p.on && head < kv.Hkv;

  bool in_range = slot >= 0 && slot < kv.capacity();
  const int page = kv.page_table[int64_t(r) * kv.max_pages + (in_range ? int(slot) >> kv.page_shift : 0)];
  in_range &= page >= 0 && page < kv.P;
  const int64_t own = slot + (lane & 15) - from;  // lane t looks at token t
  const bool called = own >= 0 && own < n;
  bool fine = called && in_range;
  if (fine && dst.page_size) {
    const int to = dst.page_table[int64_t(r) * dst.max_pages + own / dst.page_size];
    fine = to >= 0 && to < dst.num_pages;
  }
  const uint32_t asked = __ballot_sync(kAll, called) & 0xFFFFu, now = __ballot_sync(kAll, fine) & 0xFFFFu;
  if (now != asked && lane == 0 && head0 == 0) flag_status(status, CONDUIT_FLAG_INDEX);
  if (now == 0) return;
  const uint8_t* block = fp8_block(kv, l, on ? head : 0, page, int(slot));
  const float2 scale = *reinterpret_cast<const float2*>(block + 32 * kv.d);
  auto row_at = [&](int t) { return dst.row(l, on ? head : 0, r, int64_t(t0) + slot + t - from, int(slot + t - from)); };
  for (int u = p.u; u < (kv.d + 127) / 128 * 16; u += 16) {
    const bool live = on && u < kv.d / 8;
    uint2 kw[8];
    uint4 vw[4];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int t = 2 * i + p.c;
      kw[i] = make_uint2(0, 0);
      if (live) kw[i] = __ldcs(reinterpret_cast<const uint2*>(block + (t >> 3) * 8 * kv.d + (u >> 1) * 128 + (t & 7) * 16 + (u & 1) * 8));
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      vw[j] = make_uint4(0, 0, 0, 0);
      if (live) vw[j] = __ldcs(reinterpret_cast<const uint4*>(block + 16 * kv.d + (8 * u + 4 * p.c + j) * 16));
    }
    // dims of this lane's parity: halfword a of w[dim] holds tokens 2 a + c and 2 a + 8 + c
    uint32_t w[8][2];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t even[2] = {__byte_perm(vw[j].x, vw[j].y, 0x6420), __byte_perm(vw[j].z, vw[j].w, 0x6420)};
      const uint32_t odd[2] = {__byte_perm(vw[j].x, vw[j].y, 0x7531), __byte_perm(vw[j].z, vw[j].w, 0x7531)};
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t keep = p.c ? odd[h] : even[h];
        const uint32_t got = __shfl_xor_sync(kAll, p.c ? even[h] : odd[h], 16);
        w[j][h] = p.c ? got : keep;
        w[j + 4][h] = p.c ? keep : got;
      }
    }
    if (!live) continue;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int t = 2 * i + p.c;
      if (!(now >> t & 1u)) continue;
      const int64_t at = row_at(t) + 8 * u;
      float x[8], y[8];
      const float2 z[4] = {floats_lo(kw[i].x), floats_hi(kw[i].x), floats_lo(kw[i].y), floats_hi(kw[i].y)};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 a = tc::fmul2(z[e], make_float2(scale.x, scale.x));
        x[2 * e] = a.x, x[2 * e + 1] = a.y;
      }
      store8(static_cast<T*>(dst.k) + at, x);
      // token 2 i + c: halfword a = i % 4, its low byte for i < 4
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float2 pair = (i & 1) ? floats_hi(w[e][(i & 3) >> 1]) : floats_lo(w[e][(i & 3) >> 1]);
        y[e] = (i < 4 ? pair.x : pair.y) * scale.y;
      }
      store8(static_cast<T*>(dst.v) + at, y);
    }
  }
}

template <typename T, bool kWide, int kPairing>
cudaError_t append_with(const PackedDev& kv, const SeqsDev& s, const RopeDev& rope, const RowsDev& k, const RowsDev& v,
                        const RowsDev& q, const RowsDev& q_out, int32_t* status, cudaStream_t stream) {
  const int hp = heads_per_warp(kv.d), groups = (kv.Hkv + hp - 1) / hp;
  const int blocks = (s.max_rows + 15) / 16 + 1;  // a call's rows begin anywhere in a block
  constexpr int kWarps = kThreads / 32, VEC = kWide ? 16 / int(sizeof(T)) : 1;
  const int64_t q_threads = q.p ? int64_t(s.max_rows) * kv.Hq * units_per_row<VEC>(rope, kv.d) : 0;
  const int q_grid = int((q_threads + kThreads - 1) / kThreads);
  // Units of a warp: as many as leave four CTAs for each place of the device, at most seven (28 layers of 8 192 tokens, append
  // and read: four 300 us, seven 282, fourteen 284). Three CTAs an SM: with four, which spill, 327 us, with two 286.
  const int64_t warps = (int64_t(groups) * kv.L + kWarps - 1) / kWarps;
  const int64_t most = std::max<int64_t>(1, int64_t(blocks) * s.R * warps / (4 * 3 * 152));
  const int per = int(std::min<int64_t>({most, warps, 7}));
  const dim3 grid(unsigned(blocks + q_grid), s.R, unsigned(std::min<int64_t>((warps + per - 1) / per, 65535)));
  const int smem = (kPairing == kNoTurn ? 0 : 2 * kBlockTokens * kv.d * int(sizeof(float))) +
                   kWarps * 2 * kBlockTokens * hp * kv.d * int(sizeof(T));
  auto run = [&](auto kernel) {
    if (smem > 48 * 1024) {  // (a microsecond of a decoding step's call otherwise)
      cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
      if (err) return err;
    }
    kernel<<<grid, kThreads, smem, stream>>>(kv, s, rope, blocks, k, v, q, q_out, status);
    count_launches(1);
    return cudaGetLastError();
  };
  return kv.d <= 128 ? run(fp8_append_kernel<T, kWide, kPairing, 1>) : run(fp8_append_kernel<T, kWide, kPairing, 2>);
}

template <typename T, bool kWide>
cudaError_t append(const PackedDev& kv, const SeqsDev& s, const RopeDev& rope, const RowsDev& k, const RowsDev& v,
                   const RowsDev& q, const RowsDev& q_out, int32_t* status, cudaStream_t stream) {
  switch (pairing(rope)) {
    case kNoTurn: return append_with<T, kWide, kNoTurn>(kv, s, rope, k, v, q, q_out, status, stream);
    case kChunks: return append_with<T, kWide, kChunks>(kv, s, rope, k, v, q, q_out, status, stream);
    case kNeighbours: return append_with<T, kWide, kNeighbours>(kv, s, rope, k, v, q, q_out, status, stream);
    default: return append_with<T, kWide, kAnywhere>(kv, s, rope, k, v, q, q_out, status, stream);
  }
}

}  // namespace

cudaError_t launch_fp8_append(const PackedDev& kv, const SeqsDev& s, const RopeDev& rope, int dtype, const RowsDev& k,
                              const RowsDev& v, const RowsDev& q, const RowsDev& q_out, int32_t* status,
                              cudaStream_t stream) {
  // 16-byte copies where every row of the call allows them (queries: and their pairs come in whole chunks)
  const int vec = dtype == CONDUIT_BF16 ? 8 : 4;
  const bool wide = rows_aligned(k, vec) && rows_aligned(v, vec) &&
                    (!q.p || (dims_in_chunks(rope, kv.d, vec) && rows_aligned(q, vec) && rows_aligned(q_out, vec)));
  if (dtype == CONDUIT_BF16)
    return wide ? append<__nv_bfloat16, true>(kv, s, rope, k, v, q, q_out, status, stream)
                : append<__nv_bfloat16, false>(kv, s, rope, k, v, q, q_out, status, stream);
  return wide ? append<float, true>(kv, s, rope, k, v, q, q_out, status, stream)
              : append<float, false>(kv, s, rope, k, v, q, q_out, status, stream);
}

cudaError_t launch_fp8_read(const PackedDev& kv, const int32_t* first, const KvDev& dst, const BatchDev& b,
                            int max_tokens, int32_t* status, cudaStream_t stream) {
  const int hp = heads_per_warp(kv.d), groups = (kv.Hkv + hp - 1) / hp;
  const int64_t units = (int64_t(max_tokens + 15) / 16 + 1) * groups;
  constexpr int kWarps = kThreads / 32;
  const dim3 grid(unsigned((units + kWarps - 1) / kWarps), b.R, kv.L);
  if (dst.dtype == CONDUIT_BF16)
    fp8_read_kernel<__nv_bfloat16><<<grid, kThreads, 0, stream>>>(kv, first, dst, b, status);
  else
    fp8_read_kernel<float><<<grid, kThreads, 0, stream>>>(kv, first, dst, b, status);
  count_launches(1);
  return cudaGetLastError();
}

}  // namespace conduit
