// Attention over the 4-bit cache for few rows (decoding, drafts): warp-level tensor
// cores, one pass over the packed keys and values.
//
// Mathematics. A group of 32 dims of token t is m_t + s_t c, c in -8..7. Logits come
// group by group: x = sum_g s_tg (sum c q) + m_tg (sum q), with the codes exact in fp16 and
// the queries exact too (bf16 scaled to fp16's range by a power of two per row), so
// only fp32 sums round. Values are formed as fp16 m + s c (2^-11 relative), weights
// rounded to fp16: both below the rounding of a bf16 output.
//
// Shape. mma m16n8k16 with the tokens (then the dims) as the 16 rows and up to 8
// (row, query head) columns as n, so that a KV head's group of 7 or 8 query heads
// wastes nothing. The logits' accumulators hold tokens by lane / 4; movmatrix turns them
// into the operand of the value product. Each warp owns tiles of 32 tokens with a ring
// of its own: bulk copies of whole page runs, so no block-wide barrier is met before the
// end, where the warps' results are joined.
//
// Bound: 1.25 d bytes per token and KV head from HBM; next to it the unpacking, about
// two instructions a value and lane.
#include "packed_attn.cuh"

namespace conduit {
namespace {

constexpr int kWarps = 8;
constexpr int kStages = 2;
constexpr int kTile = 32;  // tokens of a tile
constexpr int kBoxBytes(int d) { return kTile * (d + d / 4); }

__device__ __forceinline__ uint32_t h2u(__half2 h) { return *reinterpret_cast<uint32_t*>(&h); }
__device__ __forceinline__ __half2 u2h(uint32_t u) { return *reinterpret_cast<__half2*>(&u); }

// Codes of two nibbles as fp16: bits 0-3 and 16-19 (lo) or 4-7 and 20-23 (hi) of w.
// 0x6400 | n is 1024 + n (or 1024 + 16 n), so one fp16 instruction gives n - 8 exactly.
__device__ __forceinline__ uint32_t codes_lo(uint32_t w) {
  return h2u(__hadd2(u2h((w & 0x000F000Fu) | 0x64006400u), __float2half2_rn(-1032.f)));
}
__device__ __forceinline__ uint32_t codes_hi(uint32_t w) {
  return h2u(__hfma2(u2h((w & 0x00F000F0u) | 0x64006400u), __float2half2_rn(0.0625f), __float2half2_rn(-72.f)));
}

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                        uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
               "l"(src), "r"(bytes), "r"(tc::smem_u32(bar))
               : "memory");
}

// N consecutive 32-bit words, N * 4 bytes aligned to the widest load that divides them.
template <int N>
__device__ __forceinline__ void load_words(const uint8_t* p, uint32_t (&w)[N]) {
  if constexpr (N % 4 == 0) {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      const uint4 x = reinterpret_cast<const uint4*>(p)[i];
      w[4 * i] = x.x, w[4 * i + 1] = x.y, w[4 * i + 2] = x.z, w[4 * i + 3] = x.w;
    }
  } else if constexpr (N % 2 == 0) {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      const uint2 x = reinterpret_cast<const uint2*>(p)[i];
      w[2 * i] = x.x, w[2 * i + 1] = x.y;
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = reinterpret_cast<const uint32_t*>(p)[i];
  }
}

// N 16-bit words in the low halves (even) and high halves (odd) of (N + 1) / 2 words.
template <int N>
__device__ __forceinline__ void load_halves(const uint8_t* p, uint32_t (&w)[(N + 1) / 2]) {
  if constexpr (N % 2 == 0) {
    load_words<N / 2>(p, w);
  } else {
    const uint16_t* h = reinterpret_cast<const uint16_t*>(p);
#pragma unroll
    for (int i = 0; i < N / 2; ++i) w[i] = h[2 * i] | uint32_t(h[2 * i + 1]) << 16;
    w[N / 2] = h[N - 1];
  }
}

__device__ __forceinline__ bool finite_pair(uint32_t p) {
  return (p & 0x7C00u) != 0x7C00u && (p & 0x7C000000u) != 0x7C000000u;
}

template <int NG>
__global__ void __launch_bounds__(kWarps * 32, 2) packed_attn_mma(AttnArgs a) {
  constexpr int D = NG * 32, kBox = kBoxBytes(D);
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ uint64_t full[kWarps][kStages];
  Item it;
  if (!item_of(a, &it)) return;
  const int w = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int c = lane & 3, q = lane >> 2;
  // a row of the logits' accumulator is the token row_of(lane / 4) of its half tile; with
  // this order the value loads of a warp touch two banks' halves evenly
  const int key_lo = (q & 1) ? (4 + (q >> 1)) ^ 1 : q >> 1;

  // keys that this lane's two columns see; columns past the last see all (their result is dropped)
  int lim[2], most = 0, least = INT32_MAX;
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int j = it.cb * kCols + 2 * c + e;
    lim[e] = j < it.n * a.kv.G ? limit_of(a, it, j) : INT32_MAX;
    if (lim[e] != INT32_MAX) most = max(most, lim[e]);
    least = min(least, lim[e]);
  }
#pragma unroll
  for (int s = 1; s < 4; s <<= 1) {
    most = max(most, __shfl_xor_sync(0xffffffffu, most, s));
    least = min(least, __shfl_xor_sync(0xffffffffu, least, s));
  }
  const int k0 = it.chunk * a.chunk, k1 = min(k0 + a.chunk, most);
  const int tiles = k1 > k0 ? (k1 - k0 + kTile - 1) / kTile : 0;
  const int mine = tiles > w ? (tiles - w + kWarps - 1) / kWarps : 0;

  uint8_t* ring = smem + w * kStages * kBox;
  if (lane == 0) {
#pragma unroll
    for (int s = 0; s < kStages; ++s) tc::mbar_init(&full[w][s], 1);
    tc::fence_barrier_init();
  }
  __syncwarp();

  const int run = min(kTile, 1 << a.kv.page_shift);  // tokens of a tile that lie in one page
  auto fill = [&](int stage, int tile) {
    const int kb = k0 + tile * kTile;
    const int runs = (min(k1 - kb, kTile) + run - 1) / run;
    if (lane == 0) tc::mbar_arrive_expect_tx(&full[w][stage], uint32_t(runs * run * (D + D / 4)));
    __syncwarp();
    if (lane < 4 * runs) {
      const int part = lane & 3, j = kb + (lane >> 2) * run, row = j & ((1 << a.kv.page_shift) - 1);
      const uint8_t* at = a.kv.page(it.l, it.g, page_of(a, it.r, j));
      const uint32_t base = tc::smem_u32(ring + stage * kBox);
      const int at_tile = (lane >> 2) * run;
      if (part < 2)
        bulk_load(base + (part * kTile + at_tile) * (D / 2), at + a.kv.codes(part, row), run * (D / 2), &full[w][stage]);
      else
        bulk_load(base + kTile * D + ((part - 2) * kTile + at_tile) * (D / 8), at + a.kv.params(part - 2, row),
                  run * (D / 8), &full[w][stage]);
    }
  };
#pragma unroll
  for (int s = 0; s < kStages; ++s)
    if (s < mine) fill(s, w + s * kWarps);

  // Queries of column q (operand layout), scaled to [256, 512) at most by 2^-shift.
  uint32_t bq[NG][4];
  float qsum[NG][2], to_log2[2];
  {
    const int j = it.cb * kCols + q;
    float x[NG][8], top = 0.f;
    const bool live = j < it.n * a.kv.G;
    const int i = live ? j / a.kv.G : 0, h = live ? it.g * a.kv.G + j % a.kv.G : 0;
    const __nv_bfloat16* src =
        static_cast<const __nv_bfloat16*>(a.q.p) + it.l * a.q.ls + int64_t(it.t0 + i) * a.q.rs + h * a.q.hs + 8 * c;
    const bool wide = ((reinterpret_cast<uintptr_t>(a.q.p) | uint64_t(2 * (a.q.ls | a.q.rs | a.q.hs))) & 15u) == 0;
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      __nv_bfloat16 v[8];
      if (!live) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = __float2bfloat16_rn(0.f);
      } else if (wide) {
        *reinterpret_cast<uint4*>(v) = *reinterpret_cast<const uint4*>(src + 32 * g);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = src[32 * g + e];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[g][e] = __bfloat162float(v[e]);
        top = fmaxf(top, fabsf(x[g][e]));
      }
    }
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
    int shift = int(__float_as_uint(top) >> 23) - 127 - 8;  // top < 2^(shift + 9)
    if (!(top < INFINITY) || top == 0.f) shift = 0;
    // 2^-shift in two factors, each a normal number
    const float f1 = __uint_as_float(uint32_t(127 - shift / 2) << 23);
    const float f2 = __uint_as_float(uint32_t(127 - (shift - shift / 2)) << 23);
    const float g1 = __uint_as_float(uint32_t(127 + shift / 2) << 23);
    const float g2 = __uint_as_float(uint32_t(127 + (shift - shift / 2)) << 23);
    const float back = a.scale * kLog2e * g1 * g2;
    float part[NG];
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      part[g] = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[g][e] = x[g][e] * f1 * f2;
        part[g] += x[g][e];
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) bq[g][e] = h2u(__floats2half2_rn(x[g][e], x[g][e + 4]));
      part[g] += __shfl_xor_sync(0xffffffffu, part[g], 1);
      part[g] += __shfl_xor_sync(0xffffffffu, part[g], 2);
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      to_log2[e] = __shfl_sync(0xffffffffu, back, 4 * (2 * c + e));
#pragma unroll
      for (int g = 0; g < NG; ++g) qsum[g][e] = __shfl_sync(0xffffffffu, part[g], 4 * (2 * c + e));
    }
  }

  float m[2] = {-INFINITY, -INFINITY}, sum[2] = {0.f, 0.f};
  float o[2 * NG][4];
#pragma unroll
  for (int t = 0; t < 2 * NG; ++t)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[t][e] = 0.f;

  bool ok = true;
  for (int n = 0; n < mine && ok; ++n) {
    const int stage = n % kStages, kb = k0 + (w + n * kWarps) * kTile;
    if (!tc::mbar_wait(&full[w][stage], uint32_t(n / kStages) & 1u)) {
      ok = false;
      break;
    }
    const uint8_t* box = ring + stage * kBox;
    const uint8_t *kc = box, *vc = box + kTile * (D / 2), *kp = box + kTile * D, *vp = kp + kTile * (D / 8);
    const bool edge = kb + kTile > least;  // some column does not see the whole tile

    float x[2][4];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int lo = 16 * t + key_lo, hi = lo + 8;
      uint32_t wl[NG], wh[NG], pl[NG], ph[NG];
      load_words<NG>(kc + lo * (D / 2) + c * (D / 8), wl);
      load_words<NG>(kc + hi * (D / 2) + c * (D / 8), wh);
      load_words<NG>(kp + lo * (D / 8), pl);
      load_words<NG>(kp + hi * (D / 8), ph);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[t][e] = 0.f;
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        float acc[4] = {0.f, 0.f, 0.f, 0.f};
        mma_f16(acc, codes_lo(wl[g]), codes_lo(wh[g]), codes_hi(wl[g]), codes_hi(wh[g]), bq[g][0], bq[g][1]);
        const uint32_t l8 = wl[g] >> 8, h8 = wh[g] >> 8;
        mma_f16(acc, codes_lo(l8), codes_lo(h8), codes_hi(l8), codes_hi(h8), bq[g][2], bq[g][3]);
        const float2 fl = __half22float2(u2h(pl[g])), fh = __half22float2(u2h(ph[g]));
        x[t][0] = fmaf(fl.x, acc[0], fmaf(fl.y, qsum[g][0], x[t][0]));
        x[t][1] = fmaf(fl.x, acc[1], fmaf(fl.y, qsum[g][1], x[t][1]));
        x[t][2] = fmaf(fh.x, acc[2], fmaf(fh.y, qsum[g][0], x[t][2]));
        x[t][3] = fmaf(fh.x, acc[3], fmaf(fh.y, qsum[g][1], x[t][3]));
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[t][e] *= to_log2[e & 1];
        if (edge && kb + (e < 2 ? lo : hi) >= lim[e & 1]) x[t][e] = -INFINITY;
      }
    }
    float corr[2];
    bool moved = false;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float top = fmaxf(fmaxf(x[0][e], x[0][e + 2]), fmaxf(x[1][e], x[1][e + 2]));
#pragma unroll
      for (int s = 4; s < 32; s <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, s));
      const float mn = fmaxf(m[e], top), base = mn == -INFINITY ? 0.f : mn;
      corr[e] = tc::ex2(m[e] - base);
      moved |= mn != m[e];
      m[e] = mn;
      sum[e] *= corr[e];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        x[t][e] = tc::ex2(x[t][e] - base);
        x[t][e + 2] = tc::ex2(x[t][e + 2] - base);
        sum[e] += x[t][e] + x[t][e + 2];
      }
    }
    if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
      for (int t = 0; t < 2 * NG; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[t][e] *= corr[e & 1];
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const uint32_t b0 = transpose8x8(h2u(__floats2half2_rn(x[t][0], x[t][1])));
      const uint32_t b1 = transpose8x8(h2u(__floats2half2_rn(x[t][2], x[t][3])));
      // tokens of this lane's operand slots 2 c, 2 c + 1, and eight on
      uint32_t v[4][(NG + 1) / 2], p[4][NG];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int key = 16 * t + (e & 1 ? (4 + c) ^ 1 : c) + (e & 2 ? 8 : 0);
        load_halves<NG>(vc + key * (D / 2) + q * (D / 16), v[e]);
        load_words<NG>(vp + key * (D / 8), p[e]);
        if (edge) {
          // tokens that some column does not see: their weight there is 0, and 0 times NaN must not be
#pragma unroll
          for (int g = 0; g < NG; ++g)
            if (kb + key >= k1 || (kb + key >= least && !finite_pair(p[e][g]))) p[e][g] = 0;
        }
      }
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        const uint32_t pick = g & 1 ? 0x7632u : 0x5410u;
        const uint32_t xl = __byte_perm(v[0][g / 2], v[1][g / 2], pick), xh = __byte_perm(v[2][g / 2], v[3][g / 2], pick);
        const __half2 sl = u2h(__byte_perm(p[0][g], p[1][g], 0x5410)), ml = u2h(__byte_perm(p[0][g], p[1][g], 0x7632));
        const __half2 sh = u2h(__byte_perm(p[2][g], p[3][g], 0x5410)), mh = u2h(__byte_perm(p[2][g], p[3][g], 0x7632));
        auto value = [](uint32_t code, __half2 s, __half2 mid) { return h2u(__hfma2(s, u2h(code), mid)); };
        mma_f16(o[2 * g], value(codes_lo(xl), sl, ml), value(codes_hi(xl), sl, ml), value(codes_lo(xh), sh, mh),
                value(codes_hi(xh), sh, mh), b0, b1);
        const uint32_t yl = xl >> 8, yh = xh >> 8;
        mma_f16(o[2 * g + 1], value(codes_lo(yl), sl, ml), value(codes_hi(yl), sl, ml), value(codes_lo(yh), sh, mh),
                value(codes_hi(yh), sh, mh), b0, b1);
      }
    }
    if (edge) {
      // a value that is not finite makes the outputs of the columns that see it NaN
      uint32_t poison = 0;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int key = 8 * t + key_lo;
        uint32_t p[NG];
        load_words<NG>(vp + key * (D / 8), p);
#pragma unroll
        for (int g = 0; g < NG; ++g)
#pragma unroll
          for (int e = 0; e < 2; ++e)
            if (kb + key < min(lim[e], k1) && !finite_pair(p[g])) poison |= 1u << (2 * g + e);
      }
#pragma unroll
      for (int s = 4; s < 32; s <<= 1) poison |= __shfl_xor_sync(0xffffffffu, poison, s);
      if (poison) {
#pragma unroll
        for (int t = 0; t < 2 * NG; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (poison >> (2 * (t / 2) + (e & 1)) & 1u) o[t][e] = NAN;
      }
    }
    __syncwarp();
    if (n + kStages < mine) fill(stage, w + (n + kStages) * kWarps);
  }
  if (!ok) {  // bounded waits for the copies that are still under way
    flag_status(a.status, CONDUIT_FLAG_TIMEOUT | CONDUIT_SITE_LOAD);
    for (int s = 0; s < kStages; ++s) tc::mbar_wait(&full[w][s], 0), tc::mbar_wait(&full[w][s], 1);
  }

  // Join of the warps.
#pragma unroll
  for (int e = 0; e < 2; ++e)
#pragma unroll
    for (int s = 4; s < 32; s <<= 1) sum[e] += __shfl_xor_sync(0xffffffffu, sum[e], s);
  __syncthreads();
  constexpr int kRow = D + 4;
  float* ow = reinterpret_cast<float*>(smem);          // [warps][columns][kRow]
  float2* st = reinterpret_cast<float2*>(ow + kWarps * kCols * kRow);  // [warps][columns] (M, sum)
  static_assert(kWarps * kCols * (kRow * 4 + 8) <= kWarps * kStages * kBox, "the join fits the ring");
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int col = 2 * c + e;
    if (q == 0) st[w * kCols + col] = make_float2(m[e], sum[e]);
#pragma unroll
    for (int g = 0; g < NG; ++g)
      *reinterpret_cast<float4*>(ow + (w * kCols + col) * kRow + 32 * g + 4 * q) =
          make_float4(o[2 * g][e], o[2 * g][e + 2], o[2 * g + 1][e], o[2 * g + 1][e + 2]);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < kCols * D; e += kWarps * 32) {
    const int col = e / D, dd = e % D, j = it.cb * kCols + col;
    if (j >= it.n * a.kv.G) break;
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) top = fmaxf(top, st[i * kCols + col].x);
    const float base = top == -INFINITY ? 0.f : top;
    float total = 0.f, out = 0.f;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) {
      const float2 s = st[i * kCols + col];
      const float wgt = tc::ex2(s.x - base);
      total = fmaf(wgt, s.y, total);
      out = fmaf(wgt, ow[(i * kCols + col) * kRow + dd], out);
    }
    store_out<__nv_bfloat16>(a, it, j, dd, out, total);
    if (dd == 0) store_stats(a, it, j, top, total);
  }
}

template <int NG>
cudaError_t launch(const AttnArgs& a, int64_t items, cudaStream_t stream) {
  constexpr int kSmem = kWarps * kStages * kBoxBytes(NG * 32);
  cudaError_t err = cudaFuncSetAttribute(packed_attn_mma<NG>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
  if (err) return err;
  packed_attn_mma<NG><<<unsigned(items), kWarps * 32, kSmem, stream>>>(a);
  count_launches(1);
  return cudaGetLastError();
}

}  // namespace

bool packed_attn_mma_supported(const PackedDev& kv, int dtype) {
  return dtype == CONDUIT_BF16 && (kv.d == 64 || kv.d == 96 || kv.d == 128);
}

cudaError_t launch_packed_attn_mma(const AttnArgs& a, int64_t items, cudaStream_t stream) {
  switch (a.kv.d) {
    case 64: return launch<2>(a, items, stream);
    case 96: return launch<3>(a, items, stream);
    default: return launch<4>(a, items, stream);
  }
}

}  // namespace conduit
