// Attention over the 4-bit cache for few rows (decoding, drafts): warp-level tensor
// cores, one pass over the packed keys and values.
//
// Mathematics. A group of 32 dims of token t is m_t + s_t c, c in -8..7. Logits come group by
// group: x = sum_g s_tg (sum c q) + m_tg (sum q), with the codes exact in fp16 and the
// queries exact too (bf16 scaled by a power of two per row to fp16's range) down to 2^-25 of their
// row's largest and within 2^-33 of it below, so beside that only fp32 sums round (to 6 x 10^-8 of a log-sum-exp). Values are formed as fp16 m + s c (2^-11 relative),
// weights rounded to fp16: both below the rounding of a bf16 output. (Codes with their offset
// left on, taken off in fp32, cost no instruction less on the pipe that counts and lost
// precision: fp16's 1024 + u 6 x 10^-6 of a log-sum-exp, bf16's 128 + u 178 us for the batch of
// 64 where this took 172.)
//
// Shape. mma with the tokens (then the dims) as the 16 rows and up to 8 (row, query head)
// columns as n, so that a KV head's group of 7 or 8 query heads wastes nothing. The
// logits' accumulators hold tokens by lane / 4; movmatrix turns them into the operand of
// the value product. Each warp owns tiles of 32 tokens with a ring of its own, so no
// block-wide barrier is met before the end, where the warps' results are joined. A tile
// comes in bulk copies of whole pages, or of four parts of a longer page: the lanes issue
// theirs one after the other, about 100 cycles each. (Four parts of every page: 168 us for
// the batch of 64 with pages of 16 tokens where this takes 157; 16-byte copies lane by lane,
// whose instructions come out of the same issue slots, 174.)
//
// Bound: 1.25 d bytes per token and KV head from HBM; next to it the unpacking of the
// values, whose integer and fp16 instructions issue at half rate. Measured: one row each of
// 64 requests of 2 000-30 000 tokens, 28 x 4 heads of 128, 157 us with the join (4.2 TB/s, 66 %
// of the issue slots); one of 262 145 tokens, 32 x 8 heads, 73 us (4.6 TB/s).
#include "attn_warps.cuh"
#include "packed_attn.cuh"

namespace conduit {
namespace {

constexpr int kWarps = 8;
constexpr int kStages = 2;
constexpr int kTile = 32;  // tokens of a tile (2^5)
constexpr int kBoxBytes(int d) { return kTile * (d + d / 4); }

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

// The mids of groups 2 (c & 1) and + 1 of a token's parameters.
template <int NG>
__device__ __forceinline__ uint32_t mids(const uint8_t* p, int c) {
  static_assert(NG <= 4, "two lanes hold the groups");
  if constexpr (NG == 4) {
    const uint2 w = *reinterpret_cast<const uint2*>(p + 8 * (c & 1));
    return __byte_perm(w.x, w.y, 0x7632);
  } else {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(p);
    uint32_t y = __byte_perm(w[0], w[1], 0x7632);
    if (c & 1) y = NG == 3 ? w[NG - 1] >> 16 : 0;
    return y;
  }
}

// State of a warp's running softmax for the two columns of a lane.
template <int NG>
struct Running {
  float ref[2], sum[2];  // reference exponent (log2 units), sum of weights of this lane's tokens
  float o[2 * NG][4];    // dims 32 g + 4 q + {0, 1} and {2, 3} of both columns in o[2 g], o[2 g + 1]
};

// A tile in shared memory: page after page as in the pool, and of pages of more than 32 tokens
// the 32 as a page of their own. Offsets of the codes and parameters of tokens 8 i.. of K (v = 0)
// or V (v = 1); kRun: tokens of a page in the tile.
template <int NG, int kRun>
struct Box {
  static constexpr int D = NG * 32, kPage = kRun * (D + D / 4);
  __device__ static constexpr int codes(int v, int i) {
    return 8 * i / kRun * kPage + v * kRun * (D / 2) + 8 * i % kRun * (D / 2);
  }
  __device__ static constexpr int params(int v, int i) {
    return 8 * i / kRun * kPage + kRun * D + v * kRun * (D / 8) + 8 * i % kRun * (D / 8);
  }
};

// One tile of 32 tokens. kEdge: some column does not see all of it.
template <int NG, int kRun, bool kEdge>
__device__ __forceinline__ void tile_step(Running<NG>& st, const uint8_t* box, const uint32_t (&bq)[NG][4],
                                          uint32_t qsum,
                                          const float (&to_log2)[2], int kb, int k1, int least, const int (&lim)[2], int c, int q, int key_lo) {
  constexpr int D = NG * 32;
  using B = Box<NG, kRun>;
  float x[2][4];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int lo = 16 * t + key_lo, hi = lo + 8;
    const uint8_t* kp_lo = box + B::params(0, 2 * t) + key_lo * (D / 8);
    const uint8_t* kp_hi = box + B::params(0, 2 * t + 1) + key_lo * (D / 8);
    uint32_t wl[NG], wh[NG], pl[NG], ph[NG];
    load_words<NG>(box + B::codes(0, 2 * t) + key_lo * (D / 2) + c * (D / 8), wl);
    load_words<NG>(box + B::codes(0, 2 * t + 1) + key_lo * (D / 2) + c * (D / 8), wh);
    load_words<NG>(kp_lo, pl);
    load_words<NG>(kp_hi, ph);
    // sum_g m_tg (sum q): one product over the groups, the query sums in two fp16 parts
    mma_f16_first(x[t], mids<NG>(kp_lo, c), mids<NG>(kp_hi, c), 0, 0, qsum, 0);
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      float acc[4];
      mma_f16_first(acc, codes_lo(wl[g]), codes_lo(wh[g]), codes_hi(wl[g]), codes_hi(wh[g]), bq[g][0], bq[g][1]);
      const uint32_t l8 = wl[g] >> 8, h8 = wh[g] >> 8;
      mma_f16(acc, codes_lo(l8), codes_lo(h8), codes_hi(l8), codes_hi(h8), bq[g][2], bq[g][3]);
      const float sl = __low2float(u2h(pl[g])), sh = __low2float(u2h(ph[g]));
      x[t][0] = fmaf(sl, acc[0], x[t][0]);
      x[t][1] = fmaf(sl, acc[1], x[t][1]);
      x[t][2] = fmaf(sh, acc[2], x[t][2]);
      x[t][3] = fmaf(sh, acc[3], x[t][3]);
    }
    if (kEdge) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (kb + (e < 2 ? lo : hi) >= lim[e & 1]) x[t][e] = -INFINITY;
    }
  }
  float top[2];
#pragma unroll
  for (int e = 0; e < 2; ++e)
    top[e] = fmaxf(fmaxf(x[0][e], x[0][e + 2]), fmaxf(x[1][e], x[1][e + 2])) * to_log2[e];
  if (__any_sync(0xffffffffu, top[0] > st.ref[0] + kMostWeight || top[1] > st.ref[1] + kMostWeight)) {
    float corr[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
#pragma unroll
      for (int s = 4; s < 32; s <<= 1) top[e] = fmaxf(top[e], __shfl_xor_sync(0xffffffffu, top[e], s));
      const float moved = fmaxf(st.ref[e], top[e] - kBias);
      corr[e] = moved == -INFINITY ? 1.f : tc::ex2(st.ref[e] - moved);
      st.ref[e] = moved;
      st.sum[e] *= corr[e];
    }
#pragma unroll
    for (int t = 0; t < 2 * NG; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) st.o[t][e] *= corr[e & 1];
  }
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const float base = kEdge && st.ref[e] == -INFINITY ? 0.f : st.ref[e];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      x[t][e] = tc::ex2(fmaf(x[t][e], to_log2[e], -base));
      x[t][e + 2] = tc::ex2(fmaf(x[t][e + 2], to_log2[e], -base));
      st.sum[e] += x[t][e] + x[t][e + 2];
    }
  }
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const uint32_t b0 = transpose8x8(h2u(__floats2half2_rn(x[t][0], x[t][1])));
    const uint32_t b1 = transpose8x8(h2u(__floats2half2_rn(x[t][2], x[t][3])));
    // tokens of this lane's operand slots 2 c, 2 c + 1, and eight on
    uint32_t v[4][(NG + 1) / 2], p[4][NG];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int block = 2 * t + (e >> 1), in = e & 1 ? (4 + c) ^ 1 : c, key = 8 * block + in;
      load_halves<NG>(box + B::codes(1, block) + in * (D / 2) + q * (D / 16), v[e]);
      load_words<NG>(box + B::params(1, block) + in * (D / 8), p[e]);
      if (kEdge) {
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
      mma_f16(st.o[2 * g], value(codes_lo(xl), sl, ml), value(codes_hi(xl), sl, ml), value(codes_lo(xh), sh, mh),
              value(codes_hi(xh), sh, mh), b0, b1);
      const uint32_t yl = xl >> 8, yh = xh >> 8;
      mma_f16(st.o[2 * g + 1], value(codes_lo(yl), sl, ml), value(codes_hi(yl), sl, ml), value(codes_lo(yh), sh, mh),
              value(codes_hi(yh), sh, mh), b0, b1);
    }
  }
  if (kEdge) {
    // a value that is not finite makes the outputs of the columns that see it NaN
    uint32_t poison = 0;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int key = 8 * t + key_lo;
      uint32_t p[NG];
      load_words<NG>(box + B::params(1, t) + key_lo * (D / 8), p);
#pragma unroll
      for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int e = 0; e < 2; ++e)
          if (kb + key < min(lim[e], k1) && !finite_pair(p[g])) poison |= 1u << (2 * g + e);
    }
    poison = __reduce_or_sync(0x11111111u << c, poison);
    if (poison) {
#pragma unroll
      for (int t = 0; t < 2 * NG; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (poison >> (2 * (t / 2) + (e & 1)) & 1u) st.o[t][e] = NAN;
    }
  }
}

// kCluster: the CTAs of a cluster take the chunks of a context and join them in shared memory.
template <int NG, int kRun, bool kCluster>
__global__ void __launch_bounds__(kWarps * 32, 2) packed_attn_mma(AttnArgs a) {
  using B = Box<NG, kRun>;
  constexpr int D = NG * 32, kBox = kBoxBytes(D);
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ uint64_t full[kWarps][kStages];
  if (!kCluster) let_join_start();
  Item it;
  place_of<kCluster>(a, &it);
  const int w = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int c = lane & 3, q = lane >> 2;
  // a row of the logits' accumulator is the token key_lo (+ 8) of its half tile; with this
  // order the value loads of a warp are spread evenly over the banks
  const int key_lo = (q & 1) ? (4 + (q >> 1)) ^ 1 : q >> 1;

  // The page of this lane's first copy is looked up beside the request's rows and length, whether
  // or not the context reaches it (8.0 us instead of 8.15 for one row over 1 025 keys), then the
  // column's query. A copy: a whole page (lane r page r of a tile), or a part of 32 tokens of a
  // longer one (lane p: K codes, V codes, K and V parameters).
  const bool whole = a.kv.page_shift <= 5;
  const int copies = whole ? kTile / kRun : 4, at_tile = whole ? lane * kRun : 0, k0 = it.chunk * a.chunk;
  const int first_j = k0 + w * kTile + at_tile;
  int next_page = lane < copies && first_j < a.kv.capacity() ? page_entry(a, it.r, first_j) : 0;
  if (!rows_of<kCluster>(a, &it)) return;
  uint4 qv[NG];
  {
    const int j = it.cb * kCols + q;
    const bool live = j < it.n * a.kv.G;
    const int i = live ? j / a.kv.G : 0, h = live ? it.g * a.kv.G + j % a.kv.G : 0;
    const __nv_bfloat16* src =
        static_cast<const __nv_bfloat16*>(a.q.p) + it.l * a.q.ls + int64_t(it.t0 + i) * a.q.rs + h * a.q.hs + 8 * c;
    const bool wide = ((reinterpret_cast<uintptr_t>(a.q.p) | uint64_t(2 * (a.q.ls | a.q.rs | a.q.hs))) & 15u) == 0;
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      qv[g] = make_uint4(0, 0, 0, 0);
      if (live && wide) {
        qv[g] = *reinterpret_cast<const uint4*>(src + 32 * g);
      } else if (live) {
        __nv_bfloat16 v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = src[32 * g + e];
        qv[g] = *reinterpret_cast<uint4*>(v);
      }
    }
  }

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
  const int k1 = min(k0 + a.chunk, most);  // at or before k0 for a chunk past the context
  const int tiles = k1 > k0 ? (k1 - k0 + kTile - 1) / kTile : 0;
  const int mine = tiles > w ? (tiles - w + kWarps - 1) / kWarps : 0;

  uint8_t* ring = smem + w * kStages * kBox;
  if (lane == 0) {
#pragma unroll
    for (int s = 0; s < kStages; ++s) tc::mbar_init(&full[w][s], 1);
    tc::fence_barrier_init();
  }
  __syncwarp();

  const int row_bytes = whole ? 0 : lane < 2 ? D / 2 : D / 8;
  const uint32_t bytes = whole ? B::kPage : kTile * row_bytes;
  const uint32_t dst = tc::smem_u32(ring) + (whole     ? lane * B::kPage
                                             : lane < 2 ? lane * kTile * (D / 2)
                                                        : kTile * D + (lane - 2) * kTile * (D / 8));
  const uint8_t* from = a.kv.page(it.l, it.g, 0) + (whole ? 0 : lane < 2 ? a.kv.codes(lane, 0) : a.kv.params(lane - 2, 0));
  const int64_t page_stride = a.kv.Hkv * a.kv.page_bytes;
  const int page_mask = (1 << a.kv.page_shift) - 1;
  // the page of this lane's copy in a tile, looked up one fill ahead
  auto page_in = [&](int n) {
    const int j = k0 + (w + n * kWarps) * kTile + at_tile;
    return n < mine && j < k1 && lane < copies ? page_entry(a, it.r, j) : 0;
  };
  auto fill = [&](int n) {
    const int stage = n % kStages, kb = k0 + (w + n * kWarps) * kTile;
    const int tokens = min(k1 - kb, kTile);
#ifdef CONDUIT_TEST_HOOKS
    if (n == a.withhold) {  // neither copies nor an arrive: the wait for this tile runs out
      next_page = page_in(n + 1);
      return;
    }
#endif
    if (lane == 0)  // whole runs
      tc::mbar_arrive_expect_tx(&full[w][stage], uint32_t((tokens + kRun - 1) & -kRun) * (D + D / 4));
    __syncwarp();
    if (lane < copies && at_tile < tokens)
      bulk_load(dst + stage * kBox, from + page_in_pool(a, next_page) * page_stride + (kb & page_mask) * row_bytes, bytes,
                &full[w][stage]);
    next_page = page_in(n + 1);
  };
#pragma unroll
  for (int s = 0; s < kStages; ++s)
    if (s < mine) fill(s);

  // Queries of column q in the operand layout, scaled by 2^-shift so that the largest lies in
  // [256, 512): their sums then fit fp16.
  uint32_t bq[NG][4];
  uint32_t qsum = 0;
  float to_log2[2];
  {
    float x[NG][8], top = 0.f;
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const __nv_bfloat16* v = reinterpret_cast<const __nv_bfloat16*>(&qv[g]);
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
    // 2^-shift and 2^shift in two factors, each a normal number
    const float f1 = __uint_as_float(uint32_t(127 - shift / 2) << 23);
    const float f2 = __uint_as_float(uint32_t(127 - (shift - shift / 2)) << 23);
    const float g1 = __uint_as_float(uint32_t(127 + shift / 2) << 23);
    const float g2 = __uint_as_float(uint32_t(127 + (shift - shift / 2)) << 23);
    // positive, so that a masked logit stays -inf under it
    const float back = fmaxf(a.scale * kLog2e * g1 * g2, 1.1754944e-38f);
#pragma unroll
    for (int e = 0; e < 2; ++e) to_log2[e] = __shfl_sync(0xffffffffu, back, 4 * (2 * c + e));
#pragma unroll
    for (int g = 0; g < NG; ++g) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[g][e] = x[g][e] * f1 * f2;
      float total = ((x[g][0] + x[g][1]) + (x[g][2] + x[g][3])) + ((x[g][4] + x[g][5]) + (x[g][6] + x[g][7]));
#pragma unroll
      for (int s = 1; s < 4; s <<= 1) total += __shfl_xor_sync(0xffffffffu, total, s);
#pragma unroll
      for (int e = 0; e < 4; ++e) {  // word e: dims e and e + 4
        bq[g][e] = h2u(__floats2half2_rn(x[g][e], x[g][e + 4]));
      }
      // slots 2 c, 2 c + 1 of the product with the mids: groups 0, 1, 2, 3, then the same in a second part
      const float first = __half2float(__float2half_rn(total));
      if (g / 2 == (c & 1))
        qsum |= uint32_t(__half_as_ushort(__float2half_rn(c < 2 ? first : total - first))) << (16 * (g & 1));
    }
  }

  Running<NG> st;
#pragma unroll
  for (int e = 0; e < 2; ++e) st.ref[e] = -INFINITY, st.sum[e] = 0.f;
#pragma unroll
  for (int t = 0; t < 2 * NG; ++t)
#pragma unroll
    for (int e = 0; e < 4; ++e) st.o[t][e] = 0.f;

  bool ok = true;
  for (int n = 0; n < mine; ++n) {
    const int stage = n % kStages, kb = k0 + (w + n * kWarps) * kTile;
    // lanes time their waits apart; the products and votes below need all of them or none
    ok = __all_sync(0xffffffffu, tc::mbar_wait(&full[w][stage], uint32_t(n / kStages) & 1u));
    if (!ok) break;
    const uint8_t* box = ring + stage * kBox;
    if (kb + kTile > least)
      tile_step<NG, kRun, true>(st, box, bq, qsum, to_log2, kb, k1, least, lim, c, q, key_lo);
    else
      tile_step<NG, kRun, false>(st, box, bq, qsum, to_log2, kb, k1, least, lim, c, q, key_lo);
    __syncwarp();
    if (n + kStages < mine) fill(n + kStages);
  }
  if (!ok) {  // bounded waits for the copies that are still under way
    flag_status(a.status, CONDUIT_FLAG_TIMEOUT | CONDUIT_SITE_LOAD);
    for (int s = 0; s < kStages; ++s) tc::mbar_wait(&full[w][s], 0), tc::mbar_wait(&full[w][s], 1);
  }

  // Join of the warps.
#pragma unroll
  for (int e = 0; e < 2; ++e)
#pragma unroll
    for (int s = 4; s < 32; s <<= 1) st.sum[e] += __shfl_xor_sync(0xffffffffu, st.sum[e], s);
  __syncthreads();
  constexpr int kRow = join_row(D);
  float* ow = reinterpret_cast<float*>(smem);          // [warps][columns][kRow]
  float2* ml = reinterpret_cast<float2*>(ow + kWarps * kCols * kRow);  // [warps][columns] (reference, sum)
  static_assert(join_bytes(D, kWarps) <= kWarps * kStages * kBox, "the join fits the ring");
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int col = 2 * c + e;
    if (q == 0) ml[w * kCols + col] = make_float2(st.ref[e] + kBias, st.sum[e] * kUnbias);
#pragma unroll
    for (int g = 0; g < NG; ++g)
      *reinterpret_cast<float4*>(ow + (w * kCols + col) * kRow + 32 * g + 4 * q) =
          make_float4(st.o[2 * g][e], st.o[2 * g][e + 2], st.o[2 * g + 1][e], st.o[2 * g + 1][e + 2]);
  }
  join_warps<D, kWarps, kCluster>(a, it, ow, ml);
}

template <int NG, int kRun, bool kCluster>
cudaError_t launch(const AttnArgs& a, int64_t items, cudaStream_t stream) {
  constexpr int kSmem = kWarps * kStages * kBoxBytes(NG * 32);
  cudaError_t err =
      cudaFuncSetAttribute(packed_attn_mma<NG, kRun, kCluster>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
  if (err) return err;
  cudaLaunchAttribute cluster{};
  cluster.id = cudaLaunchAttributeClusterDimension;
  cluster.val.clusterDim.x = kCluster ? a.chunks : 1;
  cluster.val.clusterDim.y = cluster.val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(unsigned(items));
  cfg.blockDim = dim3(kWarps * 32);
  cfg.dynamicSmemBytes = kSmem;
  cfg.stream = stream;
  cfg.attrs = &cluster;
  cfg.numAttrs = kCluster ? 1 : 0;
  count_launches(1);
  return cudaLaunchKernelEx(&cfg, packed_attn_mma<NG, kRun, kCluster>, a);
}

template <int NG>
cudaError_t launch(const AttnArgs& a, int64_t items, bool cluster, cudaStream_t stream) {
  switch (a.kv.page_shift) {
    case 3: return cluster ? launch<NG, 8, true>(a, items, stream) : launch<NG, 8, false>(a, items, stream);
    case 4: return cluster ? launch<NG, 16, true>(a, items, stream) : launch<NG, 16, false>(a, items, stream);
    default: return cluster ? launch<NG, 32, true>(a, items, stream) : launch<NG, 32, false>(a, items, stream);
  }
}

}  // namespace

cudaError_t launch_packed_attn_mma(const AttnArgs& a, int64_t items, bool cluster, cudaStream_t stream) {
  switch (a.kv.d) {
    case 64: return launch<2>(a, items, cluster, stream);
    case 96: return launch<3>(a, items, cluster, stream);
    default: return launch<4>(a, items, cluster, stream);
  }
}

}  // namespace conduit
