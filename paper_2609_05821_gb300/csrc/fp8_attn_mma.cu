// Attention over the 8-bit cache for few rows (decoding, drafts): warp-level tensor cores, one pass over
// the codes.
//
// Mathematics. Codes are exact in fp16, and so are the queries (bf16, scaled by a power of two per row so that the largest lies
// in [2^15, 2^16)) down to 2^-32 of their row's largest; what is smaller is off by 2^-40 of it at most, fp16's step at its
// low end. Beside that only fp32 sums round; a block's key scale multiplies its logits. The scale of its values, 2^v, joins the exponent of its
// weights: w_j = 2^(x_j + v - reference), with which the codes themselves are summed, while the denominator takes
// w_j 2^-v. The reference follows the largest x + v, so that fp16's range of weights goes to what counts in the output.
// Where w_j would leave fp32's range (value scales 2^60 apart and more) the denominator takes 2^(x - reference) itself.
//
// Shape. mma with the tokens (then the dims) as the 16 rows and up to 8 (row, query head) columns as n. A block of
// 16 tokens is one bulk copy; its K codes lie in the pool as the 8 x 16-byte tiles that ldmatrix reads without bank conflicts, its
// V codes dim by dim with the tokens in the order in which a lane's weights come out of movmatrix, so that a
// code costs half a conversion and nothing else. Each warp owns blocks with a ring of its own, so no
// block-wide barrier is met before the end, where the warps' results are joined.
//
// Bound: 2 d + 1 bytes per token and KV head from HBM. Measured: one row each of 64 requests of 2 000-30 000 tokens, 28 x 4
// heads of 128, 176 us with the join (6.0 TB/s, 88 % of the copy rate; 38 % of the issue slots); one of 262 145 tokens, 32 x 8
// heads, 93 us (5.8 TB/s). Two or four column blocks in a CTA of their own SM share the conversions but leave half of the
// warps: 2 rows of 64 requests of about 4 000 tokens 83 us with blocks of their own, 99 and 136 so.
#include "attn_warps.cuh"
#include "fp8.cuh"
#include "packed_attn.cuh"

namespace conduit {
namespace {

constexpr int kWarps = 8;
constexpr int kStages = 3;

__device__ __forceinline__ void ldmatrix4(uint32_t at, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(at)
               : "memory");
}

// State of a warp's running softmax for the two columns of a lane.
template <int NG>
struct Running {
  float ref[2], sum[2];  // reference exponent (log2 units, of weight times value scale), sum of weights of this lane's tokens
  float o[2 * NG][4];    // dims 16 t + q of both columns, then dims 8 on
};

// One block. kEdge: some column does not see all of it.
template <int NG, bool kEdge>
__device__ __forceinline__ void block_step(Running<NG>& st, const uint8_t* box, uint32_t at, const uint32_t (&bq)[2 * NG][2],
                                           const float (&to_log2)[2], int kb, int k1, int least, const int (&lim)[2], int lane) {
  constexpr int D = NG * 32;
  const int c = lane & 3, q = lane >> 2;
  const float2 scale = *reinterpret_cast<const float2*>(box + 32 * D);
  const int v_exp = exponent_of(scale.y);
  const float v_log2 = float(v_exp), v_down = power_of_two(-v_exp);
  float x[4], odd[4];
  // tiles: tokens 0-7 and 8-15 of a chunk of 16 dims, then of the next
  const uint32_t k_at = at + (lane >> 3 & 1) * 8 * D + (lane >> 4) * 128 + (lane & 7) * 16;
#pragma unroll
  for (int i = 0; i < NG; ++i) {
    uint32_t r[4];
    ldmatrix4(k_at + 256 * i, r);
    // a lane's word: dims 4 c .. 4 c + 3 of the chunk
    if (i == 0) {
      mma_f16_first(x, halves_lo(r[0]), halves_lo(r[1]), halves_hi(r[0]), halves_hi(r[1]), bq[0][0], bq[0][1]);
      mma_f16_first(odd, halves_lo(r[2]), halves_lo(r[3]), halves_hi(r[2]), halves_hi(r[3]), bq[1][0], bq[1][1]);
    } else {
      mma_f16(x, halves_lo(r[0]), halves_lo(r[1]), halves_hi(r[0]), halves_hi(r[1]), bq[2 * i][0], bq[2 * i][1]);
      mma_f16(odd, halves_lo(r[2]), halves_lo(r[3]), halves_hi(r[2]), halves_hi(r[3]), bq[2 * i + 1][0], bq[2 * i + 1][1]);
    }
  }
  const float f[2] = {scale.x * to_log2[0], scale.x * to_log2[1]};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[e] = (x[e] + odd[e]) * f[e & 1];
    if (kEdge && kb + q + (e < 2 ? 0 : 8) >= lim[e & 1]) x[e] = -INFINITY;
  }
  float top[2] = {fmaxf(x[0], x[2]) + v_log2, fmaxf(x[1], x[3]) + v_log2};
  if (__any_sync(0xffffffffu, top[0] > st.ref[0] + kMostWeight || top[1] > st.ref[1] + kMostWeight)) {
    float corr[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
#pragma unroll
      for (int s = 4; s < 32; s <<= 1) top[e] = fmaxf(top[e], __shfl_xor_sync(0xffffffffu, top[e], s));
      const float moved = fmaxf(st.ref[e], top[e] - kBias), by = st.ref[e] - moved;
      corr[e] = moved == -INFINITY ? 1.f : tc::ex2(by);
      st.ref[e] = moved;
      st.sum[e] = scaled_down(st.sum[e], by, corr[e]);
    }
#pragma unroll
    for (int t = 0; t < 2 * NG; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) st.o[t][e] *= corr[e & 1];
  }
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const float base = (kEdge && st.ref[e] == -INFINITY ? 0.f : st.ref[e]) - v_log2, x0 = x[e], x1 = x[e + 2];
    x[e] = tc::ex2(x0 - base);
    x[e + 2] = tc::ex2(x1 - base);
    if (top[e] < st.ref[e] - kFarBelow) {
      const float lifted = st.ref[e] - kLift;
      st.sum[e] = fmaf(tc::ex2(x0 - lifted) + tc::ex2(x1 - lifted), kUnlift, st.sum[e]);
    } else {
      st.sum[e] = fmaf(x[e] + x[e + 2], v_down, st.sum[e]);
    }
  }
  // tokens 2 c, 2 c + 1 and 8 on of column q
  const uint32_t b0 = transpose8x8(h2u(__floats2half2_rn(x[0], x[1])));
  const uint32_t b1 = transpose8x8(h2u(__floats2half2_rn(x[2], x[3])));
  uint32_t keep = 0xFFFFFFFFu;  // kEdge: bytes of tokens that the chunk has
  if (kEdge) {
    keep = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (kb + 8 * (k >> 1) + 2 * c + (k & 1) < k1) keep |= 0xFFu << (8 * k);
  }
  const uint32_t v_at = at + 16 * D + lane * 16;
#pragma unroll
  for (int i = 0; i < NG; ++i) {
    uint32_t r[4];
    ldmatrix4(v_at + 512 * i, r);
    if (kEdge) {
      // Tokens that some column does not see have weight 0 there, and 0 times NaN must not be: NaN codes become 0, and
      // a product of the places of NaN with the tokens seen says which outputs they reach.
      uint32_t nan[4], any = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        r[k] &= keep;
        nan[k] = (((r[k] & 0x7F7F7F7Fu) + 0x01010101u) >> 7) & 0x01010101u;
        any |= nan[k];
      }
      if (__any_sync(0xffffffffu, any != 0)) {
        const int lo = __shfl_sync(0xffffffffu, lim[0], q >> 1), hi = __shfl_sync(0xffffffffu, lim[1], q >> 1);
        const int own = (q & 1 ? hi : lo) - kb;  // tokens of the block that column q sees
        auto seen = [&](int t) { return (t < own ? 0x3C00u : 0u) | (t + 1 < own ? 0x3C000000u : 0u); };
        auto ones_lo = [&](uint32_t n) { return (n & 1u) * 0x3C00u | (n >> 8 & 1u) * 0x3C000000u; };
        auto ones_hi = [&](uint32_t n) { return (n >> 16 & 1u) * 0x3C00u | (n >> 24 & 1u) * 0x3C000000u; };
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float hit[4];
          mma_f16_first(hit, ones_lo(nan[2 * h]), ones_lo(nan[2 * h + 1]), ones_hi(nan[2 * h]), ones_hi(nan[2 * h + 1]),
                        seen(2 * c), seen(2 * c + 8));
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (hit[e] > 0.f) st.o[2 * i + h][e] = NAN;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) r[k] &= ~(nan[k] * 0xFFu);
      }
    }
    mma_f16(st.o[2 * i], halves_lo(r[0]), halves_lo(r[1]), halves_hi(r[0]), halves_hi(r[1]), b0, b1);
    mma_f16(st.o[2 * i + 1], halves_lo(r[2]), halves_lo(r[3]), halves_hi(r[2]), halves_hi(r[3]), b0, b1);
  }
}

// kCluster: the CTAs of a cluster take the chunks of a context and join them in shared memory.
template <int NG, bool kCluster>
__global__ void __launch_bounds__(kWarps * 32, 2) fp8_attn_mma(AttnArgs a) {
  constexpr int D = NG * 32, kBox = fp8_block_bytes(D);
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ uint64_t full[kWarps][kStages];
  if (!kCluster) let_join_start();
  Item it;
  place_of<kCluster>(a, &it);
  const int w = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int c = lane & 3, q = lane >> 2;
  const int k0 = it.chunk * a.chunk;
  // Pages of this warp's next 32 blocks, a block a lane, looked up ahead (the first ones beside the request's rows and
  // length, whether or not the context reaches them).
  auto pages_from = [&](int n) {
    const int64_t j = int64_t(k0) + int64_t(w + (n + lane) * kWarps) * kBlockTokens;
    return j < a.kv.capacity() ? page_entry(a, it.r, int(j)) : 0;
  };
  int pages = pages_from(0), later = 0;
  if (!rows_of<kCluster>(a, &it)) return;
  uint2 qv[2 * NG];
  {
    const int j = it.cb * kCols + q;
    const bool live = j < it.n * a.kv.G;
    const int i = live ? j / a.kv.G : 0, h = live ? it.g * a.kv.G + j % a.kv.G : 0;
    const __nv_bfloat16* src =
        static_cast<const __nv_bfloat16*>(a.q.p) + it.l * a.q.ls + int64_t(it.t0 + i) * a.q.rs + h * a.q.hs + 4 * c;
    const bool wide = ((reinterpret_cast<uintptr_t>(a.q.p) | uint64_t(2 * (a.q.ls | a.q.rs | a.q.hs))) & 7u) == 0;
#pragma unroll
    for (int g = 0; g < 2 * NG; ++g) {
      qv[g] = make_uint2(0, 0);
      if (live && wide) {
        qv[g] = *reinterpret_cast<const uint2*>(src + 16 * g);
      } else if (live) {
        __nv_bfloat16 v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = src[16 * g + e];
        qv[g] = *reinterpret_cast<uint2*>(v);
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
  const int blocks = k1 > k0 ? (k1 - k0 + kBlockTokens - 1) / kBlockTokens : 0;
  const int mine = blocks > w ? (blocks - w + kWarps - 1) / kWarps : 0;

  uint8_t* ring = smem + w * kStages * kBox;
  if (lane == 0) {
#pragma unroll
    for (int s = 0; s < kStages; ++s) tc::mbar_init(&full[w][s], 1);
    tc::fence_barrier_init();
  }
  __syncwarp();
  const uint32_t ring_at = tc::smem_u32(ring);
  auto fill = [&](int n) {
    const int stage = n % kStages, kb = k0 + (w + n * kWarps) * kBlockTokens;
    const int id = __shfl_sync(0xffffffffu, pages, n & 31);
    if ((n & 31) == 8 && n + 24 < mine) later = pages_from((n & ~31) + 32);
    if ((n & 31) == 31) pages = later;
#ifdef CONDUIT_TEST_HOOKS
    if (n == a.withhold) return;  // neither a copy nor an arrive: the wait for this block runs out
#endif
    if (lane == 0) {
      tc::mbar_arrive_expect_tx(&full[w][stage], kBox);
      bulk_load(ring_at + stage * kBox, fp8_block(a.kv, it.l, it.g, page_in_pool(a, id), kb), kBox, &full[w][stage]);
    }
  };
#pragma unroll
  for (int s = 0; s < kStages; ++s)
    if (s < mine) fill(s);

  // Queries of column q in the operand layout, scaled by 2^-shift so that the largest lies in [2^15, 2^16), or below that where it is
  // small: from 2^109 on every bf16 number is a multiple of fp16's least one.
  uint32_t bq[2 * NG][2];
  float to_log2[2];
  {
    float x[2 * NG][4], top = 0.f;
#pragma unroll
    for (int g = 0; g < 2 * NG; ++g) {
      const __nv_bfloat16* v = reinterpret_cast<const __nv_bfloat16*>(&qv[g]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[g][e] = __bfloat162float(v[e]);
        top = fmaxf(top, fabsf(x[g][e]));
      }
    }
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
    int shift = max(int(__float_as_uint(top) >> 23) - 127 - 15, -109);  // top < 2^(shift + 16)
    if (!(top < INFINITY) || top == 0.f) shift = 0;
    const float up = power_of_two(-shift), back = a.scale * kLog2e * power_of_two(shift);
#pragma unroll
    for (int e = 0; e < 2; ++e) to_log2[e] = __shfl_sync(0xffffffffu, back, 4 * (2 * c + e));
#pragma unroll
    for (int g = 0; g < 2 * NG; ++g) {
#pragma unroll
      for (int e = 0; e < 4; ++e) x[g][e] *= up;
      bq[g][0] = h2u(__floats2half2_rn(x[g][0], x[g][1]));
      bq[g][1] = h2u(__floats2half2_rn(x[g][2], x[g][3]));
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
    const int stage = n % kStages, kb = k0 + (w + n * kWarps) * kBlockTokens;
    // lanes time their waits apart; the products and votes below need all of them or none
    ok = __all_sync(0xffffffffu, tc::mbar_wait(&full[w][stage], uint32_t(n / kStages) & 1u));
    if (!ok) break;
    const uint8_t* box = ring + stage * kBox;
    const uint32_t at = ring_at + stage * kBox;
    if (kb + kBlockTokens > least)
      block_step<NG, true>(st, box, at, bq, to_log2, kb, k1, least, lim, lane);
    else
      block_step<NG, false>(st, box, at, bq, to_log2, kb, k1, least, lim, lane);
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
  float* ow = reinterpret_cast<float*>(smem);                          // [warps][columns][kRow]
  float2* ml = reinterpret_cast<float2*>(ow + kWarps * kCols * kRow);  // [warps][columns] (reference, sum)
  static_assert(join_bytes(D, kWarps) <= kWarps * kStages * kBox, "the join fits the ring");
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int col = 2 * c + e;
    if (q == 0) ml[w * kCols + col] = make_float2(st.ref[e] + kBias, st.sum[e] * kUnbias);
#pragma unroll
    for (int t = 0; t < 2 * NG; ++t) {
      float* to = ow + (w * kCols + col) * kRow + 16 * t + q;
      to[0] = st.o[t][e];
      to[8] = st.o[t][e + 2];
    }
  }
  join_warps<D, kWarps, kCluster>(a, it, ow, ml);
}

template <int NG, bool kCluster>
cudaError_t launch(const AttnArgs& a, int64_t items, cudaStream_t stream) {
  constexpr int kSmem = kWarps * kStages * fp8_block_bytes(NG * 32);
  cudaError_t err = cudaFuncSetAttribute(fp8_attn_mma<NG, kCluster>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
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
  return cudaLaunchKernelEx(&cfg, fp8_attn_mma<NG, kCluster>, a);
}

}  // namespace

cudaError_t launch_fp8_attn_mma(const AttnArgs& a, int64_t items, bool cluster, cudaStream_t stream) {
  switch (a.kv.d) {
    case 64: return cluster ? launch<2, true>(a, items, stream) : launch<2, false>(a, items, stream);
    case 96: return cluster ? launch<3, true>(a, items, stream) : launch<3, false>(a, items, stream);
    default: return cluster ? launch<4, true>(a, items, stream) : launch<4, false>(a, items, stream);
  }
}

}  // namespace conduit
