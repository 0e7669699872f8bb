// Attention over the 4-bit and the 8-bit cache: how a call is cut, the CUDA-core kernel (fp32
// rows, head sizes without a tensor-core kernel), and the join of key chunks.
//
// Mathematics: x_j = scale <q, K_j>, out = sum_j e^(x_j - M) V_j / sum_j e^(x_j - M) in
// one pass with a running M per (row, head); chunks of keys give (M, sum, O) that
// combine_kernel joins in order. Columns: the call's rows of a request times the G
// query heads of a KV head, column j = i G + h.
#include <algorithm>
#include <cmath>

#include "fp8.cuh"
#include "packed_attn.cuh"

namespace conduit {
namespace {

// ------------------------------------------------------------- CUDA cores
// A CTA of four warps, two columns a warp, 32 keys at a time as fp32 in shared memory: lanes are
// keys for the logits and dims for the sums. The next 32 keys' codes are on their way into
// registers meanwhile, and the pages of the 32 after them. Bound by the loads from shared memory
// beside the products (three of 16 bytes for eight products of the logits); in small calls by the
// chain of a tile. Measured, 14 x 2 heads of 64 in fp32 with the join: 1-5 rows of 3 requests over
// 1 500 keys 11.4 us (64 keys a chunk; 32: 12.5, 128: 13.4), 10-16 rows over 4 096 keys 49 us.
constexpr int kSimtKeys = 32;
constexpr int kSimtRow(int d) { return d + 4; }  // 16 bytes of eight keys in different banks

// The next 32 keys of the 4-bit cache on their way: eight dims of K and of V of a key, NG such pieces a
// thread. A key past the last stands for zeros.
template <int NG>
struct Coming4 {
  static constexpr int D = NG * 32;
  int id[NG];
  uint32_t kw[NG], vw[NG], kp[NG], vp[NG];
  __device__ __forceinline__ void look_up(const AttnArgs& a, const Item& it, int kb, int k1, int tid) {
#pragma unroll
    for (int i = 0; i < NG; ++i) {
      const int j = kb + (tid + 128 * i) / (D / 8);
      if (j < k1) id[i] = page_entry(a, it.r, j);
    }
  }
  __device__ __forceinline__ void fetch(const AttnArgs& a, const Item& it, int kb, int k1, int tid) {
#pragma unroll
    for (int i = 0; i < NG; ++i) {
      const int e = tid + 128 * i, j = kb + e / (D / 8), u = e % (D / 8), grp = u / 4, c = u % 4;
      kw[i] = vw[i] = kp[i] = vp[i] = 0;
      if (j < k1) {
        const uint8_t* at = a.kv.page(it.l, it.g, page_in_pool(a, id[i]));
        const int row = j & ((1 << a.kv.page_shift) - 1);
        kw[i] = reinterpret_cast<const uint32_t*>(at + a.kv.codes(0, row))[c * NG + grp];
        const uint16_t* vh = reinterpret_cast<const uint16_t*>(at + a.kv.codes(1, row));
        vw[i] = vh[2 * c * NG + grp] | uint32_t(vh[(2 * c + 1) * NG + grp]) << 16;
        kp[i] = reinterpret_cast<const uint32_t*>(at + a.kv.params(0, row))[grp];
        vp[i] = reinterpret_cast<const uint32_t*>(at + a.kv.params(1, row))[grp];
      }
    }
  }
  __device__ __forceinline__ static void unpack(float* to, uint32_t codes, uint32_t param) {
    const float2 sm = __half22float2(u2h(param));
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)  // 2^23 + u less 2^23 + 8, exactly
      x[e] = fmaf(sm.x, __uint_as_float(((codes >> (4 * e)) & 15u) | 0x4B000000u) - 8388616.f, sm.y);
    reinterpret_cast<float4*>(to)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4*>(to)[1] = make_float4(x[4], x[5], x[6], x[7]);
  }
  __device__ __forceinline__ void put(float* ks, float* vs, int tid) {
#pragma unroll
    for (int i = 0; i < NG; ++i) {
      const int e = tid + 128 * i, key = e / (D / 8), u = e % (D / 8);
      unpack(ks + key * kSimtRow(D) + 8 * u, kw[i], kp[i]);
      unpack(vs + key * D + 8 * u, vw[i], vp[i]);
    }
  }
};

// Values of the 8-bit cache reach 2^128 and weights 2^8, so their fp32 sums are held 2^-40 down: with 2^31 keys they stay below
// fp32's largest number, and the least value, 2^-49, is still 2^37 above its least normal one.
constexpr float kValueDown = 1.f / 1099511627776.f, kValueUp = 1099511627776.f;

// The same of the 8-bit cache, two blocks of 16 tokens: eight dims of K of a key, and a dim of V of a
// block's tokens.
template <int NG>
struct Coming8 {
  static constexpr int D = NG * 32, NV = (NG + 1) / 2;
  int kid[NG], vid[NV], seen[NV];  // seen: tokens of the block before the last key
  uint2 kw[NG];
  uint4 vw[NV];
  float kscale[NG], vscale[NV];
  __device__ __forceinline__ void look_up(const AttnArgs& a, const Item& it, int kb, int k1, int tid) {
#pragma unroll
    for (int i = 0; i < NG; ++i) {
      const int j = kb + (tid + 128 * i) / (D / 8);
      if (j < k1) kid[i] = page_entry(a, it.r, j);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int b = (tid + 128 * i) / D, j = kb + kBlockTokens * b;
      if (b < 2 && j < k1) vid[i] = page_entry(a, it.r, j);
    }
  }
  __device__ __forceinline__ void fetch(const AttnArgs& a, const Item& it, int kb, int k1, int tid) {
#pragma unroll
    for (int i = 0; i < NG; ++i) {
      const int e = tid + 128 * i, j = kb + e / (D / 8), u = e % (D / 8), t = j % kBlockTokens;
      kw[i] = make_uint2(0, 0);
      kscale[i] = 0.f;
      if (j < k1) {
        const uint8_t* at = fp8_block(a.kv, it.l, it.g, page_in_pool(a, kid[i]), j - t);
        kw[i] = *reinterpret_cast<const uint2*>(at + (t >> 3) * 8 * D + (u >> 1) * 128 + (t & 7) * 16 + (u & 1) * 8);
        kscale[i] = reinterpret_cast<const float*>(at + 32 * D)[0];
      }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int e = tid + 128 * i, b = e / D, dim = e % D, j = kb + kBlockTokens * b;
      vw[i] = make_uint4(0, 0, 0, 0);
      vscale[i] = 0.f;
      seen[i] = k1 - j;
      if (b < 2 && j < k1) {
        const uint8_t* at = fp8_block(a.kv, it.l, it.g, page_in_pool(a, vid[i]), j);
        vw[i] = *reinterpret_cast<const uint4*>(at + 16 * D + dim * 16);
        vscale[i] = reinterpret_cast<const float*>(at + 32 * D)[1] * kValueDown;
      }
    }
  }
  __device__ __forceinline__ void put(float* ks, float* vs, int tid) {
#pragma unroll
    for (int i = 0; i < NG; ++i) {
      const int e = tid + 128 * i, key = e / (D / 8), u = e % (D / 8);
      const float2 x[4] = {floats_lo(kw[i].x), floats_hi(kw[i].x), floats_lo(kw[i].y), floats_hi(kw[i].y)};
      const float s = kscale[i];
      float4* to = reinterpret_cast<float4*>(ks + key * kSimtRow(D) + 8 * u);
      to[0] = make_float4(x[0].x * s, x[0].y * s, x[1].x * s, x[1].y * s);
      to[1] = make_float4(x[2].x * s, x[2].y * s, x[3].x * s, x[3].y * s);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int e = tid + 128 * i, b = e / D, dim = e % D;
      if (b >= 2) continue;
      const uint32_t w[4] = {vw[i].x, vw[i].y, vw[i].z, vw[i].w};
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const float2 near = floats_lo(w[n]), far = floats_hi(w[n]);  // tokens 2 n, 2 n + 1 and 8 on
        const float y[4] = {near.x, near.y, far.x, far.y};
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const int t = 8 * (c >> 1) + 2 * n + (c & 1);
          vs[(kBlockTokens * b + t) * D + dim] = t < seen[i] ? y[c] * vscale[i] : 0.f;
        }
      }
    }
  }
};

template <typename T, int NG, typename Coming>
__global__ void __launch_bounds__(128) packed_attn_simt(AttnArgs a) {
  constexpr int D = NG * 32, KS = kSimtRow(D);
  extern __shared__ __align__(16) float simt_smem[];
  float *ks = simt_smem, *vs = ks + kSimtKeys * KS, *qs = vs + kSimtKeys * D;
  __shared__ float2 weights[4][kSimtKeys];
  let_join_start();
  Item it;
  place_of(a, &it);
  if (!rows_of(a, &it)) return;
  const int tid = threadIdx.x, w = tid / 32, lane = tid % 32;
  const int own_lim = lane < kCols ? limit_of(a, it, it.cb * kCols + lane) : 0;
  const int most = __reduce_max_sync(0xffffffffu, own_lim);
  int lim[2];
#pragma unroll
  for (int c = 0; c < 2; ++c) lim[c] = __shfl_sync(0xffffffffu, own_lim, 2 * w + c);
  const int k0 = it.chunk * a.chunk, k1 = min(k0 + a.chunk, most);

  Coming next;
  next.look_up(a, it, k0, k1, tid);
  for (int e = tid; e < kCols * D; e += 128) {
    const int j = it.cb * kCols + e / D;
    float x = 0.f;
    if (j < it.n * a.kv.G) {
      const int i = j / a.kv.G, h = it.g * a.kv.G + j % a.kv.G;
      x = to_float(static_cast<const T*>(a.q.p)[it.l * a.q.ls + int64_t(it.t0 + i) * a.q.rs + h * a.q.hs + e % D]);
    }
    qs[e] = x;
  }
  next.fetch(a, it, k0, k1, tid);
  next.look_up(a, it, k0 + kSimtKeys, k1, tid);

  const float to_log2 = a.scale * kLog2e;
  float m[2] = {-INFINITY, -INFINITY}, sum[2] = {0.f, 0.f}, o[2][NG];  // sum: of this lane's keys
#pragma unroll
  for (int c = 0; c < 2; ++c)
#pragma unroll
    for (int e = 0; e < NG; ++e) o[c][e] = 0.f;
  for (int kb = k0; kb < k1; kb += kSimtKeys) {
    __syncthreads();
    next.put(ks, vs, tid);
    next.fetch(a, it, kb + kSimtKeys, k1, tid);
    next.look_up(a, it, kb + 2 * kSimtKeys, k1, tid);
    __syncthreads();
    float x[2] = {0.f, 0.f};
    const float4* k = reinterpret_cast<const float4*>(ks + lane * KS);
    const float4* q0 = reinterpret_cast<const float4*>(qs + 2 * w * D);
#pragma unroll 8
    for (int e = 0; e < D / 4; ++e) {
      const float4 y = k[e];
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const float4 z = q0[c * (D / 4) + e];
        x[c] = fmaf(z.w, y.w, fmaf(z.z, y.z, fmaf(z.y, y.y, fmaf(z.x, y.x, x[c]))));
      }
    }
#pragma unroll
    for (int c = 0; c < 2; ++c) x[c] = kb + lane < lim[c] ? x[c] * to_log2 : -INFINITY;
    // the reference moves only when a logit passes it by kSimtSlack (log2 units): weights stay below 2^8
    constexpr float kSimtSlack = 8.f;
    if (__any_sync(0xffffffffu, x[0] > m[0] + kSimtSlack || x[1] > m[1] + kSimtSlack)) {
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float top = x[c];
#pragma unroll
        for (int s = 16; s > 0; s >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, s));
        const float mn = fmaxf(m[c], top), corr = mn == -INFINITY ? 1.f : exp2f(m[c] - mn);
        sum[c] *= corr;
        m[c] = mn;
#pragma unroll
        for (int e = 0; e < NG; ++e) o[c][e] *= corr;
      }
    }
    float2 p;
    p.x = exp2f(x[0] - (m[0] == -INFINITY ? 0.f : m[0]));
    p.y = exp2f(x[1] - (m[1] == -INFINITY ? 0.f : m[1]));
    sum[0] += p.x;
    sum[1] += p.y;
    weights[w][lane] = p;
    __syncwarp();
    if (kb + kSimtKeys <= min(lim[0], lim[1])) {
#pragma unroll 8
      for (int key = 0; key < kSimtKeys; ++key) {
        const float2 y = weights[w][key];
        uint32_t v[NG];
        load_words<NG>(reinterpret_cast<const uint8_t*>(vs + key * D + NG * lane), v);
#pragma unroll
        for (int e = 0; e < NG; ++e) {
          o[0][e] = fmaf(y.x, __uint_as_float(v[e]), o[0][e]);
          o[1][e] = fmaf(y.y, __uint_as_float(v[e]), o[1][e]);
        }
      }
    } else if (kb < max(lim[0], lim[1])) {
#pragma unroll 8
      for (int key = 0; key < kSimtKeys; ++key) {
        const float2 y = weights[w][key];
        const bool s0 = kb + key < lim[0], s1 = kb + key < lim[1];  // a NaN value reaches only rows that see it
        uint32_t v[NG];
        load_words<NG>(reinterpret_cast<const uint8_t*>(vs + key * D + NG * lane), v);
#pragma unroll
        for (int e = 0; e < NG; ++e) {
          if (s0) o[0][e] = fmaf(y.x, __uint_as_float(v[e]), o[0][e]);
          if (s1) o[1][e] = fmaf(y.y, __uint_as_float(v[e]), o[1][e]);
        }
      }
    }
  }
#pragma unroll
  for (int c = 0; c < 2; ++c) {
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) sum[c] += __shfl_xor_sync(0xffffffffu, sum[c], s);
    const int j = it.cb * kCols + 2 * w + c;
    if (j >= it.n * a.kv.G) continue;
#pragma unroll
    for (int e = 0; e < NG; ++e) store_out<T>(a, it, j, NG * lane + e, o[c][e], sum[c]);
    if (lane == 0) store_stats(a, it, j, m[c], sum[c], a.chunks == 1);
  }
}

constexpr int simt_smem_bytes(int d) { return (kSimtKeys * (kSimtRow(d) + d) + kCols * d) * int(sizeof(float)); }

// ---------------------------------------------------------------- the join
// Groups of threads with four dims a thread: kJoin groups share a (layer, row, head) and
// take every kJoin-th chunk of the request's context, then join in order. One group that
// walked over 147 chunks took 60 us, eight take 5; over two chunks of 73 000 (row, head)
// pairs eight groups each (six of them idle) took 200 us. Three to seven chunks (whole
// calls, one group and eight): 126 pairs 11.8 and 9.1 us, 448 pairs 12.7 and 11.7, 1 792 pairs
// 26.2 and 28.6, 4 500 pairs 47.9 and 58.6.
template <typename T, int NG, int kJoin>
__global__ void __launch_bounds__(NG * 64) combine_kernel(AttnArgs a) {
  constexpr int D = NG * 32, kLanes = NG * 8, kPer = 8 / kJoin;
  __shared__ float4 part[8][kLanes];
  __shared__ float part_sum[8];
  const int lane = threadIdx.x % kLanes, grp = threadIdx.x / kLanes, of = grp % kJoin;
  const int64_t cols = a.part_cols, col = int64_t(blockIdx.x) * kPer + grp / kJoin;
  bool on = col < cols;
  int h = 0, t = 0, l = 0, n = 0;
  if (on) {
    int r, chunk = a.chunk;
    if (a.chunks > 1) {
      h = int(col % a.kv.Hq), t = int(col / a.kv.Hq % a.s.T), l = int(col / a.kv.Hq / a.s.T);
      r = request_of(a.s.row_off, a.s.R, t);
    } else {  // a column of the tile that a request has left over from its pairs
      const int64_t unit = col / 128;
      const int g = int(unit % a.kv.Hkv);
      r = int(unit / a.kv.Hkv % a.s.R), l = int(unit / a.kv.Hkv / a.s.R);
      const int t0 = a.s.row_off[r], all = (a.s.row_off[r + 1] - t0) * a.kv.G, tiles = (all + 127) / 128;
      const int j = 128 * (tiles - 1) + int(col % 128);
      on = (tiles & 1) && j < all;
      t = t0 + j / a.kv.G, h = g * a.kv.G + j % a.kv.G, chunk = a.last_chunk;
    }
    const int len = cached_len(a.s, a.kv.capacity(), r, nullptr, false);
    n = on ? (len - 1) / chunk + 1 : 0;  // one chunk where there is no key
  }
  wait_for_chunks();
  float top = -INFINITY;
  if (kJoin == 8) {  // one column in the block: its warps look for the reference lane by lane
    for (int c = threadIdx.x % 32; c < n; c += 32) top = fmaxf(top, a.part_ml[c * cols + col].x);
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, s));
  } else {
    for (int c = 0; c < n; ++c) top = fmaxf(top, a.part_ml[c * cols + col].x);
  }
  const float base = top == -INFINITY ? 0.f : top;
  float sum = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int c = of; c < n; c += kJoin) {
    const float2 ml = a.part_ml[c * cols + col];
    const float wgt = exp2f(ml.x - base);
    sum = add_scaled(sum, ml.y, ml.x - base, wgt);
    const float4 po = *reinterpret_cast<const float4*>(a.part_o + (c * cols + col) * D + 4 * lane);
    o.x = fmaf(wgt, po.x, o.x);
    o.y = fmaf(wgt, po.y, o.y);
    o.z = fmaf(wgt, po.z, o.z);
    o.w = fmaf(wgt, po.w, o.w);
  }
  if (kJoin > 1) {
    part[grp][lane] = o;
    if (lane == 0) part_sum[grp] = sum;
    __syncthreads();
    if (of != 0 || !on) return;
#pragma unroll
    for (int c = 1; c < kJoin; ++c) {
      const float4 y = part[grp + c][lane];
      sum += part_sum[grp + c];
      o.x += y.x, o.y += y.y, o.z += y.z, o.w += y.w;
    }
  }
  if (!on) return;
  const float inv = sum == 0.f ? 0.f : a.v_up / sum;
  T* to = static_cast<T*>(a.out.p) + l * a.out.ls + int64_t(t) * a.out.rs + h * a.out.hs + 4 * lane;
  to[0] = from_float<T>(o.x * inv);
  to[1] = from_float<T>(o.y * inv);
  to[2] = from_float<T>(o.z * inv);
  to[3] = from_float<T>(o.w * inv);
  if (lane == 0 && a.lse)
    a.lse[(int64_t(l) * a.kv.Hq + h) * a.s.T + t] = sum == 0.f ? -INFINITY : kLn2 * (base + log2f(sum));
}

template <typename T, int NG, typename Coming>
cudaError_t launch_simt(const AttnArgs& a, const PackedAttnPlan& plan, cudaStream_t stream) {
  constexpr int kSmem = simt_smem_bytes(NG * 32);
  cudaError_t err = cudaFuncSetAttribute(packed_attn_simt<T, NG, Coming>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
  if (err) return err;
  packed_attn_simt<T, NG, Coming><<<unsigned(plan.items), 128, kSmem, stream>>>(a);
  count_launches(1);
  return cudaGetLastError();
}

template <typename T, int NG>
cudaError_t launch_ng(const AttnArgs& a, const PackedAttnPlan& plan, cudaStream_t stream) {
  cudaError_t err;
  if (plan.kernel == kAttnTc) {
    err = plan.bits == 8 ? launch_fp8_attn_tc(a, plan.items, stream) : launch_packed_attn_tc(a, plan.items, stream);
  } else if (plan.kernel == kAttnMma) {
    err = plan.bits == 8 ? launch_fp8_attn_mma(a, plan.items, plan.cluster, stream)
                         : launch_packed_attn_mma(a, plan.items, plan.cluster, stream);
  } else if (plan.bits == 8) {
    err = launch_simt<T, NG, Coming8<NG>>(a, plan, stream);
  } else {
    err = launch_simt<T, NG, Coming4<NG>>(a, plan, stream);
  }
  const int chunks = std::max(a.chunks, a.last_chunks);
  if (err || chunks == 1 || plan.cluster) return err;
  cudaLaunchAttribute early{};
  early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  early.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg{};
  const bool wide_join = chunks >= 8 || (chunks > 2 && a.part_cols <= 1024);
  cfg.gridDim = dim3(unsigned(wide_join ? a.part_cols : (a.part_cols + 7) / 8));
  cfg.blockDim = dim3(NG * 64);
  cfg.stream = stream;
  cfg.attrs = &early;
  cfg.numAttrs = 1;
  count_launches(1);
  return wide_join ? cudaLaunchKernelEx(&cfg, combine_kernel<T, NG, 8>, a)
                       : cudaLaunchKernelEx(&cfg, combine_kernel<T, NG, 1>, a);
}

template <typename T>
cudaError_t launch_t(const AttnArgs& a, const PackedAttnPlan& plan, cudaStream_t stream) {
  switch (a.kv.d / 32) {
    case 1: return launch_ng<T, 1>(a, plan, stream);
    case 2: return launch_ng<T, 2>(a, plan, stream);
    case 3: return launch_ng<T, 3>(a, plan, stream);
    case 4: return launch_ng<T, 4>(a, plan, stream);
    case 5: return launch_ng<T, 5>(a, plan, stream);
    case 6: return launch_ng<T, 6>(a, plan, stream);
    case 7: return launch_ng<T, 7>(a, plan, stream);
    default: return launch_ng<T, 8>(a, plan, stream);
  }
}

// Column blocks of the request with most rows. tcgen05: pairs of column tiles and a rank for
// blocks with one.
int64_t blocks_of(const PackedDev& kv, const SeqsDev& s, int kernel) {
  const int64_t cols = int64_t(s.max_rows) * kv.G;
  return kernel == kAttnTc ? (cols + 127) / 128 / 2 + 1 : (cols + kCols - 1) / kCols;
}
int64_t items_of(const PackedDev& kv, const SeqsDev& s, int kernel, int chunks, int last_chunks) {
  return int64_t(kv.L) * s.R * kv.Hkv * ((blocks_of(kv, s, kernel) - 1) * chunks + last_chunks);
}

// (reference, sum) of every chunk and column with partial results, to a multiple of 16 bytes.
size_t stats_bytes(const PackedAttnPlan& p) {
  return (size_t(std::max(p.chunks, p.last_chunks)) * p.part_cols * sizeof(float2) + 15) / 16 * 16;
}

// Time by which `places` SMs are done with `pairs` CTAs of tp each and then `singles` of ts.
double pass_time(int64_t pairs, int64_t singles, double tp, double ts) {
  constexpr int64_t places = 152;
  double at[2] = {pairs / places * tp, (pairs / places + 1) * tp};
  const int64_t n[2] = {places - pairs % places, pairs % places};
  double end = n[1] ? at[1] : at[0];
  while (singles > 0) {
    const int i = n[1] && at[1] < at[0];
    at[i] += ts;
    singles -= n[i];
    end = std::max(end, at[i]);
  }
  return end;
}

// Keys of a chunk (a multiple of step) and chunks of the longest context, from about `chunks`.
void cut(int most, int step, int* chunk, int* chunks) {
  *chunk = std::max(step, (most + *chunks - 1) / *chunks);
  *chunk = (*chunk + step - 1) / step * step;
  *chunks = most > *chunk ? (most - 1) / *chunk + 1 : 1;
}

}  // namespace

#ifdef CONDUIT_TEST_HOOKS
// Test builds only (never in libconduit.so): the next attention launches over a 4-bit cache leave out
// load n of each warp or CTA of the tensor-core kernels (n < 0: none), so that its bounded waits run out.
int32_t g_test_withhold_load = -1;
extern "C" void conduit_test_withhold_packed_load(int32_t n) { g_test_withhold_load = n; }
#endif

PackedAttnPlan packed_attn_plan(const PackedDev& kv, const SeqsDev& s, int dtype, int bits) {
  PackedAttnPlan p{};
  p.bits = bits;
  const int most = packed_attn_reach(kv, s);
  const bool mma = dtype == CONDUIT_BF16 && (kv.d == 64 || kv.d == 96 || kv.d == 128);
  // (The models here and below have the times of 128 dims; 64 and 96 go by them too.)
  // Up to eight columns: the warp-level kernel, whose one block reads the cache once. Up to 64: the
  // kernel with less time by a model, blocks of eight columns at 3.5 us and 9 ns a key on 304 places
  // after 8 us, or tiles of 128 at 11 us and 1.35 us for 128 keys (2.5 in two parts) on 152 after 18
  // (28 x 4 heads, 2 and 4 and 8 rows, warp-level / tcgen05, us: one request of 4 000 tokens 9.6 / 15.8,
  // 11.3 / 16.0, 12.5 / 16.4; 16 of about 4 000 29 / 54, 47 / 52, 84 / 58; 64 of about 1 000 37 / 81,
  // 56 / 79, 89 / 75; 64 of about 4 000 98 / 137, 159 / 133, 285 / 131).
  const int64_t columns = int64_t(s.max_rows) * kv.G;
  const double units = double(kv.L) * s.R * kv.Hkv;
  // The same with 8 bits: 5.8 ns a key (16 requests of about 4 000, 3 and 4 and 6 rows 35 / 58, 39 / 54, 65 / 62; 64 of about
  // 1 000 37 / 56, 45 / 57, 66 / 53; 64 of about 4 000 104 / 152, 131 / 154, 197 / 175; 16 of about 16 000 101 / 143, 139 / 155,
  // 158 / 143).
  const double warp_us = 8. + units * ((columns + kCols - 1) / kCols) * (3.5 + (bits == 8 ? 0.0058 : 0.009) * most) / 304.;
  const double tc_us = 18. + units * (11. + (bits == 4 && most < kExactBelow ? 2.5 : 1.35) / 128. * most) / 152.;
  const bool few = columns <= kCols || (columns <= 64 && warp_us < tc_us);
  p.kernel = !mma ? kAttnSimt : few ? kAttnMma : kAttnTc;
  const int step = p.kernel == kAttnSimt ? 64 : 256;  // least keys of a chunk
  const int64_t largest = std::max(1, (most + step - 1) / step);
  if (p.kernel == kAttnTc) {
    // One CTA per SM: the chunks with the least time by a model of the pass where every row sees
    // max_len keys, 11 us for a CTA and
    // 1.8 us for 128 keys of two column tiles (3.3 of keys in two parts), three quarters of it for
    // one, and of the join, 12 bytes a partial value at 5 TB/s after a launch of 5 us. Either all
    // blocks have the same chunks (two layers x 16 requests x 8 192 keys, 28 / 4 heads of 96: one
    // chunk 386 us, two 421) or only those with one column tile, which come last and fill up
    // what the pairs leave of the SMs (the same with 128 dims: 350 us without, 317 with; 96: 329).
    int64_t pairs = 0, singles = 0;
    for (int r = 0; r < s.R; ++r) {
      const int64_t tiles = (int64_t(s.row_off_host[r + 1] - s.row_off_host[r]) * kv.G + 127) / 128;
      pairs += tiles / 2;
      singles += tiles & 1;
    }
    const int64_t heads = int64_t(kv.L) * kv.Hkv, items = heads * (pairs + singles);
    const double per = bits == 8 ? 1.9 : most < kExactBelow ? 3.3 : 1.8;
    const double keys = per / 128. * most, all = double(kv.L) * s.T * kv.Hq;
    auto join = [&](int64_t c, double cols) { return c > 1 ? 5. + c * cols * kv.d * 12. / 5e6 : 0.; };
    // 8 bits: the mean of that and of the same contexts with lengths spread evenly up to max_len, half as many keys on as many SMs,
    // so that unequal lengths find CTAs to even them out (16 requests of 2 000-30 000 tokens, 4 rows: 210 us in two chunks, 155 so).
    auto spread = [&](int64_t n_pairs, int64_t n_singles, int64_t cp, int64_t cs, double tp, double ts) {
      const double even = pass_time(n_pairs * cp, n_singles * cs, tp, ts);
      if (bits != 8) return even;
      const double work = n_pairs * (0.5 * (cp + 1)) * tp + n_singles * (0.5 * (cs + 1)) * ts;
      return 0.5 * (even + std::max(work / 152. + 0.5 * (n_pairs ? tp : ts), n_pairs ? tp : ts));
    };
    double best = 0;
    for (int64_t c = 1; c <= std::min<int64_t>(largest, 64) && (c == 1 || items * c <= 8 * 152); ++c) {
      const double tp = 11. + keys / c, ts = 11. + 0.75 * keys / c;
      const double us = spread(heads * pairs, heads * singles, c, c, tp, ts) + join(c, all);
      if (c == 1 || us < best) best = us, p.chunks = p.last_chunks = int(c);
    }
    for (int64_t c = 2; pairs && singles && items <= 8 * 152 && c <= std::min<int64_t>(largest, 8); ++c) {
      const double us = spread(heads * pairs, heads * singles, 1, c, 11. + keys, 11. + 0.75 * keys / c) +
                        join(c, double(heads * singles * 128));
      if (us < best) best = us, p.chunks = 1, p.last_chunks = int(c);
    }
    cut(most, step, &p.last_chunk, &p.last_chunks);
  } else {
    // An SM holds two CTAs. One request: one wave of equal chunks. More, on the CUDA cores: eight
    // CTAs for each place, so that contexts of unequal lengths fill it. On the tensor cores a CTA's
    // start weighs more, so that only as long as chunks keep about 2 048 keys (the last one no fewer than
    // 1 281), and one wave else (one row,
    // 4 KV heads, us with chunks of 256 keys and so: 64 requests of about 300 tokens 18.9 and 11.5,
    // of 1 000 34.7 and 22.1, of 4 000 63.9 and 52.8, of 16 000, where both are 3 000, 157; 16 requests
    // of 4 000 34.7 and 24.5, of 16 000 56.9 and 49.7; 5 requests of 4 000 15.9 and 13.1).
    const int64_t items = std::max<int64_t>(1, items_of(kv, s, p.kernel, 1, 1)), places = 2 * 152;
    int64_t even = (8 * places + items - 1) / items;
    if (p.kernel == kAttnMma) even = std::max(places / items, std::min<int64_t>(even, (most + 1023) / 2048));
    if (s.R == 1) even = places / items;
    p.chunks = int(std::max<int64_t>(1, std::min(even, largest)));
  }
  cut(most, step, &p.chunk, &p.chunks);
  if (p.kernel != kAttnTc) p.last_chunk = p.chunk, p.last_chunks = p.chunks;
  p.items = items_of(kv, s, p.kernel, p.chunks, p.last_chunks);
  // Up to eight chunks join inside a cluster: one launch and no partial results in memory. More
  // CTAs than places and the clusters wait for one another (16 requests of 1 025 tokens: 15.8 us
  // with the join, 18.0 us in clusters; one request: 9.4 and 8.5 us).
  p.cluster = p.kernel == kAttnMma && p.chunks > 1 && p.chunks <= 8 && p.items <= 2 * 152;
  p.part_cols = p.chunks > 1 ? int64_t(kv.L) * s.T * kv.Hq : int64_t(kv.L) * s.R * kv.Hkv * 128;
  if (p.last_chunks > 1 && !p.cluster)
    p.scratch = stats_bytes(p) + size_t(std::max(p.chunks, p.last_chunks)) * p.part_cols * size_t(kv.d) * sizeof(float);
  return p;
}

cudaError_t launch_packed_attn(const PackedDev& kv, const SeqsDev& s, const PackedAttnPlan& plan, int dtype,
                               const RowsDev& q, float scale, const int32_t* limits, const RowsDev& out,
                               float* lse, void* scratch, int32_t* status, cudaStream_t stream) {
  const float v_up = plan.bits == 8 && plan.kernel == kAttnSimt ? kValueUp : 1.f;
  AttnArgs a{kv, s, q, out, lse, limits, scale, v_up, plan.chunk, plan.chunks, 0, plan.last_chunk, plan.last_chunks,
             plan.part_cols, nullptr, nullptr, status};
  a.col_blocks = int(blocks_of(kv, s, plan.kernel));
#ifdef CONDUIT_TEST_HOOKS
  a.withhold = g_test_withhold_load;
#endif
  a.part_ml = static_cast<float2*>(scratch);
  a.part_o = reinterpret_cast<float*>(static_cast<char*>(scratch) + stats_bytes(plan));
  return dtype == CONDUIT_BF16 ? launch_t<__nv_bfloat16>(a, plan, stream) : launch_t<float>(a, plan, stream);
}

}  // namespace conduit
