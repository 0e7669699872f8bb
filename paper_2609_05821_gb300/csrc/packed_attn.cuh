// What the attention kernels over the 4-bit cache share: the arguments of a call,
// a CTA's share of it, and the stores of final rows and partial results.
#pragma once

#include "cache.cuh"
#include "tc_common.cuh"

namespace conduit {
constexpr int kCols = 8;  // columns per CTA of the warp-level and CUDA-core kernels

// The tensor-core kernels' weights are fp16 numbers 2^(logit - reference): normal down to 2^-14 and
// 0 from 2^-25 on, while the fp32 sum counts every weight. So the reference stays kBias (log2 units)
// below the largest logit, which makes use of the range up to 2^15, and moves only when a logit passes it
// by kMostWeight. A weight is within 2^-11 of itself or 2^-32 of the row's largest one. (With the
// largest weight at 1, 262 144 keys of 2^-25 beside it lost 0.7 % of the output.)
constexpr float kBias = 7.f, kUnbias = 1.f / 128.f;
constexpr float kMostWeight = 15.f;

// tcgen05: a key as one fp16 number is within 2^-11 of its value, and so a logit within 2^-11 of
// scale sum |q||k|: nothing beside the rounding of a bf16 output, and in a log-sum-exp an error that falls
// with the number of keys that count (2 x 10^-4 of it for one key, 2 x 10^-6 for 8 192 of like
// weight). So a block with a column that sees fewer keys than this, if any, takes its keys as the sum of two
// fp16 numbers, a tile in both key buffers, whose logits keep fp32's precision: 170 us for 32-128 rows over 2 000 keys, where one fp16
// number takes 114. It goes by what the columns see and not by whether a log-sum-exp
// is asked for, so that outputs do not depend on that.
constexpr int kExactBelow = 2048;

struct AttnArgs {
  PackedDev kv;
  SeqsDev s;
  RowsDev q, out;
  float* lse;             // or NULL
  const int32_t* limits;  // or NULL
  float scale;
  int chunk, chunks, col_blocks;
  int last_chunk, last_chunks;  // tcgen05: of blocks with one column tile
  int64_t part_cols;      // columns with partial results: L T Hq, or L R Hkv 128 where only those blocks have them
  float2* part_ml;        // [chunks][part_cols] (M in log2 units, sum)
  float* part_o;          // [chunks][part_cols][d]
  int32_t* status;
#ifdef CONDUIT_TEST_HOOKS
  int32_t withhold;  // test builds: this load of each warp (warp-level kernel) or CTA (tcgen05) is not made (-1: none)
#endif
};

// The join is launched while the chunks are still worked on; it waits for all of them.
__device__ __forceinline__ void let_join_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_chunks() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// What a CTA works on.
struct Item {
  int l, r, g, cb, chunk, t0, n, len;
};

// The chunk, KV head, request and layer of unit x.
__device__ __forceinline__ void decode(const AttnArgs& a, uint32_t x, int chunks, Item* it) {
  it->chunk = int(x % uint32_t(chunks));
  x /= uint32_t(chunks);
  it->g = int(x % uint32_t(a.kv.Hkv));
  x /= uint32_t(a.kv.Hkv);
  it->r = int(x % uint32_t(a.s.R));
  it->l = int(x / uint32_t(a.s.R));
}
// The request's rows and length.
__device__ __forceinline__ void load_rows(const AttnArgs& a, Item* it) {
  it->t0 = a.s.row_off[it->r];
  it->n = a.s.row_off[it->r + 1] - it->t0;
  it->len = cached_len(a.s, a.kv.capacity(), it->r, a.status, threadIdx.x == 0);
}

// Column blocks of kCols, side by side so that they share the keys in L2; in clusters, the
// chunks of a context side by side. The item's place comes first, so that loads which need no
// more go out beside those of its rows; false from the second step: nothing to do.
template <bool kCluster = false>
__device__ __forceinline__ void place_of(const AttnArgs& a, Item* it) {
  const uint32_t inner = kCluster ? a.chunks : a.col_blocks;
  uint32_t x = blockIdx.x / inner;
  if (kCluster) {
    it->cb = int(x % uint32_t(a.col_blocks));
    decode(a, x / uint32_t(a.col_blocks) * a.chunks + blockIdx.x % inner, a.chunks, it);
  } else {
    it->cb = int(blockIdx.x % inner);
    decode(a, x, a.chunks, it);
  }
}
template <bool kCluster = false>
__device__ __forceinline__ bool rows_of(const AttnArgs& a, Item* it) {
  load_rows(a, it);
  if (it->cb * kCols >= it->n * a.kv.G) return false;
  return kCluster || it->chunk == 0 || it->chunk * a.chunk < it->len;
}

// Keys that column j of the item sees (0 for columns past the last).
__device__ __forceinline__ int limit_of(const AttnArgs& a, const Item& it, int j) {
  if (j >= it.n * a.kv.G) return 0;
  const int i = j / a.kv.G;
  const int lim = a.limits ? a.limits[it.t0 + i] : it.len - it.n + i + 1;
  return min(max(lim, 0), it.len);
}

// Page of token j of request r as the table has it, and the same clamped into the pool
// (out of range: flagged). Two steps, so that a lookup can be under way before its use.
__device__ __forceinline__ int page_entry(const AttnArgs& a, int r, int j) {
  return a.kv.page_table[int64_t(r) * a.kv.max_pages + (j >> a.kv.page_shift)];
}
__device__ __forceinline__ int page_in_pool(const AttnArgs& a, int id) {
  if (id >= 0 && id < a.kv.P) return id;
  flag_status(a.status, CONDUIT_FLAG_INDEX);
  return 0;
}

// Element dd of column j: of the final row if the context is one chunk, else of a partial result.
template <typename T>
__device__ __forceinline__ void store_out(const AttnArgs& a, const Item& it, int j, int dd, float o, float sum) {
  const int i = j / a.kv.G, h = it.g * a.kv.G + j % a.kv.G;
  if (a.chunks == 1) {
    T* to = static_cast<T*>(a.out.p) + it.l * a.out.ls + int64_t(it.t0 + i) * a.out.rs + h * a.out.hs;
    to[dd] = from_float<T>(sum == 0.f ? 0.f : o / sum);
  } else {
    const int64_t cols = int64_t(a.kv.L) * a.s.T * a.kv.Hq;
    const int64_t col = (int64_t(it.l) * a.s.T + it.t0 + i) * a.kv.Hq + h;
    a.part_o[(it.chunk * cols + col) * a.kv.d + dd] = o;
  }
}

// The same for dims dd .. dd + 3.
template <typename T>
__device__ __forceinline__ void store_out4(const AttnArgs& a, const Item& it, int j, int dd, float4 o, float sum,
                                           bool last) {
  const int i = j / a.kv.G, h = it.g * a.kv.G + j % a.kv.G;
  if (last) {
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    T* to = static_cast<T*>(a.out.p) + it.l * a.out.ls + int64_t(it.t0 + i) * a.out.rs + h * a.out.hs + dd;
    to[0] = from_float<T>(o.x * inv);
    to[1] = from_float<T>(o.y * inv);
    to[2] = from_float<T>(o.z * inv);
    to[3] = from_float<T>(o.w * inv);
  } else {
    const int64_t cols = int64_t(a.kv.L) * a.s.T * a.kv.Hq;
    const int64_t col = (int64_t(it.l) * a.s.T + it.t0 + i) * a.kv.Hq + h;
    *reinterpret_cast<float4*>(a.part_o + (it.chunk * cols + col) * a.kv.d + dd) = o;
  }
}

constexpr float kLn2 = 0.69314718055994531f;

__device__ __forceinline__ void store_stats(const AttnArgs& a, const Item& it, int j, float m, float sum, bool last) {
  const int i = j / a.kv.G, h = it.g * a.kv.G + j % a.kv.G;
  if (last) {
    if (a.lse)
      a.lse[(int64_t(it.l) * a.kv.Hq + h) * a.s.T + it.t0 + i] = sum == 0.f ? -INFINITY : kLn2 * (m + log2f(sum));
  } else {
    const int64_t cols = int64_t(a.kv.L) * a.s.T * a.kv.Hq;
    a.part_ml[it.chunk * cols + (int64_t(it.l) * a.s.T + it.t0 + i) * a.kv.Hq + h] = make_float2(m, sum);
  }
}

__device__ __forceinline__ uint32_t h2u(__half2 h) { return *reinterpret_cast<uint32_t*>(&h); }
__device__ __forceinline__ __half2 u2h(uint32_t u) { return *reinterpret_cast<__half2*>(&u); }

// Two nibbles u of w as fp16: 1024 + u of bits 0-3 and 16-19, 1024 + 16 u of bits 4-7 and 20-23.
__device__ __forceinline__ uint32_t masked(uint32_t w, uint32_t mask) {  // (w & mask) | 0x64006400
  uint32_t y;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(y) : "r"(w), "r"(mask), "r"(0x64006400u));
  return y;
}
__device__ __forceinline__ uint32_t raw_lo(uint32_t w) { return masked(w, 0x000F000Fu); }
__device__ __forceinline__ uint32_t raw_hi(uint32_t w) { return masked(w, 0x00F000F0u); }
// The same as u - 8, exactly.
__device__ __forceinline__ uint32_t codes_lo(uint32_t w) {
  return h2u(__hadd2(u2h(raw_lo(w)), __float2half2_rn(-1032.f)));
}
__device__ __forceinline__ uint32_t codes_hi(uint32_t w) {
  return h2u(__hfma2(u2h(raw_hi(w)), __float2half2_rn(0.0625f), __float2half2_rn(-72.f)));
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

// Neither s nor m of a parameter pair is infinite or NaN.
__device__ __forceinline__ bool finite_pair(uint32_t p) {
  return (p & 0x7C00u) != 0x7C00u && (p & 0x7C000000u) != 0x7C000000u;
}

// Warp-level tensor-core kernel (packed_attn_mma.cu) and tcgen05 kernel
// (packed_attn_tc.cu): bf16 rows, head_dim 64, 96, 128.
// `cluster`: the chunks of a context form a cluster, which joins them itself.
cudaError_t launch_packed_attn_mma(const AttnArgs& a, int64_t items, bool cluster, cudaStream_t stream);
cudaError_t launch_packed_attn_tc(const AttnArgs& a, int64_t items, cudaStream_t stream);

}  // namespace conduit
