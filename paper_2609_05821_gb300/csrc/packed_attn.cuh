// What the attention kernels over the 4-bit cache share: the arguments of a call,
// a CTA's share of it, and the stores of final rows and partial results.
#pragma once

#include "cache.cuh"
#include "tc_common.cuh"

namespace conduit {
constexpr int kCols = 8;  // columns per CTA

struct AttnArgs {
  PackedDev kv;
  SeqsDev s;
  RowsDev q, out;
  float* lse;             // or NULL
  const int32_t* limits;  // or NULL
  float scale;
  int chunk, chunks, col_blocks;
  float2* part_ml;        // [chunks][L T Hq] (M in log2 units, sum)
  float* part_o;          // [chunks][L T Hq][d]
  int32_t* status;
};

// What a CTA works on.
struct Item {
  int l, r, g, cb, chunk, t0, n, len;
};

__device__ __forceinline__ bool item_of(const AttnArgs& a, Item* it) {
  uint32_t x = blockIdx.x;
  it->cb = int(x % uint32_t(a.col_blocks));
  x /= uint32_t(a.col_blocks);
  it->chunk = int(x % uint32_t(a.chunks));
  x /= uint32_t(a.chunks);
  it->g = int(x % uint32_t(a.kv.Hkv));
  x /= uint32_t(a.kv.Hkv);
  it->r = int(x % uint32_t(a.s.R));
  it->l = int(x / uint32_t(a.s.R));
  it->t0 = a.s.row_off[it->r];
  it->n = a.s.row_off[it->r + 1] - it->t0;
  it->len = cached_len(a.s, a.kv.capacity(), it->r, a.status, threadIdx.x == 0);
  if (it->cb * kCols >= it->n * a.kv.G) return false;
  return it->chunk == 0 || it->chunk * a.chunk < it->len;
}

// Keys that column j of the item sees (0 for columns past the last).
__device__ __forceinline__ int limit_of(const AttnArgs& a, const Item& it, int j) {
  if (j >= it.n * a.kv.G) return 0;
  const int i = j / a.kv.G;
  const int lim = a.limits ? a.limits[it.t0 + i] : it.len - it.n + i + 1;
  return min(max(lim, 0), it.len);
}

// Page of token j of request r, clamped into the pool (out of range: flagged).
__device__ __forceinline__ int page_of(const AttnArgs& a, int r, int j) {
  const int id = a.kv.page_table[int64_t(r) * a.kv.max_pages + (j >> a.kv.page_shift)];
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

constexpr float kLn2 = 0.69314718055994531f;

__device__ __forceinline__ void store_stats(const AttnArgs& a, const Item& it, int j, float m, float sum) {
  const int i = j / a.kv.G, h = it.g * a.kv.G + j % a.kv.G;
  if (a.chunks == 1) {
    if (a.lse)
      a.lse[(int64_t(it.l) * a.kv.Hq + h) * a.s.T + it.t0 + i] = sum == 0.f ? -INFINITY : kLn2 * (m + log2f(sum));
  } else {
    const int64_t cols = int64_t(a.kv.L) * a.s.T * a.kv.Hq;
    a.part_ml[it.chunk * cols + (int64_t(it.l) * a.s.T + it.t0 + i) * a.kv.Hq + h] = make_float2(m, sum);
  }
}

// Warp-level tensor-core kernel (packed_attn_mma.cu): bf16 rows, head_dim 64, 96, 128.
bool packed_attn_mma_supported(const PackedDev& kv, int dtype);
cudaError_t launch_packed_attn_mma(const AttnArgs& a, int64_t items, cudaStream_t stream);

}  // namespace conduit
