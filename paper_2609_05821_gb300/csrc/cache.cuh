// Rotary positions, growing caches and the 4-bit cache: device views shared by
// rope.cu, packed.cu, packed_attn.cu and the host checks of cache_abi.cu.
#pragma once

#include <cuda_fp16.h>

#include <algorithm>

#include "internal.cuh"

namespace conduit {

constexpr int kMaxHeadDim = 256;

// Rows x[l][t][h][:]; strides in elements.
struct RowsDev {
  void* p;
  int64_t ls, rs, hs;
};

// The axis of pair p is 2 bits of word p / 16.
struct RopeDev {
  const float2* table;  // NULL: no rotation (rot == 0)
  const int32_t* pos;   // [A][T]
  int32_t len, rot, half, layout, axes, T;
  float sign;           // -1 turns back
  uint32_t axis[kMaxHeadDim / 32];
};

struct SeqsDev {
  int32_t R, T, max_len, max_rows;
  const int32_t* row_off;
  const int32_t* len;
  const int32_t* row_off_host;
};

struct PackedDev {
  uint8_t* pool;
  const int32_t* page_table;
  int32_t L, Hq, Hkv, G, d, P, max_pages, page_shift;
  int64_t page_bytes;

  __device__ __forceinline__ int capacity() const { return max_pages << page_shift; }
  __device__ __forceinline__ uint8_t* page(int l, int g, int id) const {
    return pool + ((int64_t(l) * P + id) * Hkv + g) * page_bytes;
  }
  // Offsets inside a page of row `row` of K (v = 0) or V (v = 1): codes and (s, m) pairs.
  __device__ __forceinline__ int64_t codes(int v, int row) const {
    return (int64_t(v) << page_shift) * (d / 2) + int64_t(row) * (d / 2);
  }
  __device__ __forceinline__ int64_t params(int v, int row) const {
    return (int64_t(d) << page_shift) + ((int64_t(v) << page_shift) + row) * (d / 8);
  }
};

// Cached tokens of request r, clamped to what the tables hold (out of range: flagged).
__device__ __forceinline__ int cached_len(const SeqsDev& s, int capacity, int r, int32_t* status, bool flag) {
  const int n = s.len[r], most = min(s.max_len, capacity);
  if (n >= 0 && n <= most) return n;
  if (flag) flag_status(status, CONDUIT_FLAG_INDEX);
  return n < 0 ? 0 : most;
}

cudaError_t launch_rope(const RopeDev& rope, int dtype, int L, int T, int H, int d, const RowsDev& x,
                        const RowsDev& out, int32_t* status, cudaStream_t stream);
cudaError_t launch_kv_append(const KvDev& kv, const SeqsDev& s, const RopeDev& rope, const RowsDev& k,
                             const RowsDev& v, const RowsDev& q, const RowsDev& q_out, int32_t* status,
                             cudaStream_t stream);
cudaError_t launch_packed_append(const PackedDev& kv, const SeqsDev& s, const RopeDev& rope, int dtype,
                                 const RowsDev& k, const RowsDev& v, const RowsDev& q, const RowsDev& q_out,
                                 int32_t* status, cudaStream_t stream);
cudaError_t launch_packed_read(const PackedDev& kv, const int32_t* first, const KvDev& dst, const BatchDev& b,
                               int max_tokens, int32_t* status, cudaStream_t stream);

// Attention over the 4-bit cache. A plan says how a call is cut; `scratch` bytes
// of workspace hold the partial results of `chunks` key chunks.
enum { kAttnSimt = 0, kAttnMma = 1, kAttnTc = 2 };
struct PackedAttnPlan {
  int kernel;     // CUDA cores, warp-level tensor cores, tcgen05
  int chunk;      // keys per chunk
  int chunks;     // of the longest context
  int last_chunk, last_chunks;  // tcgen05: the same of the blocks with one column tile
  int64_t part_cols;            // columns with partial results
  int64_t items;  // CTAs
  bool cluster;   // the chunks of a context join inside a cluster
  size_t scratch;
};
// Keys of the longest context that a call allows. A key's place is a 32-bit number, and so is the end of
// the last chunk, which lies less than 2^20 past the last key.
inline int packed_attn_reach(const PackedDev& kv, const SeqsDev& s) {
  return int(std::min<int64_t>(s.max_len, int64_t(kv.max_pages) << kv.page_shift));
}
constexpr int kMaxReach = INT32_MAX - (1 << 20) + 1;
PackedAttnPlan packed_attn_plan(const PackedDev& kv, const SeqsDev& s, int dtype);
cudaError_t launch_packed_attn(const PackedDev& kv, const SeqsDev& s, const PackedAttnPlan& plan, int dtype,
                               const RowsDev& q, float scale, const int32_t* limits, const RowsDev& out,
                               float* lse, void* scratch, int32_t* status, cudaStream_t stream);

}  // namespace conduit
