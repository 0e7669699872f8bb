// What the warp-level attention kernels over the 4-bit and the 8-bit cache share: their products, and the join of
// a CTA's warps and of a cluster's CTAs.
#pragma once

#include "packed_attn.cuh"

namespace conduit {

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                        uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// The same from zero, without registers for it.
__device__ __forceinline__ void mma_f16_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                              uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}

__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// The value at p's place in the shared memory of CTA `rank` of the cluster.
template <typename T>
__device__ __forceinline__ T read_of(const T* p, int rank) {
  uint32_t at;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(tc::smem_u32(p)), "r"(rank));
  T y;
  if constexpr (sizeof(T) == 8)
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(y.x), "=f"(y.y) : "r"(at) : "memory");
  else
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                 : "=f"(y.x), "=f"(y.y), "=f"(y.z), "=f"(y.w)
                 : "r"(at)
                 : "memory");
  return y;
}

constexpr int join_row(int d) { return d + 4; }
// [warps][columns][row] outputs, (reference, sum) and weights of the warps, and a cluster's own results.
constexpr int join_bytes(int d, int warps) {
  return warps * kCols * (join_row(d) * 4 + 8) + (warps + 1) * kCols * 4 + kCols * (8 + d * 4);
}

// The warps' results, ow [warps][columns][row] and ml [warps][columns] behind it, joined and stored.
template <int D, int kWarps, bool kCluster>
__device__ __forceinline__ void join_warps(const AttnArgs& a, const Item& it, const float* ow, float2* ml) {
  static_assert(kCols * D / 4 <= kWarps * 32, "four dims a thread");
  constexpr int kRow = join_row(D);
  __syncthreads();
  // weights of the warps once per column, then four dims a thread
  float* weight = reinterpret_cast<float*>(ml + kWarps * kCols);  // [warps + 1][columns], the sum last
  float2* joined_ml = reinterpret_cast<float2*>(weight + (kWarps + 1) * kCols);  // [columns] (clusters)
  float4* joined = reinterpret_cast<float4*>(joined_ml + kCols);                 // [columns][D / 4]
  if (threadIdx.x < kWarps * kCols) {
    const int col = threadIdx.x % kCols, i = threadIdx.x / kCols;
    float top = -INFINITY;
#pragma unroll
    for (int k = 0; k < kWarps; ++k) top = fmaxf(top, ml[k * kCols + col].x);
    const float base = top == -INFINITY ? 0.f : top;
    weight[i * kCols + col] = tc::ex2(ml[i * kCols + col].x - base) * kUnbias;
    if (i == 0) {
      float total = 0.f;
#pragma unroll
      for (int k = 0; k < kWarps; ++k) {
        const float by = ml[k * kCols + col].x - base;
        total = add_scaled(total, ml[k * kCols + col].y, by, tc::ex2(by));
      }
      weight[kWarps * kCols + col] = total;
      const int j = it.cb * kCols + col;
      if (kCluster)
        joined_ml[col] = make_float2(top, total);
      else if (j < it.n * a.kv.G)
        store_stats(a, it, j, top, total, a.chunks == 1);
    }
  }
  __syncthreads();
  const int col = threadIdx.x / (D / 4), dd = 4 * (threadIdx.x % (D / 4));
  if (threadIdx.x < kCols * D / 4) {
    const int j = it.cb * kCols + col;
    float4 out = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < kWarps; ++i) {
      const float wgt = weight[i * kCols + col];
      const float4 o = *reinterpret_cast<const float4*>(ow + (i * kCols + col) * kRow + dd);
      out.x = fmaf(wgt, o.x, out.x);
      out.y = fmaf(wgt, o.y, out.y);
      out.z = fmaf(wgt, o.z, out.z);
      out.w = fmaf(wgt, o.w, out.w);
    }
    if (kCluster)
      joined[threadIdx.x] = out;
    else if (j < it.n * a.kv.G)
      store_out4<__nv_bfloat16>(a, it, j, dd, out, weight[kWarps * kCols + col], a.chunks == 1);
  }
  if constexpr (kCluster) {
    // every CTA finishes a slice of the columns' dims over all chunks, in chunk order
    cluster_sync();
    constexpr int kUnits = kCols * D / 4;
    const int C = a.chunks, slice = (kUnits + C - 1) / C, u = it.chunk * slice + threadIdx.x;
    if (int(threadIdx.x) < slice && u < kUnits) {
      const int uc = u / (D / 4), ud = 4 * (u % (D / 4)), j = it.cb * kCols + uc;
      float2 st[8];
      float4 o[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {  // every load under way before the first use
        const int from = min(k, C - 1);
        st[k] = read_of<float2>(&joined_ml[uc], from);
        o[k] = read_of<float4>(&joined[u], from);
      }
      float top = -INFINITY;
#pragma unroll
      for (int k = 0; k < 8; ++k) top = fmaxf(top, st[k].x);
      const float base = top == -INFINITY ? 0.f : top;
      float total = 0.f;
      float4 out = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        if (k >= C) continue;
        const float wgt = tc::ex2(st[k].x - base);
        total = add_scaled(total, st[k].y, st[k].x - base, wgt);
        out.x = fmaf(wgt, o[k].x, out.x);
        out.y = fmaf(wgt, o[k].y, out.y);
        out.z = fmaf(wgt, o[k].z, out.z);
        out.w = fmaf(wgt, o[k].w, out.w);
      }
      if (j < it.n * a.kv.G) {
        store_out4<__nv_bfloat16>(a, it, j, ud, out, total, true);
        if (ud == 0) store_stats(a, it, j, top, total, true);
      }
    }
    cluster_sync();  // nobody leaves while its results are read
  }
}

}  // namespace conduit
