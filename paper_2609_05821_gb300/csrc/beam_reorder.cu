// Contexts follow the beams of a search: page tables are gathered and the page that has been begun is copied,
// in place, in one launch, for caches of any width.
//
// A full page is never written again, so beams share it by its number. The page that parent p has begun is its own, home[p][w];
// beam b gets the rows in use into home[b][w]. A thread owns the same 16 bytes of the begun pages of all beams of a
// group (and the same column of their tables): it reads what all of them need before it writes, which is all
// that an arbitrary map of beams asks for. What the copy reads beside that, lengths of parents and places of begun pages, the
// same launch leaves as it is.
// Bound: the rows in use of the pages begun, read once a parent and written once a child; small calls by the chain parent, length,
// page, rows. Measured: 32 groups of 8 beams, 28 layers of 4 heads of 128 in bf16, pages of 32 tokens, 38 us (47 MB from HBM, 96 MB
// written: 21 us of bytes; a parent's rows are loaded again for each child, from L2). Not HBM (30 % busy) but that chain
// at the start of each CTA, three waves of them, with the rows of about two heads behind it; one group of 4 beams 6 us.
#include <algorithm>

#include "beam.cuh"

namespace conduit {
namespace {

constexpr unsigned kAll = 0xffffffffu;
constexpr int kThreads = 256;

// kMost: beams that a thread has in hand.
template <int kMost>
__global__ void __launch_bounds__(kThreads)
    reorder_kernel(PagedPool pool, int width, const int32_t* parent, const int32_t* home, int32_t* table, int32_t* len,
                   int32_t* status) {
  const int64_t row0 = int64_t(blockIdx.y) * width;
  const int lane = threadIdx.x % 32;
  const bool beam = lane < width;
  // lane b: beam b
  const int64_t from64 = beam ? int64_t(parent[row0 + lane]) - row0 : 0;
  bool fine = from64 >= 0 && from64 < width;
  const int from = fine ? int(from64) : 0;
  const int own_n = len[row0 + from], n = __shfl_sync(kAll, own_n, 0);
  fine &= n >= 0 && int64_t(n) <= int64_t(pool.max_pages) * pool.page_size && own_n == n;
  fine = __all_sync(kAll, !beam || fine);
  const int whole = fine ? n / pool.page_size : 0, rest = fine ? n % pool.page_size : 0;
  int to = 0;
  if (rest) {
    bool own = true;
    if (beam) {
      to = home[(row0 + lane) * pool.max_pages + whole];
      own = to >= 0 && to < pool.num_pages && table[(row0 + from) * pool.max_pages + whole] == home[(row0 + from) * pool.max_pages + whole];
    }
    fine = __all_sync(kAll, own);
  }
  const int source = __shfl_sync(kAll, to, from);
  if (!fine) {
    if (blockIdx.x == 0 && threadIdx.x == 0) flag_status(status, CONDUIT_FLAG_INDEX);
    return;
  }
  if (blockIdx.x == 0) {
    for (int i0 = 0; i0 < pool.max_pages; i0 += kThreads) {
      const int i = i0 + threadIdx.x;
      const bool on = i < pool.max_pages;
      int32_t id[kMost];
#pragma unroll
      for (int b = 0; b < kMost; ++b) {
        const int p = __shfl_sync(kAll, from, b);
        if (b < width && on)
          id[b] = i < whole ? table[(row0 + p) * pool.max_pages + i] : home[(row0 + b) * pool.max_pages + i];
      }
#pragma unroll
      for (int b = 0; b < kMost; ++b)
        if (b < width && on) table[(row0 + b) * pool.max_pages + i] = id[b];
    }
    if (threadIdx.x < width && len[row0 + threadIdx.x] != n) len[row0 + threadIdx.x] = n;
    return;
  }
  if (!rest) return;
  // the beams that take another one's rows over: (page read, page written)
  __shared__ int2 moves[kMaxBeams];
  const uint32_t moved = __ballot_sync(kAll, beam && from != lane);
  if (threadIdx.x < 32 && (moved >> lane & 1u)) moves[__popc(moved & ((1u << lane) - 1u))] = make_int2(source, to);
  __syncthreads();
  const int count = __popc(moved);
  int used[4], all = 0;  // 16-byte chunks in use of a part of a head's page
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    used[k] = k < pool.parts ? ((rest + pool.part[k].tokens - 1) / pool.part[k].tokens * pool.part[k].unit + 15) / 16 : 0;
    all += used[k];
  }
  // A CTA stays for several heads: the chain of loads above costs as much as a head's rows (a CTA for each 256 chunks of the
  // page: 73 us for 32 groups of 8 beams, 28 layers).
  for (int u = blockIdx.x - 1; u < pool.L * pool.heads; u += gridDim.x - 1) {
    const int l = u / pool.heads, head = u % pool.heads;
    for (int c = threadIdx.x; c < all; c += kThreads) {
      int at = c, k = 0;
#pragma unroll
      for (int j = 0; j < 3; ++j)
        if (k == j && at >= used[j]) at -= used[j], ++k;
      const PagePart& part = pool.part[k];
      char* base = part.base + l * part.layer_stride + head * part.head_stride + int64_t(at) * 16;
      uint4 v[kMost];
#pragma unroll
      for (int b = 0; b < kMost; ++b)
        if (b < count) v[b] = *reinterpret_cast<const uint4*>(base + moves[b].x * part.page_stride);
#pragma unroll
      for (int b = 0; b < kMost; ++b)
        if (b < count) *reinterpret_cast<uint4*>(base + moves[b].y * part.page_stride) = v[b];
    }
  }
}

}  // namespace

cudaError_t launch_reorder(const PagedPool& pool, int groups, int width, const int32_t* parent, const int32_t* home,
                           int32_t* page_table, int32_t* len, int32_t* status, cudaStream_t stream) {
  // about three waves of CTAs
  const int64_t units = int64_t(pool.L) * pool.heads, most = std::max(1, 3 * 4 * 152 / groups);
  const dim3 grid(unsigned(1 + std::min(units, most)), groups);
  if (width <= 4)
    reorder_kernel<4><<<grid, kThreads, 0, stream>>>(pool, width, parent, home, page_table, len, status);
  else if (width <= 8)
    reorder_kernel<8><<<grid, kThreads, 0, stream>>>(pool, width, parent, home, page_table, len, status);
  else if (width <= 16)
    reorder_kernel<16><<<grid, kThreads, 0, stream>>>(pool, width, parent, home, page_table, len, status);
  else
    reorder_kernel<32><<<grid, kThreads, 0, stream>>>(pool, width, parent, home, page_table, len, status);
  count_launches(1);
  return cudaGetLastError();
}

}  // namespace conduit
