// Beam search's selection: the best continuations of a group over its beams and the vocabulary.
//
// Mathematics: s(b, v) = sums_b + z_bv - lse_b. Inside a row the order is that of the logits, so one pass
// over a row gives its running sum of exponentials and its n largest logits; rows meet only at the end, with their lse, in fp64,
// so that between two beams the errors of their sums decide and nothing beside them.
//
// Precision of a row's lse, with u = 2^-24: an exponential carries 2.25 |z - reference| u of its argument (difference, product, log2 e)
// and 4 u of ex2, and the same again when a reference moves; over the row's shares that is 3.25 u (ln vocab + 12) + 16 u at most. A load's
// sum is a tree, loads are added with a compensation, so the sums add 26 u whatever the vocabulary, the logarithm 2 u:
// (21 + ln vocab) 2^-22 in all, 7.8e-6 for 128 003 logits. Measured on flat levels below a peak and on slow rises: the rounding of
// the score, 5e-7 (without the compensation and with a reference that follows the maximum: 1.4e-5, 390 loads a lane).
//
// Shape: a cluster per group; its warps share the rows out in segments. While a segment streams by, a lane keeps its running
// maximum and sum, and the maximum of each of up to 16 blocks of its values: nothing about candidates. The n-th largest
// of the lanes' maxima bounds the segment's n best from below, so what can be among them lies in the few blocks that reach it, which
// are read again, 32 at a time; their values above the bound go to a small buffer and, sorted as 64-bit
// keys (logit, then the lower index), into the list of the n best across the warp's lanes. The lists and sums go to the first CTA's
// shared memory, which ranks what can still be chosen. No scratch in memory, one launch.
// Bound: the logits once, and as close behind it the exponentials, one a logit. Measured: 64 groups of 8 rows of 128 003 bf16
// logits, 16 of them chosen, 39 us (3.4 TB/s; about 10 us are its start and what follows the last logit: blocks read again, lists
// merged and ranked); 4 rows of 32 000 in fp32 9.5 us. With candidates sought at every step: 69 us.
#include "beam.cuh"
#include "tc_common.cuh"

namespace conduit {
namespace {

constexpr int kWarps = 8;
constexpr int kClusterMost = 8;
constexpr int kListsMost = kWarps * kClusterMost;
constexpr unsigned kAll = 0xffffffffu;

struct SelectArgs {
  const void* logits;
  int64_t row_stride;
  int width, vocab, n, segs;
  const float* sums;
  float* score;
  int32_t *parent, *token;
  int32_t* status;
};

constexpr int kAtOnce = 4;            // loads of 16 bytes a lane under way, beside as many in work
constexpr int kBlocks = 16;           // blocks of a lane's values
constexpr int kBuffer = 31 + 32 * 8;  // values that wait for a warp's next merge, and one load more

struct Shared {
  uint64_t list[kListsMost][kMaxBeams];  // the first CTA's: every warp's list, sorted
  float2 stats[kListsMost];              // (reference, sum of e^(z - reference))
  double base[kMaxBeams];                // sums - lse, -inf: the row is left out
  float down[kMaxBeams], up[kMaxBeams];  // bounds of it
  float sums[kMaxBeams];
  uint32_t head[kListsMost];             // keys of lower bounds of the lists' first scores
  float least;
  int count;
  union {
    struct {
      uint64_t buffer[kWarps][kBuffer + 1];  // values on their way into a warp's list
      float top[kWarps][kBlocks][32];        // largest values of blocks
      uint32_t block[kWarps][32];            // blocks to read again
    };
    struct {
      uint64_t score[kListsMost * kMaxBeams], at[kListsMost * kMaxBeams];  // what can still be chosen: rank and (beam, token)
    } cand;
  };
};

// A number that grows with x.
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);  // -0 as 0
  return u ^ ((u >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t u) {
  return __uint_as_float(u ^ ((u >> 31) ? 0x80000000u : 0xFFFFFFFFu));
}
// The same, and among equal ones the larger for a lower index; 0 stands for none.
__device__ __forceinline__ uint64_t key_of(float x, uint32_t at) { return uint64_t(ordered(x)) << 32 | (~at); }
__device__ __forceinline__ float value_of(uint64_t key) { return unordered(uint32_t(key >> 32)); }
__device__ __forceinline__ uint32_t index_of(uint64_t key) { return ~uint32_t(key); }

__device__ __forceinline__ uint64_t compare_exchange(uint64_t k, int mask, bool larger) {
  const uint64_t other = __shfl_xor_sync(kAll, k, mask);
  return (k > other) == larger ? k : other;
}

// The 32 keys of a warp in descending order by lane.
__device__ __forceinline__ uint64_t sort_down(uint64_t k, int lane) {
#pragma unroll
  for (int size = 2; size <= 32; size <<= 1)
#pragma unroll
    for (int mask = size >> 1; mask > 0; mask >>= 1) {
      const bool down = size == 32 || !(lane & size);
      k = compare_exchange(k, mask, ((lane & mask) == 0) == down);
    }
  return k;
}

// The 32 largest of two descending lists.
__device__ __forceinline__ uint64_t merge_down(uint64_t list, uint64_t k, int lane) {
  const uint64_t back = __shfl_xor_sync(kAll, k, 31);
  list = list > back ? list : back;
#pragma unroll
  for (int mask = 16; mask > 0; mask >>= 1) list = compare_exchange(list, mask, (lane & mask) == 0);
  return list;
}

// The next float below x.
__device__ __forceinline__ float below(float x) {
  const int u = __float_as_int(x);
  return x == 0.f ? __int_as_float(0x80000001) : __int_as_float(x > 0.f ? u - 1 : u + 1);
}

// What a warp knows of its segment.
struct Best {
  uint64_t list = 0;    // lane i: the i-th best
  int count = 0;        // of values in the buffer
  float m = -INFINITY;  // this lane's largest value
  float ref = -INFINITY, s = 0.f, over = 0.f;  // its sum of e^(z - ref) is s - over
};

// A list and up to 32 values of the buffer: their best. Not inlined: the code of a sort counts where every warp is
// elsewhere in it.
__device__ __noinline__ uint64_t merged(uint64_t list, const uint64_t* from, int count) {
  const int lane = threadIdx.x % 32;
  __syncwarp();
  const uint64_t k = lane < count ? from[lane] : 0;
  list = merge_down(list, sort_down(k, lane), lane);
  __syncwarp();
  return list;
}

// A lower bound of the n-th best of the lanes' largest values, as a threshold: at least n values lie above it.
__device__ __forceinline__ float bound(float top, int n, int lane) {
#pragma unroll
  for (int size = 2; size <= 32; size <<= 1)
#pragma unroll
    for (int mask = size >> 1; mask > 0; mask >>= 1) {
      const float other = __shfl_xor_sync(kAll, top, mask);
      const bool down = size == 32 || !(lane & size), larger = ((lane & mask) == 0) == down;
      top = larger ? fmaxf(top, other) : fminf(top, other);
    }
  top = __shfl_sync(kAll, top, n - 1);
  return top > -INFINITY ? below(top) : top;
}

// Values of each lane, at `at` on, above `limit` into the buffer, and 32 of those at a time into the list.
template <int N>
__device__ __forceinline__ void keep(Best& b, const float (&x)[N], uint32_t at, float limit, uint64_t* buffer, int lane) {
#pragma unroll
  for (int e = 0; e < N; ++e) {
    const bool in = x[e] > limit;
    const uint32_t who = __ballot_sync(kAll, in);
    if (in) buffer[b.count + __popc(who & ((1u << lane) - 1u))] = key_of(x[e], at + e);
    b.count += __popc(who);
  }
#pragma unroll 1
  while (b.count >= 32) {
    b.count -= 32;
    b.list = merged(b.list, buffer + b.count, 32);
  }
}

// N values' part of a lane's maximum and sum. The reference moves by more than kSlack or not at all: a row that rises slowly
// would otherwise scale its sum at every load, and each time is another error of the exponential's.
constexpr float kSlack = 4.f;
template <int N>
__device__ __forceinline__ void add_up(Best& b, const float (&x)[N], float top) {
  const bool moves = top > b.ref + kSlack;
  const float ref = moves ? top : b.ref, base = ref == -INFINITY ? 0.f : ref;
  // the difference first: its rounding, and not that of z log2(e), is what the exponential sees
  constexpr int kSums = N >= 8 ? 4 : 1;
  float2 add[kSums];
#pragma unroll
  for (int e = 0; e < N / 2; ++e) {
    const float2 d = tc::fadd2(make_float2(x[2 * e], x[2 * e + 1]), make_float2(-base, -base));
    const float2 y = tc::fmul2(d, make_float2(kLog2e, kLog2e)), w = make_float2(tc::ex2(y.x), tc::ex2(y.y));
    add[e % kSums] = e < kSums ? w : tc::fadd2(add[e % kSums], w);
  }
  if constexpr (kSums == 4) add[0] = tc::fadd2(tc::fadd2(add[0], add[1]), tc::fadd2(add[2], add[3]));
  const float corr = tc::ex2((b.ref - base) * kLog2e);  // 1 where it stays
  const float was = b.s * corr, more = add[0].x + add[0].y - b.over * corr;
  b.s = was + more;
  b.over = (b.s - was) - more;
  b.ref = ref;
  b.m = fmaxf(b.m, top);
}

template <typename T>
__device__ __forceinline__ void unpack(const uint4& w, bool on, float (&x)[16 / sizeof(T)]) {
  const T* v = reinterpret_cast<const T*>(&w);
#pragma unroll
  for (int e = 0; e < int(16 / sizeof(T)); ++e) x[e] = on ? to_float(v[e]) : -INFINITY;
}

// A number that grows with a score.
__device__ __forceinline__ uint64_t rank_of(double s) {
  const uint64_t u = uint64_t(__double_as_longlong(s));
  return u ^ (u >> 63 ? ~uint64_t(0) : uint64_t(1) << 63);
}
__device__ __forceinline__ double score_of(uint64_t r) {
  return __longlong_as_double(int64_t(r ^ (r >> 63 ? uint64_t(1) << 63 : ~uint64_t(0))));
}
// Descending by score, then by (beam, token).
__device__ __forceinline__ bool before(uint64_t s, uint64_t at, uint64_t t, uint64_t other) {
  return s > t || (s == t && at < other);
}

__device__ __forceinline__ uint32_t in_first_cta(const void* p) {
  uint32_t at;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(tc::smem_u32(p)), "r"(0));
  return at;
}

template <typename T>
__global__ void __launch_bounds__(kWarps * 32, 2) beam_select_kernel(SelectArgs a) {
  constexpr int N = 16 / sizeof(T);
  extern __shared__ __align__(16) uint8_t select_smem[];
  Shared& sh = *reinterpret_cast<Shared*>(select_smem);
  uint32_t rank, ctas;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(ctas));
  asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");  // the first CTA runs before it is written to
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const int64_t g = blockIdx.x / ctas;
  const int id = int(rank) * kWarps + warp, beam = id / a.segs, seg = id % a.segs;
  uint64_t* buffer = sh.buffer[warp];
  Best b;
  if (rank == 0 && threadIdx.x < kMaxBeams) sh.sums[threadIdx.x] = int(threadIdx.x) < a.width ? a.sums[g * a.width + threadIdx.x] : 0.f;
  if (beam < a.width) {
    const T* row = static_cast<const T*>(a.logits) + (g * a.width + beam) * a.row_stride;
    // 16-byte loads from the first boundary on; the first segment takes what lies before it, the last what lies behind
    const int head = min(int((16 - (reinterpret_cast<uintptr_t>(row) & 15u)) % 16 / sizeof(T)), a.vocab);
    const int vecs = (a.vocab - head) / N, tail = head + vecs * N;
    const int v0 = int(int64_t(vecs) * seg / a.segs), v1 = int(int64_t(vecs) * (seg + 1) / a.segs);
    const uint4* from = reinterpret_cast<const uint4*>(row + head);
    // elements of their own: before the first boundary, behind the last
    const float ends[2][2] = {{seg == 0 && lane < head ? to_float(row[lane]) : -INFINITY, -INFINITY},
                              {seg == a.segs - 1 && lane < a.vocab - tail ? to_float(row[int64_t(tail) + lane]) : -INFINITY, -INFINITY}};
    add_up<2>(b, ends[0], ends[0][0]);
    add_up<2>(b, ends[1], ends[1][0]);
    const int loads = (v1 - v0 + 32 * kAtOnce - 1) / (32 * kAtOnce), per_block = max(1, (loads + kBlocks - 1) / kBlocks);
    auto load = [&](int i, uint4 (&w)[kAtOnce]) {
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        const int v = v0 + 32 * (kAtOnce * i + k) + lane;
        if (v < v1) w[k] = __ldcs(from + v);
      }
    };
    float block_top = -INFINITY;
    int left = per_block, at_block = 0;
    auto work = [&](int i, const uint4 (&w)[kAtOnce]) {
      float x[kAtOnce * N];
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        float y[N];
        unpack<T>(w[k], v0 + 32 * (kAtOnce * i + k) + lane < v1, y);
#pragma unroll
        for (int e = 0; e < N; ++e) x[k * N + e] = y[e];
      }
      float top = x[0];
#pragma unroll
      for (int e = 1; e + 1 < kAtOnce * N; e += 2) top = tc::fmax3(top, x[e], x[e + 1]);
      top = fmaxf(top, x[kAtOnce * N - 1]);
      add_up<kAtOnce * N>(b, x, top);
      block_top = fmaxf(block_top, top);
      if (--left == 0 || i == loads - 1) {
        sh.top[warp][at_block++][lane] = block_top;
        block_top = -INFINITY;
        left = per_block;
      }
    };
    {
      uint4 w0[kAtOnce], w1[kAtOnce];  // in turn, so that no copy of one waits for its loads
      load(0, w0);
#pragma unroll 1
      for (int i = 0; i < loads; i += 2) {
        load(i + 1, w1);
        work(i, w0);
        if (i + 1 >= loads) break;
        load(i + 2, w0);
        work(i + 1, w1);
      }
    }
    // What can be among the n best. In the order of the indexes up to a batch of blocks, so that a value that equals the worst of a full
    // list from batches before has n better ones.
    float limit = bound(b.m, a.n, lane);
    auto tighten = [&] {
      const uint64_t worst = __shfl_sync(kAll, b.list, a.n - 1);
      if (worst) limit = fmaxf(limit, value_of(worst));
    };
    if (seg == 0) keep<2>(b, ends[0], uint32_t(lane), limit, buffer, lane);
    uint32_t* ids = sh.block[warp];
    int found = 0;
#pragma unroll 1
    for (int j = 0; j <= at_block; ++j) {
      const bool in = j < at_block && sh.top[warp][j][lane] > limit;
      const uint32_t who = __ballot_sync(kAll, in);
      if (found > 0 && (j == at_block || found + __popc(who) > 32)) {
        __syncwarp();
        const uint32_t id = lane < found ? ids[lane] : 0;
        const int i0 = int(id >> 5) * per_block, i1 = min(i0 + per_block, loads);
#pragma unroll 1
        for (int i = 0; i < per_block; ++i) {
          uint4 w[kAtOnce];
          const int v = v0 + 32 * kAtOnce * (i0 + i) + int(id & 31u);
          const bool on = lane < found && i0 + i < i1;
#pragma unroll
          for (int k = 0; k < kAtOnce; ++k)
            if (on && v + 32 * k < v1) w[k] = from[v + 32 * k];
#pragma unroll
          for (int k = 0; k < kAtOnce; ++k) {
            float y[N];
            unpack<T>(w[k], on && v + 32 * k < v1, y);
            keep<N>(b, y, uint32_t(head) + uint32_t(v + 32 * k) * N, limit, buffer, lane);
          }
        }
        tighten();
        found = 0;
        __syncwarp();
      }
      // (a block that the tightened limit leaves out holds nothing above it)
      if (in) ids[found + __popc(who & ((1u << lane) - 1u))] = uint32_t(j) << 5 | uint32_t(lane);
      found += __popc(who);
    }
    if (seg == a.segs - 1) keep<2>(b, ends[1], uint32_t(tail) + lane, limit, buffer, lane);
    if (b.count > 0) b.list = merged(b.list, buffer, b.count);
    // the lanes' sums, in the order of a butterfly
    float m = b.ref;
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) m = fmaxf(m, __shfl_xor_sync(kAll, m, s));
    b.s = (b.s - b.over) * tc::ex2((b.ref - (m == -INFINITY ? 0.f : m)) * kLog2e);
    b.ref = m;
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) b.s += __shfl_xor_sync(kAll, b.s, s);
  }
  asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
  {
    const uint32_t list = in_first_cta(&sh.list[id][lane]), stats = in_first_cta(&sh.stats[id]);
    asm volatile("st.shared::cluster.b64 [%0], %1;" ::"r"(list), "l"(b.list) : "memory");
    if (lane == 0) asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(stats), "f"(b.ref), "f"(b.s) : "memory");
  }
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  if (rank != 0) return;

  // ------------------------------------------------- one CTA: rows' sums, then the best of the lists
  if (threadIdx.x == 0) {
    sh.count = 0;
    sh.least = -INFINITY;
  }
  for (int w = warp; w < a.width; w += kWarps) {
    float m = -INFINITY;
    for (int i = lane; i < a.segs; i += 32) m = fmaxf(m, sh.stats[w * a.segs + i].x);
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) m = fmaxf(m, __shfl_xor_sync(kAll, m, s));
    const float from = m == -INFINITY ? 0.f : m;
    float sum = 0.f;
    for (int i = lane; i < a.segs; i += 32) {
      const float2 y = sh.stats[w * a.segs + i];
      sum += y.y * tc::ex2((y.x - from) * kLog2e);
    }
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) sum += __shfl_xor_sync(kAll, sum, s);
    if (lane == 0) {
      const float before_row = sh.sums[w];
      const bool wild = !(sum < INFINITY) || !(before_row < INFINITY);
      if (wild) flag_status(a.status, CONDUIT_FLAG_NONFINITE);
      double base = -INFINITY;
      if (!wild && sum > 0.f && before_row > -INFINITY) {
        // ln sum = k ln 2 + ln(1 + f): a float's rounding on a number below 1 alone
        const int k = int(__float_as_uint(sum) >> 23) - 127;
        const float f = __uint_as_float((__float_as_uint(sum) & 0x7FFFFFu) | 0x3F800000u) - 1.f;
        base = double(before_row) - (double(m) + (k * 0.69314718055994530942 + double(log1pf(f))));
      }
      sh.base[w] = base;
      sh.down[w] = __double2float_rd(base);
      sh.up[w] = __double2float_ru(base);
    }
  }
  __syncthreads();
  // The n-th best of the lists' first entries bounds what can be chosen; in fp32, rounded down, against scores rounded up.
  const int lists = a.width * a.segs;
  if (threadIdx.x < kListsMost) {
    const int list = threadIdx.x;
    const uint64_t key = list < lists ? sh.list[list][0] : 0;
    const float low = key ? __fadd_rd(sh.down[list / a.segs], value_of(key)) : -INFINITY;
    sh.head[list] = low > -INFINITY ? ordered(low) : 0;
  }
  __syncthreads();
  if (threadIdx.x < kListsMost) {
    const uint32_t own = sh.head[threadIdx.x];
    int place = 0;
#pragma unroll 16
    for (int i = 0; i < kListsMost; ++i) place += sh.head[i] > own || (sh.head[i] == own && i < int(threadIdx.x));
    if (place == a.n - 1 && own) sh.least = unordered(own);
  }
  __syncthreads();
  constexpr int kPer = kWarps * 32 / kListsMost;  // threads of a list
  const int list = threadIdx.x / kPer, w = list / a.segs;
  if (list < lists && sh.up[w] > -INFINITY) {
    const float least = sh.least, up = sh.up[w];
    const double base = sh.base[w];
    for (int i = threadIdx.x % kPer; i < a.n; i += kPer) {
      const uint64_t key = sh.list[list][i];
      if (!key || __fadd_ru(up, value_of(key)) < least) break;  // the list goes down
      const double score = base + double(value_of(key));
      if (!(score > -INFINITY)) break;
      const int to = atomicAdd(&sh.count, 1);
      sh.cand.score[to] = rank_of(score);
      sh.cand.at[to] = uint64_t(w) << 32 | index_of(key);
    }
  }
  __syncthreads();
  const int count = sh.count;
  const int64_t out = g * a.n;
  for (int i = threadIdx.x; i < count; i += kWarps * 32) {
    const uint64_t own = sh.cand.score[i], own_at = sh.cand.at[i];
    int place = 0;
    for (int j = 0; j < count; ++j) place += before(sh.cand.score[j], sh.cand.at[j], own, own_at);
    if (place < a.n) {
      a.score[out + place] = float(score_of(own));
      a.parent[out + place] = int32_t(g * a.width + int64_t(own_at >> 32));
      a.token[out + place] = int32_t(uint32_t(own_at));
    }
  }
  for (int i = count + threadIdx.x; i < a.n; i += kWarps * 32) {
    a.score[out + i] = -INFINITY;
    a.parent[out + i] = int32_t(g * a.width);
    a.token[out + i] = 0;
  }
}

template <typename T>
cudaError_t launch(SelectArgs a, int groups, cudaStream_t stream) {
  cudaError_t err = cudaFuncSetAttribute(beam_select_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(sizeof(Shared)));
  if (err) return err;
  cudaLaunchAttribute cluster{};
  cluster.id = cudaLaunchAttributeClusterDimension;
  // Two CTAs of 112 registers a thread on an SM: clusters of eight while all of them run at a time, else of four (64 groups of
  // 8 rows of 128 003: 39 us, 45 in clusters of eight; four CTAs an SM with half of the loads under way 43).
  const int ctas = groups * kClusterMost <= 2 * 152 ? kClusterMost : kClusterMost / 2;
  cluster.val.clusterDim.x = ctas;
  cluster.val.clusterDim.y = cluster.val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(unsigned(groups) * ctas);
  cfg.blockDim = dim3(kWarps * 32);
  cfg.dynamicSmemBytes = sizeof(Shared);
  cfg.stream = stream;
  cfg.attrs = &cluster;
  cfg.numAttrs = 1;
  a.segs = ctas * kWarps / a.width;
  count_launches(1);
  return cudaLaunchKernelEx(&cfg, beam_select_kernel<T>, a);
}

}  // namespace

cudaError_t launch_beam_select(const void* logits, int dtype, int64_t row_stride, int groups, int width, int vocab,
                               const float* sums, int num_out, float* score, int32_t* parent, int32_t* token,
                               int32_t* status, cudaStream_t stream) {
  const SelectArgs a{logits, row_stride, width, vocab, num_out, 0, sums, score, parent, token, status};
  return dtype == CONDUIT_BF16 ? launch<__nv_bfloat16>(a, groups, stream) : launch<float>(a, groups, stream);
}

}  // namespace conduit
