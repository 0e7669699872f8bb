// Attention over the 8-bit cache for many rows (query prefixes, recomputed rows): tcgen05.
//
// Mathematics: as in fp8_attn_mma.cu: codes exact in fp16, queries as there, the scales of keys on the logits, those of
// values in the exponents of the weights, which are rounded to fp16; logits, statistics and outputs in fp32
// (tensor memory).
//
// Shape. A CTA holds two tiles of 128 columns (A and B: rows of the call times query
// heads of one KV head) and walks over the keys in tiles of 128. Each key tile's codes become fp16 once in shared
// memory for both, keys token by token and values dim by dim, as they lie in the pool, both with the
// dimension that is summed over contiguous. Roles (512 threads):
//   warp 0            MMAs: P_x(t) V(t), then S_x(t + 1), for x = A, B; one lane issues.
//   warp 1            bulk copies of blocks of 16 tokens into a small ring, two at a time
//   warps 2-7         conversion: 16 codes a lane and step
//   warps 8-11, 12-15 softmax of A and of B: a thread owns a column and all 128 keys
// One column tile's softmax runs beside the other's MMAs. MMAs of one thread complete in
// order, so S_x(t + 1) may overwrite P_x(t), and S_x(t + 1) says that P_x(t) V(t) is done.
// TMEM: S_A, S_B at columns [0, 256) with P over their upper halves,
// O_A, O_B at [256, 512). A block with one column tile: A takes the even key tiles, B the odd ones.
//
// Bound: the chain S, softmax, P V, next S of each column tile beside the other's, and under it the shared memory that
// feeds the MMAs (a key tile: 192 KB of operands and 128 KB of codes in, out and widened). Measured: 32-128
// rows of 16 requests over 8 192 keys, two layers of 28 x 4 heads of 128, 331 us (0.96 PFLOP/s, tensor pipe 44 % busy); causal
// prompts, one layer: 8 192 tokens 514 us, four of 4 096 tokens 610. Three loads under way instead of four, and the
// guarded values in the usual loop: 395 us.
#include <type_traits>

#include "fp8.cuh"
#include "packed_attn.cuh"

namespace conduit {
namespace {

constexpr int kThreads = 512;
constexpr int kKeys = 128;                    // keys of a tile
constexpr int kTileCols = 128;                // columns of a tile
constexpr int kTcCols = 2 * kTileCols;
constexpr int kMmaWarp = 0, kLoadWarp = 1, kUnpackWarp = 2, kUnpackWarps = 6, kSoftWarp = 8;
constexpr uint32_t kBlock = 128 * 128;        // 128 rows of 64 fp16, swizzled
constexpr uint32_t kSCols = 128, kPCol = 64, kOCol = 256;
constexpr int kLoadKeys = 2 * kBlockTokens;   // keys of a load
constexpr int kLoads = kKeys / kLoadKeys;     // loads of a key tile
constexpr int kRing = 4;                      // loads under way
constexpr int kBlocks = kKeys / kBlockTokens; // blocks of a key tile
// While no value scale is above 2^kNear, all lie within 2^80 of each other, and a weight down to 2^-46 of its column's largest stays
// in fp32's range. From the first key tile on that has a larger one the denominator goes by weigh_apart.
constexpr float kNear = 40.f;

template <int NG>
struct Sizes {
  static constexpr int D = 32 * NG;
  static constexpr uint32_t kTile = (D + 63) / 64 * kBlock;  // a query or key tile
  static constexpr uint32_t kValues = D * 256;               // a value tile: D rows of 128 tokens
  static constexpr uint32_t kBox = fp8_block_bytes(D);
  static constexpr uint32_t kRaw = 2 * kBox;                 // a load
  static constexpr uint32_t kSmem = 1024 + 4 * kTile + 2 * kValues + kRing * kRaw;
};

struct Bars {
  uint64_t raw_full[kRing], raw_free[kRing];
  uint64_t k_full[2], k_free[2], v_full[2], v_free[2];
  uint64_t q_full, s_full[2], p_full[2], o_full[2], joined, drained;
};

// The larger of two pairs of non-negative bf16, a NaN losing to a number.
__device__ __forceinline__ uint32_t bf16_max2(uint32_t a, uint32_t b) {
  const __nv_bfloat162 y = __hmax2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&y);
}
// kind::f16 with fp16 operands, fp32 sums, the dimension that is summed over contiguous.
constexpr uint32_t idesc_f16(int m, int n) { return (1u << 4) | (uint32_t(n >> 3) << 17) | (uint32_t(m >> 4) << 24); }

// Bounded wait of a converged warp; false after a second or once another role gave up.
__device__ __forceinline__ bool wait_warp(uint64_t* bar, uint32_t parity, volatile int* abort) {
  bool ok = tc::mbar_probe(bar, parity);
  if (!ok) {
    const uint64_t t0 = tc::globaltimer_ns();
    for (uint32_t i = 1; !ok && i < tc::kSpinLimit; ++i) {
      ok = tc::mbar_try_wait(bar, parity);
      if (!ok && (i & 7u) == 0 && (*abort || tc::globaltimer_ns() - t0 > tc::kWaitNs)) break;
    }
  }
  return __all_sync(0xffffffffu, ok);
}

__device__ __forceinline__ void give_up(const AttnArgs& a, volatile int* abort, int32_t site) {
  if (!*abort) flag_status(a.status, CONDUIT_FLAG_TIMEOUT | site);
  *abort = 1;
}

// The item of this CTA: a.col_blocks - 1 ranks of blocks with two column tiles, then one rank
// of blocks with one.
__device__ __forceinline__ bool tc_item(const AttnArgs& a, Item* it) {
  const uint32_t pairs = a.col_blocks - 1, units = uint32_t(a.chunks) * a.kv.Hkv * a.s.R * a.kv.L;
  const bool single = blockIdx.x >= units * pairs;
  uint32_t x = single ? blockIdx.x - units * pairs : blockIdx.x / pairs;
  const int rank = single ? 0 : int(blockIdx.x % pairs);
  decode(a, x, single ? a.last_chunks : a.chunks, it);
  load_rows(a, it);
  const int tiles = (it->n * a.kv.G + kTileCols - 1) / kTileCols;  // column tiles of the request
  it->cb = single ? tiles / 2 : rank;
  if (single ? !(tiles & 1) : rank >= tiles / 2) return false;
  return it->chunk == 0 || it->chunk * (single ? a.last_chunk : a.chunk) < it->len;
}

// 16 codes in order as 32 bytes of fp16: words' halves near, far, near, far ... (keys), or all near ones
// first (values, whose words hold tokens 2 n, 2 n + 1 and 8 on).
template <bool kValues>
__device__ __forceinline__ void widen(const uint4& w, uint4* first, uint4* second) {
  if (kValues) {
    *first = make_uint4(halves_lo(w.x), halves_lo(w.y), halves_lo(w.z), halves_lo(w.w));
    *second = make_uint4(halves_hi(w.x), halves_hi(w.y), halves_hi(w.z), halves_hi(w.w));
  } else {
    *first = make_uint4(halves_lo(w.x), halves_hi(w.x), halves_lo(w.y), halves_hi(w.y));
    *second = make_uint4(halves_lo(w.z), halves_hi(w.z), halves_lo(w.w), halves_hi(w.w));
  }
}

// A dim's values of a block whose tokens are not all seen by every column (tokens j0 ..): codes past the keys become 0;
// so does a NaN that some column does not see (its weight there is 0, and 0 times NaN must not be), and its first token is noted.
__device__ __forceinline__ uint4 guard(uint4 w, int dim, int j0, int k1, int least, int* poison, int* poison_any) {
  uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int n = 0; n < 4; ++n) {
    uint32_t keep = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (j0 + 8 * (k >> 1) + 2 * n + (k & 1) < k1) keep |= 0xFFu << (8 * k);
    x[n] &= keep;
    const uint32_t nan = (((x[n] & 0x7F7F7F7Fu) + 0x01010101u) >> 7) & 0x01010101u;
    if (nan) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int j = j0 + 8 * (k >> 1) + 2 * n + (k & 1);
        if ((nan >> (8 * k) & 1u) && j >= least) {
          atomicMin(&poison[dim], j);
          atomicMin(poison_any, j);
          x[n] &= ~(0xFFu << (8 * k));
        }
      }
    }
  }
  return make_uint4(x[0], x[1], x[2], x[3]);
}

// A block's scales: of its keys, log2 of that of its values, and 2^- of it.
using Scales = float4;

// Weights 2^(x + v + low) of the 128 logits at sb, x = s times the key scale: packed into p; their sum without v into
// add; returns the largest x + v. kEdge: only the first `left` are seen.
template <bool kEdge>
__device__ __forceinline__ float weigh(uint32_t sb, const Scales* scales, float to_log2, float low, int left, uint32_t (&p)[4][16],
                                       float* add) {
  float top = -INFINITY;
  *add = 0.f;
#pragma unroll
  for (int b = 0; b < 4; ++b) {
    float s[32];
    tc::tmem_ld32(sb + 32 * b, s);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const Scales sc = scales[2 * b + h];
      // positive, so that a masked logit stays -inf under it
      const float up1 = fmaxf(sc.x * to_log2, 1.1754944e-38f), down1 = sc.y + low;
      const float2 up = make_float2(up1, up1), down = make_float2(down1, down1);
      float block_top = -INFINITY;
      float2 sum = make_float2(0.f, 0.f);
#pragma unroll
      for (int e = 16 * h; e < 16 * h + 16; e += 2) {
        if (kEdge) {
          if (32 * b + e >= left) s[e] = -INFINITY;
          if (32 * b + e + 1 >= left) s[e + 1] = -INFINITY;
        }
        block_top = tc::fmax3(block_top, s[e], s[e + 1]);
        const float2 y = tc::ffma2(make_float2(s[e], s[e + 1]), up, down);
        const float2 w = make_float2(tc::ex2(y.x), tc::ex2(y.y));
        sum = tc::fadd2(sum, w);
        p[b][e / 2] = h2u(__float22half2_rn(w));
      }
      top = fmaxf(top, fmaf(block_top, up1, sc.y));
      *add = fmaf(sum.x + sum.y, sc.z, *add);
    }
  }
  return top;
}

// Their sum without v alone, for value scales that lie far apart: a block whose weights are all far below the reference counts by
// its logits, others as in weigh.
__device__ __forceinline__ float weigh_apart(uint32_t sb, const Scales* scales, float to_log2, float low, int left) {
  float add = 0.f;
#pragma unroll 1
  for (int b = 0; b < kBlocks; ++b, left -= kBlockTokens) {
    float s[kBlockTokens];
    tc::tmem_ld16(sb + kBlockTokens * b, s);
    const Scales sc = scales[b];
    const float up1 = fmaxf(sc.x * to_log2, 1.1754944e-38f);
    float block_top = -INFINITY;
#pragma unroll
    for (int e = 0; e < kBlockTokens; ++e) {
      if (e >= left) s[e] = -INFINITY;
      block_top = fmaxf(block_top, s[e]);
    }
    const bool far = fmaf(block_top, up1, sc.y) < -low - kFarBelow;
    const float down1 = (far ? kLift : sc.y) + low;
    float2 sum = make_float2(0.f, 0.f);
#pragma unroll
    for (int e = 0; e < kBlockTokens; e += 2) {
      const float2 y = tc::ffma2(make_float2(s[e], s[e + 1]), make_float2(up1, up1), make_float2(down1, down1));
      sum = tc::fadd2(sum, make_float2(tc::ex2(y.x), tc::ex2(y.y)));
    }
    add = fmaf(sum.x + sum.y, far ? kUnlift : sc.z, add);
  }
  return add;
}

template <int NG>
__global__ void __launch_bounds__(kThreads, 1) fp8_attn_tc(AttnArgs a) {
  using Z = Sizes<NG>;
  constexpr int D = Z::D;
  extern __shared__ uint8_t dynamic[];
  __shared__ Bars bars;
  __shared__ uint32_t tmem_slot;
  __shared__ int seen_most, seen_least, poison[D], poison_any, abort_flag;
  __shared__ Scales scales[4][kBlocks];  // of four key tiles
  let_join_start();
  // Blocks with two column tiles come first and those with one, which take half of the time, last.
  Item it;
  if (!tc_item(a, &it)) return;
  // One column tile: A takes its even key tiles and B its odd ones, joined at the end.
  const bool split = it.cb * kTcCols + kTileCols >= it.n * a.kv.G;
  const int chunk = split ? a.last_chunk : a.chunk;
  const bool partial = (split ? a.last_chunks : a.chunks) > 1;
  uint8_t* base = dynamic + (1024 - (tc::smem_u32(dynamic) & 1023u)) % 1024;
  uint8_t *qt = base, *kt = qt + 2 * Z::kTile, *vt = kt + 2 * Z::kTile, *raw = vt + 2 * Z::kValues;
  float2* of_b = reinterpret_cast<float2*>(qt + Z::kTile);  // split: B's (reference, sum), where there is no second query tile
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid / 32, 0), lane = tid % 32;
  volatile int* abort = &abort_flag;

  if (tid == 0) {
    for (int s = 0; s < kRing; ++s) {
      tc::mbar_init(&bars.raw_full[s], 1);
      tc::mbar_init(&bars.raw_free[s], kUnpackWarps);
    }
    for (int s = 0; s < 2; ++s) {
      tc::mbar_init(&bars.k_full[s], kLoads);
      tc::mbar_init(&bars.v_full[s], kLoads);
      tc::mbar_init(&bars.k_free[s], 1);
      tc::mbar_init(&bars.v_free[s], 1);
      tc::mbar_init(&bars.s_full[s], 1);
      tc::mbar_init(&bars.p_full[s], 4);
      tc::mbar_init(&bars.o_full[s], 1);
    }
    tc::mbar_init(&bars.q_full, 8);
    tc::mbar_init(&bars.joined, 4);
    tc::mbar_init(&bars.drained, 1);
    tc::fence_barrier_init();
    seen_most = 0;
    seen_least = poison_any = INT32_MAX;
    abort_flag = 0;
  }
  if (tid < D) poison[tid] = INT32_MAX;
  if (warp == kMmaWarp) tc::tmem_alloc(&tmem_slot, 512);
  __syncthreads();
  // keys that a column sees; columns past the last see all (their result is dropped)
  const int at = tid - 32 * kSoftWarp, col = it.cb * kTcCols + (split ? at & (kTileCols - 1) : at);
  const bool live = at >= 0 && col < it.n * a.kv.G;
  const int lim = live ? limit_of(a, it, col) : INT32_MAX;
  if (warp >= kSoftWarp) {
    const int hi = __reduce_max_sync(0xffffffffu, live ? lim : 0), lo = __reduce_min_sync(0xffffffffu, lim);
    if (lane == 0) {
      atomicMax(&seen_most, hi);
      atomicMin(&seen_least, lo);
    }
  }
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  const uint32_t tmem = tmem_slot;
  const int least = seen_least, k0 = it.chunk * chunk, k1 = min(k0 + chunk, seen_most);
  const int tiles = k1 > k0 ? (k1 - k0 + kKeys - 1) / kKeys : 0;

  // 128 registers a thread at launch: 2 x 88 + 2 x 168 per four warpgroups
  if (warp < kSoftWarp) {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 88;" ::: "memory");
  if (warp == kLoadWarp) {
    // ---------------------------------------------------------------- copies
    // A load: two blocks, a lane each. Pages of the next 32 blocks are looked up ahead, a block a lane.
    auto pages_from = [&](int block) {
      const int64_t j = int64_t(k0) + int64_t(block + lane) * kBlockTokens;
      return j < k1 ? page_entry(a, it.r, int(j)) : 0;
    };
    const int loads = kLoads * tiles;
    const uint32_t dst = tc::smem_u32(raw) + lane * Z::kBox;
    int issued = 0, pages = pages_from(0), later = 0;
    bool ok = true;
    for (; issued < loads; ++issued) {
      const int in = issued & 15, slot = issued % kRing, j = k0 + issued * kLoadKeys + lane * kBlockTokens;
      const int id = __shfl_sync(0xffffffffu, pages, 2 * in + (lane & 1));
      if (in == 2) later = pages_from(2 * (issued - in) + 32);
      if (in == 15) pages = later;
      const bool mine = lane < 2 && j < k1;
      const uint8_t* src = fp8_block(a.kv, it.l, it.g, mine ? page_in_pool(a, id) : 0, mine ? j : 0);
      if (issued >= kRing && !(ok = wait_warp(&bars.raw_free[slot], (issued / kRing - 1) & 1, abort))) break;
#ifdef CONDUIT_TEST_HOOKS
      if (issued == a.withhold) continue;  // neither copies nor an arrive: the waits for this load run out
#endif
      const uint32_t copies = __popc(__ballot_sync(0xffffffffu, mine));
      if (lane == 0) tc::mbar_arrive_expect_tx(&bars.raw_full[slot], copies * Z::kBox);
      __syncwarp();
      if (mine) bulk_load(dst + slot * Z::kRaw, src, Z::kBox, &bars.raw_full[slot]);
    }
    if (!ok && lane == 0) give_up(a, abort, CONDUIT_SITE_MMA);
    for (int n = max(0, issued - kRing); n < issued; ++n)  // the last copies (all have landed unless a role gave up)
      tc::mbar_wait(&bars.raw_full[n % kRing], (n / kRing) & 1);
  } else if (warp != kMmaWarp) {
    // ------------------------------------------------------------ conversion
    // A unit is a load's keys, then its values; six warps take them in turn.
    // Every warp sees every load land and says so before its slot is used again, also where
    // others convert it: none can take a phase of a slot for the one two before it.
    int unit = warp - kUnpackWarp;  // the next one of this warp
    for (int load = 0; load < kLoads * tiles; ++load) {
      const int t = load / kLoads, v = unit & 1, stage = t & 1, slot = load % kRing;
      bool ok = wait_warp(&bars.raw_full[slot], (load / kRing) & 1, abort);
      const bool mine = unit < 2 * load + 2;
      const int kb = k0 + load * kLoadKeys, tile_key = (load % kLoads) * kLoadKeys;
      // Keys: 16 dims of a token; eight lanes a tile of 8 tokens. Values: 16 tokens of a dim.
      const uint8_t* box = raw + slot * Z::kRaw;
      const uint8_t* from = box + (v ? 16 * D : 0) + lane * 16;
      const bool edge = v && kb + kLoadKeys > least;  // values that some column does not see
      // A buffer is free once its last tile but one has been used. (When a load lands, every warp has
      // stored all units of the tile two before it, and so has passed the wait for the use before
      // that: this wait cannot mistake its phase either.)
      auto buffer_free = [&] {
        return t < 2 || wait_warp(v ? &bars.v_free[stage] : &bars.k_free[stage], ((t >> 1) - 1) & 1, abort);
      };
      auto put_values = [&](const uint4& w, int i) {
        const int dim = (i % NG) * 32 + lane, block = tile_key / kBlockTokens + i / NG;
        uint4 first, second;
        widen<true>(w, &first, &second);
        uint8_t* to = vt + stage * Z::kValues + (block >> 2) * (D * 128);
        *reinterpret_cast<uint4*>(to + tc::sw128_offset(dim, 2 * block & 7)) = first;
        *reinterpret_cast<uint4*>(to + tc::sw128_offset(dim, (2 * block + 1) & 7)) = second;
      };
      if (ok && mine && edge) {
        // apart from the usual loop, which its code would stretch
        ok = buffer_free();
#pragma unroll 1
        for (int i = 0; ok && i < 2 * NG; ++i) {
          const uint4 w = *reinterpret_cast<const uint4*>(from + (i / NG) * Z::kBox + (i % NG) * 512);
          put_values(guard(w, (i % NG) * 32 + lane, kb + (i / NG) * kBlockTokens, k1, least, poison, &poison_any), i);
        }
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&bars.raw_free[slot]);
      } else if (ok) {
        // into registers first, so that the next copy into the slot starts while this one is converted
        uint4 x[2 * NG];
        float2 sc = make_float2(1.f, 1.f);
        if (mine) {
#pragma unroll
          for (int i = 0; i < 2 * NG; ++i)
            x[i] = *reinterpret_cast<const uint4*>(from + (i / NG) * Z::kBox + (i % NG) * 512);
          if (!v && lane < 2 && kb + lane * kBlockTokens < k1)
            sc = *reinterpret_cast<const float2*>(box + lane * Z::kBox + 32 * D);
        }
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&bars.raw_free[slot]);
        if (mine && (ok = buffer_free())) {
          if (v) {
#pragma unroll
            for (int i = 0; i < 2 * NG; ++i) put_values(x[i], i);
          } else {
            if (lane < 2) {
              const int e = exponent_of(sc.y);
              scales[t & 3][tile_key / kBlockTokens + lane] = make_float4(sc.x, float(e), power_of_two(-e), 0.f);
            }
            // piece 32 i + lane of a block: chunks of 16 dims within halves of 8 tokens
#pragma unroll
            for (int i = 0; i < 2 * NG; ++i) {
              const int piece = (i % NG) * 32 + lane, half = piece / (D / 2), ch = piece % (D / 2) / 8;
              const int token = tile_key + (i / NG) * kBlockTokens + 8 * half + (piece & 7);
              uint4 first, second;
              widen<false>(x[i], &first, &second);
              uint8_t* to = kt + stage * Z::kTile + (ch >> 2) * kBlock;
              *reinterpret_cast<uint4*>(to + tc::sw128_offset(token, 2 * ch & 7)) = first;
              *reinterpret_cast<uint4*>(to + tc::sw128_offset(token, (2 * ch + 1) & 7)) = second;
            }
          }
        }
      }
      if (!ok) {
        if (lane == 0) give_up(a, abort, CONDUIT_SITE_LOAD);
        break;
      }
      if (!mine) continue;
      unit += kUnpackWarps;
      tc::fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(v ? &bars.v_full[stage] : &bars.k_full[stage]);
    }
  } else if (warp == kMmaWarp) {
    // ------------------------------------------------------------------ MMAs
    // the whole warp walks the schedule on values from one lane, so that the operands live in
    // uniform registers
    const uint32_t leader = lane == 0;
    const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
    const int all = __shfl_sync(0xffffffffu, tiles, 0);
    const bool halves = __shfl_sync(0xffffffffu, int(split), 0) != 0;
    const uint32_t q_at = __shfl_sync(0xffffffffu, tc::smem_u32(qt), 0);
    const uint32_t k_at = q_at + 2 * Z::kTile, v_at = k_at + 2 * Z::kTile;
    constexpr uint32_t idesc_s = idesc_f16(kTileCols, kKeys), idesc_o = idesc_f16(kTileCols, D);
    const uint64_t dq = tc::desc_sw128(q_at);
    // S_x = Q K^T for the key tile `tile`; a tile's keys and values are waited for by the first
    // stream that reads it and freed by the last.
    bool ok = true;
    auto score = [&](int x, int tile) {
      const int stage = tile & 1;
      if (halves || x == 0) {
        if (!(ok = wait_warp(&bars.k_full[stage], (tile >> 1) & 1, abort))) return;
        tc::tc_fence_after();
      }
      const uint64_t dk = tc::desc_sw128(k_at + stage * Z::kTile);
      const uint64_t dx = dq + (halves ? 0 : (x * Z::kTile) >> 4);
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk) {
        const uint32_t off = ((kk >> 2) * kBlock + (kk & 3) * 32) >> 4;
        tc::mma_bf16_if(leader, tm + x * kSCols, dx + off, dk + off, idesc_s, kk > 0);
      }
      tc::mma_commit_if(leader, &bars.s_full[x]);
      if (halves || x == 1) tc::mma_commit_if(leader, &bars.k_free[stage]);
    };
    const int count[2] = {halves ? (all + 1) / 2 : all, halves ? all / 2 : all};
    if (all > 0 && (ok = wait_warp(&bars.q_full, 0, abort))) {
      score(0, 0);
      if (ok && count[1] > 0) score(1, halves ? 1 : 0);
    }
    for (int t = 0; ok && t < count[0]; ++t) {
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        if (t >= count[x]) break;
        const int tile = halves ? 2 * t + x : t, stage = tile & 1;
        if ((halves || x == 0) && !(ok = wait_warp(&bars.v_full[stage], (tile >> 1) & 1, abort))) break;
        if (!(ok = wait_warp(&bars.p_full[x], t & 1, abort))) break;
        tc::tc_fence_after();
        const uint64_t dv = tc::desc_sw128(v_at + stage * Z::kValues);
#pragma unroll
        for (int kk = 0; kk < kKeys / 16; ++kk)
          tc::mma_bf16_ts_if(leader, tm + kOCol + x * kSCols, tm + x * kSCols + kPCol + kk * 8,
                             dv + (((kk >> 2) * (D * 128) + (kk & 3) * 32) >> 4), idesc_o, t > 0 || kk > 0);
        if (halves || x == 1) tc::mma_commit_if(leader, &bars.v_free[stage]);
        if (t + 1 < count[x])
          score(x, halves ? tile + 2 : tile + 1);
        else
          tc::mma_commit_if(leader, &bars.o_full[x]);
        if (!ok) break;
      }
    }
    if (!ok && lane == 0) give_up(a, abort, CONDUIT_SITE_MMA);
    tc::mma_commit_if(leader, &bars.drained);  // every MMA issued above is done once this arrives
    tc::mbar_wait(&bars.drained, 0);
    __syncwarp();
  }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 168;" ::: "memory");
    // --------------------------------------------------------------- softmax
    const int x = (warp - kSoftWarp) >> 2;
    const bool owner = !split || x == 0;  // of the column: its query and its output row
    uint8_t* tile = qt + (split ? 0 : x) * Z::kTile;  // the queries, and at the end the rows on their way out
    const int row0 = (warp & 3) * 32;   // this warp's columns of the tile
    // Where this thread's column lies; a row moves by sixteen lanes together, which ask its lane.
    const int own_i = live ? col / a.kv.G : 0, own_h = it.g * a.kv.G + (live ? col % a.kv.G : 0);
    const uint32_t rows = __ballot_sync(0xffffffffu, live);
    const int part = lane & 15, side = lane >> 4;
    float to_log2;
    {
      // Queries into the swizzled tile, two columns at a time, each scaled by a power of two so that
      // its largest lies in [2^15, 2^16) (or below, if that takes more than 2^109).
      constexpr int kUse = D / 8;  // lanes with eight dims of a column
      const bool wide = ((reinterpret_cast<uintptr_t>(a.q.p) | uint64_t(2 * (a.q.ls | a.q.rs | a.q.hs))) & 15u) == 0;
      const int64_t own = it.l * a.q.ls + int64_t(it.t0 + own_i) * a.q.rs + own_h * a.q.hs;
      uint4 v[16];
      // The usual loads stand apart: instructions that are not in a row come from memory one line
      // after the other once the keys have passed through L2 (loads of both kinds side by side: 13 000
      // cycles until the last was issued).
      if (wide) {
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          const int r = 2 * k + side;
          const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(a.q.p) + __shfl_sync(0xffffffffu, own, r) + 8 * part;
          v[k] = make_uint4(0, 0, 0, 0);
          if (part < kUse && (rows >> r & 1u)) v[k] = *reinterpret_cast<const uint4*>(src);
        }
      } else {
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          const int r = 2 * k + side;
          const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(a.q.p) + __shfl_sync(0xffffffffu, own, r) + 8 * part;
          __nv_bfloat16 e8[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) e8[e] = part < kUse && (rows >> r & 1u) ? src[e] : __nv_bfloat16(0.f);
          v[k] = *reinterpret_cast<uint4*>(e8);
        }
      }
      int own_shift = 0;
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        const uint32_t w[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
        // the largest |q|; a NaN counts where the row has nothing else
        uint32_t top = bf16_max2(bf16_max2(w[0] & 0x7FFF7FFFu, w[1] & 0x7FFF7FFFu), bf16_max2(w[2] & 0x7FFF7FFFu, w[3] & 0x7FFF7FFFu));
#pragma unroll
        for (int o = 1; o < 16; o <<= 1) top = bf16_max2(top, __shfl_xor_sync(0xffffffffu, top, o));
        top = max(top & 0xFFFFu, top >> 16);
        int shift = max(int(top >> 7) - 127 - 15, -109);
        if (top >= 0x7F80u || top == 0) shift = 0;
        const int got = __shfl_sync(0xffffffffu, shift, (lane & 1) << 4);
        if (lane >> 1 == k) own_shift = got;
        const float up = __uint_as_float(uint32_t(127 - shift) << 23);
        float f[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          f[2 * e] = __uint_as_float(w[e] << 16) * up;
          f[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u) * up;
        }
        uint4 y;
        y.x = h2u(__floats2half2_rn(f[0], f[1]));
        y.y = h2u(__floats2half2_rn(f[2], f[3]));
        y.z = h2u(__floats2half2_rn(f[4], f[5]));
        y.w = h2u(__floats2half2_rn(f[6], f[7]));
        if (part < kUse && owner)
          *reinterpret_cast<uint4*>(tile + (part >> 3) * kBlock + tc::sw128_offset(row0 + 2 * k + side, part & 7)) = y;
      }
      to_log2 = a.scale * kLog2e * __uint_as_float(uint32_t(127 + own_shift) << 23);
      tc::fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(&bars.q_full);
    }
    const uint32_t lanes = uint32_t((warp & 3) * 32) << 16;
    const uint32_t sb = tmem + lanes + x * kSCols, ob = tmem + lanes + kOCol + x * kSCols;
    float ref = -INFINITY;
    float sum = 0.f;
    bool ok = true;
    const int count = split ? (tiles + 1 - x) / 2 : tiles;
    int t = 0;
    // One key tile after the other. kFar: value scales may lie anywhere; else it ends at the first tile that has one above
    // kNear. Two loops: in one, what the second needs beside the first's weights cost the kernel 3 % of its time, so 1.5 %.
    auto walk = [&](auto far) {
      constexpr bool kFar = decltype(far)::value;
      for (; t < count; ++t) {
        if (!(ok = wait_warp(&bars.s_full[x], t & 1, abort))) break;
        tc::tc_fence_after();
        const int tile_id = split ? 2 * t + x : t, kb = k0 + tile_id * kKeys;
        const Scales* sc = scales[tile_id & 3];
        if (!kFar && __any_sync(0xffffffffu, sc[lane & (kBlocks - 1)].y > kNear)) break;
        const int left = lim - kb;  // keys of the tile that the column sees
        const bool edge = kb + kKeys > least;
        uint32_t p[4][16];
        float add;
        for (int pass = 0;; ++pass) {
          const float low = ref == -INFINITY ? 0.f : -ref;
          const float top = kFar || edge ? weigh<true>(sb, sc, to_log2, low, left, p, &add)
                                 : weigh<false>(sb, sc, to_log2, low, left, p, &add);
          if (pass || !__any_sync(0xffffffffu, top > ref + kMostWeight)) break;
          // the reference moves: what was summed so far is scaled, and the weights are taken again
          const float moved = fmaxf(ref, top - kBias), by = ref - moved, corr = moved == -INFINITY ? 1.f : tc::ex2(by);
          ref = moved;
          sum = kFar ? scaled_down(sum, by, corr) : sum * corr;
          if (t > 0) {
#pragma unroll 1
            for (int b = 0; b < D / 32; ++b) {
              float o[32];
              tc::tmem_ld32(ob + 32 * b, o);
#pragma unroll
              for (int e = 0; e < 32; ++e) o[e] *= corr;
              tc::tmem_st32(ob + 32 * b, o);
            }
          }
        }
        if (kFar) add = weigh_apart(sb, sc, to_log2, ref == -INFINITY ? 0.f : -ref, left);
        sum += add;
#pragma unroll
        for (int b = 0; b < 4; ++b) tc::tmem_st16_nowait(sb + kPCol + 16 * b, p[b]);
        tc::tmem_wait_st();
        tc::tc_fence_before();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&bars.p_full[x]);
      }
    };
    walk(std::false_type{});
    if (ok && t < count) walk(std::true_type{});
    // without keys there is nothing to wait for but the other warps' queries, over which the rows go out
    if (ok) ok = count > 0 ? wait_warp(&bars.o_full[x], 0, abort) : wait_warp(&bars.q_full, 0, abort);
    ref += kBias;
    float total = sum * kUnbias, own_w = kUnbias, b_w = 0.f;
    bool join = false;
    if (split) {
      if (x == 1) {
        of_b[at & (kTileCols - 1)] = make_float2(ref, total);
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&bars.joined);
      } else if (ok && (ok = wait_warp(&bars.joined, 0, abort)) && tiles > 1) {
        ok = wait_warp(&bars.o_full[1], 0, abort);
        join = true;
        const float2 b = of_b[at];
        const float top = fmaxf(ref, b.x), base = top == -INFINITY ? 0.f : top;
        const float wa = tc::ex2(ref - base), wb = tc::ex2(b.x - base);
        if (fminf(ref, b.x) - base < kLeastFactor)
          total = add_scaled(scaled_down(total, ref - base, wa), b.y, b.x - base, wb);
        else
          total = wa * total + wb * b.y;
        own_w = wa * kUnbias;
        b_w = wb * kUnbias;
        ref = top;
      }
    }
    if (!ok && lane == 0) give_up(a, abort, CONDUIT_SITE_FINAL);
    tc::tc_fence_after();
    if (owner) {
    // this column among those with partial results
    const int64_t part_col = a.chunks > 1 ? (int64_t(it.l) * a.s.T + it.t0 + own_i) * a.kv.Hq + own_h
                                          : ((int64_t(it.l) * a.s.R + it.r) * a.kv.Hkv + it.g) * kTileCols + row0 + lane;
    if (live) {
      if (partial)
        a.part_ml[it.chunk * a.part_cols + part_col] = make_float2(ref, total);
      else
        store_stats(a, it, col, ref, total, true);
    }
    const float inv = partial ? 1.f : total == 0.f ? 0.f : 1.f / total;
    own_w *= inv;
    b_w *= inv;
    // The rows go out through the query tile (every product that read it is done), so that
    // neighbouring lanes write neighbouring dims.
    const bool by_16 = ((reinterpret_cast<uintptr_t>(a.out.p) | uint64_t(2 * (a.out.ls | a.out.rs | a.out.hs))) & 15u) == 0;
    const int row = row0 + lane;
    // 16-byte chunk c of a row, in a place that spreads the rows over the banks
    constexpr int kRowBytes = D == 64 ? 128 : 256;  // 128 rows fit the tile
    auto chunk_at = [&](int r, int c) { return tile + r * kRowBytes + ((c ^ (r & 7)) << 4); };
    const int64_t own = partial ? (it.chunk * a.part_cols + part_col) * D
                                : it.l * a.out.ls + int64_t(it.t0 + own_i) * a.out.rs + own_h * a.out.hs;
    const bool tainted = __any_sync(0xffffffffu, poison_any < lim);  // a NaN value reaches the columns that see it
#pragma unroll
    for (int b = 0; b < D / 32; ++b) {
      float o[32];
      if (ok && count > 0) {
        tc::tmem_ld32(ob + 32 * b, o);
#pragma unroll
        for (int e = 0; e < 32; ++e) o[e] *= own_w;
      } else {
#pragma unroll
        for (int e = 0; e < 32; ++e) o[e] = 0.f;
      }
      if (ok && join) {
        float other[32];
        tc::tmem_ld32(ob + kSCols + 32 * b, other);
#pragma unroll
        for (int e = 0; e < 32; ++e) o[e] = fmaf(other[e], b_w, o[e]);
      }
      if (tainted) {
#pragma unroll
        for (int e = 0; e < 32; ++e)
          if (poison[32 * b + e] < lim) o[e] = NAN;
      }
      if (!partial) {
#pragma unroll
        for (int n = 0; n < 4; ++n) {
          __nv_bfloat162 z[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) z[e] = __floats2bfloat162_rn(o[8 * n + 2 * e], o[8 * n + 2 * e + 1]);
          *reinterpret_cast<uint4*>(chunk_at(row, 4 * b + n)) = *reinterpret_cast<const uint4*>(z);
        }
        continue;
      }
#pragma unroll
      for (int n = 0; n < 8; ++n)
        *reinterpret_cast<float4*>(chunk_at(row, n)) = make_float4(o[4 * n], o[4 * n + 1], o[4 * n + 2], o[4 * n + 3]);
      __syncwarp();
#pragma unroll 1
      for (int k = 0; k < 8; ++k) {  // four rows at a time, eight lanes a row
        const int r = 4 * k + (lane >> 3), n = lane & 7;
        float* to = a.part_o + __shfl_sync(0xffffffffu, own, r) + 32 * b + 4 * n;
        if (rows >> r & 1u) *reinterpret_cast<float4*>(to) = *reinterpret_cast<const float4*>(chunk_at(row0 + r, n));
      }
      __syncwarp();
    }
    if (!partial) {
      __syncwarp();
#pragma unroll 4
      for (int k = 0; k < 16; ++k) {
        const int r = 2 * k + side;
        __nv_bfloat16* to = static_cast<__nv_bfloat16*>(a.out.p) + __shfl_sync(0xffffffffu, own, r) + 8 * part;
        if ((rows >> r & 1u) && part < D / 8) {
          const uint4 y = *reinterpret_cast<const uint4*>(chunk_at(row0 + r, part));
          if (by_16) {
            *reinterpret_cast<uint4*>(to) = y;
          } else {
            const __nv_bfloat16* e8 = reinterpret_cast<const __nv_bfloat16*>(&y);
#pragma unroll
            for (int e = 0; e < 8; ++e) to[e] = e8[e];
          }
        }
      }
    }
    }
    tc::tc_fence_before();
  }
  __syncthreads();
  if (warp == kMmaWarp) {
    tc::tc_fence_after();
    tc::tmem_dealloc(tmem, 512);
  }
}

template <int NG>
cudaError_t launch(const AttnArgs& a, int64_t items, cudaStream_t stream) {
  constexpr uint32_t kSmem = Sizes<NG>::kSmem;
  cudaError_t err = cudaFuncSetAttribute(fp8_attn_tc<NG>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
  if (err) return err;
  fp8_attn_tc<NG><<<unsigned(items), kThreads, kSmem, stream>>>(a);
  count_launches(1);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_fp8_attn_tc(const AttnArgs& a, int64_t items, cudaStream_t stream) {
  switch (a.kv.d) {
    case 64: return launch<2>(a, items, stream);
    case 96: return launch<3>(a, items, stream);
    default: return launch<4>(a, items, stream);
  }
}

}  // namespace conduit
