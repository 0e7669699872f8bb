// Attention over the 4-bit cache for many rows (query prefixes, recomputed rows): tcgen05.
//
// Mathematics: as in packed_attn_mma.cu, with keys and values as fp16 m + s c (2^-11
// relative), the query scaled by a power of two per row into fp16, weights rounded to
// fp16; logits, statistics and outputs in fp32 (tensor memory).
//
// Shape. A CTA holds two tiles of 128 columns (A and B: rows of the call times query
// heads of one KV head) and walks over the keys in tiles of 128. Each key tile is
// unpacked once into shared memory for both. Roles (512 threads):
//   warp 0            MMAs: P_x(t) V(t), then S_x(t + 1), for x = A, B; one lane issues.
//                     The first warp, because the schedulers favour it: as warp 13 it took
//                     120 cycles to issue an MMA of 64
//   warp 1            bulk copies of pages into a small ring, half a key tile at a time
//   warps 2-7         unpack: four lanes a token, a word of eight codes at a time
//   warps 8-11, 12-15 softmax of A and of B: a thread owns a column and all 128 keys
// One column tile's softmax runs beside the other's MMAs. MMAs of one thread complete in
// order, so S_x(t + 1) may overwrite P_x(t), and S_x(t + 1) says that P_x(t) V(t) is done.
// The dims of keys and queries are permuted alike (a word's nibbles come out as dims
// e, e + 4), those of the values as they unpack (two groups side by side); the output rows
// are put back in order. TMEM: S_A, S_B at columns [0, 256) with P over their upper halves,
// O_A, O_B at [256, 512).
//
// Bound: the chain S, softmax, P V, next S of each column tile, beside the other's. A key tile
// of two column tiles takes 3 600 cycles: 2 960 of MMAs (95 each, held up by the operands in
// shared memory), 1 200-1 500 of softmax, 1 000 for each 32 tokens of keys or values that a warp
// unpacks; with keys in two parts 6 700. A CTA another 20 000-28 000 (item and limits 2 600, queries
// 8 000-13 000, first logits 1 400-2 000, rows out 6 000-11 000, the next CTA's launch 2 000). Measured: 32-128 rows of 16 requests over 8 192 keys, two layers of
// 28 x 4 heads of 128, 325 us (0.98 PFLOP/s); 96 dims 339, 64 dims 250. Causal prompts, one layer: 8 192
// tokens 552, four of 4 096 tokens 831.
#include <type_traits>

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
constexpr int kHalf = kKeys / 2;              // keys of a load
constexpr int kRing = 3;                      // loads under way

template <int NG>
struct Sizes {
  static constexpr int D = 32 * NG;
  static constexpr uint32_t kTile = (D + 63) / 64 * kBlock;  // a query, key or value tile
  static constexpr uint32_t kRaw = kHalf * (D + D / 4);      // packed keys and values of half a tile
  static constexpr uint32_t kSmem = 1024 + 6 * kTile + kRing * kRaw;
};

struct Bars {
  uint64_t raw_full[kRing], raw_free[kRing];
  uint64_t k_full[2], k_free[2], v_full[2], v_free[2];
  uint64_t q_full, s_full[2], p_full[2], o_full[2], joined, drained;
};

// The eight values of a word: nibbles (0, 4), (1, 5), (2, 6), (3, 7).
__device__ __forceinline__ uint4 values8(uint32_t w, __half2 s, __half2 m) {
  const uint32_t w8 = w >> 8;
  return make_uint4(h2u(__hfma2(s, u2h(codes_lo(w)), m)), h2u(__hfma2(s, u2h(codes_hi(w)), m)),
                    h2u(__hfma2(s, u2h(codes_lo(w8)), m)), h2u(__hfma2(s, u2h(codes_hi(w8)), m)));
}
// The larger of two pairs of non-negative bf16, a NaN losing to a number.
__device__ __forceinline__ uint32_t bf16_max2(uint32_t a, uint32_t b) {
  const __nv_bfloat162 y = __hmax2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&y);
}
// kind::f16 with fp16 operands, fp32 sums; B key-major or dim-major.
constexpr uint32_t idesc_f16(int m, int n, bool b_mn_major) {
  return (1u << 4) | (uint32_t(b_mn_major) << 16) | (uint32_t(n >> 3) << 17) | (uint32_t(m >> 4) << 24);
}

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

// One lane's share of a packed token: NG words of codes, the parameters of its groups. Keys, and
// values of 64 and 128 dims: words NG c on; values of 96 dims: words c, c + 4, c + 8.
template <int NG>
struct Packed {
  uint32_t w[NG], p[NG];
};
template <int NG, bool kValues>
__device__ __forceinline__ Packed<NG> take(const uint8_t* codes, const uint8_t* params, int token, int c) {
  constexpr int D = 32 * NG;
  Packed<NG> x;
  const uint8_t* row = codes + token * (D / 2);
  if constexpr (kValues && NG == 3) {
#pragma unroll
    for (int n = 0; n < NG; ++n) x.w[n] = *reinterpret_cast<const uint32_t*>(row + 4 * (4 * n + c));
  } else {
    load_words<NG>(row + c * (D / 8), x.w);
  }
  load_words<NG>(params + token * (D / 8), x.p);
  return x;
}

// Keys: a word's values in chunk 4 g + c.
template <int NG>
__device__ __forceinline__ void unpack_keys(uint8_t* tile, const Packed<NG>& x, int token, int c) {
  const uint32_t(&w)[NG] = x.w;
  const uint32_t(&p)[NG] = x.p;
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    const int ch = 4 * g + c;
    *reinterpret_cast<uint4*>(tile + (ch >> 3) * kBlock + tc::sw128_offset(token, ch & 7)) =
        values8(w[g], u2h(__byte_perm(p[g], p[g], 0x1010)), u2h(__byte_perm(p[g], p[g], 0x3232)));
  }
}

// The same in two parts: hi is the value in fp16, lo what is missing from it.
template <int NG>
__device__ __forceinline__ void unpack_keys_exact(uint8_t* hi, uint8_t* lo, const Packed<NG>& x, int token, int c) {
  const uint32_t(&w)[NG] = x.w;
  const uint32_t(&p)[NG] = x.p;
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    const float2 sm = __half22float2(u2h(p[g])), s2 = make_float2(sm.x, sm.x), m2 = make_float2(sm.y, sm.y);
    const uint32_t w8 = w[g] >> 8, u[4] = {codes_lo(w[g]), codes_hi(w[g]), codes_lo(w8), codes_hi(w8)};
    uint32_t h[4], l[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float2 x = tc::ffma2(s2, __half22float2(u2h(u[e])), m2);
      const __half2 top = __float22half2_rn(x);
      h[e] = h2u(top);
      l[e] = h2u(__float22half2_rn(tc::ffma2(__half22float2(top), make_float2(-1.f, -1.f), x)));
    }
    const int ch = 4 * g + c;
    const uint32_t at = (ch >> 3) * kBlock + tc::sw128_offset(token, ch & 7);
    *reinterpret_cast<uint4*>(hi + at) = make_uint4(h[0], h[1], h[2], h[3]);
    *reinterpret_cast<uint4*>(lo + at) = make_uint4(l[0], l[1], l[2], l[3]);
  }
}

// Values. kEdge: the tile holds tokens that some column does not see. Their weight there is 0,
// and 0 times NaN must not be: a parameter pair that is not finite becomes 0 and its first
// token is noted for the group.
template <int NG, bool kEdge>
__device__ __forceinline__ void unpack_values(uint8_t* tile, Packed<NG> x, int token, int c, int kb, int k1, int least,
                                              int* poison) {
  const uint32_t(&w)[NG] = x.w;
  uint32_t(&p)[NG] = x.p;
  if (kEdge) {
    const int j = kb + token;
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      if (j >= least && j < k1 && !finite_pair(p[g])) atomicMin(&poison[g], j), p[g] = 0;
      if (j >= k1) p[g] = 0;
    }
  }
#pragma unroll
  for (int n = 0; n < NG; ++n) {
    // word ch of the row: the groups g0 and g1 side by side
    int ch = NG * c + n;
    uint32_t word = w[n], p0 = p[2 * n % NG], p1 = p[(2 * n + 1) % NG];
    if constexpr (NG == 4) {  // the lanes of a token in different banks
      ch = 4 * c + (n ^ (c & 2));
      word = c & 2 ? w[n ^ 2] : w[n];
    } else if constexpr (NG == 3) {
      ch = 4 * n + c;
      const int g0 = 2 * ch % 3, g1 = (2 * ch + 1) % 3;
      p0 = g0 == 0 ? p[0] : g0 == 1 ? p[1] : p[2];
      p1 = g1 == 0 ? p[0] : g1 == 1 ? p[1] : p[2];
    }
    *reinterpret_cast<uint4*>(tile + (ch >> 3) * kBlock + tc::sw128_offset(token, ch & 7)) =
        values8(word, u2h(__byte_perm(p0, p1, 0x5410)), u2h(__byte_perm(p0, p1, 0x7632)));
  }
}

// Weights 2^(s up + down) of the 128 logits at sb: packed into p, summed into add; returns the
// largest logit (unscaled). kEdge: only the first `left` are seen.
template <bool kEdge>
__device__ __forceinline__ float weigh(uint32_t sb, float2 up, float2 down, int left, uint32_t (&p)[4][16], float2* add) {
  float top = -INFINITY;
  *add = make_float2(0.f, 0.f);
#pragma unroll
  for (int b = 0; b < 4; ++b) {
    float s[32];
    tc::tmem_ld32(sb + 32 * b, s);
#pragma unroll
    for (int e = 0; e < 32; e += 2) {
      if (kEdge) {
        if (32 * b + e >= left) s[e] = -INFINITY;
        if (32 * b + e + 1 >= left) s[e + 1] = -INFINITY;
      }
      top = tc::fmax3(top, s[e], s[e + 1]);
      const float2 y = tc::ffma2(make_float2(s[e], s[e + 1]), up, down);
      const float2 w = make_float2(tc::ex2(y.x), tc::ex2(y.y));
      *add = tc::fadd2(*add, w);
      p[b][e / 2] = h2u(__float22half2_rn(w));
    }
  }
  return top;
}

template <int NG>
__global__ void __launch_bounds__(kThreads, 1) packed_attn_tc(AttnArgs a) {
  using Z = Sizes<NG>;
  constexpr int D = Z::D;
  extern __shared__ uint8_t dynamic[];
  __shared__ Bars bars;
  __shared__ uint32_t tmem_slot;
  __shared__ int seen_most, seen_least, seen_few, poison[NG], abort_flag;
  __shared__ float2 of_b[kTileCols];  // split: B's (reference, sum)
  let_join_start();
  // Blocks with two column tiles come first and those with one, which take half of the time, last.
  Item it;
  if (!tc_item(a, &it)) return;
  // One column tile: A takes its even key tiles and B its odd ones, joined at the end.
  const bool split = it.cb * kTcCols + kTileCols >= it.n * a.kv.G;
  const int chunk = split ? a.last_chunk : a.chunk;
  const bool partial = (split ? a.last_chunks : a.chunks) > 1;
  uint8_t* base = dynamic + (1024 - (tc::smem_u32(dynamic) & 1023u)) % 1024;
  uint8_t *qt = base, *kt = qt + 2 * Z::kTile, *vt = kt + 2 * Z::kTile, *raw = vt + 2 * Z::kTile;
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid / 32, 0), lane = tid % 32;
  volatile int* abort = &abort_flag;

  if (tid == 0) {
    for (int s = 0; s < kRing; ++s) {
      tc::mbar_init(&bars.raw_full[s], 1);
      tc::mbar_init(&bars.raw_free[s], kUnpackWarps);
    }
    for (int s = 0; s < 2; ++s) {
      tc::mbar_init(&bars.k_full[s], 4);
      tc::mbar_init(&bars.v_full[s], 4);
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
    seen_least = seen_few = INT32_MAX;
    for (int g = 0; g < NG; ++g) poison[g] = INT32_MAX;
    abort_flag = 0;
  }
  if (warp == kMmaWarp) tc::tmem_alloc(&tmem_slot, 512);
  __syncthreads();
  // keys that a column sees; columns past the last see all (their result is dropped)
  const int at = tid - 32 * kSoftWarp, col = it.cb * kTcCols + (split ? at & (kTileCols - 1) : at);
  const bool live = at >= 0 && col < it.n * a.kv.G;
  const int lim = live ? limit_of(a, it, col) : INT32_MAX;
  if (warp >= kSoftWarp) {
    const int hi = __reduce_max_sync(0xffffffffu, live ? lim : 0), lo = __reduce_min_sync(0xffffffffu, lim);
    const int few = __reduce_min_sync(0xffffffffu, lim > 0 ? lim : INT32_MAX);
    if (lane == 0) {
      atomicMax(&seen_most, hi);
      atomicMin(&seen_least, lo);
      atomicMin(&seen_few, few);
    }
  }
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  const uint32_t tmem = tmem_slot;
  const int least = seen_least, k0 = it.chunk * chunk, k1 = min(k0 + chunk, seen_most);
  const int tiles = k1 > k0 ? (k1 - k0 + kKeys - 1) / kKeys : 0;
  // keys in two parts, whatever the chunk
  const bool exact = __shfl_sync(0xffffffffu, int(seen_few < kExactBelow), 0) != 0;

  // 128 registers a thread at launch: 2 x 88 + 2 x 168 per four warpgroups
  if (warp < kSoftWarp) {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 88;" ::: "memory");
  if (warp == kLoadWarp) {
    // ---------------------------------------------------------------- copies
    // A load: the packed keys and values of half a tile, in copies of whole pages (lane r page r)
    // or, of a longer page, of four parts (lane p: K codes, V codes, K and V parameters). The lanes
    // issue theirs one after the other, about 100 cycles each: with codes and parameters of keys
    // and of values apart, a tile took as long to issue as its MMAs (377 us for 8 192 keys at 16
    // tokens a page, 344 at 64).
    const bool whole = a.kv.page_shift <= 6;
    const int run_shift = min(6, a.kv.page_shift), copies = whole ? kHalf >> run_shift : 4;
    const int at_half = whole ? lane << run_shift : 0, row_bytes = whole ? 0 : lane < 2 ? D / 2 : D / 8;
    const uint32_t bytes = whole ? uint32_t(a.kv.page_bytes) : kHalf * row_bytes;
    const uint32_t dst = tc::smem_u32(raw) + (whole     ? lane * bytes
                                              : lane < 2 ? lane * kHalf * (D / 2)
                                                         : kHalf * D + (lane - 2) * kHalf * (D / 8));
    const uint8_t* from = a.kv.page(it.l, it.g, 0) + (whole ? 0 : lane < 2 ? a.kv.codes(lane, 0) : a.kv.params(lane - 2, 0));
    const int64_t page_stride = a.kv.Hkv * a.kv.page_bytes;
    auto page_at = [&](int load) {  // page of this lane's copy, looked up a load ahead
      const int j = k0 + load * kHalf + at_half;
      return lane < copies && j < k1 ? page_entry(a, it.r, j) : 0;
    };
    int issued = 0, next = page_at(0);
    bool ok = true;
    for (; issued < 2 * tiles; ++issued) {
      const int kb = k0 + issued * kHalf, tokens = max(0, min(k1 - kb, kHalf)), slot = issued % kRing;
      const bool mine = lane < copies && at_half < tokens;
      const uint8_t* src = from + (mine ? page_in_pool(a, next) : 0) * page_stride +
                           (kb & ((1 << a.kv.page_shift) - 1)) * row_bytes;
      next = page_at(issued + 1);
      if (issued >= kRing && !(ok = wait_warp(&bars.raw_free[slot], (issued / kRing - 1) & 1, abort))) break;
#ifdef CONDUIT_TEST_HOOKS
      if (issued == a.withhold) continue;  // neither copies nor an arrive: the waits for this load run out
#endif
      if (lane == 0)  // whole runs
        tc::mbar_arrive_expect_tx(&bars.raw_full[slot],
                                  uint32_t((tokens + (1 << run_shift) - 1) >> run_shift << run_shift) * (D + D / 4));
      __syncwarp();
      if (mine) bulk_load(dst + slot * Z::kRaw, src, bytes, &bars.raw_full[slot]);
    }
    if (!ok && lane == 0) give_up(a, abort, CONDUIT_SITE_MMA);
    for (int n = max(0, issued - kRing); n < issued; ++n)  // the last copies (all have landed unless a role gave up)
      tc::mbar_wait(&bars.raw_full[n % kRing], (n / kRing) & 1);
  } else if (warp != kMmaWarp) {
    // ---------------------------------------------------------------- unpack
    // A unit is a half (32 tokens) of a load's keys, then of its values; six warps take them in
    // turn. Four lanes a token. Keys: the two tokens of eight lanes are four apart, so
    // that their chunks fall into different banks of the swizzled tile; values: side by side.
    // Every warp sees every copy land and says so before its slot is used again, also where
    // another four warps unpack it: none can take a phase of a slot for the one two before it.
    // Either form of the keys has a copy of this loop (one copy that asks at every tile: 333 us for
    // 8 192 keys instead of 325, 357 instead of 339 with 96 dims).
    auto unpack = [&](auto form) {
    constexpr bool kExact = decltype(form)::value;
    const int c = lane & 3, i8 = lane >> 2, run_shift = min(6, a.kv.page_shift);
    int unit = warp - kUnpackWarp;  // the next one of this warp
    for (int load = 0; load < 2 * tiles; ++load) {
      const int t = load >> 1, v = unit >> 1 & 1, stage = t & 1, slot = load % kRing;
      bool ok = wait_warp(&bars.raw_full[slot], (load / kRing) & 1, abort);
      const bool mine = unit < 4 * load + 4;
      const int in8 = v && NG != 3 ? i8 : (i8 & 1) * 4 + (i8 >> 1), token = kHalf * (load & 1) + 32 * (unit & 1) + in8;
      // Into registers first, so that the next copy into the slot starts while this one is unpacked
      // (held until the end, the ring gave the pace: 126 us for 8 192 keys of two column tiles).
      Packed<NG> x[4];
      if (ok) {
        const uint8_t* box = raw + slot * Z::kRaw;
        if (mine) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {  // page after page as in the pool
            const int at = 32 * (unit & 1) + 8 * i, in_run = at & ((1 << run_shift) - 1);
            const uint8_t* page = box + (at - in_run) * (D + D / 4);
            const uint8_t* codes = page + ((v << run_shift) + in_run) * (D / 2);
            const uint8_t* params = page + (D << run_shift) + ((v << run_shift) + in_run) * (D / 8);
            x[i] = v ? take<NG, true>(codes, params, in8, c) : take<NG, false>(codes, params, in8, c);
          }
        }
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&bars.raw_free[slot]);
        // A buffer is free once its last tile but one has been used. (When a load lands, every warp is
        // done with the load four before it, of the buffer's last tile, and so with the wait for the
        // use before that: this wait cannot mistake its phase either.)
        if (mine && t >= 2 && !(kExact && !v))
          ok = wait_warp(v ? &bars.v_free[stage] : &bars.k_free[stage], ((t >> 1) - 1) & 1, abort);
        // keys in two parts have one buffer, whose every use every warp sees
        if (kExact && ok && t >= 1 && !(load & 1)) ok = wait_warp(&bars.k_free[0], (t - 1) & 1, abort);
      }
      if (!ok) {
        if (lane == 0) give_up(a, abort, CONDUIT_SITE_LOAD);
        break;
      }
      if (!mine) continue;
      unit += kUnpackWarps;
      uint8_t* tile = v ? vt + stage * Z::kTile : kExact ? kt : kt + stage * Z::kTile;
      const int kb = k0 + t * kKeys;
      if (!v) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if constexpr (kExact)
            unpack_keys_exact<NG>(tile, tile + Z::kTile, x[i], token + 8 * i, c);
          else
            unpack_keys<NG>(tile, x[i], token + 8 * i, c);
        }
      } else if (kb + kKeys > least) {  // some column does not see the whole tile
#pragma unroll
        for (int i = 0; i < 4; ++i) unpack_values<NG, true>(tile, x[i], token + 8 * i, c, kb, k1, least, poison);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) unpack_values<NG, false>(tile, x[i], token + 8 * i, c, kb, k1, least, poison);
      }
      tc::fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(v ? &bars.v_full[stage] : &bars.k_full[kExact ? 0 : stage]);
    }
    };
    if (exact)
      unpack(std::true_type{});
    else
      unpack(std::false_type{});
  } else if (warp == kMmaWarp) {
    // ------------------------------------------------------------------ MMAs
    // the whole warp walks the schedule on values from one lane, so that the operands live in
    // uniform registers
    const uint32_t leader = lane == 0;
    const int one = __shfl_sync(0xffffffffu, exact ? 0 : 1, 0);  // 0: keys in two parts, in one buffer
    const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
    const int all = __shfl_sync(0xffffffffu, tiles, 0);
    const bool halves = __shfl_sync(0xffffffffu, int(split), 0) != 0;
    const uint32_t q_at = __shfl_sync(0xffffffffu, tc::smem_u32(qt), 0);
    const uint32_t k_at = q_at + 2 * Z::kTile, v_at = k_at + 2 * Z::kTile;
    constexpr uint32_t idesc_s = idesc_f16(kTileCols, kKeys, false), idesc_o = idesc_f16(kTileCols, D, true);
    const uint64_t dq = tc::desc_sw128(q_at);
    // S_x = Q K^T for the key tile `tile`; a tile's keys and values are waited for by the first
    // stream that reads it and freed by the last.
    bool ok = true;
    auto score = [&](int x, int tile) {
      const int stage = tile & one;
      if (halves || x == 0) {
        if (!(ok = wait_warp(&bars.k_full[stage], (tile >> one) & 1, abort))) return;
        tc::tc_fence_after();
      }
      const uint64_t dk = tc::desc_sw128(k_at + stage * Z::kTile);
      const uint64_t dx = dq + (halves ? 0 : (x * Z::kTile) >> 4);
      // One short loop for both forms of the keys. Its code counts where blocks of both are at work at a time:
      // with a copy for either, 8 192 keys took 317 us instead of 325, but causal prompts of 4 x 4 096 tokens
      // 902 instead of 831 and 32-128 rows over 2 100 keys 233 instead of 203.
#pragma unroll 1
      for (int part = 0; part < 2 - one; ++part) {  // the second: what the keys' first parts left out
        const uint64_t dp = dk + (part ? Z::kTile >> 4 : 0);
#pragma unroll 4
        for (int kk = 0; kk < D / 16; ++kk) {
          const uint32_t off = ((kk >> 2) * kBlock + (kk & 3) * 32) >> 4;
          tc::mma_bf16_if(leader, tm + x * kSCols, dx + off, dp + off, idesc_s, kk > 0 || part > 0);
        }
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
        const uint64_t dv = tc::desc_sw128_mn(v_at + stage * Z::kTile, kBlock);
#pragma unroll
        for (int kk = 0; kk < kKeys / 16; ++kk)
          tc::mma_bf16_ts_if(leader, tm + kOCol + x * kSCols, tm + x * kSCols + kPCol + kk * 8, dv + kk * (2048 >> 4),
                             idesc_o, t > 0 || kk > 0);
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
      // its largest lies in [256, 512) (or below, if that takes more than 2^126).
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
        int shift = max(int(top >> 7) - 127 - 8, -126);
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
        uint4 y;  // in the order in which a word's nibbles unpack
        y.x = h2u(__floats2half2_rn(f[0], f[4]));
        y.y = h2u(__floats2half2_rn(f[1], f[5]));
        y.z = h2u(__floats2half2_rn(f[2], f[6]));
        y.w = h2u(__floats2half2_rn(f[3], f[7]));
        if (part < kUse && owner)
          *reinterpret_cast<uint4*>(tile + (part >> 3) * kBlock + tc::sw128_offset(row0 + 2 * k + side, part & 7)) = y;
      }
      // positive, so that a masked logit stays -inf under it
      to_log2 = fmaxf(a.scale * kLog2e * __uint_as_float(uint32_t(127 + own_shift) << 23), 1.1754944e-38f);
      tc::fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(&bars.q_full);
    }
    const uint32_t lanes = uint32_t((warp & 3) * 32) << 16;
    const uint32_t sb = tmem + lanes + x * kSCols, ob = tmem + lanes + kOCol + x * kSCols;
    float ref = -INFINITY;
    float2 sum = make_float2(0.f, 0.f);
    const float2 up = make_float2(to_log2, to_log2);
    bool ok = true;
    const int count = split ? (tiles + 1 - x) / 2 : tiles;
    for (int t = 0; t < count; ++t) {
      if (!(ok = wait_warp(&bars.s_full[x], t & 1, abort))) break;
      tc::tc_fence_after();
      const int kb = k0 + (split ? 2 * t + x : t) * kKeys;
      const int left = lim - kb;  // keys of the tile that the column sees
      const bool edge = kb + kKeys > least;
      uint32_t p[4][16];
      float2 add;
      for (int pass = 0;; ++pass) {
        const float low = ref == -INFINITY ? 0.f : -ref;
        const float2 down = make_float2(low, low);
        float top = edge ? weigh<true>(sb, up, down, left, p, &add) : weigh<false>(sb, up, down, left, p, &add);
        top *= to_log2;
        if (pass || !__any_sync(0xffffffffu, top > ref + kMostWeight)) break;
        // the reference moves: what was summed so far is scaled, and the weights are taken again
        const float moved = fmaxf(ref, top - kBias), corr = moved == -INFINITY ? 1.f : tc::ex2(ref - moved);
        ref = moved;
        sum = make_float2(sum.x * corr, sum.y * corr);
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
      sum = tc::fadd2(sum, add);
#pragma unroll
      for (int b = 0; b < 4; ++b) tc::tmem_st16_nowait(sb + kPCol + 16 * b, p[b]);
      tc::tmem_wait_st();
      tc::tc_fence_before();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(&bars.p_full[x]);
    }
    // without keys there is nothing to wait for but the other warps' queries, over which the rows go out
    if (ok) ok = count > 0 ? wait_warp(&bars.o_full[x], 0, abort) : wait_warp(&bars.q_full, 0, abort);
    ref += kBias;
    float total = (sum.x + sum.y) * kUnbias, own_w = kUnbias, b_w = 0.f;
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
    bool tainted[NG], any_tainted = false;  // a value that is not finite reaches the columns that see it
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      tainted[g] = poison[g] < lim;
      any_tainted |= tainted[g];
    }
    any_tainted = __any_sync(0xffffffffu, any_tainted);
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
#pragma unroll
      for (int n = 0; n < 8; ++n) {
        // four neighbouring dims of group g: every other column of a word of the value rows
        const int word = 4 * b + n / 2, hw = 2 * word + (n & 1), g = hw % NG, dim = 32 * g + 4 * (hw / NG);
        float y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          y[e] = o[8 * (n / 2) + 2 * e + (n & 1)];
          if (any_tainted && tainted[g]) y[e] = NAN;
        }
        if (partial) {  // a block's 32 dims, in the order in which they come
          *reinterpret_cast<float4*>(chunk_at(row, n)) = make_float4(y[0], y[1], y[2], y[3]);
        } else {
          const __nv_bfloat162 z[2] = {__floats2bfloat162_rn(y[0], y[1]), __floats2bfloat162_rn(y[2], y[3])};
          *reinterpret_cast<uint2*>(chunk_at(row, dim / 8) + (dim & 4) * 2) = *reinterpret_cast<const uint2*>(z);
        }
      }
      if (!partial) continue;
      __syncwarp();
#pragma unroll 1
      for (int k = 0; k < 8; ++k) {  // four rows at a time, eight lanes a row
        const int r = 4 * k + (lane >> 3), n = lane & 7;
        const int hw = 2 * (4 * b + n / 2) + (n & 1), dim = 32 * (hw % NG) + 4 * (hw / NG);
        float* to = a.part_o + __shfl_sync(0xffffffffu, own, r) + dim;
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
  cudaError_t err = cudaFuncSetAttribute(packed_attn_tc<NG>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
  if (err) return err;
  packed_attn_tc<NG><<<unsigned(items), kThreads, kSmem, stream>>>(a);
  count_launches(1);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_packed_attn_tc(const AttnArgs& a, int64_t items, cudaStream_t stream) {
  switch (a.kv.d) {
    case 64: return launch<2>(a, items, stream);
    case 96: return launch<3>(a, items, stream);
    default: return launch<4>(a, items, stream);
  }
}

}  // namespace conduit
