// Rotary positions with several axes, and the append to a paged cache that
// rotates keys (and queries) on the way.
//
// Mathematics: y1 = x1 c - x2 s, y2 = x2 c + x1 s for each pair, in fp32, rounded
// once. Bound: every row is read once and written once; the cosines of a row
// (8 bytes a pair) are shared by all of its heads.
#include "rotate.cuh"

namespace conduit {
namespace {

constexpr int kThreads = 256;

struct AppendArgs {
  SeqsDev s;
  KvDev kv;
};

// A thread owns a unit (VEC pairs) of a row and walks over heads hg, hg + HG, ...
// Heads count q, then (append) k, then v.
template <typename T, int VEC, bool kAppend>
__global__ void __launch_bounds__(kThreads)
    rotate_kernel(RopeDev rope, AppendArgs ap, int T_rows, int nq, int d, int HG, RowsDev x, RowsDev out, RowsDev k,
                  RowsDev v, int32_t* status) {
  using C = Chunk<T, VEC>;
  const int nu = units_per_row<VEC>(rope, d);
  const uint32_t lin = blockIdx.x * uint32_t(kThreads) + threadIdx.x;
  const uint32_t rest = lin / uint32_t(nu);
  const int u = int(lin - rest * nu);
  const int i = int(rest / uint32_t(HG)), hg = int(rest % uint32_t(HG));
  const int r = blockIdx.y, l = blockIdx.z;
  int64_t t = i, slot_off = 0;
  bool ok = true;
  if (kAppend) {
    const int t0 = ap.s.row_off[r], n = ap.s.row_off[r + 1] - t0;
    if (i >= n) return;
    t = t0 + i;
    const int len = ap.s.len[r], slot = len - n + i;
    ok = slot >= 0 && slot < ap.s.max_len && slot / ap.kv.page_size < ap.kv.max_pages;
    if (ok) {
      const int page = ap.kv.page_table[int64_t(r) * ap.kv.max_pages + slot / ap.kv.page_size];
      ok = page >= 0 && page < ap.kv.num_pages;
      slot_off = ((int64_t(l) * ap.kv.num_pages + page) * ap.kv.Hkv * ap.kv.page_size + slot % ap.kv.page_size) * d;
    }
  } else if (i >= T_rows) {
    return;
  }
  const Unit un = unit_of<VEC>(rope, u);
  float2 cs[VEC];
  if (rope.rot && ok) {
    // a unit that only copies checks the positions too: a row is written whole or not at all
    ok = load_turn<VEC>(rope, t, un.turns ? u * VEC : 0, cs);
  }
  if (!ok) {
    if (u == 0 && hg == 0) flag_status(status, CONDUIT_FLAG_INDEX);
    return;
  }
  const int Hkv = kAppend ? ap.kv.Hkv : 0, H = nq + 2 * Hkv;
#pragma unroll 4
  for (int h = hg; h < H; h += HG) {
    const T* src;
    T* dst;
    bool turns = un.turns;
    if (h < nq) {
      src = static_cast<const T*>(x.p) + l * x.ls + t * x.rs + h * x.hs;
      dst = static_cast<T*>(out.p) + l * out.ls + t * out.rs + h * out.hs;
    } else {
      const bool is_v = h >= nq + Hkv;
      const int g = is_v ? h - nq - Hkv : h - nq;
      const RowsDev& from = is_v ? v : k;
      src = static_cast<const T*>(from.p) + l * from.ls + t * from.rs + g * from.hs;
      dst = static_cast<T*>(is_v ? ap.kv.v : ap.kv.k) + slot_off + int64_t(g) * ap.kv.page_size * d;
      turns &= !is_v;
    }
    C a = *reinterpret_cast<const C*>(src + un.a);
    if (un.turns) {
      C b = *reinterpret_cast<const C*>(src + un.b);
      if (turns) turn_chunks<T, VEC>(rope, cs, a, b);
      *reinterpret_cast<C*>(dst + un.b) = b;
    }
    *reinterpret_cast<C*>(dst + un.a) = a;
  }
}

template <typename T, int VEC, bool kAppend>
cudaError_t launch(const RopeDev& rope, const AppendArgs& ap, int L, int R, int rows, int nq, int d, const RowsDev& x,
                   const RowsDev& out, const RowsDev& k, const RowsDev& v, int32_t* status, cudaStream_t stream) {
  const int H = nq + (kAppend ? 2 * ap.kv.Hkv : 0), nu = units_per_row<VEC>(rope, d);
  const int HG = H;
  const int64_t threads = int64_t(rows) * HG * nu;
  const dim3 grid(unsigned((threads + kThreads - 1) / kThreads), R, L);
  rotate_kernel<T, VEC, kAppend><<<grid, kThreads, 0, stream>>>(rope, ap, rows, nq, d, HG, x, out, k, v, status);
  count_launches(1);
  return cudaGetLastError();
}

template <bool kAppend>
cudaError_t dispatch(const RopeDev& rope, const AppendArgs& ap, int dtype, int L, int R, int rows, int nq, int d,
                     const RowsDev& x, const RowsDev& out, const RowsDev& k, const RowsDev& v, int32_t* status,
                     cudaStream_t stream) {
  const int vec = dtype == CONDUIT_BF16 ? 8 : 4;
  const bool wide = dims_in_chunks(rope, d, vec) && (nq == 0 || (rows_aligned(x, vec) && rows_aligned(out, vec))) &&
                    (!kAppend || (rows_aligned(k, vec) && rows_aligned(v, vec)));
  if (dtype == CONDUIT_BF16)
    return wide ? launch<__nv_bfloat16, 8, kAppend>(rope, ap, L, R, rows, nq, d, x, out, k, v, status, stream)
                : launch<__nv_bfloat16, 1, kAppend>(rope, ap, L, R, rows, nq, d, x, out, k, v, status, stream);
  return wide ? launch<float, 4, kAppend>(rope, ap, L, R, rows, nq, d, x, out, k, v, status, stream)
              : launch<float, 1, kAppend>(rope, ap, L, R, rows, nq, d, x, out, k, v, status, stream);
}

}  // namespace

cudaError_t launch_rope(const RopeDev& rope, int dtype, int L, int T, int H, int d, const RowsDev& x,
                        const RowsDev& out, int32_t* status, cudaStream_t stream) {
  return dispatch<false>(rope, AppendArgs{}, dtype, L, 1, T, H, d, x, out, RowsDev{}, RowsDev{}, status, stream);
}

cudaError_t launch_kv_append(const KvDev& kv, const SeqsDev& s, const RopeDev& rope, const RowsDev& k,
                             const RowsDev& v, const RowsDev& q, const RowsDev& q_out, int32_t* status,
                             cudaStream_t stream) {
  return dispatch<true>(rope, AppendArgs{s, kv}, kv.dtype, kv.L, s.R, s.max_rows, q.p ? kv.Hq : 0, kv.d, q, q_out, k,
                        v, status, stream);
}

}  // namespace conduit
