// Rotary positions with several axes, and the append to a paged cache that
// rotates keys (and queries) on the way.
//
// Rows move in chunks of 16 bytes where pairs and passing dims come in whole chunks and rows are
// aligned, else (heads of 72 dims in bf16, for instance) element by element.
//
// Mathematics: y1 = x1 c - x2 s, y2 = x2 c + x1 s for each pair, in fp32, rounded
// once. Bound: every row is read once and written once; the cosines of a row
// (8 bytes a pair) are shared by all of its heads. Measured: 28 heads of 128 dims, 16 384 tokens
// in 44 us (5.5 TB/s); 22 000 tokens appended to 4-head pages with 28 query heads in 78 us
// (5.0 TB/s); 9 001 fp32 rows of 16 heads of 80 dims in 18 us (5.1 TB/s).
#include <algorithm>

#include "rotate.cuh"

namespace conduit {
namespace {

constexpr int kThreads = 64;

struct AppendArgs {
  SeqsDev s;
  KvDev kv;
};

// A thread owns a unit (VEC pairs) of a row and walks over heads hg, hg + HG, ...
// Heads count q, then (append) k, then v.
template <typename T, int VEC, bool kAppend>
__global__ void __launch_bounds__(kThreads, 12)
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
  int slot = 0, pos[CONDUIT_MAX_AXES];
  bool ok = true;
  // Loads that do not wait for one another go out together: a row's length, then its
  // positions and its page, then its cosines and the first head.
  if (kAppend) {
    const int t0 = ap.s.row_off[r], t1 = ap.s.row_off[r + 1], len = ap.s.len[r];
    if (i >= t1 - t0) return;
    t = t0 + i;
    slot = len - (t1 - t0) + i;
    const int in_req = slot / ap.kv.page_size;
    ok = slot >= 0 && slot < ap.s.max_len && in_req < ap.kv.max_pages;
    const int page = ap.kv.page_table[int64_t(r) * ap.kv.max_pages + (ok ? in_req : 0)];
    ok &= page >= 0 && page < ap.kv.num_pages;
    slot_off = ((int64_t(l) * ap.kv.num_pages + page) * ap.kv.Hkv * ap.kv.page_size + slot % ap.kv.page_size) * d;
  } else if (i >= T_rows) {
    return;
  }
  const Unit un = unit_of<VEC>(rope, d, u);
  const int Hkv = kAppend ? ap.kv.Hkv : 0, H = nq + 2 * Hkv;
  C a, b;
  auto load = [&](int h) {
    const bool is_q = h < nq, is_k = h < nq + Hkv;
    const RowsDev& from = is_q ? x : is_k ? k : v;
    const T* src = static_cast<const T*>(from.p) + l * from.ls + t * from.rs + (is_q ? h : is_k ? h - nq : h - nq - Hkv) * from.hs;
    a = load_once<T, VEC>(src + un.a);
    if (un.b >= 0) b = load_once<T, VEC>(src + un.b);
  };
  if (rope.rot) ok &= load_positions(rope, t, pos);
  load(hg);
  if (!ok) {  // the row is left out, in all of its parts
    if (u == 0 && hg == 0) flag_status(status, CONDUIT_FLAG_INDEX);
    return;
  }
  float2 cs[VEC];
  if (un.turns) load_turn<VEC>(rope, pos, u * VEC, cs);
  for (int h = hg; h < H; h += HG) {
    C y = a, z = b;
    if (h + HG < H) load(h + HG);
    if (un.turns && h < nq + Hkv) turn_chunks<T, VEC>(rope, cs, y, z);
    T* dst;
    if (h < nq)
      dst = static_cast<T*>(out.p) + l * out.ls + t * out.rs + h * out.hs;
    else if (h < nq + Hkv)
      dst = static_cast<T*>(ap.kv.k) + slot_off + int64_t(h - nq) * ap.kv.page_size * d;
    else
      dst = static_cast<T*>(ap.kv.v) + slot_off + int64_t(h - nq - Hkv) * ap.kv.page_size * d;
    store_once<T, VEC>(dst + un.a, y);
    if (un.b >= 0) store_once<T, VEC>(dst + un.b, z);
  }
}

template <typename T, int VEC, bool kAppend>
cudaError_t launch(const RopeDev& rope, const AppendArgs& ap, int L, int R, int rows, int nq, int d, const RowsDev& x,
                   const RowsDev& out, const RowsDev& k, const RowsDev& v, int32_t* status, cudaStream_t stream) {
  const int H = nq + (kAppend ? 2 * ap.kv.Hkv : 0), nu = units_per_row<VEC>(rope, d);
  // Heads per thread: one while the launch does not fill the SMs, then up to nine on one set of
  // cosines (28 query heads, 16 384 tokens: one 102 us, four 52, nine 44, sixteen 46; with 36 heads
  // into a paged cache: 205, 100, 78, 82).
  const int64_t wide = int64_t(rows) * R * L * H * nu / (152 * 2048);
  const int per = int(std::min<int64_t>(9, std::max<int64_t>(1, wide)));
  const int HG = (H + per - 1) / per;
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
