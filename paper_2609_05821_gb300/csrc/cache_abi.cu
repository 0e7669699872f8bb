// C ABI of the rotary positions, the growing paged cache and the 4-bit cache:
// host-side argument checks and launches. Every check runs before anything is
// enqueued; nothing here allocates.
#include <cmath>

#include "abi_checks.cuh"
#include "cache.cuh"

using namespace conduit;
using namespace conduit::abi;

namespace {

constexpr int kMaxGrid = 65535;  // grid.y, grid.z

conduit_status check_dtype(int32_t dtype) {
  if (dtype != CONDUIT_F32 && dtype != CONDUIT_BF16)
    return fail(CONDUIT_ERR_INVALID_ARG, "dtype must be CONDUIT_F32 or CONDUIT_BF16");
  return CONDUIT_OK;
}

conduit_status make_rope(const conduit_rotary* r, const int32_t* pos, int64_t rows, int d, bool inverse, RopeDev* out) {
  *out = RopeDev{};
  if (!r) return CONDUIT_OK;
  if (r->rot_dim < 2 || r->rot_dim % 2 || r->rot_dim > d)
    return fail(CONDUIT_ERR_INVALID_ARG, "rot_dim must be even, in [2, head_dim]");
  if (r->num_axes < 1 || r->num_axes > CONDUIT_MAX_AXES)
    return fail(CONDUIT_ERR_INVALID_ARG, "num_axes must be in [1, %d]", CONDUIT_MAX_AXES);
  if (r->layout != CONDUIT_ROPE_HALVES && r->layout != CONDUIT_ROPE_PAIRS)
    return fail(CONDUIT_ERR_INVALID_ARG, "layout must be CONDUIT_ROPE_HALVES or _PAIRS");
  if (r->table_len < 1 || !r->table || !r->axis)
    return fail(CONDUIT_ERR_INVALID_ARG, "the rotary table, its length and axis are required");
  if (!aligned16(r->table)) return fail(CONDUIT_ERR_INVALID_ARG, "the rotary table must be 16-byte aligned");
  if (rows > 0 && !pos) return fail(CONDUIT_ERR_INVALID_ARG, "pos is NULL");
  if (reinterpret_cast<uintptr_t>(pos) % 4) return fail(CONDUIT_ERR_INVALID_ARG, "pos must be 4-byte aligned");
  for (int p = 0; p < r->rot_dim / 2; ++p) {
    if (r->axis[p] < 0 || r->axis[p] >= r->num_axes)
      return fail(CONDUIT_ERR_INVALID_ARG, "axis[%d] is outside [0, num_axes)", p);
    out->axis[p / 16] |= uint32_t(r->axis[p]) << (2 * (p % 16));
  }
  out->table = reinterpret_cast<const float2*>(r->table);
  out->pos = pos;
  out->len = r->table_len;
  out->rot = r->rot_dim;
  out->half = r->rot_dim / 2;
  out->layout = r->layout;
  out->axes = r->num_axes;
  out->T = int(rows);
  out->sign = inverse ? -1.f : 1.f;
  return CONDUIT_OK;
}

conduit_status make_rows(const conduit_rows* r, const char* name, int dtype, RowsDev* out) {
  if (!r || !r->data) return fail(CONDUIT_ERR_INVALID_ARG, "%s is NULL", name);
  if (r->layer_stride < 0 || r->row_stride < 0 || r->head_stride < 0)
    return fail(CONDUIT_ERR_INVALID_ARG, "%s has a negative stride", name);
  if (reinterpret_cast<uintptr_t>(r->data) % (dtype == CONDUIT_BF16 ? 2 : 4))
    return fail(CONDUIT_ERR_INVALID_ARG, "%s is not aligned to its element", name);
  *out = RowsDev{r->data, r->layer_stride, r->row_stride, r->head_stride};
  return CONDUIT_OK;
}

// Rows that are written: distinct rows may not share memory, so no stride of a
// dimension with more than one entry is below the row's length.
conduit_status check_written(const conduit_rows* r, const char* name, int64_t L, int64_t T, int64_t H, int d) {
  if ((L > 1 && r->layer_stride < d) || (T > 1 && r->row_stride < d) || (H > 1 && r->head_stride < d))
    return fail(CONDUIT_ERR_INVALID_ARG, "%s has rows that overlap", name);
  return CONDUIT_OK;
}

conduit_status make_seqs(const conduit_seqs* s, SeqsDev* out) {
  if (!s) return fail(CONDUIT_ERR_INVALID_ARG, "seqs is NULL");
  if (s->num_requests < 1) return fail(CONDUIT_ERR_INVALID_ARG, "num_requests must be >= 1");
  if (s->num_requests > kMaxGrid) return fail(CONDUIT_ERR_UNSUPPORTED, "more than %d requests", kMaxGrid);
  if (s->max_len < 0) return fail(CONDUIT_ERR_INVALID_ARG, "max_len must be >= 0");
  if (!s->row_off || !s->row_off_dev || !s->len_dev)
    return fail(CONDUIT_ERR_INVALID_ARG, "row_off, row_off_dev and len_dev are required");
  if (s->row_off[0] != 0) return fail(CONDUIT_ERR_INVALID_ARG, "row_off must start at 0");
  *out = SeqsDev{s->num_requests, 0, s->max_len, 0, s->row_off_dev, s->len_dev, s->row_off};
  for (int r = 0; r < s->num_requests; ++r) {
    if (s->row_off[r + 1] < s->row_off[r])
      return fail(CONDUIT_ERR_INVALID_ARG, "row_off must be non-decreasing (request %d)", r);
    out->max_rows = std::max(out->max_rows, s->row_off[r + 1] - s->row_off[r]);
  }
  out->T = s->row_off[s->num_requests];
  return CONDUIT_OK;
}

// Threads of a launch are counted in 32 bits.
conduit_status check_threads(int64_t rows, int64_t per_row, int64_t L) {
  if (rows * per_row > int64_t(1) << 31) return fail(CONDUIT_ERR_UNSUPPORTED, "a request has too many rows");
  if (L > kMaxGrid) return fail(CONDUIT_ERR_UNSUPPORTED, "more than %d layers", kMaxGrid);
  return CONDUIT_OK;
}

conduit_status make_packed(const conduit_packed_kv* kv, PackedDev* out) {
  if (!kv) return fail(CONDUIT_ERR_INVALID_ARG, "kv is NULL");
  if (kv->num_layers < 1 || kv->num_q_heads < 1 || kv->num_kv_heads < 1)
    return fail(CONDUIT_ERR_INVALID_ARG, "layer and head counts must be >= 1");
  if (kv->num_q_heads % kv->num_kv_heads)
    return fail(CONDUIT_ERR_INVALID_ARG, "num_q_heads must be a multiple of num_kv_heads");
  const int64_t bytes = conduit_packed_page_bytes(kv->head_dim, kv->page_size);
  if (bytes < 0)
    return fail(CONDUIT_ERR_UNSUPPORTED,
                "head_dim must be a multiple of 32 in [32, 256], page_size a power of two in [8, 1024]");
  if (kv->num_pages < 1 || kv->max_pages_per_req < 1 || !kv->page_table)
    return fail(CONDUIT_ERR_INVALID_ARG, "page_table, num_pages and max_pages_per_req are required");
  if (int64_t(kv->max_pages_per_req) * kv->page_size > INT32_MAX)
    return fail(CONDUIT_ERR_UNSUPPORTED, "a page-table row holds more than 2^31 - 1 tokens");
  if (!kv->pool) return fail(CONDUIT_ERR_INVALID_ARG, "pool is NULL");
  if (!aligned16(kv->pool)) return fail(CONDUIT_ERR_INVALID_ARG, "pool must be 16-byte aligned");
  int shift = 0;
  while ((1 << shift) < kv->page_size) ++shift;
  *out = PackedDev{static_cast<uint8_t*>(kv->pool), kv->page_table, kv->num_layers, kv->num_q_heads,
                   kv->num_kv_heads, kv->num_q_heads / kv->num_kv_heads, kv->head_dim, kv->num_pages,
                   kv->max_pages_per_req, shift, bytes};
  return CONDUIT_OK;
}

conduit_status check_reach(const PackedDev& kv, const SeqsDev& s) {
  if (packed_attn_reach(kv, s) > kMaxReach)
    return fail(CONDUIT_ERR_UNSUPPORTED, "contexts of more than %d tokens (min of max_len and a page-table row)", kMaxReach);
  return CONDUIT_OK;
}

// The rows of an append: k, v and, both or neither, q and q_out.
struct AppendRows {
  RowsDev k, v, q, q_out;
};

conduit_status make_append_rows(const conduit_rows* k, const conduit_rows* v, const conduit_rows* q,
                                const conduit_rows* q_out, int dtype, int64_t L, int64_t T, int64_t Hq, int d,
                                AppendRows* out) {
  conduit_status st;
  *out = AppendRows{};
  if ((st = make_rows(k, "k", dtype, &out->k)) || (st = make_rows(v, "v", dtype, &out->v))) return st;
  if ((q != nullptr) != (q_out != nullptr))
    return fail(CONDUIT_ERR_INVALID_ARG, "q and q_out are given together or not at all");
  if (!q) return CONDUIT_OK;
  if ((st = make_rows(q, "q", dtype, &out->q)) || (st = make_rows(q_out, "q_out", dtype, &out->q_out)) ||
      (st = check_written(q_out, "q_out", L, T, Hq, d)))
    return st;
  return CONDUIT_OK;
}

}  // namespace

extern "C" {

conduit_status conduit_rope(const conduit_rotary* rope, const int32_t* pos, int32_t num_layers,
                            int32_t num_rows, int32_t num_heads, int32_t head_dim, int32_t dtype,
                            const conduit_rows* x, const conduit_rows* out, int32_t inverse,
                            int32_t* status, void* stream) {
  conduit_status st;
  if (!rope) return fail(CONDUIT_ERR_INVALID_ARG, "rope is NULL");
  if (num_layers < 1 || num_heads < 1 || num_rows < 0)
    return fail(CONDUIT_ERR_INVALID_ARG, "layers and heads must be >= 1, rows >= 0");
  if (head_dim < 2 || head_dim > kMaxHeadDim)
    return fail(CONDUIT_ERR_UNSUPPORTED, "head_dim must be in [2, %d]", kMaxHeadDim);
  RopeDev rd;
  RowsDev xd, od;
  if ((st = check_dtype(dtype)) || (st = make_rope(rope, pos, num_rows, head_dim, inverse != 0, &rd))) return st;
  if (num_rows == 0) return CONDUIT_OK;
  if ((st = make_rows(x, "x", dtype, &xd)) || (st = make_rows(out, "out", dtype, &od)) ||
      (st = check_written(out, "out", num_layers, num_rows, num_heads, head_dim)) ||
      (st = check_threads(num_rows, int64_t(num_heads) * head_dim, num_layers)))
    return st;
  cudaError_t err = launch_rope(rd, dtype, num_layers, num_rows, num_heads, head_dim, xd, od, status,
                                static_cast<cudaStream_t>(stream));
  if (err) return cuda_fail(err, "rope");
  return CONDUIT_OK;
}

conduit_status conduit_kv_append(const conduit_kv* kv, const conduit_seqs* seqs,
                                 const conduit_rotary* rope, const int32_t* pos,
                                 const conduit_rows* k, const conduit_rows* v, const conduit_rows* q,
                                 const conduit_rows* q_out, int32_t* status, void* stream) {
  conduit_status st;
  SeqsDev sd;
  if ((st = make_seqs(seqs, &sd))) return st;
  // the checks of a cache that a batch reads; the token counts are on the device here
  conduit_batch none{};
  if ((st = check_kv(kv, &none))) return st;
  if (kv->page_size == 0) return fail(CONDUIT_ERR_UNSUPPORTED, "append needs a paged cache");
  if (int64_t(kv->max_pages_per_req) * kv->page_size > INT32_MAX)
    return fail(CONDUIT_ERR_UNSUPPORTED, "a page-table row holds more than 2^31 - 1 tokens");
  RopeDev rd;
  AppendRows rows;
  if ((st = make_rope(rope, pos, sd.T, kv->head_dim, false, &rd))) return st;
  if (sd.T == 0) return CONDUIT_OK;
  const int64_t heads = kv->num_q_heads + 2 * int64_t(kv->num_kv_heads);
  if ((st = make_append_rows(k, v, q, q_out, kv->dtype, kv->num_layers, sd.T, kv->num_q_heads, kv->head_dim, &rows)) ||
      (st = check_threads(sd.max_rows, heads * kv->head_dim, kv->num_layers)))
    return st;
  KvDev kd{};
  kd.k = kv->k;
  kd.v = kv->v;
  kd.L = kv->num_layers;
  kd.Hq = kv->num_q_heads;
  kd.Hkv = kv->num_kv_heads;
  kd.d = kv->head_dim;
  kd.G = kv->num_q_heads / kv->num_kv_heads;
  kd.dtype = kv->dtype;
  kd.page_size = kv->page_size;
  kd.num_pages = kv->num_pages;
  kd.max_pages = kv->max_pages_per_req;
  kd.page_table = kv->page_table;
  cudaError_t err = launch_kv_append(kd, sd, rd, rows.k, rows.v, rows.q, rows.q_out, status,
                                     static_cast<cudaStream_t>(stream));
  if (err) return cuda_fail(err, "kv_append");
  return CONDUIT_OK;
}

int64_t conduit_packed_page_bytes(int32_t head_dim, int32_t page_size) {
  if (head_dim < 32 || head_dim > kMaxHeadDim || head_dim % 32) return -1;
  if (page_size < 8 || page_size > 1024 || (page_size & (page_size - 1))) return -1;
  return int64_t(page_size) * (head_dim + head_dim / 4);
}

conduit_status conduit_packed_append(const conduit_packed_kv* kv, const conduit_seqs* seqs,
                                     const conduit_rotary* rope, const int32_t* pos, int32_t dtype,
                                     const conduit_rows* k, const conduit_rows* v,
                                     const conduit_rows* q, const conduit_rows* q_out,
                                     int32_t* status, void* stream) {
  conduit_status st;
  PackedDev kd;
  SeqsDev sd;
  RopeDev rd;
  AppendRows rows;
  if ((st = make_packed(kv, &kd)) || (st = make_seqs(seqs, &sd)) || (st = check_dtype(dtype)) ||
      (st = make_rope(rope, pos, sd.T, kd.d, false, &rd)))
    return st;
  if (sd.T == 0) return CONDUIT_OK;
  if ((st = make_append_rows(k, v, q, q_out, dtype, kd.L, sd.T, kd.Hq, kd.d, &rows)) ||
      (st = check_threads(sd.max_rows, (kd.Hq + 2 * int64_t(kd.Hkv)) * kd.d, kd.L)))
    return st;
  cudaError_t err = launch_packed_append(kd, sd, rd, dtype, rows.k, rows.v, rows.q, rows.q_out, status,
                                         static_cast<cudaStream_t>(stream));
  if (err) return cuda_fail(err, "packed_append");
  return CONDUIT_OK;
}

conduit_status conduit_packed_read(const conduit_packed_kv* kv, const int32_t* first,
                                   const conduit_kv* dst, const conduit_batch* batch,
                                   int32_t* status, void* stream) {
  conduit_status st;
  PackedDev kd;
  if ((st = make_packed(kv, &kd)) || (st = check_batch(batch)) || (st = check_kv(dst, batch))) return st;
  if (dst->num_layers != kd.L || dst->num_kv_heads != kd.Hkv || dst->head_dim != kd.d)
    return fail(CONDUIT_ERR_INVALID_ARG, "dst must have the packed cache's layers, KV heads and head_dim");
  if (batch->num_requests > kMaxGrid) return fail(CONDUIT_ERR_UNSUPPORTED, "more than %d requests", kMaxGrid);
  int most = 0;
  for (int r = 0; r < batch->num_requests; ++r) most = std::max(most, batch->tok_off[r + 1] - batch->tok_off[r]);
  if ((st = check_threads(most, int64_t(kd.Hkv) * kd.d, kd.L))) return st;
  cudaError_t err = launch_packed_read(kd, first, make_kv(dst, batch), make_batch(batch), most, status,
                                       static_cast<cudaStream_t>(stream));
  if (err) return cuda_fail(err, "packed_read");
  return CONDUIT_OK;
}

conduit_status conduit_packed_attn_workspace_size(const conduit_packed_kv* kv, const conduit_seqs* seqs,
                                                  int32_t dtype, size_t* bytes) {
  conduit_status st;
  PackedDev kd;
  SeqsDev sd;
  if (!bytes) return fail(CONDUIT_ERR_INVALID_ARG, "bytes is NULL");
  if ((st = make_packed(kv, &kd)) || (st = make_seqs(seqs, &sd)) || (st = check_dtype(dtype)) ||
      (st = check_reach(kd, sd)))
    return st;
  *bytes = align_up(packed_attn_plan(kd, sd, dtype).scratch);
  return CONDUIT_OK;
}

conduit_status conduit_packed_attn(const conduit_packed_kv* kv, const conduit_seqs* seqs, int32_t dtype,
                                   const conduit_rows* q, float scale, const int32_t* limits,
                                   const conduit_rows* out, float* lse, void* workspace,
                                   size_t workspace_bytes, int32_t* status, void* stream) {
  conduit_status st;
  PackedDev kd;
  SeqsDev sd;
  RowsDev qd, od;
  if ((st = make_packed(kv, &kd)) || (st = make_seqs(seqs, &sd)) || (st = check_dtype(dtype)) ||
      (st = check_reach(kd, sd)))
    return st;
  if (!(scale >= 0.f) || !std::isfinite(scale))
    return fail(CONDUIT_ERR_INVALID_ARG, "scale must be finite and >= 0 (0: 1/sqrt(head_dim))");
  if (sd.T == 0) return CONDUIT_OK;
  if ((st = make_rows(q, "q", dtype, &qd)) || (st = make_rows(out, "out", dtype, &od)) ||
      (st = check_written(out, "out", kd.L, sd.T, kd.Hq, kd.d)))
    return st;
  if (reinterpret_cast<uintptr_t>(limits) % 4 || reinterpret_cast<uintptr_t>(lse) % 4)
    return fail(CONDUIT_ERR_INVALID_ARG, "limits and lse must be 4-byte aligned");
  const PackedAttnPlan plan = packed_attn_plan(kd, sd, dtype);
  if ((st = check_workspace(workspace, workspace_bytes, align_up(plan.scratch)))) return st;
  if (plan.items > INT32_MAX) return fail(CONDUIT_ERR_UNSUPPORTED, "too many rows, heads and layers for one call");
  if (scale == 0.f) scale = 1.f / std::sqrt(float(kd.d));
  cudaError_t err = launch_packed_attn(kd, sd, plan, dtype, qd, scale, limits, od, lse, workspace, status,
                                       static_cast<cudaStream_t>(stream));
  if (err) return cuda_fail(err, "packed_attn");
  return CONDUIT_OK;
}

}  // extern "C"
