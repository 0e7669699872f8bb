// Beam search: launchers of the selection over beams and vocabulary, and of the contexts' reordering.
#pragma once

#include "cache.cuh"

namespace conduit {

constexpr int kMaxBeams = 32;  // beams of a group, candidates of a selection

cudaError_t launch_beam_select(const void* logits, int dtype, int64_t row_stride, int groups, int width, int vocab,
                               const float* sums, int num_out, float* score, int32_t* parent, int32_t* token,
                               int32_t* status, cudaStream_t stream);

// A part of what a page holds of one layer and head: rows of `unit` bytes for `tokens` tokens each.
struct PagePart {
  char* base;
  int64_t layer_stride, page_stride, head_stride;  // bytes
  int32_t unit, tokens, bytes;                     // bytes: of a whole page
};
struct PagedPool {
  PagePart part[4];
  int32_t parts, L, heads, page_size, num_pages, max_pages;
};
cudaError_t launch_reorder(const PagedPool& pool, int groups, int width, const int32_t* parent, const int32_t* home,
                           int32_t* page_table, int32_t* len, int32_t* status, cudaStream_t stream);

}  // namespace conduit
