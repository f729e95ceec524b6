// Internal declarations of the paged K/V cache and of rotary positions (h2o_pages_*, h2o_rotate).
#pragma once
#include "store.cuh"

// The handle: host memory only.
struct h2o_pages {
  h2o_pages_config_t cfg;  // strides filled in
  uint32_t polls;          // of a wait before it gives up
  // bfloat16: tensor maps (opaque here) for few query rows and for many, and the rows of their boxes
  alignas(64) unsigned char few_k[128], few_v[128], many_k[128], many_v[128];
  int few_box, many_box;
};

namespace h2o {

// Rotation angles: of pair i, position * frequency[i].
struct Turn {
  const double* frequency;  // dev [half]
  const uint8_t* axis;      // dev [half], or null: axis 0
  const int64_t* positions; // dev [axes][tokens], or null: the token's row
  int64_t position_stride;
  int half, axes, halves, inverse;  // pairs; axes; 1: a pair is channels i and i + half, 0: 2 i and 2 i + 1; 1: by -angle
};

// What one launch of the rotating kernel moves: heads of q to q_out, heads of k and v to their rows of the pages.
struct MoveArgs {
  const void *q, *k, *v;
  void* q_out;
  int64_t q_stride, q_out_stride, kv_stride, n_tokens;  // elements between tokens
  int q_heads, kv_heads, dim;                           // kv_heads 0: no cache
  int q_turn, k_turn;                                   // 1: rotated
  Turn turn;
  // the cache
  void *pk, *pv;
  int64_t page_stride, row_stride, head_stride, table_stride;
  const int32_t *table, *length, *cu;
  int n_pages, page_size, max_pages, max_length, batch;
  int32_t* status;
};
int pages_tc_tile_keys();
cudaError_t launch_pages_tc(const AttendView& a, const void* map_k, const void* map_v, cudaStream_t stream);
cudaError_t launch_move(const MoveArgs& a, int dtype, cudaStream_t stream);

}  // namespace h2o
