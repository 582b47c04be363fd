// Parameters of the calls that rearrange requests' rows (paged_rows.cu).
#pragma once
#include <type_traits>

#include "paged4.cuh"

namespace heatkv {

constexpr int ROWS_CHUNKS = 592;               // chunks of the pool's pages, a CTA each: four on an SM

struct RowsParams {
  const int32_t *parents, *keep_len;           // fork
  const uint8_t* mask;                         // compact: 0 where a token leaves
  int64_t mask_stride;
  int32_t mask_width;
  const int32_t *lengths, *table, *state_in;
  int64_t table_stride, out_stride;
  int32_t *free_pages, *lengths_out, *table_out, *state_out, *move_from, *move_to;
  int32_t n_seq, table_pages, n_pages, n_moves;
  // workspace; row_stay, `was` and `is` are zero before the first call
  uint32_t *marks, *claims;                    // [n_pages] of large pools
  int2* row_moves;                             // [n_seq] fork: {page with the last tokens, length}, then {that page, fresh page}
  int2* row_stay;                              // [2][4096] compact: {table_pages - first page that something leaves (0: none), tokens that stay}
  int32_t *was, *is;                           // calls of compact so far, in turn
  int32_t *chunk_sums, *totals, *page_stay;    // page_stay [n_seq][table_pages]: tokens that stay
  int32_t chunk, chunks;
};
struct MoveParams {
  void *k, *v;                                 // (a cache in 4 bits: its blocks, and strides in bytes)
  const int32_t *from, *to;
  int64_t page_stride, head_stride, row_stride;
  int32_t n_moves, n_pages, Hkv, d;
};

uint64_t rows_workspace_bytes(int n_seq, int table_pages, int n_pages);
void place_rows_workspace(void* ws, RowsParams* p);
cudaError_t launch_paged_fork(const RowsParams& p, cudaStream_t stream);
cudaError_t launch_paged_compact(const RowsParams& p, cudaStream_t stream);
cudaError_t launch_paged_move(const MoveParams& p, int bits, cudaStream_t stream);

}  // namespace heatkv
