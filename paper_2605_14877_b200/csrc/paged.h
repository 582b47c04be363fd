// What the translation units of the paged cache (requests of any length) share.
#pragma once
#include <cuda.h>
#include <cudaTypedefs.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "device_common.cuh"
#include "heatkv.h"

namespace heatkv {

constexpr int PAGE = HEATKV_PAGE_TOKENS;
constexpr int PAGED_MAX_SEQ = 4096;            // requests of a call: their prefix sums fit one CTA's shared memory
constexpr int PAGED_MAX_TABLE = 1 << 19;       // pages of a block table row
constexpr int PAGED_MAX_PAGES = 1 << 25;       // pages of a pool: slot numbers have 31 bits
constexpr int PAGED_MAX_SELECT_PAGES = 32768;  // pages of a context whose scores one CTA keeps in shared memory

// Selected pages are attended to for many tokens at once from so many new tokens a request and selected pages in all: 8 requests x 32 tokens
// x 4 heads x 16 pages take 59 us token by token and 64 together, x 64 tokens 100 and 69, 16 heads x 16 tokens 98 and 81.  What is gained hangs on how
// much the lists of neighbouring tokens have in common, which no size says.  2001 tokens, 4 kv heads of 8 heads, 16 of 500 pages: where 40 neighbours
// have the same list 396 and 84 us, where every token has a list of its own 370 and 490 (heads of their own, G = 1: 337 and 76, 335 and 346);
// a chunk of 300 beside 64 single tokens, 8 kv heads of 4 heads: 153 and 112, 150 and 179.
constexpr int PAGED_SPARSE_CHUNK = 8, PAGED_SPARSE_PAGES = 24576;

// Workspace: 64 words (word 0: status of bounded waits), then arrival counters, then partial results.
constexpr int PAGED_WS_HEAD_WORDS = 64;
constexpr int PAGED_WS_CTRS = 1024;            // times 8: one for every run of paged_tc_kernel and 32 rows; the first also counts pieces (paged_small_kernel),
                                               // the last CTAs (union_kernel)
constexpr int PAGED_WS_PARTIALS = (PAGED_WS_HEAD_WORDS + PAGED_WS_CTRS * 8) * 4;

// SMs that a launch is laid out for at most: a run's counters and, in paged_small_kernel, pieces of a unit (16 bits) are counted by it.
constexpr int PAGED_MOST_SMS = 240;
static_assert(PAGED_MOST_SMS < PAGED_WS_CTRS, "counters of every run, and a ticket");

struct PagedDevice {
  PFN_cuTensorMapEncodeTiled_v12000 encode = nullptr;
  int n_sm = 0;
};

struct TablesParams {
  const int32_t *new_tokens, *past_tokens, *free_pages, *state_in;
  int32_t *state_out, *block_table, *q_begin, *kv_len, *slot_map, *positions;
  int64_t table_stride;
  int32_t n_seq, n_pages, table_pages, n_tokens;
};
struct ReleaseParams {
  const int32_t *kv_len, *keep_len, *block_table, *state_in;
  int32_t *free_pages, *state_out;
  int64_t table_stride;
  int32_t n_seq, n_pages, table_pages;
};
struct StoreParams {
  const void *k_new, *v_new;
  void *k, *v;
  int8_t* k_code;
  float* k_scale;
  const int32_t* slot_map;
  int64_t tok, head, page_stride, head_stride, row_stride;
  int32_t n_tokens, n_pages, Hkv, d, fp16;
  int32_t copy_blocks;
};
struct SelectParams {
  const void* q;
  int64_t q_tok, q_head;
  const int32_t *q_begin, *kv_len, *block_table;
  int64_t table_stride;
  const int8_t* k_code;
  const float* k_scale;
  int32_t* sel;
  int32_t n_seq, table_pages, n_tokens, n_pages, Hkv, G, d, fp16, sink, local, n_sel;
};
struct PagedParams {
  const void* q;
  void* out;
  float* lse;                       // [n_tokens][H] or null
  int64_t q_tok, q_head, o_tok, o_head;
  const int32_t *q_begin, *kv_len, *block_table;
  int64_t table_stride;
  int32_t n_seq, table_pages, n_tokens, n_pages;
  int32_t H, Hkv, G;
  int32_t causal;
  int32_t tile_tokens;              // tokens of a row tile: tile_tokens * G rows
  float scale_log2;                 // sm_scale * log2(e)
  uint32_t* status;
  uint32_t* counters;
  float* partials;
  const int32_t* sel;               // selected pages [n_tokens][Hkv][n_sel], or null: all
  int32_t n_sel;
  int32_t max_new;
};

// the 4-bit cache
struct Store4Params {
  const void *k_new, *v_new;        // (read back: written)
  unsigned char* blocks;
  const int32_t* slot_map;
  int64_t tok, head, page_stride, head_stride;      // strides of the blocks in bytes
  int32_t n_tokens, n_pages, Hkv, fp16, k_exp, v_exp;
};
struct Paged4Params {
  PagedParams a;                    // scale_log2 holds what the numbers of K are to be multiplied by
  const unsigned char* blocks;
  int64_t page_stride, head_stride; // bytes
  float v_unit;                     // .. and those of V
  int32_t fp16;                     // type of q and out
};

cudaError_t launch_paged_tables(const TablesParams& p, cudaStream_t stream);
cudaError_t launch_paged_release(const ReleaseParams& p, cudaStream_t stream);
cudaError_t launch_paged_store(StoreParams p, cudaStream_t stream);
cudaError_t launch_paged_summaries(const StoreParams& p, cudaStream_t stream);
cudaError_t launch_paged_select(const SelectParams& p, int max_new, int n_sm, cudaStream_t stream);
// warp-level kernel: row tiles of up to 64 rows
uint64_t paged_small_partial_bytes(int d, int n_sm, int Hkv, int n_tokens);
cudaError_t launch_paged_small(const PagedParams& p, const heatkv_paged_pool& pool, const PagedDevice& dev, cudaStream_t stream);
// tensor-memory kernel: row tiles of up to 128 rows
uint64_t paged_tc_partial_bytes(int d, int n_sm, int G, int Hkv, int n_tokens, int n_seq);
bool paged_tc_takes_lists(int G, int Hkv, int n_sel, int table_pages, int n_tokens, int n_seq);
cudaError_t launch_paged_tc(const PagedParams& p, const heatkv_paged_pool& pool, const PagedDevice& dev, cudaStream_t stream);

cudaError_t launch_paged4_rows(const Store4Params& p, bool load, int d, cudaStream_t stream);
uint64_t paged4_small_partial_bytes(int d, int n_sm);
cudaError_t launch_paged4_tc(const Paged4Params& p, int d, const PagedDevice& dev, cudaStream_t stream);
cudaError_t launch_paged4_small(const Paged4Params& p, int d, const PagedDevice& dev, cudaStream_t stream);

// A tensor map with four dimensions of 16-bit numbers, 128-byte swizzle.
inline bool paged_encode(const PagedDevice& dev, CUtensorMap* m, void* base, int dtype, const cuuint64_t* dims, const cuuint64_t* strides,
                         const cuuint32_t* box) {
  const cuuint32_t unit[4] = {1, 1, 1, 1};
  return encode_in_context([&] {
    return dev.encode(m, dtype == HEATKV_DTYPE_FP16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, base, dims, strides, box,
                      unit, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                      CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
  });
}

// boxes of 64 columns x 64 rows of one page and head: (column, row, head, page)
inline bool paged_encode_pool(const PagedDevice& dev, CUtensorMap* m, void* base, const heatkv_paged_pool& pool) {
  const cuuint64_t dims[4] = {(cuuint64_t)pool.d, PAGE, (cuuint64_t)pool.n_kv_heads, (cuuint64_t)pool.n_pages};
  const cuuint64_t strides[3] = {(cuuint64_t)pool.row_stride * 2, (cuuint64_t)pool.head_stride * 2, (cuuint64_t)pool.page_stride * 2};
  const cuuint32_t box[4] = {64, PAGE, 1, 1};
  return paged_encode(dev, m, base, pool.dtype, dims, strides, box);
}

// query rows: boxes of 64 columns x the G heads of a kv head x tile_tokens tokens: (column, head, token)
inline bool paged_encode_q(const PagedDevice& dev, CUtensorMap* m, const PagedParams& p, const heatkv_paged_pool& pool) {
  const cuuint64_t dims[4] = {(cuuint64_t)pool.d, (cuuint64_t)p.H, (cuuint64_t)p.n_tokens, 1};
  const cuuint64_t strides[3] = {(cuuint64_t)p.q_head * 2, (cuuint64_t)p.q_tok * 2, 16};
  const cuuint32_t box[4] = {64, (cuuint32_t)p.G, (cuuint32_t)p.tile_tokens, 1};
  return paged_encode(dev, m, const_cast<void*>(p.q), pool.dtype, dims, strides, box);
}

}  // namespace heatkv
