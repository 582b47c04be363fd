// Entry points of the paged cache: checks of arguments and kernel choice.
#include <atomic>

#include "paged_wait.cuh"

namespace heatkv {
namespace {

constexpr int MAX_DEVICES = 64;

// The current device's SM count and the driver's tensor-map encoder.
bool paged_device(PagedDevice* out) {
  static std::atomic<int> sms[MAX_DEVICES];
  static std::atomic<void*> encode{nullptr};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= MAX_DEVICES) return false;
  int n = sms[dev].load(std::memory_order_relaxed);
  if (n == 0) {
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) return false;
    sms[dev].store(n, std::memory_order_relaxed);
  }
  void* fn = encode.load(std::memory_order_relaxed);
  if (!fn) {
    cudaDriverEntryPointQueryResult res;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &res) != cudaSuccess || res != cudaDriverEntryPointSuccess || !fn)
      return false;
    encode.store(fn, std::memory_order_relaxed);
  }
  out->n_sm = n < PAGED_MOST_SMS ? n : PAGED_MOST_SMS;
  out->encode = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(fn);
  return true;
}

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

int check_pool(const heatkv_paged_pool* p) {
  if (!p || !p->k || !p->v || p->n_pages < 1 || p->n_kv_heads < 1) return HEATKV_ERR_INVALID_ARG;
  if ((p->d != 64 && p->d != 128) || (p->dtype != HEATKV_DTYPE_BF16 && p->dtype != HEATKV_DTYPE_FP16)) return HEATKV_ERR_INVALID_ARG;
  if (p->n_pages > PAGED_MAX_PAGES || p->n_kv_heads > 4096) return HEATKV_ERR_TOO_LARGE;
  if (!aligned(p->k, 16) || !aligned(p->v, 16) || ((p->page_stride | p->head_stride | p->row_stride) & 7)) return HEATKV_ERR_INVALID_ARG;
  if (p->page_stride < p->d || p->head_stride < p->d || p->row_stride < p->d) return HEATKV_ERR_INVALID_ARG;
  if ((p->k_code == nullptr) != (p->k_scale == nullptr) || !aligned(p->k_code, 16)) return HEATKV_ERR_INVALID_ARG;
  return HEATKV_OK;
}

int check_batch(const heatkv_paged_pool* pool, const heatkv_paged_batch* b, int n_heads) {
  const int rc = check_pool(pool);
  if (rc != HEATKV_OK) return rc;
  if (!b || !b->q_begin || !b->kv_len || !b->block_table || b->n_seq < 1 || b->n_tokens < 1 || b->table_pages < 1 || b->max_new < 1)
    return HEATKV_ERR_INVALID_ARG;
  if (b->table_stride < b->table_pages) return HEATKV_ERR_INVALID_ARG;
  if (b->n_seq > PAGED_MAX_SEQ || b->table_pages > PAGED_MAX_TABLE) return HEATKV_ERR_TOO_LARGE;
  if (((int64_t)b->n_tokens + b->n_seq) * pool->n_kv_heads > (1 << 30)) return HEATKV_ERR_TOO_LARGE;        // units have 31-bit numbers
  if (n_heads < 1 || n_heads % pool->n_kv_heads != 0 || n_heads / pool->n_kv_heads > 128) return HEATKV_ERR_SHAPE_MISMATCH;
  return HEATKV_OK;
}

// Fills the part of the parameters that all calls over a batch share.
int attention_params(const heatkv_paged_pool* pool, const heatkv_paged_batch* b, int n_heads, const void* q, const heatkv_token_strides* st,
                     float sm_scale, void* out, float* lse, PagedParams* p) {
  const int rc = check_batch(pool, b, n_heads);
  if (rc != HEATKV_OK) return rc;
  const int64_t row = (int64_t)n_heads * pool->d;
  const heatkv_token_strides s = st ? *st : heatkv_token_strides{row, pool->d, row, pool->d};
  if (!q || !out || !aligned(q, 16) || !aligned(out, 16) || ((s.q_tok | s.q_head | s.o_tok | s.o_head) & 7)) return HEATKV_ERR_INVALID_ARG;
  if (s.q_tok < pool->d || s.q_head < pool->d || s.o_tok < pool->d || s.o_head < pool->d) return HEATKV_ERR_INVALID_ARG;
  if (!(sm_scale == sm_scale) || sm_scale > 1e30f) return HEATKV_ERR_INVALID_ARG;
  *p = PagedParams{};
  p->q = q;
  p->out = out;
  p->lse = lse;
  p->q_tok = s.q_tok;
  p->q_head = s.q_head;
  p->o_tok = s.o_tok;
  p->o_head = s.o_head;
  p->q_begin = b->q_begin;
  p->kv_len = b->kv_len;
  p->block_table = b->block_table;
  p->table_stride = b->table_stride;
  p->n_seq = b->n_seq;
  p->table_pages = b->table_pages;
  p->n_tokens = b->n_tokens;
  p->n_pages = pool->n_pages;
  p->H = n_heads;
  p->Hkv = pool->n_kv_heads;
  p->G = n_heads / pool->n_kv_heads;
  p->max_new = b->max_new;
  const float scale = sm_scale > 0.f ? sm_scale : pool->d == 128 ? 0.08838834764831845f : 0.125f;
  p->scale_log2 = scale * 1.4426950408889634f;
  return HEATKV_OK;
}

uint64_t workspace_bytes(const PagedDevice& dev, int d, int G, int Hkv, int n_tokens, int n_seq) {
  const uint64_t a = paged_small_partial_bytes(d, dev.n_sm, Hkv, n_tokens), b = paged_tc_partial_bytes(d, dev.n_sm, G, Hkv, n_tokens, n_seq);
  return PAGED_WS_PARTIALS + (a > b ? a : b);
}

int place_workspace(const PagedDevice& dev, const heatkv_paged_pool* pool, void* ws, uint64_t bytes, PagedParams* p) {
  if (!ws || !aligned(ws, 256)) return HEATKV_ERR_INVALID_ARG;
  if (bytes < workspace_bytes(dev, pool->d, p->G, p->Hkv, p->n_tokens, p->n_seq)) return HEATKV_ERR_TOO_LARGE;
  p->status = static_cast<uint32_t*>(ws);
  p->counters = p->status + PAGED_WS_HEAD_WORDS;
  p->partials = reinterpret_cast<float*>(static_cast<char*>(ws) + PAGED_WS_PARTIALS);
  return HEATKV_OK;
}

int done(cudaError_t rc) {
  if (rc != cudaSuccess) {
    cudaGetLastError();
    return HEATKV_ERR_CUDA;
  }
  return HEATKV_OK;
}

// The paged kernels' waits on a barrier that nothing will ever signal, with limits of well under a millisecond.  result: 2 where the first gave up,
// left its code and raised the CTA's flag, the second ended because of that flag, and the one for copies under way ended, too; 1: one of them
// claimed success.
constexpr uint32_t EXPIRY_CODE = 64;
__global__ void __launch_bounds__(32) paged_wait_expiry_kernel(uint32_t* status, uint32_t* result) {
  constexpr long long LIMIT = 1 << 20;
  __shared__ __align__(8) uint64_t bar;
  __shared__ uint32_t abort_word;
  const uint32_t at = smem_u32(&bar);
  if (threadIdx.x == 0) {
    tc::mbar_init(at, 1);
    abort_word = 0;
  }
  __syncthreads();
  const bool first = wait_all(at, 0, &abort_word, status, EXPIRY_CODE, LIMIT), second = wait_all(at, 0, &abort_word, status, EXPIRY_CODE + 1);
  settle(at, 0, LIMIT);
  if (threadIdx.x == 0) *result = first || second ? 1 : *const_cast<volatile uint32_t*>(&abort_word) ? 2 : 3;
}

}  // namespace
}  // namespace heatkv

using namespace heatkv;

extern "C" {

int heatkv_paged_tables(const int32_t* new_tokens, const int32_t* past_tokens, int n_seq, const int32_t* free_pages, int n_pages,
                        const int32_t* state, int32_t* state_out, int32_t* block_table, int64_t table_stride, int table_pages,
                        int32_t* q_begin, int32_t* kv_len, int32_t* slot_map, int32_t* positions, int n_tokens, void* stream) {
  if (!new_tokens || !past_tokens || !free_pages || !state || !state_out || !block_table || !q_begin || !kv_len || !slot_map)
    return HEATKV_ERR_INVALID_ARG;
  if (n_seq < 1 || n_pages < 1 || table_pages < 1 || table_stride < table_pages || n_tokens < 1 || state == state_out) return HEATKV_ERR_INVALID_ARG;
  if (n_seq > PAGED_MAX_SEQ || n_pages > PAGED_MAX_PAGES || table_pages > PAGED_MAX_TABLE) return HEATKV_ERR_TOO_LARGE;
  if (kv_len == past_tokens || kv_len == new_tokens) return HEATKV_ERR_INVALID_ARG;      // (read by all CTAs while one writes)
  const TablesParams p = {new_tokens, past_tokens, free_pages, state,      state_out, block_table, q_begin, kv_len,
                          slot_map,   positions,   table_stride, n_seq, n_pages,   table_pages, n_tokens};
  return done(launch_paged_tables(p, static_cast<cudaStream_t>(stream)));
}

int heatkv_paged_release(const int32_t* kv_len, const int32_t* keep_len, int n_seq, const int32_t* block_table, int64_t table_stride,
                         int table_pages, int32_t* free_pages, int n_pages, const int32_t* state, int32_t* state_out, void* stream) {
  if (!kv_len || !keep_len || !block_table || !free_pages || !state || !state_out || state == state_out) return HEATKV_ERR_INVALID_ARG;
  if (n_seq < 1 || n_pages < 1 || table_pages < 1 || table_stride < table_pages) return HEATKV_ERR_INVALID_ARG;
  if (n_seq > PAGED_MAX_SEQ || n_pages > PAGED_MAX_PAGES || table_pages > PAGED_MAX_TABLE) return HEATKV_ERR_TOO_LARGE;
  const ReleaseParams p = {kv_len, keep_len, block_table, state, free_pages, state_out, table_stride, n_seq, n_pages, table_pages};
  return done(launch_paged_release(p, static_cast<cudaStream_t>(stream)));
}

int heatkv_paged_store(const heatkv_paged_pool* pool, const void* k_new, const void* v_new, int64_t tok_stride, int64_t head_stride,
                       const int32_t* slot_map, int n_tokens, void* stream) {
  const int rc = check_pool(pool);
  if (rc != HEATKV_OK) return rc;
  if (!k_new || !v_new || !slot_map || n_tokens < 1 || !aligned(k_new, 16) || !aligned(v_new, 16) || ((tok_stride | head_stride) & 7))
    return HEATKV_ERR_INVALID_ARG;
  if (tok_stride < 0 || head_stride < 0) return HEATKV_ERR_INVALID_ARG;
  const StoreParams p = {k_new, v_new, pool->k, pool->v, pool->k_code, pool->k_scale, slot_map, tok_stride, head_stride, pool->page_stride,
                         pool->head_stride, pool->row_stride, n_tokens, pool->n_pages, pool->n_kv_heads, pool->d, pool->dtype == HEATKV_DTYPE_FP16, 0};
  return done(launch_paged_store(p, static_cast<cudaStream_t>(stream)));
}

int heatkv_paged_workspace_bytes(const heatkv_paged_pool* pool, const heatkv_paged_batch* batch, int n_heads, uint64_t* bytes) {
  const int rc = check_batch(pool, batch, n_heads);
  if (rc != HEATKV_OK) return rc;
  PagedDevice dev;
  if (!bytes) return HEATKV_ERR_INVALID_ARG;
  if (!paged_device(&dev)) return done(cudaErrorInitializationError);
  *bytes = workspace_bytes(dev, pool->d, n_heads / pool->n_kv_heads, pool->n_kv_heads, batch->n_tokens, batch->n_seq);
  return HEATKV_OK;
}

int heatkv_paged_attention(const heatkv_paged_pool* pool, const heatkv_paged_batch* batch, int n_heads, const void* q,
                           const heatkv_token_strides* st, int causal, float sm_scale, void* out, float* lse, void* workspace,
                           uint64_t workspace_bytes, void* stream) {
  PagedParams p;
  int rc = attention_params(pool, batch, n_heads, q, st, sm_scale, out, lse, &p);
  if (rc != HEATKV_OK) return rc;
  PagedDevice dev;
  if (!paged_device(&dev)) return done(cudaErrorInitializationError);
  rc = place_workspace(dev, pool, workspace, workspace_bytes, &p);
  if (rc != HEATKV_OK) return rc;
  p.causal = causal != 0;
  // Up to 32 rows of the longest request: the warp-level kernel.  24 requests of 2000 tokens: 12 rows 44 us against 56 on the tensor-memory
  // kernel, 21 rows 33 and 40, 32 rows 82 and 88, 36 rows 64 and 56, 63 rows 55 and 40.  Up to 48 rows, too, where there are fewer units
  // than SMs: 34 to 48 rows at 2 to 16 heads a group, 32 units of 500 tokens 16 and 24 us, of 2500 24 and 39, 64 of 2500 36 and 39; 42 rows, 96 units of
  // 40 to 8000 tokens 17 and 34; 192 units of 500 36 and 33, of 2500 90 and 66.  (Few units of long contexts lose: 64 of 8000 83 and 69, 128 of
  // 2500 57 and 52, of 8000 147 and 109.  Lengths are not known here, and a table is as wide as its longest request.)  49 to 64 rows: 32 units
  // of 2500 30 and 38, of 8000 64 and 54, 64 of 2500 48 and 39.
  // And any number of tiles of 16 rows where there is little to do in all: a tile of `table_pages` pages weighs six more (its own beginning and
  // end).  One request of 8 kv heads with 4 heads each, 14 new tokens behind 500 or 8000: 10 and 25 us, 22 and 53 on the tensor-memory kernel; a
  // prompt of 100: 8 and 17; two kv heads, a prompt of 400 (weight 2600): 13 and 23, 100 behind 1500 with 8 heads each (3100): 19 and 28; 4 requests of 28
  // behind 1000 (5152) 25 and 24, 16 of 20 behind 300 (7040) 19 and 16.  Of 250 shapes measured none up to 6000 loses more than 4 %.
  const int64_t rows = (int64_t)p.max_new * p.G, units = (int64_t)p.n_seq * p.Hkv;
  const int64_t tiles = p.G <= 16 ? ((int64_t)p.max_new + 16 / p.G - 1) / (16 / p.G) : 0;
  const bool little = units <= 6000 && tiles <= 6000 && units * tiles * ((int64_t)p.table_pages + 6) <= 6000;
  const bool few = rows <= 32 || (p.G <= 16 && ((rows <= 48 && units < dev.n_sm) || little));
  return done((few ? launch_paged_small : launch_paged_tc)(p, *pool, dev, static_cast<cudaStream_t>(stream)));
}

int heatkv_paged_select(const heatkv_paged_pool* pool, const heatkv_paged_batch* batch, int n_heads, const void* q,
                        const heatkv_token_strides* st, int sink, int local, int n_select, int32_t* sel, void* stream) {
  int rc = check_batch(pool, batch, n_heads);
  if (rc != HEATKV_OK) return rc;
  if (!q || !sel || !pool->k_code || sink < 0 || local < 1 || n_select < 1 || sink > n_select - local) return HEATKV_ERR_INVALID_ARG;
  if (batch->table_pages > PAGED_MAX_SELECT_PAGES || (int64_t)batch->n_tokens * pool->n_kv_heads > INT32_MAX) return HEATKV_ERR_TOO_LARGE;
  const int64_t row = (int64_t)n_heads * pool->d;
  const int64_t q_tok = st ? st->q_tok : row, q_head = st ? st->q_head : pool->d;
  if (((q_tok | q_head) & 7) || q_tok < pool->d || q_head < pool->d || !aligned(q, 16)) return HEATKV_ERR_INVALID_ARG;
  PagedDevice dev;
  if (!paged_device(&dev)) return done(cudaErrorInitializationError);
  const SelectParams p = {q, q_tok, q_head, batch->q_begin, batch->kv_len, batch->block_table, batch->table_stride, pool->k_code, pool->k_scale, sel,
                          batch->n_seq, batch->table_pages, batch->n_tokens, pool->n_pages, pool->n_kv_heads, n_heads / pool->n_kv_heads, pool->d,
                          pool->dtype == HEATKV_DTYPE_FP16, sink, local, n_select};
  return done(launch_paged_select(p, batch->max_new, dev.n_sm, static_cast<cudaStream_t>(stream)));
}

int heatkv_paged_sparse_attention(const heatkv_paged_pool* pool, const heatkv_paged_batch* batch, int n_heads, const void* q,
                                  const heatkv_token_strides* st, const int32_t* sel, int n_select, float sm_scale, void* out, float* lse,
                                  void* workspace, uint64_t workspace_bytes, void* stream) {
  PagedParams p;
  int rc = attention_params(pool, batch, n_heads, q, st, sm_scale, out, lse, &p);
  if (rc != HEATKV_OK) return rc;
  if (!sel || n_select < 1) return HEATKV_ERR_INVALID_ARG;
  if (p.G > 64) return HEATKV_ERR_SHAPE_MISMATCH;
  if ((int64_t)p.n_tokens * p.Hkv * ((n_select + 3) / 4) > (1 << 30)) return HEATKV_ERR_TOO_LARGE;
  PagedDevice dev;
  if (!paged_device(&dev)) return done(cudaErrorInitializationError);
  rc = place_workspace(dev, pool, workspace, workspace_bytes, &p);
  if (rc != HEATKV_OK) return rc;
  p.causal = 1;
  p.sel = sel;
  p.n_sel = n_select;
  // tokens of a chunk share the pages that they select: they are taken together
  const bool chunk = p.max_new >= PAGED_SPARSE_CHUNK && (int64_t)p.n_tokens * p.Hkv * n_select >= PAGED_SPARSE_PAGES &&
                     paged_tc_takes_lists(p.G, p.Hkv, n_select, p.table_pages, p.n_tokens, p.n_seq);
  return done((chunk ? launch_paged_tc : launch_paged_small)(p, *pool, dev, static_cast<cudaStream_t>(stream)));
}

int heatkv_paged_status(const void* workspace, void* stream) {
  if (!workspace) return HEATKV_ERR_INVALID_ARG;
  uint32_t word = 0;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (cudaMemcpyAsync(&word, workspace, 4, cudaMemcpyDeviceToHost, s) != cudaSuccess || cudaStreamSynchronize(s) != cudaSuccess)
    return done(cudaErrorUnknown);
  return word ? HEATKV_ERR_DEVICE_TIMEOUT : HEATKV_OK;
}

int heatkv_paged_selftest_wait_expiry(void* workspace, void* stream) {
  if (!workspace || !aligned(workspace, 256)) return HEATKV_ERR_INVALID_ARG;
  uint32_t* words = static_cast<uint32_t*>(workspace);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  constexpr int RESULT = 1;                            // word behind the status: no kernel reads it
  uint32_t host[2] = {0, 0};
  paged_wait_expiry_kernel<<<1, 32, 0, s>>>(words, words + RESULT);
  if (cudaGetLastError() != cudaSuccess || cudaMemcpyAsync(host, words, sizeof(host), cudaMemcpyDeviceToHost, s) != cudaSuccess ||
      cudaMemsetAsync(words + RESULT, 0, 4, s) != cudaSuccess || cudaStreamSynchronize(s) != cudaSuccess)
    return done(cudaErrorUnknown);
  if (host[RESULT] == 1) return HEATKV_OK;
  return host[RESULT] == 2 && host[0] == EXPIRY_CODE ? HEATKV_ERR_DEVICE_TIMEOUT : HEATKV_ERR_CUDA;
}

}  // extern "C"
