// Rows of a block table between steps: rows that go on as copies of others, are cut back or end (fork), tokens that leave a request (compact), and
// the moves of K and V that either takes.
//
// Which pages are shared is nowhere kept: both calls mark the pages that the old table lists and those that the new one does, and what is only in
// the first goes to the ring of free pages, in page order, so that the result does not depend on which CTA came first.  All of it is chains of a few
// loads over tables of some thousand entries: what bounds it is the number of launches and of dependent loads.
#include <algorithm>

#include "paged_rows.cuh"

namespace heatkv {
namespace {

constexpr int RT = 256;                        // threads of a CTA
constexpr int DECIDE_THREADS = 1024;
enum Mark : uint32_t { OLD = 1, WHOLE = 2, PART = 4 };   // listed by the old table; by the new one, all of the page or its first rows

__device__ __forceinline__ int pages_of(int tokens) { return (tokens + PAGE - 1) / PAGE; }
__device__ __forceinline__ int length_of(const RowsParams& p, int i) { return min(max(p.lengths[i], 0), p.table_pages * PAGE); }
__device__ __forceinline__ bool valid(const RowsParams& p, int page) { return page >= 0 && page < p.n_pages; }
__device__ __forceinline__ int ring_at(const RowsParams& p, int64_t i) { return p.free_pages[(int)(i % p.n_pages)]; }
__device__ __forceinline__ int ring_head(const RowsParams& p) { return (p.state_in[0] % p.n_pages + p.n_pages) % p.n_pages; }
__device__ __forceinline__ int ring_count(const RowsParams& p) { return min(max(p.state_in[1], 0), p.n_pages); }

// Exclusive sum over a CTA of W warps; `all` gets the sum.
template <int W>
__device__ __forceinline__ int64_t exclusive_sum(int64_t v, int64_t* sums, int64_t& all) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int64_t inc = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t up = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += up;
  }
  __syncthreads();
  if (lane == 31) sums[warp] = inc;
  __syncthreads();
  int64_t before = 0;
  all = 0;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    const int64_t x = sums[w];
    if (w < warp) before += x;
    all += x;
  }
  return before + inc - v;
}

// ------------------------------------------------------------------------------------------------ fork
// The row that a partly filled page stays with: one that goes on as itself before the others, then the lowest; larger is better, 0 is none.
__device__ __forceinline__ uint32_t claim(int parent, int row) { return 2 * PAGED_MAX_SEQ - (parent == row ? row : PAGED_MAX_SEQ + row); }

// CTA (x, i): row i's entries; marks of the old and the new lists.
__global__ void __launch_bounds__(RT) fork_mark_kernel(const RowsParams p) {
  pdl_trigger();
  pdl_wait();
  const int i = blockIdx.y, had = pages_of(length_of(p, i));
  const int parent = p.parents[i];
  const bool on = parent >= 0 && parent < p.n_seq;
  const int length = on ? min(length_of(p, parent), p.keep_len ? max(p.keep_len[i], 0) : INT32_MAX) : 0, whole = length / PAGE, rest = length % PAGE;
  for (int j = blockIdx.x * RT + threadIdx.x; j < p.table_pages; j += gridDim.x * RT) {
    if (j < had) {
      const int page = p.table[i * p.table_stride + j];
      if (valid(p, page)) atomicOr(p.marks + page, OLD);
    }
    int page = -1;
    if (j < whole + (rest > 0)) {
      page = p.table[parent * p.table_stride + j];
      if (valid(p, page)) {
        atomicOr(p.marks + page, j < whole ? WHOLE : PART);
        if (j == whole) atomicMax(p.claims + page, claim(parent, i));
      }
    }
    p.table_out[i * p.out_stride + j] = page;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) p.lengths_out[i] = length;
}

// Pages of chunk c that go back.
__device__ __forceinline__ bool goes_back(const RowsParams& p, int page) { return (p.marks[page] & (OLD | WHOLE | PART)) == OLD; }

// CTA 0: who gets a page of its own for its last tokens; the others: how many pages of each chunk go back.
__global__ void __launch_bounds__(DECIDE_THREADS) fork_decide_kernel(const RowsParams p) {
  __shared__ int64_t sums[DECIDE_THREADS / 32];
  pdl_trigger();
  pdl_wait();
  int64_t all;
  if (blockIdx.x > 0) {
    const int c = blockIdx.x - 1;
    const int64_t first = (int64_t)c * p.chunk, end = min(first + p.chunk, (int64_t)p.n_pages);
    int64_t mine = 0;
    for (int64_t page = first + threadIdx.x; page < end; page += DECIDE_THREADS) mine += goes_back(p, (int)page);
    exclusive_sum<DECIDE_THREADS / 32>(mine, sums, all);
    if (threadIdx.x == 0) p.chunk_sums[c] = (int)all;
    return;
  }
  constexpr int PER = PAGED_MAX_SEQ / DECIDE_THREADS;
  const int i0 = threadIdx.x * PER, head = ring_head(p), free = ring_count(p);
  int page[PER];
  int64_t mine = 0;
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    const int i = i0 + u;
    page[u] = -1;
    if (i >= p.n_seq) continue;
    const int length = p.lengths_out[i];
    if (length % PAGE == 0) continue;
    const int last = p.table_out[i * p.out_stride + length / PAGE];
    if (!valid(p, last)) continue;
    if ((p.marks[last] & WHOLE) || p.claims[last] != claim(p.parents[i], i)) {
      page[u] = last;
      ++mine;
    }
  }
  int64_t rank = exclusive_sum<DECIDE_THREADS / 32>(mine, sums, all);
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    const int i = i0 + u;
    if (i >= p.n_seq) continue;
    int2 move = make_int2(-1, -1);
    if (page[u] >= 0) {
      const int length = p.lengths_out[i];
      int fresh = -1;
      if (rank < free) {
        fresh = ring_at(p, head + rank);
        move = make_int2(page[u], fresh);
      } else {
        p.lengths_out[i] = length / PAGE * PAGE;
      }
      p.table_out[i * p.out_stride + length / PAGE] = fresh;
      ++rank;
    }
    p.row_moves[i] = move;
  }
  if (threadIdx.x == 0) {
    const int taken = (int)min(all, (int64_t)free);
    p.totals[0] = taken;
    p.totals[1] = (int)(all - taken);
  }
}

// Pages that go back to the ring's end, chunk by chunk in page order; marks made zero for the next call.  Gives the number of all of them.
__device__ __forceinline__ int64_t give_back(const RowsParams& p, int64_t* sums) {
  int64_t before = 0, all, total;
  const int c = blockIdx.x;
  int64_t mine = 0, upto = 0;
  for (int x = threadIdx.x; x < p.chunks; x += RT) {
    const int n = p.chunk_sums[x];
    mine += n;
    if (x < c) upto += n;
  }
  exclusive_sum<RT / 32>(mine, sums, total);
  exclusive_sum<RT / 32>(upto, sums, before);
  const int head = ring_head(p), free = ring_count(p);
  if (c < p.chunks) {
    const int64_t first = (int64_t)c * p.chunk, end = min(first + p.chunk, (int64_t)p.n_pages);
    for (int64_t base = first; base < end; base += RT) {
      const int64_t page = base + threadIdx.x;
      const bool back = page < end && goes_back(p, (int)page);
      const int64_t at = before + exclusive_sum<RT / 32>(back, sums, all);
      if (back) p.free_pages[(int)((head + free + at) % p.n_pages)] = (int)page;
      if (page < end) p.marks[page] = p.claims[page] = 0;
      before += all;
    }
  }
  return total;
}

__global__ void __launch_bounds__(RT) fork_end_kernel(const RowsParams p) {
  __shared__ int64_t sums[RT / 32];
  pdl_trigger();
  pdl_wait();
  const int64_t back = give_back(p, sums);
  for (int64_t x = (int64_t)blockIdx.x * RT + threadIdx.x; x < (int64_t)p.n_seq * PAGE; x += (int64_t)gridDim.x * RT) {
    const int i = (int)(x / PAGE), r = (int)(x % PAGE);
    const int2 move = p.row_moves[i];
    const bool moves = move.y >= 0 && r < p.lengths_out[i] % PAGE;
    p.move_from[x] = moves ? move.x * PAGE + r : -1;
    p.move_to[x] = moves ? move.y * PAGE + r : -1;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    const int taken = p.totals[0];
    p.state_out[0] = (int)(((int64_t)ring_head(p) + taken) % p.n_pages);
    p.state_out[1] = (int)(ring_count(p) - taken + back);
    p.state_out[2] = p.totals[1];
    p.state_out[3] = (int)back;
  }
}

// ------------------------------------------------------------------------------------------------ compact
// The tokens of a page that stay, as bits: lane l looks at tokens l and l + 32.
__device__ __forceinline__ uint64_t staying(const RowsParams& p, int i, int j, int length, int lane) {
  uint64_t bits = 0;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int t = j * PAGE + u * 32 + lane;
    const bool stays = t < length && (t >= p.mask_width || p.mask[i * p.mask_stride + t] != 0);
    bits |= (uint64_t)__ballot_sync(0xffffffffu, stays) << (32 * u);
  }
  return bits;
}

// A warp per page: how many of its tokens stay, and the old table's marks.
__global__ void __launch_bounds__(RT) compact_count_kernel(const RowsParams p) {
  pdl_trigger();
  pdl_wait();
  const int i = blockIdx.y, length = length_of(p, i), pages = pages_of(length), lane = threadIdx.x & 31;
  for (int j = blockIdx.x * (RT / 32) + (threadIdx.x >> 5); j < pages; j += gridDim.x * (RT / 32)) {
    const int stay = __popcll(staying(p, i, j, length, lane));
    if (lane == 0) {
      p.page_stay[(int64_t)i * p.table_pages + j] = stay;
      const int page = p.table[i * p.table_stride + j];
      if (valid(p, page)) atomicOr(p.marks + page, OLD);
    }
  }
}

// A CTA per row: its first page that something leaves, and the tokens before every page from there on.
__global__ void __launch_bounds__(RT) compact_row_kernel(const RowsParams p) {
  __shared__ int64_t sums[RT / 32];
  __shared__ int first;
  pdl_trigger();
  pdl_wait();
  const int i = blockIdx.x, length = length_of(p, i), pages = pages_of(length);
  int32_t* stay = p.page_stay + (int64_t)i * p.table_pages;
  if (threadIdx.x == 0) first = INT32_MAX;
  __syncthreads();
  for (int j = threadIdx.x; j < pages; j += RT)
    if (stay[j] < min(PAGE, length - j * PAGE)) {
      atomicMin(&first, j);
      break;
    }
  __syncthreads();
  const int j0 = first;
  int64_t before = 0, all;
  for (int base = min(j0, pages); base < pages; base += RT) {
    const int j = base + threadIdx.x, n = j < pages ? stay[j] : 0;
    const int64_t at = before + exclusive_sum<RT / 32>(n, sums, all);
    if (j < pages) stay[j] = (int)at;
    before += all;
  }
  if (threadIdx.x == 0) p.row_moves[i] = make_int2(j0 == INT32_MAX ? -1 : j0, (int)before);
}

// What the rows before row i take, and whether it is served: every CTA sums up for itself.
struct RowPlan {
  int first, moved;                            // first page that changes (-1: none, or refused), tokens that move
  int64_t page_rank, move_rank;                // fresh pages and moves of the rows before
};
__device__ __forceinline__ RowPlan plan_row(const RowsParams& p, int i, int64_t* sums, bool last, int64_t (&totals)[3]) {
  // (rows before i; with `last`, all rows, and the totals: pages taken, rows refused, moves)
  const int free = ring_count(p), n = last ? p.n_seq : i + 1, per = (n + RT - 1) / RT, x0 = min((int)threadIdx.x * per, n), x1 = min(x0 + per, n);
  __shared__ RowPlan mine;
  int64_t need = 0, moves = 0, all_need, all_moves;
  for (int x = x0; x < x1; ++x) {
    const int2 r = p.row_moves[x];
    if (r.x >= 0) {
      need += pages_of(r.y);
      moves += r.y;
    }
  }
  int64_t a = exclusive_sum<RT / 32>(need, sums, all_need), b = exclusive_sum<RT / 32>(moves, sums, all_moves);
  int64_t taken = 0, refused = 0, moved = 0;
  for (int x = x0; x < x1; ++x) {
    const int2 r = p.row_moves[x];
    const int want = r.x >= 0 ? pages_of(r.y) : 0;
    const bool served = r.x >= 0 && (want == 0 || (a + want <= free && b + r.y <= p.n_moves));
    if (x == i) mine = {served ? r.x : -1, r.y, a, b};
    if (want > 0) {
      taken = served ? a + want : taken;
      moved = served ? b + r.y : moved;
      refused += !served;
      a += want;
      b += r.y;
    }
  }
  __syncthreads();
  if (last) {
    __shared__ unsigned long long most[2];
    if (threadIdx.x == 0) most[0] = most[1] = 0;
    __syncthreads();
    atomicMax(&most[0], (unsigned long long)taken);
    atomicMax(&most[1], (unsigned long long)moved);
    exclusive_sum<RT / 32>(refused, sums, totals[1]);
    __syncthreads();
    totals[0] = (int64_t)most[0];
    totals[2] = (int64_t)most[1];
  }
  return mine;
}

// CTA (x, i): row i's new entries, marks and moves.
__global__ void __launch_bounds__(RT) compact_place_kernel(const RowsParams p) {
  __shared__ int64_t sums[RT / 32];
  pdl_trigger();
  pdl_wait();
  const int i = blockIdx.y, length = length_of(p, i), pages = pages_of(length), lane = threadIdx.x & 31, head = ring_head(p);
  int64_t totals[3];
  const RowPlan r = plan_row(p, i, sums, false, totals);
  const int32_t* stay = p.page_stay + (int64_t)i * p.table_pages;
  const int first = r.first >= 0 ? r.first : pages, fresh = r.first >= 0 ? pages_of(r.moved) : 0;
  for (int j = blockIdx.x * RT + threadIdx.x; j < p.table_pages; j += gridDim.x * RT) {
    int page = -1;
    if (j < first) {
      page = p.table[i * p.table_stride + j];
      if (valid(p, page)) atomicOr(p.marks + page, WHOLE);
    } else if (j < first + fresh) {
      page = ring_at(p, head + r.page_rank + (j - first));
    }
    p.table_out[i * p.out_stride + j] = page;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) p.lengths_out[i] = r.first >= 0 ? first * PAGE + r.moved : length;
  if (r.first < 0) return;
  for (int j = first + blockIdx.x * (RT / 32) + (threadIdx.x >> 5); j < pages; j += gridDim.x * (RT / 32)) {
    const uint64_t bits = staying(p, i, j, length, lane);
    const int page = p.table[i * p.table_stride + j], before = stay[j];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int at = u * 32 + lane;
      if (!(bits >> at & 1)) continue;
      const int rank = before + __popcll(bits & (((uint64_t)1 << at) - 1));
      const int to = ring_at(p, head + r.page_rank + rank / PAGE);
      const bool moves = valid(p, page) && valid(p, to);
      p.move_from[r.move_rank + rank] = moves ? page * PAGE + at : -1;
      p.move_to[r.move_rank + rank] = moves ? to * PAGE + rank % PAGE : -1;
    }
  }
}

__global__ void __launch_bounds__(DECIDE_THREADS) compact_chunk_kernel(const RowsParams p) {
  __shared__ int64_t sums[DECIDE_THREADS / 32];
  pdl_trigger();
  pdl_wait();
  const int64_t first = (int64_t)blockIdx.x * p.chunk, end = min(first + p.chunk, (int64_t)p.n_pages);
  int64_t mine = 0, all;
  for (int64_t page = first + threadIdx.x; page < end; page += DECIDE_THREADS) mine += goes_back(p, (int)page);
  exclusive_sum<DECIDE_THREADS / 32>(mine, sums, all);
  if (threadIdx.x == 0) p.chunk_sums[blockIdx.x] = (int)all;
}

__global__ void __launch_bounds__(RT) compact_end_kernel(const RowsParams p) {
  __shared__ int64_t sums[RT / 32];
  pdl_trigger();
  pdl_wait();
  const int64_t back = give_back(p, sums);
  int64_t totals[3];
  plan_row(p, 0, sums, true, totals);
  for (int64_t x = totals[2] + (int64_t)blockIdx.x * RT + threadIdx.x; x < p.n_moves; x += (int64_t)gridDim.x * RT) p.move_from[x] = p.move_to[x] = -1;
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    p.state_out[0] = (int)((ring_head(p) + totals[0]) % p.n_pages);
    p.state_out[1] = (int)(ring_count(p) - totals[0] + back);
    p.state_out[2] = (int)totals[1];
    p.state_out[3] = (int)totals[2];
  }
}

// ------------------------------------------------------------------------------------------------ moves
constexpr int MT = 256;

// Rows of K and V of all heads, 16 bytes at a time.
__global__ void __launch_bounds__(MT) move_kernel(const MoveParams p) {
  pdl_trigger();
  pdl_wait();
  const uint32_t n_slots = (uint32_t)p.n_pages * PAGE;
  const int ch = p.d / 8, words = p.Hkv * ch;
  const int64_t x = (int64_t)blockIdx.x * MT + threadIdx.x, e = x / words;
  const int w = (int)(x - e * words), h = w / ch, c = w - h * ch;
  if (e >= p.n_moves) return;
  const uint32_t from = (uint32_t)p.from[e], to = (uint32_t)p.to[e];
  if (from >= n_slots || to >= n_slots) return;
  auto at = [&](uint32_t slot) { return (int64_t)(slot / PAGE) * p.page_stride + h * p.head_stride + (int64_t)(slot % PAGE) * p.row_stride + c * 8; };
  const int64_t a = at(from), b = at(to);
  const int4 k = *reinterpret_cast<const int4*>(static_cast<const __nv_bfloat16*>(p.k) + a);
  const int4 v = *reinterpret_cast<const int4*>(static_cast<const __nv_bfloat16*>(p.v) + a);
  *reinterpret_cast<int4*>(static_cast<__nv_bfloat16*>(p.k) + b) = k;
  *reinterpret_cast<int4*>(static_cast<__nv_bfloat16*>(p.v) + b) = v;
}

// The same of a cache in 4 bits: eight words of K's codes, eight of V's and one of scales each, of d / 16 bytes.
template <int D>
__global__ void __launch_bounds__(MT) move4_kernel(const MoveParams p) {
  using B = Block4<D>;
  using Word = typename std::conditional<D == 128, uint2, uint32_t>::type;
  constexpr int WORDS = 18;
  pdl_trigger();
  pdl_wait();
  const uint32_t n_slots = (uint32_t)p.n_pages * PAGE;
  const int words = p.Hkv * WORDS;
  const int64_t x = (int64_t)blockIdx.x * MT + threadIdx.x, e = x / words;
  const int w = (int)(x - e * words), h = w / WORDS, c = w - h * WORDS;
  if (e >= p.n_moves) return;
  const uint32_t from = (uint32_t)p.from[e], to = (uint32_t)p.to[e];
  if (from >= n_slots || to >= n_slots) return;
  auto at = [&](uint32_t slot) {
    const int row = (int)(slot % PAGE);
    const int in = c < 8 ? B::K + row * B::ROW + c * (int)sizeof(Word) : c < 16 ? B::V + row * B::ROW + (c - 8) * (int)sizeof(Word)
                 : (c == 16 ? B::KS : B::VS) + row * B::SCALES;
    return reinterpret_cast<Word*>(static_cast<unsigned char*>(p.k) + (int64_t)(slot / PAGE) * p.page_stride + h * p.head_stride + in);
  };
  *at(to) = *at(from);
}

}  // namespace

uint64_t rows_workspace_bytes(int n_seq, int table_pages, int n_pages) {
  return ((uint64_t)2 * n_pages + ROWS_CHUNKS + 64 + 2 * (uint64_t)n_seq + (uint64_t)n_seq * table_pages) * 4;
}

void place_rows_workspace(void* ws, RowsParams* p) {
  p->chunk = std::max(1024, (p->n_pages + ROWS_CHUNKS - 1) / ROWS_CHUNKS);
  p->chunks = (p->n_pages + p->chunk - 1) / p->chunk;
  p->marks = static_cast<uint32_t*>(ws);
  p->claims = p->marks + p->n_pages;
  p->row_moves = reinterpret_cast<int2*>(p->claims + p->n_pages);
  p->chunk_sums = reinterpret_cast<int32_t*>(p->row_moves + p->n_seq);
  p->totals = p->chunk_sums + ROWS_CHUNKS;
  p->page_stay = p->totals + 64;
}

cudaError_t launch_paged_fork(const RowsParams& p, cudaStream_t stream) {
  cudaError_t rc = launch_pdl(fork_mark_kernel, dim3((unsigned)std::min(64, (p.table_pages + RT - 1) / RT), p.n_seq), dim3(RT), 0, stream, p);
  if (rc != cudaSuccess) return rc;
  rc = launch_pdl(fork_decide_kernel, dim3(1 + p.chunks), dim3(DECIDE_THREADS), 0, stream, p);
  if (rc != cudaSuccess) return rc;
  return launch_pdl(fork_end_kernel, dim3(std::max(p.chunks, std::min(148, (p.n_seq * PAGE + RT - 1) / RT))), dim3(RT), 0, stream, p);
}

cudaError_t launch_paged_compact(const RowsParams& p, cudaStream_t stream) {
  const dim3 by_page((unsigned)std::min(512, (p.table_pages + RT / 32 - 1) / (RT / 32)), p.n_seq);
  cudaError_t rc = launch_pdl(compact_count_kernel, by_page, dim3(RT), 0, stream, p);
  if (rc != cudaSuccess) return rc;
  rc = launch_pdl(compact_row_kernel, dim3(p.n_seq), dim3(RT), 0, stream, p);
  if (rc != cudaSuccess) return rc;
  rc = launch_pdl(compact_place_kernel, by_page, dim3(RT), 0, stream, p);
  if (rc != cudaSuccess) return rc;
  rc = launch_pdl(compact_chunk_kernel, dim3(p.chunks), dim3(DECIDE_THREADS), 0, stream, p);
  if (rc != cudaSuccess) return rc;
  return launch_pdl(compact_end_kernel, dim3(std::max(p.chunks, 64)), dim3(RT), 0, stream, p);
}

cudaError_t launch_paged_move(const MoveParams& p, int bits, cudaStream_t stream) {
  const int64_t words = (int64_t)p.n_moves * p.Hkv * (bits == 4 ? 18 : p.d / 8), blocks = (words + MT - 1) / MT;
  if (blocks > INT32_MAX) return cudaErrorInvalidValue;
  const dim3 grid((unsigned)blocks);
  if (bits == 16) return launch_pdl(move_kernel, grid, dim3(MT), 0, stream, p);
  return p.d == 128 ? launch_pdl(move4_kernel<128>, grid, dim3(MT), 0, stream, p) : launch_pdl(move4_kernel<64>, grid, dim3(MT), 0, stream, p);
}

}  // namespace heatkv
