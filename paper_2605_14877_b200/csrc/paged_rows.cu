// Rows of a block table between steps: rows that go on as copies of others, are cut back or end (fork), tokens that leave a request (compact), and
// the moves of K and V that either takes.
//
// Which pages are shared is nowhere kept: both calls mark the pages that the old table lists and those that the new one does, and what is only in
// the first goes to the ring of free pages, in page order, so that the result does not depend on which CTA came first.  All of it is chains of a few
// loads over tables of some thousand entries: what bounds it is the number of launches and of dependent loads.  So small pools and tables (one_cta) have their
// marks in one CTA's shared memory: a fork is one launch, where that CTA decides while others copy the entries that no
// decision changes (32 rows of 1 to 40 pages 4.9 us, in three launches with marks in global memory 10.1; 97 rows of 141 pages 7.4, by one CTA alone 10.3),
// and a compaction two, one CTA of the second seeing to the marks while the others list the moves (100 000 tokens of one row 9.0 us, 40 rows of 50 to 9000
// 8.4; the first with marks in global memory 16.8).
#include <algorithm>

#include "paged_rows.cuh"

namespace heatkv {
namespace {

constexpr int RT = 256;                        // threads of a CTA
constexpr int DECIDE_THREADS = 1024;
constexpr int PLACE_THREADS = 512, PLACE_PAGES = 32;                // .. that lists the moves of so many pages of a row at a time
// What one CTA sees to, with the pages' marks in its shared memory.  Its time grows with the rows (64 moves each, by that CTA alone) and the entries, that of the
// launches of many CTAs with the pages: a fork takes 0.5 to 0.9 of theirs with 4 to 96 rows, over 4000 pages 1.0 with 128, 1.15 with 160, 1.5 with 256, over 16 384
// pages 0.7, 0.85 and 1.1, and with 16 000 to 32 768 entries 0.8 to 1.0, with more 1.1 to 2.5; compactions the same of rows, and 0.7 to 0.9 below 8000 entries,
// 0.95 to 1.1 at 8000 to 16 000, 1.05 to 1.2 at 16 000 to 32 768.
constexpr int SMALL_PAGES = 16384, FORK_ENTRIES = 32768, COMPACT_ENTRIES = 12000;
__host__ __device__ constexpr int small_rows(int n_pages) { return 112 + n_pages / 192; }
inline bool one_cta(const RowsParams& p, int entries) {
  return p.n_pages <= SMALL_PAGES && p.n_seq <= small_rows(p.n_pages) && (int64_t)p.n_seq * p.table_pages <= entries;
}
static_assert(small_rows(SMALL_PAGES) <= DECIDE_THREADS, "a thread a row");
enum Mark : uint32_t { OLD = 1, WHOLE = 2, PART = 4 };   // listed by the old table; by the new one, all of the page or its first rows

__device__ __forceinline__ int pages_of(int tokens) { return (tokens + PAGE - 1) / PAGE; }
__device__ __forceinline__ int length_of(const RowsParams& p, int i) { return min(max(p.lengths[i], 0), p.table_pages * PAGE); }
__device__ __forceinline__ bool valid(const RowsParams& p, int page) { return page >= 0 && page < p.n_pages; }
// the ring's entry `i` places behind the oldest, i up to twice the pages (a table that lists pages which a full ring has, too)
__device__ __forceinline__ uint32_t ring_place(const RowsParams& p, int head, int64_t i) {
  uint32_t at = (uint32_t)head + (uint32_t)i;
#pragma unroll
  for (int u = 0; u < 2; ++u) at -= at < (uint32_t)p.n_pages ? 0u : (uint32_t)p.n_pages;
  return at;
}
__device__ __forceinline__ int ring_at(const RowsParams& p, int head, int64_t i) { return p.free_pages[ring_place(p, head, i)]; }
__device__ __forceinline__ int ring_head(const RowsParams& p) { return (p.state_in[0] % p.n_pages + p.n_pages) % p.n_pages; }
__device__ __forceinline__ int ring_count(const RowsParams& p) { return min(max(p.state_in[1], 0), p.n_pages); }

// Exclusive sums over a CTA of W warps, of K numbers of each thread; `all` gets the sums.  `sums` has K * W entries.
template <int W, int K>
__device__ __forceinline__ void exclusive_sums(int64_t (&v)[K], int64_t* sums, int64_t (&all)[K]) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  __shared__ int64_t total[K];
  auto scan = [&](int64_t x) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t up = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += up;
    }
    return x;
  };
  int64_t inc[K];
#pragma unroll
  for (int k = 0; k < K; ++k) inc[k] = scan(v[k]);
  __syncthreads();
#pragma unroll
  for (int k = 0; k < K; ++k)
    if (lane == 31) sums[k * W + warp] = inc[k];
  __syncthreads();
  if (warp < K) {                                // (every thread adding up all warps' sums took longer than this and another barrier)
    const int64_t x = lane < W ? sums[warp * W + lane] : 0, s = scan(x);
    if (lane < W) sums[warp * W + lane] = s - x;
    if (lane == 31) total[warp] = s;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < K; ++k) {
    all[k] = total[k];
    v[k] = sums[k * W + warp] + inc[k] - v[k];
  }
}
template <int W>
__device__ __forceinline__ int64_t exclusive_sum(int64_t v, int64_t* sums, int64_t& all) {
  int64_t x[1] = {v}, total[1];
  exclusive_sums<W>(x, sums, total);
  all = total[0];
  return x[0];
}

// Marks of up to SMALL_PAGES pages in shared memory, eight a word.
// (rows of a family list the same pages: a look is cheaper than the next atomic on the same word)
__device__ __forceinline__ void mark(uint32_t* flags, int page, uint32_t what) {
  uint32_t* word = flags + (page >> 3);
  what <<= (page & 7) * 4;
  if ((*const_cast<volatile uint32_t*>(word) & what) != what) atomicOr(word, what);
}
__device__ __forceinline__ int flag_words(int n_pages) { return (n_pages + 7) / 8; }
__device__ __forceinline__ bool goes_back(uint32_t mark) { return (mark & (OLD | WHOLE | PART)) == OLD; }
// row.use(j, row.load(j)) for all rows, row = make(its number), and j below `pages`, by a CTA of T threads: a row by a warp, or by all of them where
// rows are few.  Eight loads are on their way before the first is used.
template <int T, typename Make>
__device__ __forceinline__ void for_rows(int rows, int pages, Make make) {
  constexpr int AHEAD = 8;
  const bool few = rows < T / 64;
  const int at = few ? threadIdx.x : threadIdx.x & 31, step = few ? T : 32;
  for (int i = few ? 0 : threadIdx.x >> 5; i < rows; i += few ? 1 : T / 32) {
    const auto row = make(i);
    for (int base = at; base < pages; base += step * AHEAD) {
      decltype(row.load(0)) x[AHEAD];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u)
        if (base + u * step < pages) x[u] = row.load(base + u * step);
#pragma unroll
      for (int u = 0; u < AHEAD; ++u)
        if (base + u * step < pages) row.use(base + u * step, x[u]);
    }
  }
}
// Pages that go back to the ring's end, in page order, by a CTA of T threads; their number.
template <int T>
__device__ __forceinline__ int give_back_small(const RowsParams& p, const uint32_t* flags, int64_t* sums, int head, int free) {
  int64_t before = 0, all;
  const int words = flag_words(p.n_pages);
  for (int base = 0; base < words; base += T) {
    const int w = base + threadIdx.x;
    const uint32_t x = w < words ? flags[w] : 0;
    uint32_t back = 0;                           // (pages past the last have no marks)
#pragma unroll
    for (int u = 0; u < 8; ++u) back |= (uint32_t)goes_back(x >> 4 * u) << u;
    int64_t at = before + exclusive_sum<T / 32>(__popc(back), sums, all);
    for (; back; back &= back - 1) p.free_pages[ring_place(p, head, free + at++)] = w * 8 + __ffs(back) - 1;
    before += all;
  }
  return (int)before;
}

// ------------------------------------------------------------------------------------------------ fork
// The row that a partly filled page stays with: one that goes on as itself before the others, then the lowest; larger is better, 0 is none.
__device__ __forceinline__ uint32_t claim(int parent, int row) { return 2 * PAGED_MAX_SEQ - (parent == row ? row : PAGED_MAX_SEQ + row); }

// What a row lists, and how much of it rows that go on from it have whole: its marks.
struct ForkMarks {
  const int32_t* table;
  uint32_t* flags;
  int n_pages, pages, whole;
  __device__ __forceinline__ int load(int j) const { return j < pages ? table[j] : -1; }
  __device__ __forceinline__ void use(int j, int page) const {
    if ((uint32_t)page < (uint32_t)n_pages) mark(flags, page, j < whole ? OLD | WHOLE : OLD);
  }
};
struct ForkCopy {
  const int32_t* table;
  int32_t* out;
  int pages, last;                               // last: the entry of a page that is not full, which is not written here
  __device__ __forceinline__ int load(int j) const { return j < pages ? table[j] : -1; }
  __device__ __forceinline__ void use(int j, int page) const {
    if (j != last) out[j] = page;
  }
};
// A fork of few rows (one_cta): CTA 0 decides, the others copy full pages' entries, so many rows each.
__host__ __device__ constexpr int copied_rows(int n_seq) { return n_seq < DECIDE_THREADS / 64 ? 1 : DECIDE_THREADS / 32; }
__global__ void __launch_bounds__(DECIDE_THREADS) fork_small_kernel(const RowsParams p) {
  extern __shared__ uint32_t sm[];
  uint32_t* flags = sm;                                            // [flag_words]
  uint32_t* claims = flags + flag_words(p.n_pages);                // [n_pages]
  int32_t* had = reinterpret_cast<int32_t*>(claims + p.n_pages);   // [n_seq] tokens; then pages
  int32_t* length = had + p.n_seq;                                 // [n_seq] of the row that goes on
  int32_t* wholes = length + p.n_seq;                              // [n_seq] the most pages of the row that one which goes on from it has whole
  int2* move = reinterpret_cast<int2*>(sm + (flag_words(p.n_pages) + p.n_pages + 3 * p.n_seq + 1) / 2 * 2);    // [n_seq] {page with the last tokens, page to copy it to}
  __shared__ int64_t sums[DECIDE_THREADS / 32];
  pdl_trigger();
  if (blockIdx.x > 0) {
    pdl_wait();
    const int rows = copied_rows(p.n_seq), first = (blockIdx.x - 1) * rows;
    for_rows<DECIDE_THREADS>(min(rows, p.n_seq - first), p.table_pages, [&](int row) {
      const int i = first + row, of = p.parents[i];
      const bool on = of >= 0 && of < p.n_seq;
      const int n = on ? min(length_of(p, of), p.keep_len ? max(p.keep_len[i], 0) : INT32_MAX) : 0;
      return ForkCopy{p.table + (on ? of : 0) * p.table_stride, p.table_out + i * p.out_stride, pages_of(n), n % PAGE ? n / PAGE : -1};
    });
    return;
  }
  for (int i = threadIdx.x; i < flag_words(p.n_pages) + p.n_pages; i += DECIDE_THREADS) sm[i] = 0;
  pdl_wait();
  const int head = ring_head(p), free = ring_count(p), i = threadIdx.x;
  int of = -1, keep = INT32_MAX;
  if (i < p.n_seq) {
    had[i] = length_of(p, i);
    of = p.parents[i];
    if (p.keep_len) keep = max(p.keep_len[i], 0);
    if (of >= p.n_seq || of < 0) of = -1;
    wholes[i] = 0;
  }
  __syncthreads();
  int n = 0, last = -1, listed = -1;                               // this thread's row: its tokens, and the page with the last ones if that is not full
  if (i < p.n_seq && of >= 0) {
    n = min(had[of], keep);
    atomicMax(wholes + of, n / PAGE);
    if (n % PAGE) listed = p.table[of * p.table_stride + n / PAGE];
    if (valid(p, listed)) last = listed;
  }
  if (i < p.n_seq) length[i] = n;
  __syncthreads();
  if (last >= 0) {
    mark(flags, last, PART);
    atomicMax(claims + last, claim(of, i));
  }
  for_rows<DECIDE_THREADS>(p.n_seq, p.table_pages, [&](int row) {
    return ForkMarks{p.table + row * p.table_stride, flags, p.n_pages, pages_of(had[row]), wholes[row]};
  });
  __syncthreads();
  // who gets a page of its own for its last tokens
  const bool wants = last >= 0 && ((flags[last >> 3] >> (last & 7) * 4 & WHOLE) || claims[last] != claim(of, i));
  int64_t all;
  const int64_t rank = exclusive_sum<DECIDE_THREADS / 32>(wants, sums, all);
  if (i < p.n_seq) {
    int fresh = -1;
    if (wants && rank < free) fresh = ring_at(p, head, rank);
    if (n % PAGE) p.table_out[i * p.out_stride + n / PAGE] = wants ? fresh : listed;
    if (wants && fresh < 0) length[i] = n = n / PAGE * PAGE;
    move[i] = make_int2(last, fresh);
    p.lengths_out[i] = n;
  }
  const int back = give_back_small<DECIDE_THREADS>(p, flags, sums, head, free), taken = (int)min(all, (int64_t)free);
  __syncthreads();
  for (int x = threadIdx.x; x < p.n_seq * PAGE; x += DECIDE_THREADS) {
    const int row = x / PAGE, r = x % PAGE;
    const int2 m = move[row];
    const bool moves = m.y >= 0 && r < length[row] % PAGE;
    p.move_from[x] = moves ? m.x * PAGE + r : -1;
    p.move_to[x] = moves ? m.y * PAGE + r : -1;
  }
  if (threadIdx.x == 0) {
    p.state_out[0] = ring_place(p, head, taken);
    p.state_out[1] = free - taken + back;
    p.state_out[2] = (int)(all - taken);
    p.state_out[3] = back;
  }
}

// The others, in launches of many CTAs with their marks in global memory.
__global__ void __launch_bounds__(DECIDE_THREADS) zero_marks_kernel(const RowsParams p) {
  pdl_trigger();
  pdl_wait();
  for (int64_t x = (int64_t)blockIdx.x * DECIDE_THREADS + threadIdx.x; x < p.n_pages; x += (int64_t)gridDim.x * DECIDE_THREADS) p.marks[x] = p.claims[x] = 0;
}
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
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    p.lengths_out[i] = length;
    const int last = rest > 0 ? p.table[parent * p.table_stride + whole] : -1;
    p.row_moves[i] = make_int2(valid(p, last) ? last : -1, length);          // the page with its last tokens, if that is not full
  }
}

// Who gets a page of its own for its last tokens: a CTA with all rows, up to four a thread.
__global__ void __launch_bounds__(DECIDE_THREADS) fork_decide_kernel(const RowsParams p) {
  __shared__ int64_t sums[DECIDE_THREADS / 32];
  pdl_trigger();
  pdl_wait();
  int64_t all;
  constexpr int PER = PAGED_MAX_SEQ / DECIDE_THREADS;
  const int per = (p.n_seq + DECIDE_THREADS - 1) / DECIDE_THREADS, i0 = threadIdx.x * per, head = ring_head(p), free = ring_count(p);
  int2 row[PER];
  int64_t mine = 0;
#pragma unroll
  for (int u = 0; u < PER; ++u) row[u] = u < per && i0 + u < p.n_seq ? p.row_moves[i0 + u] : make_int2(-1, 0);
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    if (row[u].x < 0) continue;
    const uint32_t mark = p.marks[row[u].x], best = p.claims[row[u].x];
    if (!(mark & WHOLE) && best == claim(p.parents[i0 + u], i0 + u)) row[u].x = -1;          // it keeps the page
    else ++mine;
  }
  int64_t rank = exclusive_sum<DECIDE_THREADS / 32>(mine, sums, all);
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    const int i = i0 + u;
    if (u >= per || i >= p.n_seq) continue;
    int2 move = make_int2(-1, -1);
    if (row[u].x >= 0) {
      int fresh = -1;
      if (rank < free) {
        fresh = ring_at(p, head, rank);
        move = make_int2(row[u].x, fresh);
      } else {
        p.lengths_out[i] = row[u].y / PAGE * PAGE;
      }
      p.table_out[i * p.out_stride + row[u].y / PAGE] = fresh;
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

// Pages of a chunk of the pool, where there is more than one, that go back: how many.
__global__ void __launch_bounds__(RT) chunk_kernel(const RowsParams p) {
  __shared__ int64_t sums[RT / 32];
  pdl_trigger();
  pdl_wait();
  const int64_t first = (int64_t)blockIdx.x * p.chunk, end = min(first + p.chunk, (int64_t)p.n_pages);
  int64_t mine = 0, all;
  for (int64_t page = first + threadIdx.x; page < end; page += RT) mine += goes_back(p.marks[page]);
  exclusive_sum<RT / 32>(mine, sums, all);
  if (threadIdx.x == 0) p.chunk_sums[blockIdx.x] = (int)all;
}
// Pages that go back to the ring's end, chunk by chunk in page order, by CTAs of 1024 threads.  Gives the number of all of them to CTA 0.
__device__ __forceinline__ int64_t give_back(const RowsParams& p, int64_t* sums) {
  int64_t before = 0, all, total = 0;
  const int c = blockIdx.x;
  if (c >= p.chunks) return 0;
  if (p.chunks > 1) {
    int64_t mine = 0, upto = 0;
    for (int x = threadIdx.x; x < p.chunks; x += DECIDE_THREADS) {
      const int n = p.chunk_sums[x];
      mine += n;
      if (x < c) upto += n;
    }
    exclusive_sum<DECIDE_THREADS / 32>(mine, sums, total);
    exclusive_sum<DECIDE_THREADS / 32>(upto, sums, before);
  }
  const int head = ring_head(p), free = ring_count(p);
  const int64_t first = (int64_t)c * p.chunk, end = min(first + p.chunk, (int64_t)p.n_pages);
  constexpr int PER = 4;                       // neighbouring pages of a thread
  for (int64_t base = first; base < end; base += DECIDE_THREADS * PER) {
    const int64_t page0 = base + threadIdx.x * PER;
    bool back[PER];
    int n = 0;
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      back[u] = page0 + u < end && goes_back(p.marks[page0 + u]);
      n += back[u];
    }
    int64_t at = before + exclusive_sum<DECIDE_THREADS / 32>(n, sums, all);
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      if (back[u]) p.free_pages[ring_place(p, head, free + at++)] = (int)(page0 + u);
    }
    before += all;
  }
  return p.chunks > 1 ? total : before;
}

__global__ void __launch_bounds__(DECIDE_THREADS) fork_end_kernel(const RowsParams p) {
  __shared__ int64_t sums[DECIDE_THREADS / 32];
  pdl_trigger();
  pdl_wait();
  const int64_t back = give_back(p, sums);
  for (int x = blockIdx.x * DECIDE_THREADS + threadIdx.x; x < p.n_seq * PAGE; x += gridDim.x * DECIDE_THREADS) {
    const int i = x / PAGE, r = x % PAGE;
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

// What the rows' tokens are counted in is there twice: a call counts in one and makes the other zero for the next.  Its number is what both kernels go
// by: the first reads `was` and writes `is`, the second the other way round, so that no CTA reads a word that another is writing.
__device__ __forceinline__ int2* row_stay(const RowsParams& p, int call) { return p.row_stay + (call & 1) * PAGED_MAX_SEQ; }

// A warp per page: how many of its tokens stay; per row, how many stay in all and the first page that something leaves (pages before it are full,
// so that says how many move).
__global__ void __launch_bounds__(RT) compact_count_kernel(const RowsParams p) {
  pdl_trigger();
  pdl_wait();
  const int i = blockIdx.y, length = length_of(p, i), pages = pages_of(length), lane = threadIdx.x & 31, call = *p.was + 1;
  int2* row = row_stay(p, call) + i;
  for (int j = blockIdx.x * (RT / 32) + (threadIdx.x >> 5); j < pages; j += gridDim.x * (RT / 32)) {
    const int stay = __popcll(staying(p, i, j, length, lane));
    if (lane == 0) {
      p.page_stay[(int64_t)i * p.table_pages + j] = stay;
      atomicAdd(&row->y, stay);
      if (stay < min(PAGE, length - j * PAGE)) atomicMax(&row->x, p.table_pages - j);
    }
  }
  if (blockIdx.x == 0 && i == 0 && threadIdx.x == 0) *p.is = call;
}

// The rows' plan, by a CTA of T threads that calls row(number, first page that changes (-1: none, or refused), tokens that move, fresh pages and moves of
// the rows before) for rows 0 .. n - 1, and is together again behind it.  totals, if it is not null: what the rows take, {pages, rows refused, moves}.
template <int T, typename Row>
__device__ __forceinline__ void plan_rows(const RowsParams& p, int call, int n, int free, int64_t* sums, Row row, int64_t* totals) {
  const int2* stay = row_stay(p, call);
  const int per = (n + T - 1) / T, x0 = min((int)threadIdx.x * per, n), x1 = min(x0 + per, n);
  auto change = [&](int x) {
    const int2 r = __ldcg(stay + x);
    const int first = p.table_pages - r.x;
    return r.x > 0 ? make_int2(first, r.y - first * PAGE) : make_int2(-1, 0);
  };
  int64_t before[2] = {0, 0}, all[2];            // pages and moves
  for (int x = x0; x < x1; ++x) {
    const int2 r = change(x);
    before[0] += pages_of(r.y);
    before[1] += r.y;
  }
  exclusive_sums<T / 32>(before, sums, all);
  __shared__ unsigned long long most[2];
  __shared__ unsigned int turned_down;
  if (threadIdx.x == 0) most[0] = most[1] = turned_down = 0;
  int64_t taken = 0, refused = 0, moved = 0;
  for (int x = x0; x < x1; ++x) {
    const int2 r = change(x);
    const int want = pages_of(r.y);
    const bool served = r.x >= 0 && (want == 0 || (before[0] + want <= free && before[1] + r.y <= p.n_moves));
    row(x, served ? r.x : -1, r.y, before[0], before[1]);
    if (want > 0) {
      before[0] += want;
      before[1] += r.y;
      if (served) {
        taken = before[0];
        moved = before[1];
      } else {
        ++refused;
      }
    }
  }
  __syncthreads();
  if (!totals) return;
  // rows that are served are the first ones of those that want pages: the most that any thread saw
  if (taken > 0) {
    atomicMax(&most[0], (unsigned long long)taken);
    atomicMax(&most[1], (unsigned long long)moved);
  }
  if (refused > 0) atomicAdd(&turned_down, (unsigned)refused);
  __syncthreads();
  totals[0] = (int64_t)most[0];
  totals[1] = turned_down;
  totals[2] = (int64_t)most[1];
}
__device__ __forceinline__ void compact_state(const RowsParams& p, int head, int free, const int64_t (&totals)[3], int64_t back) {
  p.state_out[0] = ring_place(p, head, totals[0]);
  p.state_out[1] = (int)(free - totals[0] + back);
  p.state_out[2] = (int)totals[1];
  p.state_out[3] = (int)totals[2];
}

struct CompactRow {
  const int32_t* table;
  uint32_t* flags;
  int n_pages, pages, first;
  __device__ __forceinline__ int load(int j) const { return j < pages ? table[j] : -1; }
  __device__ __forceinline__ void use(int j, int page) const {
    if ((uint32_t)page < (uint32_t)n_pages) mark(flags, page, j < first ? OLD | WHOLE : OLD);
  }
};
// CTA (x, i): row i's new entries and its moves.  SMALL: CTA (0, n_seq) sees to the pages that go back, else they are marked in global memory.
// What does not hang on the other rows is loaded before their sums.
template <bool SMALL>
__global__ void __launch_bounds__(PLACE_THREADS) compact_place_kernel(const RowsParams p) {
  extern __shared__ uint32_t flags[];                              // SMALL: [flag_words], then [n_seq] rows' first pages that change, and lengths
  constexpr int T = PLACE_THREADS, W = T / 32, PER = PLACE_PAGES / W;
  __shared__ int64_t sums[2 * W];
  pdl_trigger();
  if (SMALL && (int)blockIdx.y == p.n_seq)
    for (int x = threadIdx.x; x < flag_words(p.n_pages); x += T) flags[x] = 0;
  pdl_wait();
  const int call = *p.is, head = ring_head(p), free = ring_count(p), lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int64_t totals[3];
  if ((int)blockIdx.y == p.n_seq) {
    if (blockIdx.x > 0) return;
    int32_t* firsts = reinterpret_cast<int32_t*>(flags + (SMALL ? flag_words(p.n_pages) : 0));
    int32_t* lengths = firsts + p.n_seq;
    if (SMALL)
      for (int x = threadIdx.x; x < p.n_seq; x += T) lengths[x] = length_of(p, x);
    plan_rows<T>(p, call, p.n_seq, free, sums, [&](int x, int first, int, int64_t, int64_t) { if (SMALL) firsts[x] = first; }, totals);
    for (int x = threadIdx.x; x < PAGED_MAX_SEQ; x += T) row_stay(p, call + 1)[x] = make_int2(0, 0);
    if (threadIdx.x == 0) *p.was = call;
    if (SMALL) {
      for_rows<T>(p.n_seq, p.table_pages, [&](int x) {
        return CompactRow{p.table + x * p.table_stride, flags, p.n_pages, pages_of(lengths[x]), firsts[x] >= 0 ? firsts[x] : INT32_MAX};
      });
      __syncthreads();
      const int back = give_back_small<T>(p, flags, sums, head, free);
      if (threadIdx.x == 0) compact_state(p, head, free, totals, back);
    } else if (threadIdx.x < 3) {
      p.totals[threadIdx.x] = (int)(threadIdx.x == 0 ? totals[0] : threadIdx.x == 1 ? totals[1] : totals[2]);
    }
    return;
  }
  const int i = blockIdx.y, length = length_of(p, i), pages = pages_of(length);
  const int32_t* stay = p.page_stay + (int64_t)i * p.table_pages;
  // PLACE_PAGES pages at a time: this thread's part of the tokens that stay in pages before them, lane's page's; its warp's pages' tokens and entries
  int64_t mine;
  int n, entry[PER];
  uint64_t bits[PER];
  auto fetch = [&](int c0) {
    mine = n = 0;
    if (c0 >= pages) return;
#pragma unroll 4
    for (int j = threadIdx.x; j < c0; j += T) mine += stay[j];
    if (c0 + lane < pages) n = stay[c0 + lane];
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      const int j = c0 + warp + u * W;
      if (j >= pages) break;
      entry[u] = p.table[i * p.table_stride + j];
      bits[u] = staying(p, i, j, length, lane);
    }
  };
  int c0 = blockIdx.x * PLACE_PAGES;
  fetch(c0);
  __shared__ int first_page, moved;
  __shared__ int64_t page_rank, move_rank;
  const bool all_rows = blockIdx.x == 0 && i == 0;                 // (this CTA's moves past the last need the totals)
  plan_rows<T>(p, call, all_rows ? p.n_seq : i + 1, free, sums, [&](int x, int first, int m, int64_t a, int64_t b) {
    if (x != i) return;
    first_page = first;
    moved = m;
    page_rank = a;
    move_rank = b;
  }, all_rows ? totals : nullptr);
  if (all_rows)
    for (int64_t x = totals[2] + threadIdx.x; x < p.n_moves; x += T) p.move_from[x] = p.move_to[x] = -1;
  const int first = first_page >= 0 ? first_page : pages, fresh = first_page >= 0 ? pages_of(moved) : 0;
  for (int j = blockIdx.x * T + threadIdx.x; j < p.table_pages; j += gridDim.x * T) {
    int page = -1;
    if (j < max(first, SMALL ? 0 : pages)) {
      page = p.table[i * p.table_stride + j];
      if (!SMALL && valid(p, page)) atomicOr(p.marks + page, j < first ? OLD | WHOLE : OLD);
    }
    if (j >= first) page = j < first + fresh ? ring_at(p, head, page_rank + (j - first)) : -1;
    p.table_out[i * p.out_stride + j] = page;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) p.lengths_out[i] = first_page >= 0 ? first * PAGE + moved : length;
  if (first_page < 0) return;
  // the tokens that move before each of a CTA's pages; all of the pages before the first that changes are full
  __shared__ int before_page[PLACE_PAGES];
  for (; c0 < pages; c0 += gridDim.x * PLACE_PAGES, fetch(c0)) {
    if (c0 + PLACE_PAGES <= first) continue;
    int64_t upto;
    exclusive_sum<W>(mine, sums, upto);
    if (threadIdx.x < 32) {
      int inc = n;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += up;
      }
      before_page[lane] = (int)upto + inc - n - first * PAGE;
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      const int j = c0 + warp + u * W;
      if (j < first || j >= pages) continue;
      const int page = entry[u], before = before_page[j - c0];
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int at = half * 32 + lane;
        if (!(bits[u] >> at & 1)) continue;
        const int rank = before + __popcll(bits[u] & (((uint64_t)1 << at) - 1));
        const int to = ring_at(p, head, page_rank + rank / PAGE);
        const bool moves = valid(p, page) && valid(p, to);
        p.move_from[move_rank + rank] = moves ? page * PAGE + at : -1;
        p.move_to[move_rank + rank] = moves ? to * PAGE + rank % PAGE : -1;
      }
    }
    __syncthreads();
  }
}

__global__ void __launch_bounds__(DECIDE_THREADS) compact_end_kernel(const RowsParams p) {
  __shared__ int64_t sums[DECIDE_THREADS / 32];
  pdl_trigger();
  pdl_wait();
  const int64_t back = give_back(p, sums);
  const int64_t totals[3] = {p.totals[0], p.totals[1], p.totals[2]};
  if (blockIdx.x == 0 && threadIdx.x == 0) compact_state(p, ring_head(p), ring_count(p), totals, back);
}

// ------------------------------------------------------------------------------------------------ moves
constexpr int MT = 256, MOVE_UNROLL = 4;

// Words of K and V of all heads of an entry, MOVE_UNROLL of them per thread, whose loads are all on their way at once (two or eight, or hints that the
// words are used once, are no better).  What bounds it is reading and writing: 30 000 tokens of 8 heads of 128 in 16 bits, 247 MB, take 41 us (6.0 TB/s).
// In 4 bits a row is 64 bytes of codes and 8 of scales: of rows that lie apart DRAM brings their neighbours, too (33 000 tokens, two in five of their pages':
// 76 MB read for 38, 21.5 us).
// A cache of 16 bits: 16 bytes of K and of V.
struct Words16 {
  using Word = int4;
  __device__ static int words(const MoveParams& p) { return p.Hkv * (p.d / 8); }
  __device__ static int64_t at(const MoveParams& p, uint32_t slot, int w, int) {
    const int ch = p.d / 8, h = w / ch, c = w - h * ch;
    return ((int64_t)(slot / PAGE) * p.page_stride + h * p.head_stride + (int64_t)(slot % PAGE) * p.row_stride + c * 8) * 2;
  }
  __device__ static char* base(const MoveParams& p, int part) { return static_cast<char*>(part ? p.v : p.k); }
};
// .. of 4 bits: the codes of K or V, four lanes a row (16 bytes each for d = 128)
template <int D>
struct Codes4 {
  using Word = typename std::conditional<D == 128, int4, int2>::type;
  __device__ static int words(const MoveParams& p) { return p.Hkv * 4; }
  __device__ static int64_t at(const MoveParams& p, uint32_t slot, int w, int part) {
    using B = Block4<D>;
    return (int64_t)(slot / PAGE) * p.page_stride + (w >> 2) * p.head_stride + (part ? B::V : B::K) + (int)(slot % PAGE) * B::ROW + (w & 3) * (int)sizeof(Word);
  }
  __device__ static char* base(const MoveParams& p, int) { return static_cast<char*>(p.k); }
};
// .. and the scales
template <int D>
struct Scales4 {
  using Word = typename std::conditional<D == 128, int2, int>::type;
  __device__ static int words(const MoveParams& p) { return p.Hkv; }
  __device__ static int64_t at(const MoveParams& p, uint32_t slot, int w, int part) {
    using B = Block4<D>;
    return (int64_t)(slot / PAGE) * p.page_stride + w * p.head_stride + (part ? B::VS : B::KS) + (int)(slot % PAGE) * B::SCALES;
  }
  __device__ static char* base(const MoveParams& p, int) { return static_cast<char*>(p.k); }
};

template <typename W>
__device__ __forceinline__ void move_words(const MoveParams& p, int block) {
  const uint32_t n_slots = (uint32_t)p.n_pages * PAGE, words = W::words(p);
  const int64_t first = (int64_t)block * (MT * MOVE_UNROLL), e0 = first / words;
  const uint32_t w0 = (uint32_t)(first - e0 * words);
  typename W::Word x[MOVE_UNROLL][2];
  int64_t to[MOVE_UNROLL][2];
#pragma unroll
  for (int u = 0; u < MOVE_UNROLL; ++u) {
    const uint32_t i = w0 + threadIdx.x + u * MT, de = i / words, w = i - de * words;
    to[u][0] = -1;
    if (e0 + de >= p.n_moves) continue;
    const uint32_t a = (uint32_t)p.from[e0 + de], b = (uint32_t)p.to[e0 + de];
    if (a >= n_slots || b >= n_slots) continue;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      x[u][k] = *reinterpret_cast<const typename W::Word*>(W::base(p, k) + W::at(p, a, w, k));
      to[u][k] = W::at(p, b, w, k);
    }
  }
#pragma unroll
  for (int u = 0; u < MOVE_UNROLL; ++u) {
    if (to[u][0] < 0) continue;
#pragma unroll
    for (int k = 0; k < 2; ++k) *reinterpret_cast<typename W::Word*>(W::base(p, k) + to[u][k]) = x[u][k];
  }
}
__global__ void __launch_bounds__(MT) move_kernel(const MoveParams p) {
  pdl_trigger();
  pdl_wait();
  move_words<Words16>(p, blockIdx.x);
}
// the first blocks move codes, the others scales
template <int D>
__global__ void __launch_bounds__(MT) move4_kernel(const MoveParams p, int code_blocks) {
  pdl_trigger();
  pdl_wait();
  if ((int)blockIdx.x < code_blocks) move_words<Codes4<D>>(p, blockIdx.x);
  else move_words<Scales4<D>>(p, blockIdx.x - code_blocks);
}

}  // namespace

// (the words that must be zero before the first call come first, and are of one size, so that calls of all sizes may share a workspace)
uint64_t rows_workspace_bytes(int n_seq, int table_pages, int n_pages) {
  return ((uint64_t)6 * PAGED_MAX_SEQ + ROWS_CHUNKS + 64 + 2 * (uint64_t)n_pages + (uint64_t)n_seq * table_pages) * 4;
}

void place_rows_workspace(void* ws, RowsParams* p) {
  p->chunk = std::max(16384, (p->n_pages + ROWS_CHUNKS - 1) / ROWS_CHUNKS);
  p->chunks = (p->n_pages + p->chunk - 1) / p->chunk;
  p->row_stay = static_cast<int2*>(ws);
  p->row_moves = p->row_stay + 2 * PAGED_MAX_SEQ;
  p->chunk_sums = reinterpret_cast<int32_t*>(p->row_moves + PAGED_MAX_SEQ);
  p->totals = p->chunk_sums + ROWS_CHUNKS;
  p->was = p->totals + 32;
  p->is = p->totals + 33;
  p->marks = reinterpret_cast<uint32_t*>(p->totals + 64);
  p->claims = p->marks + p->n_pages;
  p->page_stay = reinterpret_cast<int32_t*>(p->claims + p->n_pages);
}

namespace {
cudaError_t launch_zero_marks(const RowsParams& p, cudaStream_t stream) {
  return launch_pdl(zero_marks_kernel, dim3(std::min(592, (p.n_pages + DECIDE_THREADS - 1) / DECIDE_THREADS)), dim3(DECIDE_THREADS), 0, stream, p);
}
cudaError_t launch_chunks(const RowsParams& p, cudaStream_t stream) {
  return p.chunks > 1 ? launch_pdl(chunk_kernel, dim3(p.chunks), dim3(RT), 0, stream, p) : cudaSuccess;
}
}  // namespace

cudaError_t launch_paged_fork(const RowsParams& p, cudaStream_t stream) {
  cudaError_t rc;
  if (one_cta(p, FORK_ENTRIES)) {
    auto bytes = [](int n_pages, int n_seq) { return ((n_pages + 7) / 8 + n_pages + 5 * n_seq + 2) * 4; };
    // (always the most that any call takes: the limit is the process's, and another thread may set it before this launch; 47 KB need no limit raised)
    rc = bytes(p.n_pages, p.n_seq) <= 47 * 1024 ? cudaSuccess
                                                : cudaFuncSetAttribute(fork_small_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes(SMALL_PAGES, small_rows(SMALL_PAGES)));
    return rc != cudaSuccess ? rc : launch_pdl(fork_small_kernel, dim3(1 + (p.n_seq + copied_rows(p.n_seq) - 1) / copied_rows(p.n_seq)), dim3(DECIDE_THREADS), bytes(p.n_pages, p.n_seq), stream, p);
  }
  rc = launch_zero_marks(p, stream);
  if (rc != cudaSuccess) return rc;
  rc = launch_pdl(fork_mark_kernel, dim3((unsigned)std::min(64, (p.table_pages + RT - 1) / RT), p.n_seq), dim3(RT), 0, stream, p);
  if (rc != cudaSuccess) return rc;
  rc = launch_pdl(fork_decide_kernel, dim3(1), dim3(DECIDE_THREADS), 0, stream, p);
  if (rc == cudaSuccess) rc = launch_chunks(p, stream);
  if (rc != cudaSuccess) return rc;
  const int writers = std::min(148, (p.n_seq * PAGE + DECIDE_THREADS - 1) / DECIDE_THREADS);
  return launch_pdl(fork_end_kernel, dim3(std::max(p.chunks, writers)), dim3(DECIDE_THREADS), 0, stream, p);
}

cudaError_t launch_paged_compact(const RowsParams& p, cudaStream_t stream) {
  auto ctas = [&](int pages, int more) { return dim3((unsigned)std::min(256, (p.table_pages + pages - 1) / pages), p.n_seq + more); };
  const bool small = one_cta(p, COMPACT_ENTRIES);
  cudaError_t rc = small ? cudaSuccess : launch_zero_marks(p, stream);
  if (rc == cudaSuccess) rc = launch_pdl(compact_count_kernel, ctas(RT / 32, 0), dim3(RT), 0, stream, p);
  if (rc != cudaSuccess) return rc;
  if (small) return launch_pdl(compact_place_kernel<true>, ctas(PLACE_PAGES, 1), dim3(PLACE_THREADS), ((p.n_pages + 7) / 8 + 2 * p.n_seq) * 4, stream, p);
  rc = launch_pdl(compact_place_kernel<false>, ctas(PLACE_PAGES, 1), dim3(PLACE_THREADS), 0, stream, p);
  if (rc == cudaSuccess) rc = launch_chunks(p, stream);
  if (rc != cudaSuccess) return rc;
  return launch_pdl(compact_end_kernel, dim3(p.chunks), dim3(DECIDE_THREADS), 0, stream, p);
}

cudaError_t launch_paged_move(const MoveParams& p, int bits, cudaStream_t stream) {
  auto blocks = [&](int words) { return ((int64_t)p.n_moves * words + MT * MOVE_UNROLL - 1) / (MT * MOVE_UNROLL); };
  const int64_t rows = blocks(p.Hkv * (bits == 16 ? p.d / 8 : 4)), scales = bits == 16 ? 0 : blocks(p.Hkv);
  if (rows + scales > INT32_MAX) return cudaErrorInvalidValue;
  const dim3 grid((unsigned)(rows + scales));
  if (bits == 16) return launch_pdl(move_kernel, grid, dim3(MT), 0, stream, p);
  return p.d == 128 ? launch_pdl(move4_kernel<128>, grid, dim3(MT), 0, stream, p, (int)rows) : launch_pdl(move4_kernel<64>, grid, dim3(MT), 0, stream, p, (int)rows);
}

}  // namespace heatkv
