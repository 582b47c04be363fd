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
constexpr int PLACE_PAGES = 32;                // pages of a row whose moves a CTA lists
enum Mark : uint32_t { OLD = 1, WHOLE = 2, PART = 4 };   // listed by the old table; by the new one, all of the page or its first rows

__device__ __forceinline__ int pages_of(int tokens) { return (tokens + PAGE - 1) / PAGE; }
__device__ __forceinline__ int length_of(const RowsParams& p, int i) { return min(max(p.lengths[i], 0), p.table_pages * PAGE); }
__device__ __forceinline__ bool valid(const RowsParams& p, int page) { return page >= 0 && page < p.n_pages; }
// the ring's entry `i` places behind the oldest, i below twice the pages
__device__ __forceinline__ uint32_t ring_place(const RowsParams& p, int head, int64_t i) {
  const uint32_t at = (uint32_t)head + (uint32_t)i;
  return at < (uint32_t)p.n_pages ? at : at - (uint32_t)p.n_pages;
}
__device__ __forceinline__ int ring_at(const RowsParams& p, int head, int64_t i) { return p.free_pages[ring_place(p, head, i)]; }
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
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    p.lengths_out[i] = length;
    const int last = rest > 0 ? p.table[parent * p.table_stride + whole] : -1;
    p.row_moves[i] = make_int2(valid(p, last) ? last : -1, length);          // the page with its last tokens, if that is not full
  }
}

// Pages of chunk c that go back.
__device__ __forceinline__ bool goes_back(const RowsParams& p, int page) { return (p.marks[page] & (OLD | WHOLE | PART)) == OLD; }

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

// Pages that go back.
__device__ __forceinline__ bool goes_back(uint32_t mark) { return (mark & (OLD | WHOLE | PART)) == OLD; }
// .. of a chunk of the pool, where there is more than one: how many
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
// Pages that go back to the ring's end, chunk by chunk in page order, by CTAs of 1024 threads; marks made zero for the next call.  Gives the number of all of
// them to CTA 0.
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
      if (back[u]) p.free_pages[(head + free + at++) % p.n_pages] = (int)(page0 + u);
      if (page0 + u < end) p.marks[page0 + u] = p.claims[page0 + u] = 0;
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

// A warp per page: how many of its tokens stay, and the old table's marks; per row, how many stay in all and the first page that something leaves
// (pages before it are full, so that says how many move).
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
      atomicAdd(&p.row_stay[i].y, stay);
      if (stay < min(PAGE, length - j * PAGE)) atomicMax(&p.row_stay[i].x, p.table_pages - j);
    }
  }
}

// The first page of row i that changes (-1: none) and the tokens that move.
__device__ __forceinline__ int2 row_change(const RowsParams& p, int i) {
  const int2 r = p.row_stay[i];
  const int first = p.table_pages - r.x;
  return r.x > 0 ? make_int2(first, r.y - first * PAGE) : make_int2(-1, 0);
}

// What the rows before row i take, and whether it is served: every CTA sums up for itself.
struct RowPlan {
  int first, moved;                            // first page that changes (-1: none, or refused), tokens that move
  int64_t page_rank, move_rank;                // fresh pages and moves of the rows before
};
template <int T>
__device__ __forceinline__ RowPlan plan_row(const RowsParams& p, int i, int64_t* sums, bool last, int64_t (&totals)[3]) {
  // (rows before i; with `last`, all rows, and the totals: pages taken, rows refused, moves)
  const int free = ring_count(p), n = last ? p.n_seq : i + 1, per = (n + T - 1) / T, x0 = min((int)threadIdx.x * per, n), x1 = min(x0 + per, n);
  __shared__ RowPlan mine;
  int64_t need = 0, moves = 0, all_need, all_moves;
  for (int x = x0; x < x1; ++x) {
    const int2 r = row_change(p, x);
    if (r.x >= 0) {
      need += pages_of(r.y);
      moves += r.y;
    }
  }
  int64_t a = exclusive_sum<T / 32>(need, sums, all_need), b = exclusive_sum<T / 32>(moves, sums, all_moves);
  int64_t taken = 0, refused = 0, moved = 0;
  for (int x = x0; x < x1; ++x) {
    const int2 r = row_change(p, x);
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
    exclusive_sum<T / 32>(refused, sums, totals[1]);
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
  const bool all_rows = blockIdx.x == 0 && i == 0;                 // this CTA says what all rows take, for the last kernel
  const RowPlan r = plan_row<RT>(p, i, sums, all_rows, totals);
  if (all_rows && threadIdx.x < 3) p.totals[threadIdx.x] = (int)totals[threadIdx.x];
  const int32_t* stay = p.page_stay + (int64_t)i * p.table_pages;
  const int first = r.first >= 0 ? r.first : pages, fresh = r.first >= 0 ? pages_of(r.moved) : 0;
  for (int j = blockIdx.x * RT + threadIdx.x; j < p.table_pages; j += gridDim.x * RT) {
    int page = -1;
    if (j < first) {
      page = p.table[i * p.table_stride + j];
      if (valid(p, page)) atomicOr(p.marks + page, WHOLE);
    } else if (j < first + fresh) {
      page = ring_at(p, head, r.page_rank + (j - first));
    }
    p.table_out[i * p.out_stride + j] = page;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) p.lengths_out[i] = r.first >= 0 ? first * PAGE + r.moved : length;
  if (r.first < 0) return;
  // a CTA's pages lie together: the tokens that move before them, and before each of them
  __shared__ int before_page[PLACE_PAGES];
  for (int c0 = first / PLACE_PAGES * PLACE_PAGES + blockIdx.x * PLACE_PAGES; c0 < pages; c0 += gridDim.x * PLACE_PAGES) {
    const int c1 = min(c0 + PLACE_PAGES, pages);
    int64_t mine = 0, upto;
#pragma unroll 4
    for (int j = first + threadIdx.x; j < c0; j += RT) mine += stay[j];
    exclusive_sum<RT / 32>(mine, sums, upto);
    if (threadIdx.x < 32) {
      const int j = c0 + lane, n = j >= first && j < c1 ? stay[j] : 0;
      int inc = n;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += up;
      }
      before_page[lane] = (int)upto + inc - n;
    }
    __syncthreads();
    for (int j = max(first, c0) + (threadIdx.x >> 5); j < c1; j += RT / 32) {
      const uint64_t bits = staying(p, i, j, length, lane);
      const int page = p.table[i * p.table_stride + j], before = before_page[j - c0];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int at = u * 32 + lane;
        if (!(bits >> at & 1)) continue;
        const int rank = before + __popcll(bits & (((uint64_t)1 << at) - 1));
        const int to = ring_at(p, head, r.page_rank + rank / PAGE);
        const bool moves = valid(p, page) && valid(p, to);
        p.move_from[r.move_rank + rank] = moves ? page * PAGE + at : -1;
        p.move_to[r.move_rank + rank] = moves ? to * PAGE + rank % PAGE : -1;
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
  for (int64_t x = totals[2] + (int64_t)blockIdx.x * DECIDE_THREADS + threadIdx.x; x < p.n_moves; x += (int64_t)gridDim.x * DECIDE_THREADS)
    p.move_from[x] = p.move_to[x] = -1;
  // zero again for the next call: what the rows' tokens were counted in
  for (int i = blockIdx.x; i < p.n_seq; i += gridDim.x) {
    const int pages = pages_of(length_of(p, i));
    for (int j = threadIdx.x; j < pages; j += DECIDE_THREADS) p.page_stay[(int64_t)i * p.table_pages + j] = 0;
    if (threadIdx.x == 0) p.row_stay[i] = make_int2(0, 0);
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    p.state_out[0] = (int)((ring_head(p) + totals[0]) % p.n_pages);
    p.state_out[1] = (int)(ring_count(p) - totals[0] + back);
    p.state_out[2] = (int)totals[1];
    p.state_out[3] = (int)totals[2];
  }
}

// ------------------------------------------------------------------------------------------------ moves
constexpr int MT = 256, MOVE_UNROLL = 4;

// Words of K and V of all heads of an entry, MOVE_UNROLL of them per thread, whose loads are all on their way at once.  What bounds it is reading
// and writing.
// A cache of 16 bits: 16 bytes of K and of V.
struct Words16 {
  using Word = int4;
  static constexpr int PARTS = 2;
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
  static constexpr int PARTS = 2;
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
  static constexpr int PARTS = 2;
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

// First what any call has, of one size, so that calls of all sizes may share a workspace: what lies behind it is zero between calls.
uint64_t rows_workspace_bytes(int n_seq, int table_pages, int n_pages) {
  return ((uint64_t)4 * PAGED_MAX_SEQ + ROWS_CHUNKS + 64 + 2 * (uint64_t)n_pages + (uint64_t)n_seq * table_pages) * 4;
}

void place_rows_workspace(void* ws, RowsParams* p) {
  p->chunk = std::max(16384, (p->n_pages + ROWS_CHUNKS - 1) / ROWS_CHUNKS);
  p->chunks = (p->n_pages + p->chunk - 1) / p->chunk;
  p->row_stay = static_cast<int2*>(ws);
  p->row_moves = p->row_stay + PAGED_MAX_SEQ;
  p->chunk_sums = reinterpret_cast<int32_t*>(p->row_moves + PAGED_MAX_SEQ);
  p->totals = p->chunk_sums + ROWS_CHUNKS;
  p->marks = reinterpret_cast<uint32_t*>(p->totals + 64);
  p->claims = p->marks + p->n_pages;
  p->page_stay = reinterpret_cast<int32_t*>(p->claims + p->n_pages);
}

namespace {
cudaError_t launch_chunks(const RowsParams& p, cudaStream_t stream) {
  return p.chunks > 1 ? launch_pdl(chunk_kernel, dim3(p.chunks), dim3(RT), 0, stream, p) : cudaSuccess;
}
}  // namespace

cudaError_t launch_paged_fork(const RowsParams& p, cudaStream_t stream) {
  cudaError_t rc = launch_pdl(fork_mark_kernel, dim3((unsigned)std::min(64, (p.table_pages + RT - 1) / RT), p.n_seq), dim3(RT), 0, stream, p);
  if (rc != cudaSuccess) return rc;
  rc = launch_pdl(fork_decide_kernel, dim3(1), dim3(DECIDE_THREADS), 0, stream, p);
  if (rc == cudaSuccess) rc = launch_chunks(p, stream);
  if (rc != cudaSuccess) return rc;
  const int writers = std::min(148, (p.n_seq * PAGE + DECIDE_THREADS - 1) / DECIDE_THREADS);
  return launch_pdl(fork_end_kernel, dim3(std::max(p.chunks, writers)), dim3(DECIDE_THREADS), 0, stream, p);
}

cudaError_t launch_paged_compact(const RowsParams& p, cudaStream_t stream) {
  auto ctas = [&](int pages) { return dim3((unsigned)std::min(256, (p.table_pages + pages - 1) / pages), p.n_seq); };
  cudaError_t rc = launch_pdl(compact_count_kernel, ctas(RT / 32), dim3(RT), 0, stream, p);
  if (rc != cudaSuccess) return rc;
  rc = launch_pdl(compact_place_kernel, ctas(PLACE_PAGES), dim3(RT), 0, stream, p);
  if (rc == cudaSuccess) rc = launch_chunks(p, stream);
  if (rc != cudaSuccess) return rc;
  return launch_pdl(compact_end_kernel, dim3(std::max(p.chunks, std::min(p.n_seq, 148))), dim3(DECIDE_THREADS), 0, stream, p);
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
