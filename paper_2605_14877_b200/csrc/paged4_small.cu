// Attention of few query rows (decode, drafted tokens) over a paged cache in 4 bits, on warp-level MMA.
//
// A request's new tokens times the G query heads of one kv head are its rows, token by token; a row tile is 8 or 16 of them, a unit a row tile of one
// request and kv head, and its pages come one after another.  The pages of all units, request by request, head by head, are dealt out in equal runs, one a
// CTA, and a run's pages in equal ranges, one a warp.  A warp works through its range by itself, from the copies that it sends for (9216 bytes, a ring of
// its own) to the product with V, and never waits for another: units that lie in its range whole it writes out, of the at most two that its
// range's ends cut it leaves unnormalised rows, which the CTA's warps add up when all are done, in page order.  A unit that a run's border cuts leaves
// the sum in the workspace, and the CTA that leaves the last part of it adds them up, in page order again.  (With page x of a run taken by warp x mod 8, so that the warps met wherever a unit
// ended, a decode of 64 requests took 68 us: a unit's end and beginning cost 6000 cycles, and the SM with the shortest units was the last.)
//
// The products are transposed, S^T = K Q^T and O^T = V^T P^T, so that the cache is the operand with 16 rows and the queries the one with 8: a group of up to
// eight heads costs half of what it would the other way round.  Which columns a step of a product takes is free as long as both operands take the
// same, so a lane's part of K is what lies next to each other: 32 codes of one key (16 bytes) with their two scales, and of V 16 codes of one
// key with their scale.  Codes become fp16 numbers in registers, exactly (Steps4): queries are scaled, row by row, to fp16's range by a power of
// two, and probabilities are fp16 for either type.
//
// What bounds it: long contexts the reading and, nearly as much, the instructions that make numbers of codes (64 requests of 12 000 tokens, 8 kv heads of four:
// 885 MB in 164 us, 5.4 TB/s; a page takes an SM 370 to 440 cycles); ordinary ones the ends of the call: 64 requests of 300 to 12 000 are 35.2 us for
// 101 MB, of which 4.4 pass before the first page (lengths, runs, table, pages: one load behind another) and 4 to 5 after most warps' last (the SMs' differences,
// parts added up, a fence and a counter).  One token over 200 keys is 7.7 us, the same chain.
#include <algorithm>
#include <climits>
#include <type_traits>

#include "paged4.cuh"
#include "paged_wait.cuh"

namespace heatkv {
namespace {

using namespace tc;

constexpr int MOST_WARPS = 12;
constexpr int MAX_STAGES = 6;
// A row's reference is set 2^BELOW under its maximum and moves when a maximum passes it by more than 2^MOVE: probabilities fit fp16, and the smallest that do
// not round to nothing there are 2^-(25 + BELOW) of the largest.  (With references at the maximum a key 2^25.5 under it counted in the sum and not in the
// output: 260 000 such keys beside a heavy one are half a percent of it, and were missing.)
constexpr float BELOW = 7.f, MOVE = 15.f;
constexpr int SHARE = 4;                       // pages of a run at least
constexpr int WHOLE = 8;                       // units of up to so many pages are never cut by a run's border
constexpr int MIN_PART = 4;                    // pages of a part
constexpr int UNIT_END = 1;                    // what a unit weighs beyond its pages: its rows in, its sums and rows out

struct Small4Params {
  Paged4Params q;
  float* ends;                                 // [CTAs][warps] rows of the unit that a warp's range begins inside of
  int32_t stages;
  uint32_t inverse;                            // 2^32 / CTAs
};

// c += a x b for one 16 x 8 x 16 product of fp16
__device__ __forceinline__ void mma_half(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
template <bool F16>
__device__ __forceinline__ uint32_t pack_out(float lo, float hi) {
  return F16 ? pack_half(lo, hi) : pack_bf16(lo, hi);
}

__host__ __device__ constexpr int64_t slot_floats(int rows, int d) { return (int64_t)rows * (d + 2); }

// Requests, in shared memory: what the units before them weigh, how many units those are; first new token, number of new tokens, tokens in all.
struct Requests {
  int64_t* pre;
  int32_t *units, *first, *count, *keys;
  __device__ Requests(unsigned char* at, int n_seq) {
    pre = reinterpret_cast<int64_t*>(at);
    units = reinterpret_cast<int32_t*>(pre + n_seq + 1);
    first = units + n_seq + 1;
    count = first + n_seq;
    keys = count + n_seq;
  }
  static constexpr int bytes(int n_seq) { return n_seq * 24 + 16; }
  __device__ int64_t pages(int i) const { return pre[i] - (int64_t)UNIT_END * units[i]; }      // before request i
};
// The runs: CTA c's begins where what came before weighs raw(c), or near there.
struct Runs {
  int64_t all, share;                          // a run's share in 2^-16
  int grid;
  // (without a division of 64-bit numbers: a call with that much has as many runs as there are CTAs, whose reciprocal is `inverse` 2^-32)
  __device__ void deal(int64_t all_, int ctas, uint32_t inverse) {
    all = all_;
    if (all < (1 << 15)) {
      grid = max(min(ctas, ((int)all + SHARE - 1) / SHARE), 1);
      share = ((uint32_t)all << 16) / (uint32_t)grid;
    } else {
      grid = ctas;
      share = all * inverse >> 16;
    }
  }
  __device__ int64_t raw(int c) const { return share * c >> 16; }
  // a border inside a unit of `pages` pages from `begin` on: not near its ends, not in a short one
  __device__ static int64_t snap(int64_t y, int64_t begin, int pages) {
    const int64_t at = y - begin, end = begin + pages + UNIT_END;
    if (pages <= WHOLE) return 2 * at < pages ? begin : end;
    return at < MIN_PART ? begin : pages - at < MIN_PART ? end : y;
  }
};
// The last of 0 .. n - 1 where f is not above y[k], by a whole warp, 32 places at a time (f ascends from f(0) <= y[k]; lane by lane, halving: decode of 64
// requests 35.7 us instead of 35.2).
template <int K, typename F>
__device__ __forceinline__ void last_not_above(int n, F f, const int64_t (&y)[K], int (&at)[K]) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int k = 0; k < K; ++k) at[k] = 0;
  for (int size = n; size > 1;) {
    const int step = (size + 31) / 32, off = lane * step;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int i = at[k] + off;
      const bool not_above = off < size && i < n && f(i) <= y[k];
      at[k] += max(__popc(__ballot_sync(0xffffffffu, not_above)) - 1, 0) * step;
    }
    size = step;
  }
}
__device__ __forceinline__ int divide(int64_t a, int b) { return a >> 31 ? (int)(a / b) : (int)((uint32_t)a / (uint32_t)b); }

// A unit, and the pages of it that some row sees.
template <int ROWS>
struct Unit {
  int seq, head, tile, pages, tiles;           // row tiles of the request
  int seen;
  int row0, rows;                              // of the tile
  int kv, pos0, tok0;                          // tokens of the request; place and number of its first new one
  __device__ void set(const Requests& q, const PagedParams& p) {
    const int n = q.count[seq];
    kv = q.keys[seq];
    tok0 = q.first[seq];
    pos0 = kv - n;
    pages = (kv + PAGE - 1) / PAGE;
    tiles = (n * p.G + ROWS - 1) / ROWS;
    row0 = tile * ROWS;
    rows = min(ROWS, n * p.G - row0);
    const int sees = p.causal ? min(pos0 + (row0 + rows - 1) / p.G + 1, kv) : kv;
    seen = (max(sees, 0) + PAGE - 1) / PAGE;
  }
  __device__ void next(const Requests& q, const PagedParams& p) {
    if (++tile == tiles) {
      tile = 0;
      if (++head == p.Hkv) {
        head = 0;
        do ++seq; while (seq < p.n_seq && (q.keys[seq] == 0 || q.count[seq] == 0));
        if (seq == p.n_seq) return;            // (behind the last unit: nothing is read there)
      }
    }
    set(q, p);
  }
};

template <int D, int NT, bool F16, int WARPS>
__global__ void __launch_bounds__(WARPS * 32, 1) paged4_small_kernel(const __grid_constant__ Small4Params sp) {
  using B = Block4<D>;
  constexpr int ROWS = 8 * NT, THREADS = WARPS * 32;
  constexpr int WORDS = D / 32;                                    // words of codes that a lane has of a key
  constexpr int MTILES = D / 16;                                   // 16-row tiles of O^T: two neighbouring columns of a lane each
  constexpr int KT = PAGE / 16;
  // (with 16 rows the registers are better used otherwise: 32 requests, 16 heads a group, 24.7 us and 25.4)
  constexpr bool UNEVEN = NT == 1;
  using Steps = typename std::conditional<UNEVEN, Steps4Uneven, Steps4>::type;
  static_assert(ROWS * (D + 2) * 4 <= B::BYTES, "a warp's rows fit a stage");
  const Paged4Params& q4 = sp.q;
  const PagedParams& p = q4.a;
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ __align__(8) uint64_t bars[WARPS * MAX_STAGES];
  __shared__ uint32_t abort_word;
  __shared__ int2 final_parts[2];                                  // of the run's first and last unit: the CTAs whose parts are there, if this one is to add them up
  __shared__ int64_t sums[WARPS];
  __shared__ int4 records[2 * WARPS];                              // a warp's two ends: {request, head, tile, what is cut}
  volatile uint32_t* abort_flag = &abort_word;
  const int stages = sp.stages;
  const Requests req(smem + WARPS * stages * B::BYTES, p.n_seq);
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  const uint32_t bar0 = smem_u32(bars);
  auto full = [&](int s) { return bar0 + (warp * MAX_STAGES + s) * 8; };

  pdl_trigger();
  if (threadIdx.x < WARPS * MAX_STAGES) mbar_init(bar0 + threadIdx.x * 8, 1);
  if (threadIdx.x < 2 * WARPS) records[threadIdx.x] = make_int4(-1, 0, 0, 0);
  if (threadIdx.x < 2) final_parts[threadIdx.x] = make_int2(0, -1);
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  pdl_wait();
  if (threadIdx.x == 0) *abort_flag = *reinterpret_cast<volatile uint32_t*>(p.status) != 0;
  // What the ranges will begin with comes to L2 while the lengths are on their way, each CTA's share of the lines, where all of it is a line a thread: the
  // table, the query rows.
  {
    const int64_t line = (int64_t)blockIdx.x * THREADS + threadIdx.x, lines = (int64_t)gridDim.x * THREADS;
    const int per_row = (p.table_pages + 31) / 32, row_lines = D / 64;
    if ((int64_t)p.n_seq * per_row <= lines && line < (int64_t)p.n_seq * per_row) {
      const int i = (int)line / per_row;
      prefetch_l2(p.block_table + i * p.table_stride + ((int)line - i * per_row) * 32);
    }
    if ((int64_t)p.n_tokens * p.H * row_lines <= lines && line < (int64_t)p.n_tokens * p.H * row_lines) {
      const int row = (int)line / row_lines, tok = row / p.H;
      prefetch_l2(static_cast<const __half*>(p.q) + tok * p.q_tok + (row - tok * p.H) * p.q_head + ((int)line - row * row_lines) * 64);
    }
  }
  // ------------------------------------------------------------------ the run, and this warp's range of it
  Runs runs;
  {
    const int per = (p.n_seq + THREADS - 1) / THREADS, i0 = min((int)threadIdx.x * per, p.n_seq), i1 = min(i0 + per, p.n_seq);
    auto units = [&](int i) { return req.keys[i] > 0 ? (req.count[i] * p.G + ROWS - 1) / ROWS * p.Hkv : 0; };
    auto weight = [&](int i) { return (int64_t)units(i) * ((req.keys[i] + PAGE - 1) / PAGE + UNIT_END); };
    // what comes before a thread's requests: the weight, and the units in a sum of their own
    int64_t mine = 0, mine_units = 0;
    for (int i = i0; i < i1; ++i) {
      const int b = max(p.q_begin[i], 0);
      req.first[i] = b;
      req.count[i] = max(min(p.q_begin[i + 1], p.n_tokens) - b, 0);
      req.keys[i] = min(max(p.kv_len[i], 0), p.table_pages * PAGE);
      mine += weight(i);
      mine_units += units(i);
    }
    int64_t inc = mine;
    int inc_units = (int)mine_units;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t up = __shfl_up_sync(0xffffffffu, inc, o);
      const int up_units = __shfl_up_sync(0xffffffffu, inc_units, o);
      if (lane >= o) {
        inc += up;
        inc_units += up_units;
      }
    }
    __shared__ int unit_sums[WARPS];
    if (lane == 31) {
      sums[warp] = inc;
      unit_sums[warp] = inc_units;
    }
    __syncthreads();
    int64_t at = inc - mine, all = 0;
    int at_units = inc_units - (int)mine_units;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
      all += sums[w];
      if (w < warp) {
        at += sums[w];
        at_units += unit_sums[w];
      }
    }
    for (int i = i0; i < i1; ++i) {
      req.pre[i] = at;
      req.units[i] = at_units;
      at += weight(i);
      at_units += units(i);
    }
    if (i0 < i1 && i1 == p.n_seq) {
      req.pre[p.n_seq] = at;
      req.units[p.n_seq] = at_units;
    }
    runs.deal(all, gridDim.x, sp.inverse);
    __syncthreads();
  }
  // rows of requests without keys
  for (int i = blockIdx.x; i < p.n_seq; i += gridDim.x) {
    if (req.keys[i] > 0) continue;
    const int64_t b = req.first[i], n = (int64_t)req.count[i] * p.H;
    for (int64_t j = threadIdx.x; j < n * D; j += THREADS) {
      const int64_t t = b + j / ((int64_t)p.H * D), hd = j / D % p.H;
      static_cast<uint16_t*>(p.out)[t * p.o_tok + hd * p.o_head + j % D] = 0;
    }
    if (p.lse)
      for (int64_t j = threadIdx.x; j < n; j += THREADS) p.lse[b * p.H + j] = -INFINITY;
  }
  if ((int)blockIdx.x >= runs.grid || runs.all == 0) return;
  // pages before the borders of this CTA and of the next, in lanes' turn
  auto border = [&](int c, int at) {
    if (c == runs.grid) return req.pages(p.n_seq);
    const int64_t y = runs.raw(c);
    const int pages = (req.keys[at] + PAGE - 1) / PAGE, number = divide(y - req.pre[at], pages + UNIT_END);
    const int64_t begin = req.pre[at] + (int64_t)number * (pages + UNIT_END);
    return req.pages(at) + (int64_t)number * pages + min(Runs::snap(y, begin, pages) - begin, (int64_t)pages);
  };
  const int64_t raw[2] = {runs.raw(blockIdx.x), runs.raw(blockIdx.x + 1)};
  int in[2];
  last_not_above(p.n_seq, [&](int i) { return req.pre[i]; }, raw, in);
  const int64_t a_border = border(blockIdx.x + (lane & 1), lane & 1 ? in[1] : in[0]), first_page = __shfl_sync(0xffffffffu, a_border, 0);
  const int n_run = (int)min(__shfl_sync(0xffffffffu, a_border, 1) - first_page, (int64_t)INT_MAX / 16);
  if (n_run <= 0) return;
  const int x0 = n_run * warp / WARPS, x1 = n_run * (warp + 1) / WARPS;
  // the unit with page y of all, one of request `seq`, and the page's number in it
  auto locate = [&](int64_t y, int seq, Unit<ROWS>& u) {
    const int64_t local = y - req.pages(seq);
    const int pages = (req.keys[seq] + PAGE - 1) / PAGE, tiles = (req.count[seq] * p.G + ROWS - 1) / ROWS, number = divide(local, pages);
    u.seq = seq;
    u.head = (int)((uint32_t)number / (uint32_t)tiles);
    u.tile = number - u.head * tiles;
    u.set(req, p);
    return (int)(local - (int64_t)number * pages);
  };
  auto pages_before = [&](int i) { return req.pages(i); };
  Unit<ROWS> unit;
  const int64_t range[1] = {first_page + min(x0, n_run - 1)};
  int range_seq[1];
  last_not_above(p.n_seq, pages_before, range, range_seq);
  int j0 = locate(range[0], range_seq[0], unit);                   // its page where the range begins
  // ------------------------------------------------------------------ copies
  unsigned char* ring = smem + warp * stages * B::BYTES;
  Unit<ROWS> ahead = unit;                                         // the page to be sent for next: number ahead_j of this unit
  int ahead_x = x0, ahead_j = j0, ahead_len = min(unit.pages - j0, x1 - x0), ahead_stop = min(j0 + ahead_len, unit.seen);
  int entry = -1, entries = 0, ahead_stage = 0, sent = 0;          // lane l: the table's entry for page `entries` + l of the unit
  bool more = true;
  auto look_up = [&]() {                                           // on to a page that is seen
    bool fresh = sent == 0;
    while (ahead_j >= ahead_stop) {
      fresh = true;
      ahead_x += ahead_len;
      if (ahead_x >= x1) {
        more = false;
        return;
      }
      ahead.next(req, p);
      ahead_j = 0;
      ahead_len = min(ahead.pages, x1 - ahead_x);
      ahead_stop = min(ahead_len, ahead.seen);
    }
    if (fresh || ahead_j - entries == 32) {
      entries = ahead_j;
      entry = ahead_j + lane < ahead_stop ? __ldg(p.block_table + ahead.seq * p.table_stride + ahead_j + lane) : -1;
    }
  };
  auto send = [&]() {
    if (!more) return;
    unsigned char* dst = ring + ahead_stage * B::BYTES;
    const int ahead_page = __shfl_sync(0xffffffffu, entry, ahead_j - entries);
    if (ahead_page >= 0 && ahead_page < p.n_pages) {
      if (lane == 0) {
        mbar_expect_tx(full(ahead_stage), B::BYTES);
        bulk_load(smem_u32(dst), q4.blocks + ahead_page * q4.page_stride + ahead.head * q4.head_stride, B::BYTES, full(ahead_stage));
      }
    } else {                                                       // no page of the pool: zeros
      for (int i = lane; i < B::BYTES / 16; i += 32) reinterpret_cast<int4*>(dst)[i] = make_int4(0, 0, 0, 0);
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");           // (before the stage's next copy)
      __syncwarp();
      if (lane == 0) mbar_arrive(full(ahead_stage));
    }
    __syncwarp();
    ahead_stage = ahead_stage + 1 == stages ? 0 : ahead_stage + 1;
    ++sent;
    ++ahead_j;
    look_up();
  };
  // a unit's query rows: they are asked for before the pages that would be in front of them, the next unit's are brought to L2
  const int gr = lane >> 2, qd = lane & 3;
  uint4 q_rows[NT][WORDS];
  auto row_at = [&](const Unit<ROWS>& u, int r) {
    const int row = u.row0 + r, tok = row / p.G;
    return static_cast<const __half*>(p.q) + (int64_t)(u.tok0 + tok) * p.q_tok + (int64_t)(u.head * p.G + row - tok * p.G) * p.q_head;
  };
  auto load_rows = [&]() {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int i = 0; i < WORDS; ++i) q_rows[nt][i] = make_uint4(0, 0, 0, 0);
      if (nt * 8 + gr < unit.rows) {
        const uint4* src = reinterpret_cast<const uint4*>(row_at(unit, nt * 8 + gr) + qd * (D / 4));
#pragma unroll
        for (int i = 0; i < WORDS; ++i) q_rows[nt][i] = __ldg(src + i);
      }
    }
  };
  if (x0 < x1) {
    look_up();
    load_rows();
  } else {
    more = false;
  }
  for (int s = 0; s < stages; ++s) send();

  // ------------------------------------------------------------------ products and softmax
  const int key_of = gr ^ ((gr >> 1) & 1);                         // keys of a block of eight in the order in which neither K's nor V's reads meet in a bank
  const int v0 = (2 * qd) ^ (qd & 1), v1 = v0 ^ 1;                 // the keys of the operands' columns 2 qd and 2 qd + 1
  int st = 0;
  uint32_t parity = 0;
  for (int x = x0; x < x1;) {
    const int len = min(unit.pages - j0, x1 - x), stop = min(j0 + len, unit.seen);
    uint32_t qf[NT][4 * WORDS];                                    // this lane's part of the query rows
    float row_scale[NT][2], m_ref[NT][2], l_sum[NT][2], o[MTILES][NT][4];
    int lim[NT][2], least = 0;                                     // keys that a row may see; the fewest
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int i = 0; i < WORDS; ++i) {
        qf[nt][4 * i] = q_rows[nt][i].x;
        qf[nt][4 * i + 1] = q_rows[nt][i].y;
        qf[nt][4 * i + 2] = q_rows[nt][i].z;
        qf[nt][4 * i + 3] = q_rows[nt][i].w;
      }
      // a row is divided by the power of two that makes its largest number 2^14 to 2^15, so that fp16 has room for it, and those that meet every second
      // pair of a word of codes by 16
      float down;                                                  // of row nt * 8 + gr: what it was divided by
      {
        float2 y[4 * WORDS];
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < 4 * WORDS; ++i) {
          y[i] = F16 ? __half22float2(as_half2(qf[nt][i])) : make_float2(__uint_as_float(qf[nt][i] << 16), __uint_as_float(qf[nt][i] & 0xffff0000u));
          top = fmaxf(top, fmaxf(fabsf(y[i].x), fabsf(y[i].y)));
        }
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        // (rows of infinities, of zeros or below 2^-86 are left as near as fp16 comes to them)
        const int e = (int)(__float_as_uint(top) >> 23);
        const int power = top == 0.f || e == 255 ? 0 : min(14 + 127 - e, 100);
        const float up = __uint_as_float((uint32_t)(127 + power) << 23);
        down = __uint_as_float((uint32_t)(127 - power) << 23);
#pragma unroll
        for (int i = 0; i < 4 * WORDS; ++i) qf[nt][i] = pack_half(y[i].x * (UNEVEN && (i & 1) ? up / 16.f : up), y[i].y * (UNEVEN && (i & 1) ? up / 16.f : up));
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        // (a normal number: 0 times a masked logit, or infinity times 0, would be none; logits below are 2^-90 then, or less)
        row_scale[nt][e] = fminf(fmaxf(p.scale_log2 * __shfl_sync(0xffffffffu, down, (2 * qd + e) * 4), 0x1p-126f), 0x1p127f);
        const int mine = nt * 8 + 2 * qd + e;
        lim[nt][e] = p.causal && mine < unit.rows ? min(unit.pos0 + (unit.row0 + mine) / p.G + 1, unit.kv) : unit.kv;
        m_ref[nt][e] = NO_MAX;
        l_sum[nt][e] = 0.f;
        least = nt + e == 0 ? lim[nt][e] : min(least, lim[nt][e]);
      }
    }
    least = __reduce_min_sync(0xffffffffu, least);
#pragma unroll
    for (int j = 0; j < MTILES; ++j)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[j][nt][i] = 0.f;
    for (int j = j0; j < stop; ++j) {
      if (!wait_all(full(st), parity, abort_flag, p.status, 1)) break;
      const unsigned char* page = ring + st * B::BYTES;
      const int first = j * PAGE;                             // key number of the page's first key
      float s[KT][NT][4];
      uint32_t kw[KT][2][WORDS], kb[KT][2];
#pragma unroll
      for (int mt = 0; mt < KT; ++mt) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[mt][nt][i] = 0.f;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int key = mt * 16 + u * 8 + key_of;
          if (D == 128) {
            const uint4 y = *reinterpret_cast<const uint4*>(page + B::K + key * B::ROW + qd * 16);
            kw[mt][u][0] = y.x, kw[mt][u][1] = y.y, kw[mt][u][WORDS - 2] = y.z, kw[mt][u][WORDS - 1] = y.w;
            kb[mt][u] = *reinterpret_cast<const uint16_t*>(page + B::KS + key * B::SCALES + qd * 2);
          } else {
            const uint2 y = *reinterpret_cast<const uint2*>(page + B::K + key * B::ROW + qd * 8);
            kw[mt][u][0] = y.x, kw[mt][u][1] = y.y;
            kb[mt][u] = page[B::KS + key * B::SCALES + qd];
          }
        }
      }
      // (the products of one tile wait for one another: the tiles take turns)
#pragma unroll
      for (int g = 0; g < WORDS / 2; ++g) {                      // sixteen columns with one scale
#pragma unroll
        for (int mt = 0; mt < KT; ++mt) {
          const Steps a(__byte_perm(kb[mt][0], 0, g ? 0x4141 : 0x4040)), b(__byte_perm(kb[mt][1], 0, g ? 0x4141 : 0x4040));
#pragma unroll
          for (int i = 2 * g; i < 2 * g + 2; ++i) {
            uint32_t ka[4], kc[4];
            values4(kw[mt][0][i], a, ka);
            values4(kw[mt][1][i], b, kc);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              mma_half(s[mt][nt], ka[0], kc[0], ka[1], kc[1], qf[nt][4 * i], qf[nt][4 * i + 1]);
              mma_half(s[mt][nt], ka[2], kc[2], ka[3], kc[3], qf[nt][4 * i + 2], qf[nt][4 * i + 3]);
            }
          }
        }
      }
      if (first + PAGE > least) {                                // some row may not see some of the keys (uniform)
#pragma unroll
        for (int mt = 0; mt < KT; ++mt)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (first + mt * 16 + (i >> 1) * 8 + key_of >= lim[nt][i & 1]) s[mt][nt][i] = -INFINITY;
      }
      bool grow = false;
      float top[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float t = fmaxf(s[0][nt][e], s[0][nt][2 + e]);
#pragma unroll
          for (int mt = 1; mt < KT; ++mt) t = fmax3(t, s[mt][nt][e], s[mt][nt][2 + e]);
          top[nt][e] = t * row_scale[nt][e];
          grow |= top[nt][e] > m_ref[nt][e] + MOVE;
        }
      if (__any_sync(0xffffffffu, grow)) {                       // new references
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float t = top[nt][e];
            t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 4));
            t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 8));
            t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 16));
            const float m_new = fmaxf(m_ref[nt][e], t - BELOW), f = exp2f(m_ref[nt][e] - m_new);
            m_ref[nt][e] = m_new;
            l_sum[nt][e] *= f;
#pragma unroll
            for (int j = 0; j < MTILES; ++j) {
              o[j][nt][e] *= f;
              o[j][nt][2 + e] *= f;
            }
          }
      }
      // probabilities: their sums take them as 32-bit numbers (a page's for themselves first: a long row's is off by an eighth of the roundings), the product
      // with V rounded to fp16, as the matrix unit wants its operands
      uint32_t pf[KT][NT][2];
      float of_page[NT][2];
#pragma unroll
      for (int mt = 0; mt < KT; ++mt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const float e0 = ex2_approx(fmaf(s[mt][nt][2 * u], row_scale[nt][0], -m_ref[nt][0]));
            const float e1 = ex2_approx(fmaf(s[mt][nt][2 * u + 1], row_scale[nt][1], -m_ref[nt][1]));
            of_page[nt][0] = mt + u == 0 ? e0 : of_page[nt][0] + e0;
            of_page[nt][1] = mt + u == 0 ? e1 : of_page[nt][1] + e1;
            pf[mt][nt][u] = transpose8(pack_half(e0, e1));
          }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) l_sum[nt][e] += of_page[nt][e];
      const int there = unit.kv - first;                         // keys of the page that exist
#pragma unroll
      for (int mt = 0; mt < KT; ++mt) {
        uint32_t w[4][WORDS / 2], bytes[4];                      // keys v0, v1 of either block of eight
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int key = mt * 16 + (u >> 1) * 8 + (u & 1 ? v1 : v0);
          if (D == 128) {
            const uint2 y = *reinterpret_cast<const uint2*>(page + B::V + key * B::ROW + gr * 8);
            w[u][0] = y.x, w[u][WORDS / 2 - 1] = y.y;
            bytes[u] = page[B::VS + key * B::SCALES + gr];
          } else {
            w[u][0] = *reinterpret_cast<const uint32_t*>(page + B::V + key * B::ROW + gr * 4);
            bytes[u] = page[B::VS + key * B::SCALES + (gr >> 1)];
          }
        }
        if (there < PAGE) {                                      // what lies behind the last key may be anything (uniform)
#pragma unroll
          for (int u = 0; u < 4; ++u)
            if (mt * 16 + (u >> 1) * 8 + (u & 1 ? v1 : v0) >= there) bytes[u] = 0;
        }
        const Steps a(bytes[0] | bytes[1] << 16), b(bytes[2] | bytes[3] << 16);
#pragma unroll
        for (int i = 0; i < WORDS / 2; ++i) {
          uint32_t a_even[4], a_odd[4], b_even[4], b_odd[4];
          values4(__byte_perm(w[0][i], w[1][i], 0x5410), a, a_even);
          values4(__byte_perm(w[0][i], w[1][i], 0x7632), a, a_odd);
          values4(__byte_perm(w[2][i], w[3][i], 0x5410), b, b_even);
          values4(__byte_perm(w[2][i], w[3][i], 0x7632), b, b_odd);
#pragma unroll
          for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma_half(o[i * 4 + n][nt], a_even[n], a_odd[n], b_even[n], b_odd[n], pf[mt][nt][0], pf[mt][nt][1]);
        }
      }
      __syncwarp();                                                // everybody has read the page
      send();
      if (++st == stages) {
        st = 0;
        parity ^= 1;
      }
    }
    // ---------------------------------------------------------------- the rows of the unit, or of the part of it
#pragma unroll
    for (int j = 1; j < (UNEVEN ? MTILES : 0); j += 2)             // (every second pair was 16 times as large)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[j][nt][i] *= 1.f / 16.f;
    const bool begins = j0 == 0, ends = j0 + len == unit.pages;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float& l = l_sum[nt][e];
        l += __shfl_xor_sync(0xffffffffu, l, 4);
        l += __shfl_xor_sync(0xffffffffu, l, 8);
        l += __shfl_xor_sync(0xffffffffu, l, 16);
      }
    if (begins && ends) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int row = nt * 8 + 2 * qd + e, of = unit.row0 + row, tok = unit.tok0 + of / p.G, hd = unit.head * p.G + of % p.G;
          if (row >= unit.rows) continue;
          const float l = l_sum[nt][e], inv = l == 0.f ? 0.f : q4.v_unit / l;
          uint4* dst = reinterpret_cast<uint4*>(static_cast<__half*>(p.out) + (int64_t)tok * p.o_tok + (int64_t)hd * p.o_head + gr * (D / 8));
#pragma unroll
          for (int c = 0; c < D / 64; ++c) {
            uint32_t y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = pack_out<F16>(o[4 * c + i][nt][e] * inv, o[4 * c + i][nt][2 + e] * inv);
            dst[c] = make_uint4(y[0], y[1], y[2], y[3]);
          }
          if (p.lse && gr == 0) p.lse[(int64_t)tok * p.H + hd] = l == 0.f ? -INFINITY : (m_ref[nt][e] + log2f(l)) * 0.6931471805599453f;
        }
    } else {
      // (a unit that goes on behind the range is its last one: all copies have landed, the ring is free)
      float* rows = begins ? reinterpret_cast<float*>(ring) : sp.ends + ((int64_t)blockIdx.x * WARPS + warp) * slot_floats(ROWS, D);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int row = nt * 8 + 2 * qd + e;
          if (gr == 0) reinterpret_cast<float2*>(rows + ROWS * D)[row] = make_float2(m_ref[nt][e], l_sum[nt][e]);
          // columns gr * D / 8 ..: words of four, their places changed so that the four lanes of a row group do not meet in a bank
#pragma unroll
          for (int c = 0; c < D / 32; ++c)
            reinterpret_cast<float4*>(rows + row * D)[(gr * (D / 32) + c) ^ qd] =
                make_float4(o[2 * c][nt][e], o[2 * c][nt][2 + e], o[2 * c + 1][nt][e], o[2 * c + 1][nt][2 + e]);
        }
      if (lane == 0) records[2 * warp + begins] = make_int4(unit.seq, unit.head, unit.tile, (begins ? 0 : 1) | (ends ? 0 : 2));
    }
    x += len;
    j0 = 0;
    if (x < x1) {
      unit.next(req, p);
      load_rows();
    }
  }
  if (*abort_flag) {
    // leaving early: every copy under way lands before the CTA exits
    for (int k = max(sent - stages, 0); k < sent; ++k) settle(full(k % stages), (k / stages) & 1);
  }
  // Warp 0, while others are still at work: the units that the run's borders cut, by lane 0 the first, by lane 1 the last, and the CTAs that have
  // parts of them.  (One unit that is both is lane 0's.)
  int c0 = blockIdx.x, c1 = -1;
  if (warp == 0) {
    const int side = lane & 1;
    Unit<ROWS> u;
    const int64_t ends[2] = {first_page, first_page + n_run - 1};
    int seqs[2];
    last_not_above(p.n_seq, pages_before, ends, seqs);
    const int j = locate(side ? ends[1] : ends[0], side ? seqs[1] : seqs[0], u);
    const bool cut = side ? j + 1 < u.pages : j > 0;
    const int64_t begin = req.pre[u.seq] + ((int64_t)u.head * u.tiles + u.tile) * (u.pages + UNIT_END), end = begin + u.pages + UNIT_END;
    // the last CTA whose run begins before `y`, a place of this unit (at its beginning: not behind it)
    auto last_before = [&](int64_t y) {
      auto before = [&](int c) {
        const int64_t raw = runs.raw(c);
        return raw < begin || (raw < end && Runs::snap(raw, begin, u.pages) < y);
      };
      int c = min(max((int)((float)y * 65536.f / (float)runs.share), 0), runs.grid - 1);
      while (c + 1 < runs.grid && before(c + 1)) ++c;
      while (c > 0 && !before(c)) --c;
      return c;
    };
    const bool same = __shfl_sync(0xffffffffu, (int)(u.seq == __shfl_xor_sync(0xffffffffu, u.seq, 1) && u.head == __shfl_xor_sync(0xffffffffu, u.head, 1) &&
                                                     u.tile == __shfl_xor_sync(0xffffffffu, u.tile, 1)), 0);
    const bool began = __shfl_sync(0xffffffffu, (int)cut, 0), goes_on = __shfl_sync(0xffffffffu, (int)cut, 1);
    if (side == 0 && began) {
      c0 = last_before(begin + 1);
      c1 = same && goes_on ? last_before(end) : (int)blockIdx.x;
    }
    if (side == 1 && goes_on && !(same && began)) c1 = last_before(end);
    if (lane >= 2) c1 = -1;
  }
  // ------------------------------------------------------------------ units that ranges' ends cut: added up by all warps, a row each
  __syncthreads();
  const int4 mine = lane < 2 * WARPS ? records[lane] : make_int4(-1, 0, 0, 0);
  const uint32_t met = __ballot_sync(0xffffffffu, mine.x >= 0);
  uint32_t left = met;
  int turn = 0;
  while (left) {
    const int head_lane = __ffs(left) - 1;
    unit.seq = __shfl_sync(0xffffffffu, mine.x, head_lane);
    unit.head = __shfl_sync(0xffffffffu, mine.y, head_lane);
    unit.tile = __shfl_sync(0xffffffffu, mine.z, head_lane);
    const uint32_t parties = __ballot_sync(0xffffffffu, mine.x == unit.seq && mine.y == unit.head && mine.z == unit.tile);
    left &= ~parties;
    const bool on = __shfl_sync(0xffffffffu, mine.w, 31 - __clz(parties)) & 2, from_before = __shfl_sync(0xffffffffu, mine.w, head_lane) & 1;
    unit.set(req, p);
    const bool cut = on || from_before;
    // a warp has at most one part of a unit: in its ring where the unit begins in its range, else in the workspace
    auto rows_of = [&](int w) {
      return parties >> (2 * w + 1) & 1 ? reinterpret_cast<const float*>(smem + w * stages * B::BYTES)
                                        : sp.ends + ((int64_t)blockIdx.x * WARPS + w) * slot_floats(ROWS, D);
    };
    float* slot = p.partials + (2 * (int64_t)blockIdx.x + (from_before ? 0 : 1)) * slot_floats(ROWS, D);
    constexpr int LANES = D / 4, AT_ONCE = 32 / LANES;             // lanes of a row, rows at once
    const int my = lane % LANES;
    for (int r0 = 0; r0 < unit.rows; r0 += AT_ONCE, ++turn) {
      if (turn % WARPS != warp) continue;
      const int row = r0 + lane / LANES;
      float4 c[WARPS];
      float2 ml[WARPS];
#pragma unroll
      for (int w = 0; w < WARPS; ++w) {
        ml[w] = make_float2(NO_MAX, 0.f);
        c[w] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (!(parties >> (2 * w) & 3)) continue;
        const float* from = rows_of(w);
        ml[w] = reinterpret_cast<const float2*>(from + ROWS * D)[row];
        c[w] = reinterpret_cast<const float4*>(from + row * D)[my];
      }
      float top = ml[0].x, sum = 0.f;
#pragma unroll
      for (int w = 1; w < WARPS; ++w) top = fmaxf(top, ml[w].x);
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < WARPS; ++w) {
        const float f = exp2f(ml[w].x - top);
        sum = fmaf(ml[w].y, f, sum);
        acc.x = fmaf(c[w].x, f, acc.x);
        acc.y = fmaf(c[w].y, f, acc.y);
        acc.z = fmaf(c[w].z, f, acc.z);
        acc.w = fmaf(c[w].w, f, acc.w);
      }
      if (row >= unit.rows) continue;
      const int col = (my ^ ((row >> 1) & 3)) * 4, of = unit.row0 + row, tok = unit.tok0 + of / p.G, hd = unit.head * p.G + of % p.G;
      if (cut) {
        __stcg(reinterpret_cast<float4*>(slot + row * D + col), acc);
        if (my == 0) __stcg(reinterpret_cast<float2*>(slot + ROWS * D) + row, make_float2(top, sum));
      } else {
        const float inv = sum == 0.f ? 0.f : q4.v_unit / sum;
        uint32_t* dst = reinterpret_cast<uint32_t*>(static_cast<__half*>(p.out) + (int64_t)tok * p.o_tok + (int64_t)hd * p.o_head + col);
        *reinterpret_cast<uint2*>(dst) = make_uint2(pack_out<F16>(acc.x * inv, acc.y * inv), pack_out<F16>(acc.z * inv, acc.w * inv));
        if (p.lse && my == 0) p.lse[(int64_t)tok * p.H + hd] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
      }
    }
  }
  // ------------------------------------------------------------------ units that the run's borders cut: added up by the CTA that leaves their last part
  const int first_lane = __ffs(met) - 1, last_lane = 31 - __clz(met);
  const bool any_cut = met && ((__shfl_sync(0xffffffffu, mine.w, first_lane) & 1) || (__shfl_sync(0xffffffffu, mine.w, last_lane) & 2));
  if (!any_cut) return;
  __syncthreads();
  if (warp == 0 && c1 >= 0) {                                      // (lanes 0 and 1)
    __threadfence();                                               // all warps' rows, behind the barrier
    const bool last = atomicAdd(p.counters + c0, 1u) == (uint32_t)(c1 - c0);
    if (last) *reinterpret_cast<volatile uint32_t*>(p.counters + c0) = 0;                // ready for the next launch
    if (last) final_parts[lane] = make_int2(c0, c1);
    __threadfence();
  }
  __syncthreads();
#pragma unroll 1
  for (int u = 0; u < 2; ++u) {
    const int c0 = final_parts[u].x, c1 = final_parts[u].y;
    if (c1 < c0) continue;
    const int of = u == 0 ? first_lane : last_lane;
    unit.seq = __shfl_sync(0xffffffffu, mine.x, of);
    unit.head = __shfl_sync(0xffffffffu, mine.y, of);
    unit.tile = __shfl_sync(0xffffffffu, mine.z, of);
    unit.set(req, p);
    for (int row = warp; row < unit.rows; row += WARPS) {
      constexpr int N = D / 32, AHEAD = 8;
      auto part = [&](int c) { return p.partials + (2 * (int64_t)c + (c == c0)) * slot_floats(ROWS, D); };
      float acc[N], l = 0.f, top = NO_MAX;
#pragma unroll
      for (int k = 0; k < N; ++k) acc[k] = 0.f;
      for (int base = c0; base <= c1; base += AHEAD) {
        float c[AHEAD][N];
        float2 ml[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
          ml[i] = make_float2(NO_MAX, 0.f);
#pragma unroll
          for (int k = 0; k < N; ++k) c[i][k] = 0.f;
          if (base + i > c1) continue;
          const float* s = part(base + i);
          ml[i] = __ldcg(reinterpret_cast<const float2*>(s + ROWS * D) + row);
          if (N == 4) {
            const float4 y = __ldcg(reinterpret_cast<const float4*>(s + row * D) + lane);
            c[i][0] = y.x, c[i][1] = y.y, c[i][N - 2] = y.z, c[i][N - 1] = y.w;
          } else {
            const float2 y = __ldcg(reinterpret_cast<const float2*>(s + row * D) + lane);
            c[i][0] = y.x, c[i][1] = y.y;
          }
        }
        float t = top;
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) t = fmaxf(t, ml[i].x);
        const float f0 = exp2f(top - t);
        top = t;
        l *= f0;
#pragma unroll
        for (int k = 0; k < N; ++k) acc[k] *= f0;
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
          const float f = exp2f(ml[i].x - top);
          l = fmaf(ml[i].y, f, l);
#pragma unroll
          for (int k = 0; k < N; ++k) acc[k] = fmaf(c[i][k], f, acc[k]);
        }
      }
      const int of = unit.row0 + row, tok = unit.tok0 + of / p.G, hd = unit.head * p.G + of % p.G;
      const float inv = l == 0.f ? 0.f : q4.v_unit / l;
      uint32_t* dst = reinterpret_cast<uint32_t*>(static_cast<__half*>(p.out) + (int64_t)tok * p.o_tok + (int64_t)hd * p.o_head + lane * N);
#pragma unroll
      for (int k = 0; k < N; k += 2) dst[k / 2] = pack_out<F16>(acc[k] * inv, acc[k + 1] * inv);
      if (p.lse && lane == 0) p.lse[(int64_t)tok * p.H + hd] = l == 0.f ? -INFINITY : (top + log2f(l)) * 0.6931471805599453f;
    }
  }
}

uint64_t slot_bytes(int d, int rows, int slots) { return ((uint64_t)slots * slot_floats(rows, d) * 4 + 255) / 256 * 256; }

template <int D, int NT, bool F16, int WARPS>
cudaError_t launch(const Paged4Params& q, int n_sm, cudaStream_t stream) {
  constexpr int stage = WARPS * Block4<D>::BYTES, room = 226 * 1024 - 1024;
  const int fixed = Requests::bytes(q.a.n_seq);
  Small4Params sp;
  sp.q = q;
  sp.ends = q.a.partials + slot_bytes(D, 8 * NT, 2 * n_sm) / 4;
  sp.inverse = (uint32_t)((1ull << 32) / (unsigned)n_sm);
  // as many pages under way as shared memory holds (of a call of 3200 requests and more one a warp)
  sp.stages = std::max(1, std::min(MAX_STAGES, (room - fixed) / stage));
  auto kernel = paged4_small_kernel<D, NT, F16, WARPS>;
  // (the kernel's limit is the process's: always the most that any call takes, as another thread may set it between this line and the launch)
  cudaError_t rc = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, room);
  if (rc != cudaSuccess) return rc;
  return launch_pdl(kernel, dim3(n_sm), dim3(WARPS * 32), fixed + sp.stages * stage, stream, sp);
}
template <int D, bool F16>
cudaError_t launch_typed(const Paged4Params& q, int rows, int n_sm, cudaStream_t stream) {
  if (rows > 8) return launch<D, 2, F16, 8>(q, n_sm, stream);
  // Twelve warps with two pages each under way where there is much to do, eight with three where the beginning and the end of a call weigh more (128-wide
  // heads).  Time of twelve over eight, one to 256 requests of 2 and 8 kv heads, by pages of the table and kv head: 1.00 to 1.12 at 4000, 1.01 at 8000, 1.00 at 9000 and
  // 10 000, 0.98 to 1.00 at 11 000 to 14 000, 0.97 to 0.99 at 16 000, 0.95 at 32 000 (requests of spread lengths 0.85 to 1.01 there).
  const bool much = D == 128 && q.a.n_seq <= 340 && (int64_t)q.a.n_seq * q.a.Hkv * q.a.table_pages >= 10000;
  return much ? launch<D, 1, F16, D == 128 ? 12 : 8>(q, n_sm, stream) : launch<D, 1, F16, 8>(q, n_sm, stream);
}

}  // namespace

uint64_t paged4_small_partial_bytes(int d, int n_sm) { return slot_bytes(d, 16, 2 * n_sm) + slot_bytes(d, 16, MOST_WARPS * n_sm); }

cudaError_t launch_paged4_small(const Paged4Params& p, int d, const PagedDevice& dev, cudaStream_t stream) {
  const int rows = (int64_t)std::max(1, p.a.max_new) * p.a.G <= 8 ? 8 : 16;
  if (p.fp16) return d == 128 ? launch_typed<128, true>(p, rows, dev.n_sm, stream) : launch_typed<64, true>(p, rows, dev.n_sm, stream);
  return d == 128 ? launch_typed<128, false>(p, rows, dev.n_sm, stream) : launch_typed<64, false>(p, rows, dev.n_sm, stream);
}

}  // namespace heatkv
