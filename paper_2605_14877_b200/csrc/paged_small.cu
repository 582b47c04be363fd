// Attention of few query rows over a paged cache (decode, drafted tokens) and over selected pages, on warp-level MMA.
//
// A row tile is tile_tokens consecutive tokens of a request times the G query heads of one kv head, up to 32 rows (64 over selected pages; where a
// request has more, several of 16); a unit is a row tile
// of one request and kv head, its keys come page by page.  What bounds it is the reading of K and V, so the work is cut by pages, not by
// requests: a unit of more than S pages is cut into equal pieces of at most S, S such that every CTA takes about PER_CTA pieces, and CTAs
// take pieces from a counter until none is left (dealt out beforehand in equal shares, the SMs with the longest way to memory decided when
// a call ended: SMs' active cycles differed by 15 %).  Pieces leave partial results (unnormalised O, maximum, sum) in the workspace, which a
// second small kernel adds up in page order; neither the pieces nor that order depends on which CTA took what.  (Added up by the CTA that
// leaves a unit's last piece, with a fence and a counter behind every piece, a decode of 64 requests took 92 us, with the second kernel 67.)
//
// One warp takes pieces and looks up what they are, one ahead; the next sends for Q, K and V (TMA, K and V of one page per stage),
// so that what a piece's beginning has to read (counter, lengths, table) is read while the pages before it arrive.  The others
// come in groups of four for 16 MT rows each; a warp takes 16 keys of a page for the logits and a quarter of the columns for the product
// with V, so no two of a group hold parts of the same result; between the two the probabilities pass through shared memory, and the one
// barrier that this takes also counts whether some row's maximum has outgrown its reference, which all four share (then, seldom, the
// page's probabilities are taken again).  Rows past a request's last key in its last page are whatever the pool holds: their logits are
// masked and their values replaced by zero.
#include <algorithm>
#include <climits>

#include <cuda_fp16.h>

#include "paged_wait.cuh"

namespace heatkv {
namespace {

using namespace tc;

constexpr int MAX_STAGES = 12;
constexpr float MOVE = 8.f;                    // a reference moves when a maximum passes it by more than 2^MOVE (P fits fp16)
// Pages of a piece.  In a small call every CTA takes one piece, of at least MIN_CHUNK pages (one token, 32 pages of 8 kv heads: 9.5 us with 4, 10.8
// with 8) and at most FULL_CHUNK (24 requests of drafted tokens: 20.1 us in two rounds of 4, 16.7 in one of up to 8; 64 requests
// of 500 tokens, 8 kv heads: 31.4 in pieces of 6, 28.5 of 8, which is whole units); in a large one PER_CTA, longer ones (64 requests of 1360 tokens on
// average: 66.9 us with 4, 67.7 with 3, 68.1 with 6 or 8).
constexpr int MIN_CHUNK = 4, FULL_CHUNK = 8;
// (and units of up to FULL_CHUNK pages stay whole: a short request then needs no second kernel, 7.3 us instead of 10)
constexpr int PER_CTA = 4;
constexpr int MERGE_WARPS = 8;

struct SmallParams {
  PagedParams a;
  uint32_t* counter;                           // pieces taken beyond every CTA's first; zero between launches
  int2* cuts;                                  // [n_tokens][Hkv] {the unit's first slot, its pieces | the token's place in it << 16}; not cut: no pieces
  int32_t stages;
};
struct SmallMaps {
  CUtensorMap q, k, v;
};

template <int D, int MT, int GROUPS>
struct SmallLayout {
  static constexpr int WARPS = 4 * GROUPS;                       // that compute
  static constexpr int THREADS = (WARPS + 2) * 32;
  static constexpr int CTAS = GROUPS == 1 ? 2 : 1;               // of an SM: one's pages arrive while the other ends a unit
  static constexpr int ROWS = 16 * MT * GROUPS;
  static constexpr uint32_t TILE = PAGE * D * 2;                 // K or V of one page
  static constexpr uint32_t Q_BYTES = ROWS * D * 2;              // two buffers
  static constexpr uint32_t P_BYTES = ROWS * PAGE * 2;           // probabilities of a page, two buffers
  static constexpr uint32_t ML = 4 * ROWS * 4;                   // maxima or sums of the four warps of a group
  static constexpr uint32_t FIXED = 2 * Q_BYTES + 2 * P_BYTES + ML;
};

// c += a x b for one 16 x 8 x 16 product of bf16 or fp16
template <bool F16>
__device__ __forceinline__ void mma16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  // (not volatile: a product depends on its operands alone and may move between the loads, which keep their order)
  if (F16)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <bool F16>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
  if (F16) {
    __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&v);
  }
  return pack_bf16(lo, hi);
}

// The four warps of a group meet; with a vote: whether any of their threads says so.
__device__ __forceinline__ bool meet_any(int group, bool mine) {
  uint32_t any;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 q, %1, 0;\n\tbar.red.or.pred p, %2, 128, q;\n\tselp.u32 %0, 1, 0, p;\n\t}"
               : "=r"(any)
               : "r"((uint32_t)mine), "r"(group + 1)
               : "memory");
  return any != 0;
}
__device__ __forceinline__ void meet(int group) { asm volatile("bar.sync %0, 128;" ::"r"(group + 1) : "memory"); }

// A partial result: rows of O, then their maxima and sums; whole 16-byte words.
__host__ __device__ constexpr int64_t slot_floats(int rows, int d) { return ((int64_t)rows * (d + 2) + 3) & ~(int64_t)3; }

__device__ __forceinline__ int chunk_of(int64_t pages, int units, int ctas) {
  const int room = ctas - units / 2;                               // (a unit's last piece is half empty on average)
  int chunk = FULL_CHUNK;
  if (room > 0 && pages < (int64_t)room * FULL_CHUNK) chunk = max(((int)pages + room - 1) / room, MIN_CHUNK);
  const int64_t share = (int64_t)ctas * PER_CTA;
  return pages <= share * chunk ? chunk : (int)((pages + share - 1) / share);
}
__device__ __forceinline__ int pieces_of(int pages, int chunk) { return pages <= FULL_CHUNK ? pages > 0 : (pages + chunk - 1) / chunk; }

enum RingWord : int { W_KIND = 0, W_HEAD, W_TOK0, W_ROWS, W_TILES, W_KV, W_POS0, W_SLOT, W_PIECE, W_PIECES, W_SEQ, W_TILE0, RING_WORDS = 12 };
constexpr int RING = 2;                        // the piece at work and the next: more would be taken from CTAs that run out

__device__ __forceinline__ int find_last(const int32_t* a, int n, int x) {     // last i in [0, n) with a[i] <= x
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a[mid] <= x) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// A part of a row's sum: columns lane * D / 32 .., relative to the maximum `top`.
template <int D>
struct RowSum {
  static constexpr int N = D / 32;
  float acc[N], top, l;
  __device__ void clear() {
    top = NO_MAX;
    l = 0.f;
#pragma unroll
    for (int k = 0; k < N; ++k) acc[k] = 0.f;
  }
};
// A row's parts in the workspace (`first`: the unit's first slot).
template <int D>
struct Parts {
  static constexpr int N = D / 32;
  const float* first;
  int64_t pitch;
  int slot_rows, row, lane;
  struct Columns {
    float v[N];
  };
  __device__ float2 stats(int i) const { return __ldcg(reinterpret_cast<const float2*>(first + i * pitch + slot_rows * D) + row); }
  __device__ Columns columns(int i) const {
    Columns c;
    const float* src = first + i * pitch + row * D + lane * N;
    if (N == 4) {
      const float4 y = __ldcg(reinterpret_cast<const float4*>(src));
      c.v[0] = y.x, c.v[1] = y.y, c.v[N - 2] = y.z, c.v[N - 1] = y.w;
    } else {
      const float2 y = __ldcg(reinterpret_cast<const float2*>(src));
      c.v[0] = y.x, c.v[1] = y.y;
    }
    return c;
  }
};
// Parts begin .. end - 1, by a warp.  The first ones' columns come with the maxima and sums, not behind them (a decode of 64 requests, up to 16
// parts: 69.1 us with 4 of them, 68.7 with 8, 66.9 with 12, 67.2 with 16; one request of 131 000 tokens 98.2, 97.8, 95.6, 96.1).
constexpr int AHEAD = 12;
template <int D>
__device__ __forceinline__ RowSum<D> sum_parts(const Parts<D>& p, int begin, int end) {
  constexpr int N = D / 32;
  RowSum<D> r;
  r.clear();
  const int n = end - begin;
  typename Parts<D>::Columns ahead[AHEAD];
#pragma unroll
  for (int i = 0; i < AHEAD; ++i)
    if (i < n) ahead[i] = p.columns(begin + i);
  float2 ml = make_float2(NO_MAX, 0.f);                            // of part begin + lane
  if (p.lane < n) ml = p.stats(begin + p.lane);
  r.top = ml.x;
  for (int i = p.lane + 32; i < n; i += 32) r.top = fmaxf(r.top, p.stats(begin + i).x);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) r.top = fmaxf(r.top, __shfl_xor_sync(0xffffffffu, r.top, o));
  for (int base = 0; base < n; base += 32) {
    if (base > 0) ml = base + p.lane < n ? p.stats(begin + base + p.lane) : make_float2(NO_MAX, 0.f);
    const float w = exp2f(ml.x - r.top), wl = ml.y * w;
    const int m = min(32, n - base);
    auto add = [&](int i, const typename Parts<D>::Columns& c) {
      const float wi = __shfl_sync(0xffffffffu, w, i);
      r.l += __shfl_sync(0xffffffffu, wl, i);
#pragma unroll
      for (int k = 0; k < N; ++k) r.acc[k] = fmaf(c.v[k], wi, r.acc[k]);
    };
    int i = 0;
    if (base == 0) {
#pragma unroll
      for (int k = 0; k < AHEAD; ++k)
        if (k < m) add(k, ahead[k]);
      i = min(AHEAD, m);
    }
#pragma unroll 4
    for (; i < m; ++i) add(i, p.columns(begin + base + i));
  }
  return r;
}
template <int D, bool F16>
__device__ __forceinline__ void put_row(const PagedParams& p, const RowSum<D>& r, int tok, int hd, int lane) {
  constexpr int N = D / 32;
  const float inv = r.l == 0.f ? 0.f : 1.f / r.l;                  // (0: no key; a sum that is NaN stays one, here and in the logarithm)
  uint32_t* dst = reinterpret_cast<uint32_t*>(static_cast<__nv_bfloat16*>(p.out) + (int64_t)tok * p.o_tok + (int64_t)hd * p.o_head + lane * N);
  if (N == 4) {
    *reinterpret_cast<uint2*>(dst) = make_uint2(pack16<F16>(r.acc[0] * inv, r.acc[1] * inv), pack16<F16>(r.acc[N - 2] * inv, r.acc[N - 1] * inv));
  } else {
    *dst = pack16<F16>(r.acc[0] * inv, r.acc[1] * inv);
  }
  if (p.lse && lane == 0) p.lse[(int64_t)tok * p.H + hd] = r.l == 0.f ? -INFINITY : (r.top + log2f(r.l)) * 0.6931471805599453f;
}

template <int D, int MT, int GROUPS, bool F16, bool SPARSE>
__global__ void __launch_bounds__((SmallLayout<D, MT, GROUPS>::THREADS), (SmallLayout<D, MT, GROUPS>::CTAS))
paged_small_kernel(const __grid_constant__ SmallParams sp, const __grid_constant__ SmallMaps maps) {
  using L = SmallLayout<D, MT, GROUPS>;
  constexpr int NCH = D / 64, ROWS = L::ROWS, WARPS = L::WARPS, THREADS = L::THREADS;
  const PagedParams& p = sp.a;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t sbase = (raw + 1023u) & ~1023u;
  unsigned char* sgen = smem_raw + (sbase - raw);
  const int stages = sp.stages;
  const uint32_t q_off = stages * 2 * L::TILE, p_off = q_off + 2 * L::Q_BYTES, ml_off = p_off + 2 * L::P_BYTES, pre_off = ml_off + L::ML;
  int32_t* chunk_begin = reinterpret_cast<int32_t*>(sgen + pre_off);            // [n_seq + 1] pieces before the request
  int32_t* slot_begin = chunk_begin + p.n_seq + 1;                              // [n_seq + 1] partial results before it
  __shared__ __align__(8) uint64_t bars[2 * MAX_STAGES + 2 * RING + 2];
  __shared__ int32_t ring[RING][RING_WORDS];
  __shared__ int32_t ring_page[RING][32], ring_place[RING][32];                 // the piece's first pages, in the pool and in the table row
  __shared__ int32_t page_of[MAX_STAGES];                                       // place in the request's table row of the page in a stage
  __shared__ uint32_t abort_word, leave_word[GROUPS];
  __shared__ int64_t sums[WARPS + 2];
  volatile uint32_t* abort_flag = &abort_word;
  const uint32_t bar0 = smem_u32(bars);
  auto full = [&](int s) { return bar0 + s * 16; };
  auto empty = [&](int s) { return bar0 + s * 16 + 8; };
  auto ring_full = [&](int s) { return bar0 + MAX_STAGES * 16 + s * 8; };
  auto ring_empty = [&](int s) { return bar0 + MAX_STAGES * 16 + (RING + s) * 8; };
  auto q_full = [&](int s) { return bar0 + MAX_STAGES * 16 + (2 * RING + s) * 8; };
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;

  pdl_trigger();
  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) {
      mbar_init(full(s), 1);
      mbar_init(empty(s), WARPS);
    }
    for (int s = 0; s < RING; ++s) {
      mbar_init(ring_full(s), 1);
      mbar_init(ring_empty(s), WARPS + 1);
    }
    for (int s = 0; s < 2; ++s) mbar_init(q_full(s), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  // rows of a tile that no copy writes stay zero
  for (uint32_t i = threadIdx.x; i < 2 * L::Q_BYTES / 16; i += THREADS) reinterpret_cast<int4*>(sgen + q_off)[i] = make_int4(0, 0, 0, 0);
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  pdl_wait();
  if (threadIdx.x == 0) *abort_flag = *reinterpret_cast<volatile uint32_t*>(p.status) != 0;
  // S, the pieces and the partial results.  (A request without keys has no pieces, and its rows get their zeros here.)
  int64_t total = 0;
  int chunk = 0, n_chunks = 0;
  if (SPARSE) {
    total = (int64_t)p.n_tokens * p.Hkv * p.n_sel;
    chunk = chunk_of(total, (int)min((int64_t)p.n_tokens * p.Hkv, (int64_t)INT_MAX), gridDim.x);
    const int pieces = pieces_of(p.n_sel, chunk);
    n_chunks = (int)min((int64_t)p.n_tokens * p.Hkv * pieces, (int64_t)INT_MAX);
    __syncthreads();
  } else {
    const int per = (p.n_seq + THREADS - 1) / THREADS, i0 = min((int)threadIdx.x * per, p.n_seq), i1 = min(i0 + per, p.n_seq);
    auto scan = [&](int64_t v, int64_t& all) {
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
      for (int w = 0; w < WARPS + 2; ++w) {
        const int64_t x = sums[w];
        if (w < warp) before += x;
        all += x;
      }
      return before + inc - v;
    };
    int64_t sum = 0;
    int units_mine = 0;
    for (int i = i0; i < i1; ++i) {
      const int b = max(p.q_begin[i], 0), n = max(min(p.q_begin[i + 1], p.n_tokens) - b, 0);
      const int kv = min(max(p.kv_len[i], 0), p.table_pages * PAGE);
      const int tiles = (kv + PAGE - 1) / PAGE, units = (n + p.tile_tokens - 1) / p.tile_tokens * p.Hkv;
      chunk_begin[i] = units;
      slot_begin[i] = tiles;
      sum += (int64_t)tiles * units;
      if (tiles > 0) units_mine = min(units_mine + units, 4096);
    }
    // pages, and above them the units, as many as matter
    constexpr int64_t PAGES = ((int64_t)1 << 43) - 1;
    scan(min(sum, PAGES / THREADS) + ((int64_t)min(units_mine, 4096) << 43), total);
    chunk = chunk_of(total & PAGES, (int)(total >> 43), gridDim.x);
    // (both in one sum: pieces in the low 40 bits, partial results, of which there are few, above)
    constexpr int64_t LOW = ((int64_t)1 << 40) - 1;
    int64_t mine = 0, all;
    for (int i = i0; i < i1; ++i) {
      const int pieces = pieces_of(slot_begin[i], chunk);
      const int64_t c = (int64_t)chunk_begin[i] * pieces;
      mine += c + (pieces > 1 ? c << 40 : 0);
    }
    int64_t at = scan(mine, all);
    for (int i = i0; i < i1; ++i) {
      const int pieces = pieces_of(slot_begin[i], chunk);
      const int64_t c = (int64_t)chunk_begin[i] * pieces;
      chunk_begin[i] = (int)min((int64_t)(at & LOW), (int64_t)INT_MAX);
      slot_begin[i] = (int)(at >> 40);
      at += c + (pieces > 1 ? c << 40 : 0);
    }
    n_chunks = (int)min((int64_t)(all & LOW), (int64_t)INT_MAX);
    if (threadIdx.x == 0) chunk_begin[p.n_seq] = n_chunks;
    __syncthreads();
    for (int i = blockIdx.x; i < p.n_seq; i += gridDim.x) {
      if (chunk_begin[i + 1] != chunk_begin[i]) continue;
      const int b = max(p.q_begin[i], 0), e = min(p.q_begin[i + 1], p.n_tokens);
      const int64_t n = (int64_t)max(e - b, 0) * p.H;
      for (int64_t j = threadIdx.x; j < n * D; j += THREADS) {
        const int64_t t = b + j / ((int64_t)p.H * D), hd = j / D % p.H;
        static_cast<uint16_t*>(p.out)[t * p.o_tok + hd * p.o_head + j % D] = 0;
      }
      if (p.lse)
        for (int64_t j = threadIdx.x; j < n; j += THREADS) p.lse[b * (int64_t)p.H + j] = -INFINITY;
      for (int64_t j = threadIdx.x; j < (int64_t)max(e - b, 0) * p.Hkv; j += THREADS) sp.cuts[b * (int64_t)p.Hkv + j] = make_int2(-1, 0);
    }
  }

  // page j of a piece that ends before page `end`: number in the pool, and place in the request's table row
  auto look_up = [&](int seq, int head, int tok0, int pos0, int j, int end) {
    int place = -1, page = -1;
    if (j < end) {
      place = j;
      if (SPARSE) {
        place = p.sel[((int64_t)tok0 * p.Hkv + head) * p.n_sel + j];
        if (pos0 < 0 || place > pos0 / PAGE) place = -1;           // nothing there that the query may see
      }
      if (place >= 0 && place < p.table_pages) page = p.block_table[seq * p.table_stride + place];
      if (page < 0 || page >= p.n_pages) page = -1;                // (a box outside of the map arrives as zeros)
    }
    if (place < 0 || place >= p.table_pages) place = 1 << 24;      // past every limit
    return make_int2(page, place);
  };
  if (warp == WARPS) {
    // ------------------------------------------------------------------ pieces
    const bool leader = elect_one();
    // The next piece is asked for while this one is looked up; every CTA that had one ends with one question too many, and the last of
    // those n_chunks questions puts the counter back.
    auto ask = [&]() {
      uint32_t next = 0;
      if (lane == 0) {
        next = atomicAdd(sp.counter, 1u);
        if (next == (uint32_t)n_chunks - 1u) *reinterpret_cast<volatile uint32_t*>(sp.counter) = 0;
      }
      return next;
    };
    int idx = blockIdx.x;
    for (uint32_t it = 0;; ++it) {
      const uint32_t slot = it % RING;
      if (it >= RING && !wait_all(ring_empty(slot), ((it / RING) - 1) & 1, abort_flag, p.status, 1)) break;
      if (idx >= n_chunks) {
        if (lane == 0) ring[slot][W_KIND] = 0;
        __syncwarp();
        if (leader) mbar_arrive(ring_full(slot));
        break;
      }
      const uint32_t next = ask();
      int seq, head, tok0, tokens, kv, pos0, tiles, piece, pieces, out_slot;
      if (SPARSE) {
        pieces = pieces_of(p.n_sel, chunk);
        const int unit = idx / pieces;
        piece = idx - unit * pieces;
        out_slot = pieces > 1 ? idx : -1;
        tok0 = unit / p.Hkv;
        head = unit - tok0 * p.Hkv;
        seq = find_last(p.q_begin, p.n_seq, tok0);
        const int e = p.q_begin[seq + 1];
        kv = p.kv_len[seq];
        tokens = tok0 >= p.q_begin[seq] && tok0 < e ? 1 : 0;       // rows past the last request's are nobody's
        pos0 = tokens ? kv - e + tok0 : -1;
        tiles = p.n_sel;
      } else {
        seq = find_last(chunk_begin, p.n_seq, idx);
        const int b = max(p.q_begin[seq], 0), n = max(min(p.q_begin[seq + 1], p.n_tokens) - b, 0);
        kv = min(max(p.kv_len[seq], 0), p.table_pages * PAGE);
        tiles = (kv + PAGE - 1) / PAGE;
        pieces = pieces_of(tiles, chunk);
        const int local = idx - chunk_begin[seq], unit = local / pieces;
        piece = local - unit * pieces;
        out_slot = pieces > 1 ? slot_begin[seq] + local : -1;
        const int first = unit / p.Hkv * p.tile_tokens;
        head = unit % p.Hkv;
        tok0 = b + first;
        tokens = min(p.tile_tokens, n - first);
        pos0 = kv - n + first;
      }
      const int size = (tiles + pieces - 1) / pieces, tile0 = min(piece * size, tiles);
      int tile1 = min(tile0 + size, tiles);
      // pages that none of the tile's tokens sees are left out (a piece of nothing else is empty): 3 prompts of 400, 4 kv heads, 16.7 us instead of 18.3
      if (!SPARSE && p.causal) tile1 = max(tile0, min(tile1, (max(pos0 + tokens, 0) + PAGE - 1) / PAGE));
      if (lane == 0) {
        int32_t* w = ring[slot];
        w[W_KIND] = 1;
        w[W_HEAD] = head;
        w[W_TOK0] = tok0;
        w[W_ROWS] = tokens * p.G;
        w[W_TILES] = tile1 - tile0;
        w[W_KV] = kv;
        w[W_POS0] = pos0;
        w[W_SLOT] = out_slot;
        w[W_PIECE] = piece;
        w[W_PIECES] = pieces;
        w[W_SEQ] = seq;
        w[W_TILE0] = tile0;
      }
      const int2 a = look_up(seq, head, tok0, pos0, tile0 + lane, tile1);
      ring_page[slot][lane] = a.x;
      ring_place[slot][lane] = a.y;
      __syncwarp();
      if (leader) mbar_arrive(ring_full(slot));
      idx = (int)gridDim.x + (int)__shfl_sync(0xffffffffu, next, 0);
    }
    return;
  }
  if (warp == WARPS + 1) {
    // ------------------------------------------------------------------ copies
    const bool leader = elect_one();
    const uint32_t q_bytes = (uint32_t)(p.tile_tokens * p.G) * 128 * NCH;
    uint32_t g = 0, it = 0;
    bool ok = true;
    for (;; ++it) {
      const uint32_t slot = it % RING, q = it & 1;
      ok = wait_all(ring_full(slot), (it / RING) & 1, abort_flag, p.status, 6);
      if (!ok) break;
      const volatile int32_t* w = ring[slot];
      if (w[W_KIND] == 0) break;
      const int tiles = w[W_TILES], tile0 = w[W_TILE0], head = w[W_HEAD], tok0 = w[W_TOK0];
      int page32 = ring_page[slot][lane], place32 = ring_place[slot][lane];
      // (the query rows' buffer was the last but one piece's)
      if (it >= 2) ok = wait_all(ring_empty((it - 2) % RING), ((it - 2) / RING) & 1, abort_flag, p.status, 7);
      if (!ok) break;
      if (leader) {
        mbar_expect_tx(q_full(q), q_bytes);
#pragma unroll
        for (int ch = 0; ch < NCH; ++ch) tma_load_4d(sbase + q_off + q * L::Q_BYTES + ch * ROWS * 128, &maps.q, ch * 64, head * p.G, tok0, 0, q_full(q));
      }
      __syncwarp();
      for (int j = 0; j < tiles; ++j, ++g) {
        if (j > 0 && (j & 31) == 0) {
          const int2 a = look_up(w[W_SEQ], head, tok0, w[W_POS0], tile0 + j + lane, tile0 + tiles);
          page32 = a.x;
          place32 = a.y;
        }
        const int page = __shfl_sync(0xffffffffu, page32, j & 31), place = __shfl_sync(0xffffffffu, place32, j & 31);
        const uint32_t st = g % stages, use = g / stages;
        if (use > 0) ok = wait_all(empty(st), (use - 1) & 1, abort_flag, p.status, 2);
        if (!ok) break;
        if (leader) {
          page_of[st] = place;
          mbar_expect_tx(full(st), 2 * L::TILE);
          const uint32_t dst = sbase + st * 2 * L::TILE;
#pragma unroll
          for (int ch = 0; ch < NCH; ++ch) tma_load_4d(dst + ch * PAGE * 128, &maps.k, ch * 64, 0, head, page, full(st));
#pragma unroll
          for (int ch = 0; ch < NCH; ++ch) tma_load_4d(dst + L::TILE + ch * PAGE * 128, &maps.v, ch * 64, 0, head, page, full(st));
        }
        __syncwarp();
      }
      if (!ok) {
        ++it;                                                      // (its query rows are under way)
        break;
      }
      if (leader) mbar_arrive(ring_empty(slot));
      __syncwarp();
    }
    if (!ok || *abort_flag) {
      // leaving early: every copy under way lands before the CTA exits
      for (uint32_t s = 0; s < (uint32_t)stages; ++s)
        if (g > s) settle(full(s), ((g - s + stages - 1) / stages - 1) & 1);
      for (uint32_t s = 0; s < 2; ++s)
        if (it > s) settle(q_full(s), ((it - s + 1) / 2 - 1) & 1);
    }
    return;
  }

  // ------------------------------------------------------------------ products and softmax
  constexpr int NT = D / 32;                                       // 8-column tiles of O that a warp holds
  constexpr bool Q_REGS = MT == 1;                                 // the unit's query fragments stay in registers
  const int group = GROUPS == 1 ? 0 : warp >> 2, quarter = warp & 3, row0 = group * 16 * MT;
  const int gr = lane >> 2, qd = lane & 3;                         // row group and column pair of the fragments
  const int key0 = quarter * 16;
  float* ml = reinterpret_cast<float*>(sgen + ml_off) + group * 4 * 16 * MT;    // [quarter][row of the group]
  // ldmatrix rows of this lane: K (keys x dims as they lie), V (transposed), P and Q (rows x keys / dims)
  const int k_row = key0 + (lane & 7) + ((lane >> 4) << 3), k_ch = (lane >> 3) & 1;
  const int v_row = (lane & 7) + (((lane >> 3) & 1) << 3), v_ch = quarter * (D / 32) + (lane >> 4);
  const int a_row = row0 + (lane & 7) + (((lane >> 3) & 1) << 3), a_ch = lane >> 4;
  int row_tok[MT][2], row_head[MT][2];                             // what the fragments' rows are
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int row = row0 + m * 16 + i * 8 + gr;
      row_tok[m][i] = row / p.G;
      row_head[m][i] = row - row_tok[m][i] * p.G;
    }
  uint32_t g = 0;
  for (uint32_t it = 0;; ++it) {
    const uint32_t slot = it % RING;
    bool ok = wait_all(ring_full(slot), (it / RING) & 1, abort_flag, p.status, 3);
    const volatile int32_t* w = ring[slot];
    if (ok && w[W_KIND] != 0) ok = wait_all(q_full(it & 1), (it >> 1) & 1, abort_flag, p.status, 4);
    if (meet_any(group, !ok)) break;                               // (all four or none)
    if (w[W_KIND] == 0) break;
    const int rows = w[W_ROWS], kv = w[W_KV], pos0 = w[W_POS0], tiles = w[W_TILES];
    const uint32_t qt = sbase + q_off + (it & 1) * L::Q_BYTES;
    int lim[MT][2], least = INT_MAX;                               // keys that a row may see; the fewest
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        lim[m][i] = p.causal ? min(pos0 + row_tok[m][i] + 1, kv) : kv;
        if (SPARSE && pos0 < 0) lim[m][i] = 0;
        if (row0 + m * 16 + i * 8 + gr < rows) least = min(least, lim[m][i]);
      }
    least = __reduce_min_sync(0xffffffffu, least);
    uint32_t qa[D / 16][4];
    auto load_q = [&](int m) {
      const int row = m * 16 + a_row;
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) ldmatrix_x4(qa[ks], qt + (ks >> 2) * ROWS * 128 + row * 128 + ((((ks * 2 + a_ch) & 7) ^ (row & 7)) << 4));
    };
    if (Q_REGS) load_q(0);
    float o[MT][NT][4], m_ref[MT][2], l_sum[MT][2];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[m][n][i] = 0.f;
      m_ref[m][0] = m_ref[m][1] = NO_MAX;
      l_sum[m][0] = l_sum[m][1] = 0.f;
    }
    bool left = false;
    for (int j = 0; j < tiles; ++j, ++g) {
      const uint32_t st = g % stages, use = g / stages;
      ok = wait_all(full(st), use & 1, abort_flag, p.status, 5);
      const int lp = *reinterpret_cast<volatile int32_t*>(&page_of[st]);
      const uint32_t kt = sbase + st * 2 * L::TILE, vt = kt + L::TILE, pt = sbase + p_off + (g & 1) * L::P_BYTES;
      const int first = lp * PAGE + key0;                          // key number of this warp's first key
      // (all loads before the products: one behind another they would each wait for the last one's product)
      uint32_t kb[D / 16][4];
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks)
        ldmatrix_x4(kb[ks], kt + (ks >> 2) * PAGE * 128 + k_row * 128 + ((((ks * 2 + k_ch) & 7) ^ (k_row & 7)) << 4));
      float s[MT][2][4];
#pragma unroll
      for (int m = 0; m < MT; ++m) {
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[m][n][i] = 0.f;
        if (!Q_REGS) load_q(m);
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
          mma16<F16>(s[m][0], qa[ks], kb[ks][0], kb[ks][1]);
          mma16<F16>(s[m][1], qa[ks], kb[ks][2], kb[ks][3]);
        }
      }
      if (first + 16 > least) {                                    // some row may not see some of the keys (uniform)
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (first + n * 8 + qd * 2 + (i & 1) >= lim[m][i >> 1]) s[m][n][i] = -INFINITY;
      }
      bool grow = !ok;
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float top = fmaxf(fmaxf(s[m][0][2 * i], s[m][0][2 * i + 1]), fmaxf(s[m][1][2 * i], s[m][1][2 * i + 1])) * p.scale_log2;
          grow |= top > m_ref[m][i] + MOVE;
        }
      // probabilities against the present references, their sums apart until these are known to serve.  The sums take them as 32-bit numbers; for the
      // product with V they are rounded to 16 bits, as the matrix unit wants its operands: next to the rounding of the result itself that
      // makes its error 1.3 times what it would be (0.0022 for 0.0017 of a bf16 result, root mean square), and a second product for the low halves
      // would double the work.
      float sum[MT][2];
      auto probabilities = [&]() {
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            sum[m][i] = 0.f;
            const int row = row0 + m * 16 + i * 8 + gr;
#pragma unroll
            for (int n = 0; n < 2; ++n) {
              const float e0 = ex2_approx(fmaf(s[m][n][2 * i], p.scale_log2, -m_ref[m][i]));
              const float e1 = ex2_approx(fmaf(s[m][n][2 * i + 1], p.scale_log2, -m_ref[m][i]));
              sum[m][i] += e0 + e1;
              asm volatile("st.shared.b32 [%0], %1;" ::"r"(pt + row * 128 + (((quarter * 2 + n) ^ (row & 7)) << 4) + qd * 4), "r"(pack16<F16>(e0, e1)) : "memory");
            }
          }
      };
      probabilities();
      // this warp's columns of the values, on their way while the warps meet
      uint32_t vb[PAGE / 16][NT / 2][4];
#pragma unroll
      for (int kk = 0; kk < PAGE / 16; ++kk)
#pragma unroll
        for (int n = 0; n < NT / 2; ++n) {
          const int c = v_ch + n * 2, row = kk * 16 + v_row;
          ldmatrix_x4_trans(vb[kk][n], vt + (c >> 3) * PAGE * 128 + row * 128 + (((c & 7) ^ (row & 7)) << 4));
        }
      if (meet_any(group, grow)) {
        // new references: the largest of the four warps' maxima
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            float top = fmaxf(fmaxf(s[m][0][2 * i], s[m][0][2 * i + 1]), fmaxf(s[m][1][2 * i], s[m][1][2 * i + 1])) * p.scale_log2;
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
            if (qd == 0) ml[quarter * 16 * MT + m * 16 + i * 8 + gr] = top;
          }
        if (quarter == 0 && lane == 0) leave_word[group] = *abort_flag;         // one thread's look at the flag is everybody's
        meet(group);
        if (*reinterpret_cast<volatile uint32_t*>(&leave_word[group])) {
          left = true;
          break;
        }
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float* t = ml + m * 16 + i * 8 + gr;
            const float m_new = fmaxf(m_ref[m][i], fmaxf(fmaxf(t[0], t[16 * MT]), fmaxf(t[32 * MT], t[48 * MT])));
            const float f = exp2f(m_ref[m][i] - m_new);
            m_ref[m][i] = m_new;
            l_sum[m][i] *= f;
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              o[m][n][2 * i] *= f;
              o[m][n][2 * i + 1] *= f;
            }
          }
        probabilities();
        meet(group);
      }
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        l_sum[m][0] += sum[m][0];
        l_sum[m][1] += sum[m][1];
      }
      // O += P V for this warp's columns; values of keys that the request does not have are whatever the pool holds
      if (lp * PAGE + PAGE > kv) {
#pragma unroll
        for (int kk = 0; kk < PAGE / 16; ++kk) {
          const int e = kv - lp * PAGE - kk * 16 - qd * 2;         // keys from this lane's first that exist
          const uint32_t keep0 = e >= 2 ? 0xffffffffu : e == 1 ? 0xffffu : 0u, keep1 = e >= 10 ? 0xffffffffu : e == 9 ? 0xffffu : 0u;
#pragma unroll
          for (int n = 0; n < NT / 2; ++n) {
            vb[kk][n][0] &= keep0;
            vb[kk][n][1] &= keep1;
            vb[kk][n][2] &= keep0;
            vb[kk][n][3] &= keep1;
          }
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(empty(st));                       // K and V of the page are in registers
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        uint32_t a[PAGE / 16][4];
        const int row = m * 16 + a_row;
#pragma unroll
        for (int kk = 0; kk < PAGE / 16; ++kk) ldmatrix_x4(a[kk], pt + row * 128 + (((kk * 2 + a_ch) ^ (row & 7)) << 4));
#pragma unroll
        for (int kk = 0; kk < PAGE / 16; ++kk)
#pragma unroll
          for (int n = 0; n < NT / 2; ++n) {
            mma16<F16>(o[m][2 * n], a[kk], vb[kk][n][0], vb[kk][n][1]);
            mma16<F16>(o[m][2 * n + 1], a[kk], vb[kk][n][2], vb[kk][n][3]);
          }
      }
    }
    if (left) break;
    // ------------------------------------------------------------------ the unit's sums, and its rows out
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float l = l_sum[m][i];
        l += __shfl_xor_sync(0xffffffffu, l, 1);
        l += __shfl_xor_sync(0xffffffffu, l, 2);
        if (qd == 0) ml[quarter * 16 * MT + m * 16 + i * 8 + gr] = l;
      }
    meet(group);
    const int out_slot = w[W_SLOT], tok0 = w[W_TOK0], head0 = w[W_HEAD] * p.G;
    if (w[W_PIECE] == 0 && (int)threadIdx.x < rows / p.G)
      sp.cuts[(int64_t)(tok0 + (int)threadIdx.x) * p.Hkv + w[W_HEAD]] = make_int2(out_slot, out_slot < 0 ? 0 : w[W_PIECES] | (int)threadIdx.x << 16);
    const int slot_rows = p.tile_tokens * p.G;
    float* part = p.partials + (int64_t)out_slot * slot_floats(slot_rows, D);
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int row = row0 + m * 16 + i * 8 + gr;
        if (row >= rows) continue;
        const float* t = ml + m * 16 + i * 8 + gr;
        const float l = (t[0] + t[16 * MT]) + (t[32 * MT] + t[48 * MT]);
        const int col = quarter * (D / 4) + qd * 2;
        if (out_slot < 0) {
          const float inv = l == 0.f ? 0.f : 1.f / l;
          const int64_t tok = tok0 + row_tok[m][i], hd = head0 + row_head[m][i];
          uint32_t* dst = reinterpret_cast<uint32_t*>(static_cast<__nv_bfloat16*>(p.out) + tok * p.o_tok + hd * p.o_head + col);
#pragma unroll
          for (int n = 0; n < NT; ++n) dst[n * 4] = pack16<F16>(o[m][n][2 * i] * inv, o[m][n][2 * i + 1] * inv);
          if (p.lse && quarter == 0 && qd == 0) p.lse[tok * p.H + hd] = l == 0.f ? -INFINITY : (m_ref[m][i] + log2f(l)) * 0.6931471805599453f;
        } else {
#pragma unroll
          for (int n = 0; n < NT; ++n) __stcg(reinterpret_cast<float2*>(part + row * D + col + n * 8), make_float2(o[m][n][2 * i], o[m][n][2 * i + 1]));
          if (quarter == 0 && qd == 0) __stcg(reinterpret_cast<float2*>(part + slot_rows * D) + row, make_float2(m_ref[m][i], l));
        }
      }
    __syncwarp();
    if (lane == 0) mbar_arrive(ring_empty(slot));
  }
}

// Partial results of a call: pieces of units of more than S pages, S at least pages / (CTAs * PER_CTA), so at most twice CTAs * PER_CTA
// (a unit of x S pages, x > 1, has fewer than 2 x pieces).
__host__ __device__ constexpr int max_slots(int ctas) { return 2 * PER_CTA * ctas; }
static_assert(max_slots(2 * PAGED_MOST_SMS) < 1 << 16, "pieces of a unit in 16 bits (at most two CTAs an SM)");

// Adds up the parts of the rows whose units were cut, in page order: a CTA per row where the rows are few, else a warp.  What bounds it is a
// chain of loads behind the end of the kernel before (cut, parts), and the start of its CTAs: one for every slot and row instead of one for 8 of
// the call's rows, as it was first, made a decode of 64 requests 71 us instead of 67.
template <int D, bool F16, bool WIDE>
__global__ void __launch_bounds__(MERGE_WARPS * 32) paged_merge_kernel(const __grid_constant__ SmallParams sp, int slots) {
  const PagedParams& p = sp.a;
  constexpr int N = D / 32;
  __shared__ float sums[MERGE_WARPS][D], tops[MERGE_WARPS], ls[MERGE_WARPS];
  pdl_trigger();
  pdl_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, slot_rows = p.tile_tokens * p.G;
  const int begin_tok = __ldg(p.q_begin), end_tok = __ldg(p.q_begin + p.n_seq);
  Parts<D> parts;
  parts.pitch = slot_floats(slot_rows, D);
  parts.slot_rows = slot_rows;
  parts.lane = lane;
  const int64_t rows = (int64_t)p.n_tokens * p.H, step = (int64_t)gridDim.x * (WIDE ? 1 : MERGE_WARPS);
  for (int64_t x = WIDE ? blockIdx.x : (int64_t)blockIdx.x * MERGE_WARPS + warp; x < rows; x += step) {
    const int tok = (int)(x / p.H), hd = (int)(x - (int64_t)tok * p.H), head = hd / p.G;
    const int2 cut = __ldcg(sp.cuts + (int64_t)tok * p.Hkv + head);
    const int pieces = cut.y & 0xffff;
    parts.row = (cut.y >> 16) * p.G + hd - head * p.G;
    // (Rows that are nobody's have an entry of some call before, or none; in a call that gave up, a request's own may be whatever the other
    // kernel left there.  No such entry leads out of the workspace.)
    if (tok < begin_tok || tok >= end_tok || pieces < 2 || pieces > slots || cut.x < 0 || cut.x > slots - pieces ||
        (uint32_t)parts.row >= (uint32_t)slot_rows)
      continue;
    parts.first = p.partials + cut.x * parts.pitch;
    if (!WIDE) {
      put_row<D, F16>(p, sum_parts<D>(parts, 0, pieces), tok, hd, lane);
      continue;
    }
    const int begin = pieces * warp / MERGE_WARPS, end = pieces * (warp + 1) / MERGE_WARPS;
    RowSum<D> r;
    r.clear();
    if (begin < end) r = sum_parts<D>(parts, begin, end);
#pragma unroll
    for (int i = 0; i < N; ++i) sums[warp][lane * N + i] = r.acc[i];
    if (lane == 0) {
      tops[warp] = r.top;
      ls[warp] = r.l;
    }
    __syncthreads();
    if (warp == 0) {
      r.clear();
      for (int i = 0; i < MERGE_WARPS; ++i) r.top = fmaxf(r.top, tops[i]);
      for (int i = 0; i < MERGE_WARPS; ++i) {
        const float w = exp2f(tops[i] - r.top);
        r.l = fmaf(ls[i], w, r.l);
#pragma unroll
        for (int j = 0; j < N; ++j) r.acc[j] = fmaf(sums[i][lane * N + j], w, r.acc[j]);
      }
      put_row<D, F16>(p, r, tok, hd, lane);
    }
    __syncthreads();
  }
}

uint64_t cut_bytes(int n_tokens, int Hkv) { return ((uint64_t)n_tokens * Hkv * 8 + 255) / 256 * 256; }

template <int D, int MT, int GROUPS, bool F16, bool SPARSE>
cudaError_t launch(const PagedParams& p, const SmallMaps& maps, int n_sm, cudaStream_t stream) {
  using L = SmallLayout<D, MT, GROUPS>;
  auto fixed_of = [](int n_seq) { return (int)(L::FIXED + (SPARSE ? 0 : (n_seq + 1) * 8) + 1024); };
  const int fixed = fixed_of(p.n_seq);
  SmallParams sp;
  sp.a = p;
  sp.counter = p.counters;
  sp.cuts = reinterpret_cast<int2*>(p.partials);
  sp.a.partials = p.partials + cut_bytes(p.n_tokens, p.Hkv) / 4;
  // as many pages under way as the CTA's share of an SM's shared memory holds
  constexpr int room = (L::CTAS == 2 ? 113 : 226) * 1024 - 768, stage = 2 * (int)L::TILE;
  sp.stages = std::max(2, std::min(MAX_STAGES, (room - fixed) / stage));
  const int smem = fixed + sp.stages * stage;
  // (the kernel's limit is the process's: always the most that any call takes, as another thread may set it between this line and the launch)
  const int most = std::max(room, fixed_of(PAGED_MAX_SEQ) + 2 * stage);
  auto kernel = paged_small_kernel<D, MT, GROUPS, F16, SPARSE>;
  cudaError_t rc = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
  if (rc != cudaSuccess) return rc;
  rc = launch_pdl(kernel, dim3(n_sm * L::CTAS), dim3(L::THREADS), smem, stream, sp, maps);
  // nothing can have been cut where no unit has more pages
  if (rc != cudaSuccess || (SPARSE ? p.n_sel : p.table_pages) <= FULL_CHUNK) return rc;
  const int64_t rows = (int64_t)p.n_tokens * p.H, pieces = (SPARSE ? p.n_sel : p.table_pages) / MIN_CHUNK;       // (of a unit, at most)
  if (rows <= 8 * n_sm && pieces > AHEAD) return launch_pdl(paged_merge_kernel<D, F16, true>, dim3((unsigned)rows), dim3(MERGE_WARPS * 32), 0, stream, sp, max_slots(L::CTAS * n_sm));
  const int64_t ctas = std::min<int64_t>((rows + MERGE_WARPS - 1) / MERGE_WARPS, 8 * n_sm);
  return launch_pdl(paged_merge_kernel<D, F16, false>, dim3((unsigned)ctas), dim3(MERGE_WARPS * 32), 0, stream, sp, max_slots(L::CTAS * n_sm));
}
template <int D, bool F16, bool SPARSE>
cudaError_t launch_rows(const PagedParams& p, int rows, const SmallMaps& maps, int n_sm, cudaStream_t stream) {
  if (rows <= 16) return launch<D, 1, 1, F16, SPARSE>(p, maps, n_sm, stream);
  // (over all pages, more than 32 rows are the tensor-memory kernel's or come in tiles of 16)
  if (rows <= 32 || !SPARSE) return launch<D, 2, 1, F16, SPARSE>(p, maps, n_sm, stream);
  return launch<D, 2, SPARSE ? 2 : 1, F16, SPARSE>(p, maps, n_sm, stream);
}
template <int D>
cudaError_t launch_typed(const PagedParams& p, bool fp16, int rows, const SmallMaps& maps, int n_sm, cudaStream_t stream) {
  if (p.sel) return fp16 ? launch_rows<D, true, true>(p, rows, maps, n_sm, stream) : launch_rows<D, false, true>(p, rows, maps, n_sm, stream);
  return fp16 ? launch_rows<D, true, false>(p, rows, maps, n_sm, stream) : launch_rows<D, false, false>(p, rows, maps, n_sm, stream);
}

}  // namespace

uint64_t paged_small_partial_bytes(int d, int n_sm, int Hkv, int n_tokens) {
  // (twice the CTAs, at most 32 rows each, or once and 64)
  return cut_bytes(n_tokens, Hkv) + (uint64_t)max_slots(2 * n_sm) * 32 * (d + 2) * 4;
}

cudaError_t launch_paged_small(const PagedParams& p, const heatkv_paged_pool& pool, const PagedDevice& dev, cudaStream_t stream) {
  // rows of a tile: up to 16, 32 or 64
  const int tokens = p.sel ? 1 : std::max(1, p.max_new);
  const int64_t wanted = (int64_t)tokens * p.G;
  // (more than 32 rows come in tiles of 16: 42 rows, 96 units, 17.5 us against 21.0 in tiles of 32)
  const int rows = wanted <= 16 || (wanted > 32 && !p.sel && p.G <= 16) ? 16 : wanted <= 32 || !p.sel ? 32 : 64;
  PagedParams q = p;
  q.tile_tokens = p.sel ? 1 : rows / p.G;
  SmallMaps maps;
  if (!paged_encode_pool(dev, &maps.k, pool.k, pool) || !paged_encode_pool(dev, &maps.v, pool.v, pool) || !paged_encode_q(dev, &maps.q, q, pool))
    return cudaErrorInvalidValue;
  const bool fp16 = pool.dtype == HEATKV_DTYPE_FP16;
  return pool.d == 128 ? launch_typed<128>(q, fp16, rows, maps, dev.n_sm, stream) : launch_typed<64>(q, fp16, rows, maps, dev.n_sm, stream);
}

}  // namespace heatkv
