// Attention of many query rows over a paged cache (chunks of prompts, an image's scale) on the tensor cores' own memory.
//
// A row tile is floor(128 / G) consecutive tokens of a request times the G query heads of one kv head; an item is two of them (A and B),
// which share the stream of key tiles (128 keys: two pages).  The key tiles of all items, request by request, head by head, in token
// order, are dealt out in equal runs, one per SM, so that every SM ends at the same time whatever the lengths; an item that a run's border
// cuts leaves unnormalised rows in the workspace, where the warp that arrives last for its 32 rows adds the parts up in key order.
// Warp roles as in attn_tc.cu:
//   warp 2       walks the CTA's run and tells the others the items, one ahead (a two-entry ring);
//   warp 0       sends for Q, K and V (TMA);
//   warp 1       issues the products: S = Q K^T and O += P V, accumulators in tensor memory;
//   warps 4-7    softmax of tile A, warps 8-11 of tile B, one thread a row; they write the item's rows, too.
// Tensor memory: S_A/P_A 0..127, S_B/P_B 128..255, O_A 256..383, O_B 384..511.  Rows past a request's last key in its last page are
// whatever the pool holds: their logits are masked, their values overwritten by zeros before the product (warp 1).
//
// Over selected pages (SPARSE) the keys of an item are the pages that any of its tokens selected, in ascending order, and a row sees a page
// if its token is among those that did: neighbouring tokens select much the same pages, so a page is read and multiplied once for all of
// them instead of once for each.  Warp 2 brings the tokens' lists into shared memory, the copy warp merges them as it goes (a
// token per lane and tile) and hands the tokens' bits to the softmax warps beside each tile.
// (A tile has at most 32 tokens there, one a bit of a word, so that groups of one or two heads fill a quarter or half of its 128 rows.)
// What bounds it: 128-wide heads the matrix unit and, back to back, power (2 sequences of 4096 new tokens over 8096 keys, 16 heads: 450 to 470 us,
// 1160 to 1200 TFLOP/s; three causal prompts of 2100 to 4096 tokens, 32 heads, whose items are short: 213 us, 880); 64-wide heads the softmax warps'
// waits for tensor memory (half the products per exponential: 32 heads of the first shape 666 us, 815 TFLOP/s; no unit is busy more than 57 %).
// Every wait is bounded in time; on expiry the CTA records which wait it was, lets its own copies land and its products end, and leaves.
#include <algorithm>

#include <cuda_fp16.h>

#include "paged_wait.cuh"

namespace heatkv {
namespace {

using namespace tc;

constexpr int BM = 128, BN = 128;
constexpr int THREADS = 384;
constexpr int KV_STAGES = 2;
// Register hand-over between warpgroups, inside what the launch allocates (checked against the compiled kernel before it runs).
constexpr int REGS_LAUNCH = 168, REGS_SMALL = 72, REGS_SOFTMAX = 216;
static_assert(128 * REGS_SMALL + 256 * REGS_SOFTMAX <= THREADS * REGS_LAUNCH, "register hand-over exceeds the CTA's allocation");
constexpr uint32_t HALF_COLS_BYTES = 128 * 128;        // one 64-column half of a 128-row tile
constexpr uint32_t SLOT_BYTES = PAGE * 128;            // a page inside one column half
constexpr uint32_t STAGE_BYTES = 2048;                 // per softmax warp: 32 rows x 32 columns on their way out

// An item's lists of selected pages: 16-bit places, and a bit for every page of a context (0xffff stands for none).
constexpr int LIST_ENTRIES = 2048, LIST_WORDS = 2048;
constexpr uint32_t LIST_BYTES = LIST_ENTRIES * 2 + LIST_WORDS * 4;

template <int D>
struct Layout {
  static constexpr int NCH = D / 64;
  static constexpr uint32_t TILE_BYTES = NCH * HALF_COLS_BYTES;
  static constexpr uint32_t SM_Q = 0;
  static constexpr uint32_t SM_K = SM_Q + 2 * TILE_BYTES;
  static constexpr uint32_t SM_V = SM_K + KV_STAGES * TILE_BYTES;
  static constexpr uint32_t SM_OUT = SM_V + KV_STAGES * TILE_BYTES;
  static constexpr uint32_t SM_BAR = SM_OUT + 8 * STAGE_BYTES;
  static constexpr uint32_t SM_LIST = SM_BAR + 512;
  static constexpr uint32_t SM_ALLOC = SM_BAR + 512 + 1024;             // (and the lists where pages are selected)
  static_assert(SM_ALLOC + LIST_BYTES + LIST_ENTRIES * 2 <= 227 * 1024, "shared memory of one CTA");
  // one part of a cut item: O of both tiles (groups of four columns outermost), then references and sums
  static constexpr int SLOT_FLOATS = 2 * BM * D + 2 * 2 * BM;
};
enum Bar : uint32_t {
  Q_FULL = 0, Q_EMPTY = 2, K_FULL = 4, K_EMPTY = 6, V_FULL = 8, V_EMPTY = 10, S_FULL = 12, P_FULL = 14, PV_DONE = 18, ITEM_FULL = 20, ITEM_EMPTY = 22,
  DRAIN = 24, N_BARS
};
constexpr uint32_t BAR_TMEM_PTR = N_BARS * 8, BAR_ABORT = BAR_TMEM_PTR + 4, BAR_RING = 256, BAR_INFO = 384;
constexpr int INFO_RING = 4;                           // key tiles whose pages and bits are kept: the copy warp is at most two ahead of the softmax
enum InfoWord : int { I_PLACE = 0, I_BITS = 2, INFO_WORDS = 8 };   // two places; bits of tile A for both, of tile B for both
enum ItemWord : int { W_KIND = 0, W_SEQ, W_HEAD, W_TOK0, W_TOKENS, W_POS0, W_KV, W_J0, W_NT, W_TILES, W_C0, W_C1, W_SEEK };

struct TcParams {
  PagedParams a;
  // the plan of the call
  int32_t* item_begin;        // [n_seq + 1] the request's first item
  int64_t* item_units;        // [items] what a request's items weigh, of one head, summed up (a long prompt of many heads a group passes 2^31)
  int32_t* item_prefix;       // SPARSE (in the same place): [items * Hkv + 1] every item's and kv head's key tiles, summed up
  int32_t* runs;              // [n_sm][RUN_WORDS] where every CTA's run starts
  uint32_t* ticket;           // CTAs of union_kernel that are done; zero between launches
  int32_t items;              // room for the items
  int32_t n_cta;
};
enum RunWord : int { R_SEQ = 0, R_HEAD, R_ITEM, R_J0, R_UNITS, R_C0_FIRST = R_UNITS + 2, R_C1_FIRST, R_C1_LAST, RUN_WORDS = 10 };
static_assert(R_UNITS % 2 == 0 && RUN_WORDS % 2 == 0 && R_C1_LAST < RUN_WORDS, "a run's units are a 64-bit number");
struct TcMaps {
  CUtensorMap q, k, v;
};

__device__ __forceinline__ int request_tokens(const PagedParams& p, int i, int& b) {
  b = max(p.q_begin[i], 0);
  return max(min(p.q_begin[i + 1], p.n_tokens) - b, 0);
}
__device__ __forceinline__ int request_keys(const PagedParams& p, int i) { return min(max(p.kv_len[i], 0), p.table_pages * PAGE); }
// Key tiles of the item that starts at token `tok` of a request: up to the last key that its last token sees, at least one (which then
// is masked whole, so that rows without keys are written like all others).
__device__ __forceinline__ int item_tiles(const PagedParams& p, int tok, int n, int kv) {
  const int upto = p.causal ? min(kv, kv - n + min(n, tok + 2 * p.tile_tokens)) : kv;
  return max(1, (upto + BN - 1) / BN);
}

// The lists of selected pages of an item's tokens, merged by a warp: lane l has token l of tile A and token l of tile B.  Whatever the
// order of a list, its entries come one after another, so every entry is met exactly once.
constexpr int NO_PAGE = 1 << 24;
struct Merge {
  const uint16_t* list;
  int a, b, a_end, b_end;                          // the next places to be read
  int va, vb, va2, vb2;                            // the lists' next entries, and those behind them (read ahead)
  __device__ int entry(int& i, int end) const {
    int v = 0xffff;
    while (i < end && (v = list[i++]) == 0xffff) {}
    return v == 0xffff ? NO_PAGE : v;
  }
  __device__ void start(const uint16_t* l, int n_sel, int tokens, int tile_tokens, int lane) {
    list = l;
    const bool in_a = lane < min(tile_tokens, tokens), in_b = lane < tile_tokens && tile_tokens + lane < tokens;
    a = lane * n_sel;
    a_end = in_a ? a + n_sel : a;
    b = (tile_tokens + lane) * n_sel;
    b_end = in_b ? b + n_sel : b;
    refill();
  }
  __device__ void refill() {
    va = entry(a, a_end);
    vb = entry(b, b_end);
    va2 = entry(a, a_end);
    vb2 = entry(b, b_end);
  }
  // ascending lists: on to the first entries that are not below `page`
  __device__ void seek(int page, int n_sel, int tile_tokens, int lane) {
    auto first = [&](int from, int end) {
      int lo = from, hi = end;
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (list[mid] < page) lo = mid + 1; else hi = mid;
      }
      return lo;
    };
    a = first(min(lane * n_sel, a_end), a_end);
    b = first(min((tile_tokens + lane) * n_sel, b_end), b_end);
    refill();
  }
  // the next page (NO_PAGE: none is left) and the tokens of each tile that selected it
  __device__ int next(uint32_t& bits_a, uint32_t& bits_b) {
    const int page = __reduce_min_sync(0xffffffffu, min(va, vb));
    const bool ha = va == page && page < NO_PAGE, hb = vb == page && page < NO_PAGE;
    bits_a = __ballot_sync(0xffffffffu, ha);
    bits_b = __ballot_sync(0xffffffffu, hb);
    if (ha) {
      va = va2;
      va2 = entry(a, a_end);
    }
    if (hb) {
      vb = vb2;
      vb2 = entry(b, b_end);
    }
    __syncwarp();
    return page;
  }
};
// An item's lists into shared memory; entries that count for nothing become 0xffff.  Returns whether all lists ascend (with nothing but
// such entries behind the last page), as heatkv_paged_select writes them.
__device__ __forceinline__ bool load_lists(const PagedParams& p, uint16_t* list, int tok0, int tokens, int pos0, int head, int lane) {
  // lanes: as many tokens at once as their lists fit a warp; longer lists in rounds
  const int at_once = max(1, 32 / p.n_sel), t_lane = lane / p.n_sel, i_lane = at_once > 1 ? lane - t_lane * p.n_sel : lane;
  const bool active = at_once == 1 || t_lane < at_once;
  const int64_t stride = (int64_t)p.Hkv * p.n_sel;
  bool ascend = true;
  for (int i0 = 0; i0 < p.n_sel; i0 += 32) {
    const int i = i0 + i_lane;
    constexpr int AHEAD = 8;
    for (int base = 0; base < tokens; base += at_once * AHEAD) {
      int place[AHEAD];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int t = base + t_lane + u * at_once;
        place[u] = active && t < tokens && i < p.n_sel ? __ldg(p.sel + (tok0 + t) * stride + head * p.n_sel + i) : -1;
      }
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int t = base + t_lane + u * at_once;
        if (pos0 + t < 0 || place[u] > (pos0 + t) / PAGE || place[u] >= p.table_pages) place[u] = -1;
        const int v = place[u] < 0 ? 0xffff : place[u], before = __shfl_up_sync(0xffffffffu, v, 1);
        if (active && t < tokens && i < p.n_sel) {
          list[t * p.n_sel + i] = (uint16_t)v;
          if (i_lane > 0) ascend &= v == 0xffff || before < v;
        }
      }
    }
  }
  __syncwarp();
  if (p.n_sel > 32)                                                // the seams between rounds
    for (int t = lane; t < tokens; t += 32)
      for (int i = 32; i < p.n_sel; i += 32) ascend &= list[t * p.n_sel + i] == 0xffff || list[t * p.n_sel + i - 1] < list[t * p.n_sel + i];
  return __all_sync(0xffffffffu, ascend);
}
// A bit for every page that some list has; `words` of them.
__device__ __forceinline__ void mark_pages(const uint16_t* list, int total, uint32_t* bits, int words, int lane) {
  for (int i = lane; i < words; i += 32) bits[i] = 0;
  __syncwarp();
  for (int i = lane; i < total; i += 32)
    if (list[i] != 0xffff) atomicOr(bits + (list[i] >> 5), 1u << (list[i] & 31));
  __syncwarp();
}
__device__ __forceinline__ int pages_words(const PagedParams& p, int last_pos) { return min(max(last_pos, 0) / PAGE + 1, p.table_pages) / 32 + 1; }
// the page with `rank` marked ones before it, by a warp (NO_PAGE: there are not so many)
__device__ __forceinline__ int page_of_rank(const uint32_t* bits, int words, int rank, int lane) {
  for (int base = 0; base < words; base += 32) {
    uint32_t w = base + lane < words ? bits[base + lane] : 0;
    int inc = __popc(w);
    const int own = inc;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int up = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += up;
    }
    const uint32_t reach = __ballot_sync(0xffffffffu, inc > rank);
    if (reach) {
      const int l = __ffs(reach) - 1;
      int skip = rank - __shfl_sync(0xffffffffu, inc - own, l);
      w = __shfl_sync(0xffffffffu, w, l);
      for (; skip > 0; --skip) w &= w - 1;
      return (base + l) * 32 + __ffs(w) - 1;
    }
    rank -= __shfl_sync(0xffffffffu, inc, 31);
  }
  return NO_PAGE;
}

// An item weighs its key tiles and as much again as its end costs (rows out, the next one's first products), in tiles.
constexpr int ITEM_END = 1;

// The runs: CTA c's is the units bound(c) .. bound(c + 1) - 1 of all.  A run has at least MIN_SHARE units, and in a call of few and long items
// more: P parts of an item of T tiles take about 1.35 T / P us, and half a microsecond each to add up, one behind another.
constexpr int MIN_SHARE = 4;
struct Shares {
  int64_t all;
  int grid;
  __device__ Shares(int64_t all_, int longest, int n_cta) : all(all_) {
    const int64_t share = max(MIN_SHARE, (int)sqrtf(0.4f * (float)longest));
    grid = (int)min((int64_t)n_cta, (all + share - 1) / share);
  }
  __device__ int64_t bound(int c) const { return all * c / grid; }
  // the CTA that holds unit y: the last c with bound(c) <= y
  __device__ int owner(int64_t y) const {
    int c = min((int)((double)y * grid / (double)all), grid - 1);  // (an estimate, put right without a division)
    while (c + 1 < grid && all * (c + 1) < (y + 1) * grid) ++c;
    while (c > 0 && all * c >= (y + 1) * grid) --c;
    return c;
  }
};
// CTA c's run.  `place(y)` says which item holds unit y; a run that would begin with an item's end begins with the next item.
// All CTAs between an item's first and last tile have tiles of it: their bounds lie inside it.
template <typename P>
__device__ __forceinline__ void write_run(const TcParams& tp, const Shares& sh, int c, P place) {
  int32_t* run = tp.runs + c * RUN_WORDS;
  int64_t* units = reinterpret_cast<int64_t*>(run + R_UNITS);
  *units = 0;
  if (c >= sh.grid) return;
  int64_t y0 = sh.bound(c);
  const int64_t y1 = sh.bound(c + 1);
  auto a = place(y0);
  if (y0 - a.begin >= a.tiles) {
    y0 = a.begin + a.tiles + ITEM_END;
    if (y0 >= y1) return;
    a = place(y0);
  }
  const auto z = place(y1 - 1);
  run[R_SEQ] = a.seq;
  run[R_HEAD] = a.head;
  run[R_ITEM] = a.item;
  run[R_J0] = (int)(y0 - a.begin);
  *units = y1 - y0;
  run[R_C0_FIRST] = sh.owner(a.begin);
  run[R_C1_FIRST] = sh.owner(a.begin + a.tiles - 1);
  run[R_C1_LAST] = sh.owner(z.begin + z.tiles - 1);
}
struct Place {
  int seq, head, item, tiles;
  int64_t begin;                                                   // the item's first unit
};
template <typename T, typename X>
__device__ __forceinline__ int last_not_above(const T* a, int n, X x) {        // last i in [0, n) with a[i] <= x
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a[mid] <= x) lo = mid; else hi = mid - 1;
  }
  return lo;
}
// Exclusive sum over a CTA of WARPS warps.
template <int WARPS>
__device__ __forceinline__ int64_t exclusive(int64_t v, int64_t* sums, int64_t& all) {
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
  for (int w = 0; w < WARPS; ++w) {
    const int64_t x = sums[w];
    if (w < warp) before += x;
    all += x;
  }
  return before + inc - v;
}

// One CTA: what every request's items weigh, and the runs.  All sums stay in shared memory (the items' as far as they fit): the kernel is
// a chain of look-ups, and through global memory it took 10 us.
constexpr int PT = 512, PLAN_ITEMS = 16384;
__global__ void __launch_bounds__(PT) plan_kernel(const __grid_constant__ TcParams tp) {
  extern __shared__ __align__(8) unsigned char plan_smem[];
  const PagedParams& p = tp.a;
  const bool fits = tp.items <= PLAN_ITEMS;
  int64_t* item_units = fits ? reinterpret_cast<int64_t*>(plan_smem) : tp.item_units;
  int64_t* seq_prefix = reinterpret_cast<int64_t*>(plan_smem) + (fits ? tp.items : 0);         // [n_seq + 1] units before the request
  int32_t* item_begin = reinterpret_cast<int32_t*>(seq_prefix + p.n_seq + 1);  // [n_seq + 1]
  int32_t* tokens = item_begin + p.n_seq + 1;                      // [n_seq]
  int32_t* keys = tokens + p.n_seq;                                // [n_seq]
  __shared__ int64_t sums[PT / 32];
  __shared__ int longest;
  pdl_trigger();
  pdl_wait();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, pair = 2 * p.tile_tokens;
  int b;
  if (tid == 0) longest = 1;
  for (int i = tid; i < p.n_seq; i += PT) {
    tokens[i] = request_tokens(p, i, b);
    keys[i] = request_keys(p, i);
  }
  __syncthreads();
  const int per = (p.n_seq + PT - 1) / PT, i0 = min(tid * per, p.n_seq), i1 = min(i0 + per, p.n_seq);
  int64_t mine = 0, all;
  for (int i = i0; i < i1; ++i) mine += (tokens[i] + pair - 1) / pair;
  int64_t at = exclusive<PT / 32>(mine, sums, all);
  for (int i = i0; i < i1; ++i) {
    tp.item_begin[i] = item_begin[i] = (int)min(at, (int64_t)tp.items);
    at += (tokens[i] + pair - 1) / pair;
  }
  if (tid == 0) tp.item_begin[p.n_seq] = item_begin[p.n_seq] = (int)min(all, (int64_t)tp.items);
  __syncthreads();
  // a warp per request: units before every item
  for (int i = warp; i < p.n_seq; i += PT / 32) {
    const int first = item_begin[i], count = item_begin[i + 1] - first;
    int64_t before = 0;
    for (int base = 0; base < count; base += 32) {
      const int w = base + lane < count ? item_tiles(p, (base + lane) * pair, tokens[i], keys[i]) + ITEM_END : 0;
      int inc = w;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += up;
      }
      if (base + lane < count) item_units[first + base + lane] = before + inc - w;
      before += __shfl_sync(0xffffffffu, inc, 31);
    }
    if (lane == 0) {
      seq_prefix[i] = before;                                      // of one head, for now
      if (count > 0) atomicMax(&longest, max(1, (keys[i] + BN - 1) / BN));
    }
  }
  __syncthreads();
  mine = 0;
  for (int i = i0; i < i1; ++i) mine += seq_prefix[i] * p.Hkv;
  at = exclusive<PT / 32>(mine, sums, all);
  for (int i = i0; i < i1; ++i) {
    const int64_t v = seq_prefix[i] * p.Hkv;
    seq_prefix[i] = at;
    at += v;
  }
  if (tid == 0) seq_prefix[p.n_seq] = all;
  __syncthreads();
  const Shares sh(all, longest, tp.n_cta);
  for (int c = tid; c < tp.n_cta; c += PT)
    write_run(tp, sh, c, [&](int64_t y) {
      Place r;
      r.seq = last_not_above(seq_prefix, p.n_seq, y);
      const int64_t s0 = seq_prefix[r.seq], per_head = (seq_prefix[r.seq + 1] - s0) / p.Hkv;
      r.head = (int)((y - s0) / per_head);
      const int64_t local = y - s0 - r.head * per_head;
      const int first = item_begin[r.seq];
      r.item = last_not_above(item_units + first, item_begin[r.seq + 1] - first, local);
      r.begin = y - (local - item_units[first + r.item]);
      r.tiles = item_tiles(p, r.item * pair, tokens[r.seq], keys[r.seq]);
      return r;
    });
}

// Key tiles of every item and kv head over selected pages: half of the pages that its tokens' lists give when merged, a warp each.  The
// CTA that is done last sums them up and writes the runs.
constexpr int UNION_WARPS = 4, UNION_THREADS = UNION_WARPS * 32;
__global__ void __launch_bounds__(UNION_THREADS) union_kernel(const __grid_constant__ TcParams tp) {
  extern __shared__ __align__(8) unsigned char union_smem[];
  const PagedParams& p = tp.a;
  int32_t* item_begin = reinterpret_cast<int32_t*>(union_smem);    // [n_seq + 1]
  unsigned char* lists = union_smem + ((p.n_seq + 1) * 4 + 15) / 16 * 16;      // a warp's lists and bits each; at last the items' sums
  __shared__ int64_t sums[UNION_WARPS];
  __shared__ uint32_t ticket;
  __shared__ int longest;
  pdl_trigger();
  pdl_wait();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, pair = 2 * p.tile_tokens;
  const int per = (p.n_seq + UNION_THREADS - 1) / UNION_THREADS, i0 = min(tid * per, p.n_seq), i1 = min(i0 + per, p.n_seq);
  int b;
  int64_t mine = 0, all;
  for (int i = i0; i < i1; ++i) mine += item_begin[i] = (request_tokens(p, i, b) + pair - 1) / pair;
  int64_t at = exclusive<UNION_WARPS>(mine, sums, all);
  for (int i = i0; i < i1; ++i) {
    const int n = item_begin[i];
    item_begin[i] = (int)min(at, (int64_t)tp.items);
    at += n;
  }
  if (tid == 0) item_begin[p.n_seq] = (int)min(all, (int64_t)tp.items);
  __syncthreads();
  if (blockIdx.x == 0)
    for (int i = tid; i <= p.n_seq; i += UNION_THREADS) tp.item_begin[i] = item_begin[i];
  const int count = item_begin[p.n_seq] * p.Hkv;
  const int64_t x = (int64_t)blockIdx.x * UNION_WARPS + warp;
  if (x < count) {
    const int item = (int)x / p.Hkv, head = (int)x - item * p.Hkv, seq = last_not_above(item_begin, p.n_seq, item);
    const int n = request_tokens(p, seq, b), kv = request_keys(p, seq), tok = (item - item_begin[seq]) * pair, tokens = min(n - tok, pair);
    uint16_t* list = reinterpret_cast<uint16_t*>(lists + warp * LIST_BYTES);
    uint32_t* bits = reinterpret_cast<uint32_t*>(list + LIST_ENTRIES);
    int pages = 0;
    if (load_lists(p, list, b + tok, tokens, kv - n + tok, head, lane)) {
      const int words = pages_words(p, kv - n + tok + tokens - 1);
      mark_pages(list, tokens * p.n_sel, bits, words, lane);
      for (int i = lane; i < words; i += 32) pages += __popc(bits[i]);
      pages = __reduce_add_sync(0xffffffffu, pages);
    } else {                                                       // a page may come more than once
      Merge merge;
      merge.start(list, p.n_sel, tokens, p.tile_tokens, lane);
      uint32_t bits_a, bits_b;
      while (merge.next(bits_a, bits_b) < NO_PAGE) ++pages;
    }
    if (lane == 0) tp.item_prefix[x] = max(1, (pages + 1) / 2);
  }
  __threadfence();
  __syncthreads();
  if (tid == 0) {
    ticket = atomicAdd(tp.ticket, 1u);
    if (ticket == gridDim.x - 1) *reinterpret_cast<volatile uint32_t*>(tp.ticket) = 0;         // ready for the next launch
  }
  __syncthreads();
  if (ticket != gridDim.x - 1) return;
  __threadfence();
  const int each = (count + UNION_THREADS - 1) / UNION_THREADS, x0 = min(tid * each, count), x1 = min(x0 + each, count);
  const bool fits = (count + 1) * 4 <= (int)(UNION_WARPS * LIST_BYTES);
  int32_t* prefix = fits ? reinterpret_cast<int32_t*>(lists) : tp.item_prefix;
  mine = 0;
  int most = 1;
  if (tid == 0) longest = 1;
#pragma unroll 4
  for (int i = x0; i < x1; ++i) {
    const int v = __ldcg(tp.item_prefix + i) + ITEM_END;
    if (fits) prefix[i] = v;
    mine += v;
    most = max(most, v);
  }
  __syncthreads();
  atomicMax(&longest, most);
  at = exclusive<UNION_WARPS>(mine, sums, all);
  for (int i = x0; i < x1; ++i) {
    const int v = fits ? prefix[i] : __ldcg(tp.item_prefix + i) + ITEM_END;
    prefix[i] = tp.item_prefix[i] = (int)at;                       // (paged_tc_takes_lists: all of them are below 2^31)
    at += v;
  }
  if (tid == 0) prefix[count] = tp.item_prefix[count] = (int)all;
  __syncthreads();
  const Shares sh(all, longest, tp.n_cta);
  for (int c = tid; c < tp.n_cta; c += UNION_THREADS)
    write_run(tp, sh, c, [&](int64_t y) {
      Place r;
      const int i = last_not_above(prefix, count, y), item = i / p.Hkv;
      r.head = i - item * p.Hkv;
      r.seq = last_not_above(item_begin, p.n_seq, item);
      r.item = item - item_begin[r.seq];
      r.begin = prefix[i];
      r.tiles = prefix[i + 1] - prefix[i] - ITEM_END;
      return r;
    });
}

__device__ __forceinline__ int ring_word(const volatile int32_t* ring, int word) { return __shfl_sync(0xffffffffu, ring[word], 0); }

// Key tiles of row tile A in this part of an item: with B's tokens behind its own it may see fewer (at least one, if need be masked whole).
template <bool SPARSE>
__device__ __forceinline__ int tiles_of_a(const PagedParams& p, const volatile int32_t* ring, int n_tiles) {
  if (SPARSE || !p.causal) return n_tiles;
  const int sees = min(ring_word(ring, W_POS0) + p.tile_tokens, ring_word(ring, W_KV));
  return max(1, min(n_tiles, (sees + BN - 1) / BN - ring_word(ring, W_J0)));
}

template <bool F16>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
  if (F16) {
    __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&v);
  }
  return pack_bf16(lo, hi);
}

// 2^x for a pair on the FMA units: x = n + f with n = round(x), f in [-1/2, 1/2]; the polynomial of degree 4 that is nearest to 2^f there
// (relative error 2.7e-6 with its 32-bit steps) gets n added to its exponent.  Below -125, where the exponent would leave its range, the result
// is zero: keys that a row does not see arrive as minus infinity, and times a value near the type's largest even 2^-125 would show.
__device__ __forceinline__ void exp2_pair(uint64_t x, float& e0, float& e1) {
  constexpr float MAGIC = 12582912.f;                  // 1.5 * 2^23: the sum's low mantissa bits hold round(x)
  float x0, x1;
  unpack2(x, x0, x1);
  const uint64_t magic = pack2(MAGIC, MAGIC), t = add2(x, magic), f = sub2(x, sub2(t, magic));
  uint64_t q = fma2(pack2(0.00957010221f, 0.00957010221f), f, pack2(0.0559178591f, 0.0559178591f));
  q = fma2(q, f, pack2(0.240247443f, 0.240247443f));
  q = fma2(q, f, pack2(0.693121791f, 0.693121791f));
  q = fma2(q, f, pack2(0.999999285f, 0.999999285f));
  float t0, t1, q0, q1;
  unpack2(t, t0, t1);
  unpack2(q, q0, q1);
  e0 = x0 >= -125.f ? __uint_as_float(__float_as_uint(q0) + (__float_as_uint(t0) << 23)) : 0.f;
  e1 = x1 >= -125.f ? __uint_as_float(__float_as_uint(q1) + (__float_as_uint(t1) << 23)) : 0.f;
}
template <int D, bool F16, bool SPARSE>
__global__ void __launch_bounds__(THREADS, 1) paged_tc_kernel(const __grid_constant__ TcParams tp, const __grid_constant__ TcMaps maps) {
  using L = Layout<D>;
  constexpr int NCH = L::NCH;
  constexpr uint32_t TILE_BYTES = L::TILE_BYTES, SM_Q = L::SM_Q, SM_K = L::SM_K, SM_V = L::SM_V, SM_OUT = L::SM_OUT, SM_BAR = L::SM_BAR;
  // How far (log2) a maximum may rise above the reference of its row's exponentials: bf16 and the 32-bit sums have room for 2^32,
  // fp16 probabilities for 2^15.
  constexpr float THRESHOLD = F16 ? 8.f : RESCALE_THRESHOLD;
  // One pair of exponentials in four on the FMA units where the exponential unit is as busy as anything (64-wide heads: a chunk of 1500
  // tokens behind 20 000, 40 heads, 439 us without, 396 with one pair in four, 438 with one in two; 128-wide heads, bound by the products:
  // no difference, and 6 % slower with one in two).
  constexpr bool POLY = D == 64;
  const PagedParams& p = tp.a;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t sbase = (raw + 1023u) & ~1023u;
  unsigned char* sgen = smem_raw + (sbase - raw);
  volatile uint32_t* abort_flag = reinterpret_cast<volatile uint32_t*>(sgen + SM_BAR + BAR_ABORT);
  volatile uint32_t* tmem_ptr_smem = reinterpret_cast<volatile uint32_t*>(sgen + SM_BAR + BAR_TMEM_PTR);
  volatile int32_t* ring_base = reinterpret_cast<volatile int32_t*>(sgen + SM_BAR + BAR_RING);
  volatile int32_t* info_base = reinterpret_cast<volatile int32_t*>(sgen + SM_BAR + BAR_INFO);
  auto bar = [&](uint32_t which) { return sbase + SM_BAR + which * 8; };
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;

  pdl_trigger();
  if (threadIdx.x == 0) {
    for (int x = 0; x < 2; ++x) {
      mbar_init(bar(Q_FULL + x), 1);
      mbar_init(bar(Q_EMPTY + x), 1);
      mbar_init(bar(S_FULL + x), 1);
      mbar_init(bar(P_FULL + 2 * x), BM);
      mbar_init(bar(P_FULL + 2 * x + 1), BM);
      mbar_init(bar(PV_DONE + x), 1);
      mbar_init(bar(ITEM_FULL + x), 1);
      mbar_init(bar(ITEM_EMPTY + x), 10);
    }
    for (int s = 0; s < KV_STAGES; ++s) {
      mbar_init(bar(K_FULL + s), 1);
      mbar_init(bar(K_EMPTY + s), 1);
      mbar_init(bar(V_FULL + s), 1);
      mbar_init(bar(V_EMPTY + s), 1);
    }
    mbar_init(bar(DRAIN), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 0) {
    __syncwarp();
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(sbase + SM_BAR + BAR_TMEM_PTR), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  pdl_wait();
  if (threadIdx.x == 0) *abort_flag = *reinterpret_cast<volatile uint32_t*>(p.status) != 0;      // an earlier CTA gave up: do not wait again
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, *tmem_ptr_smem, 0);

  if (warp < 4) {
    reg_dealloc<REGS_SMALL>();
    if (warp == 0) {
      // ---------------------------------------------------------------- copies
      const bool leader = elect_one();
      uint32_t g = 0, iq[2] = {0, 0};                              // key tiles sent for; items that loaded query tile x
      uint32_t armed_k = 0, armed_v = 0, armed_q = 0, par_k = 0, par_v = 0, par_q = 0;
      const uint32_t q_bytes = (uint32_t)(p.tile_tokens * p.G) * 128;
      bool ok = true;
      for (uint32_t it = 0; ok; ++it) {
        const uint32_t slot = it & 1;
        volatile int32_t* ring = ring_base + slot * 16;
        ok = wait_all(bar(ITEM_FULL + slot), (it >> 1) & 1, abort_flag, p.status, 1 + ITEM_FULL);
        if (!ok) break;
        if (ring_word(ring, W_KIND) == 0) break;
        const int head = ring_word(ring, W_HEAD), tok0 = ring_word(ring, W_TOK0), tokens = ring_word(ring, W_TOKENS), j0 = ring_word(ring, W_J0),
                  n_tiles = ring_word(ring, W_NT), nq = tokens > p.tile_tokens ? 2 : 1;
        const int32_t* table = p.block_table + ring_word(ring, W_SEQ) * p.table_stride;
        const int n_pages = (ring_word(ring, W_KV) + PAGE - 1) / PAGE;
        int pages = -1;
        Merge merge;
        uint32_t bits[4];
        if (SPARSE) {
          merge.start(reinterpret_cast<const uint16_t*>(sgen + L::SM_LIST) + slot * LIST_ENTRIES, p.n_sel, tokens, p.tile_tokens, lane);
          const int seek = ring_word(ring, W_SEEK);                // past the pages of the parts before this one
          if (seek > 0) merge.seek(seek, p.n_sel, p.tile_tokens, lane);
          if (seek < 0)
            for (int i = 0; i < 2 * j0; ++i) merge.next(bits[0], bits[1]);
        }
        for (int j = 0; j < n_tiles && ok; ++j, ++g) {
          if (!SPARSE && (j & 15) == 0) {                          // page numbers of 16 tiles at a time, one per lane
            const int pg = 2 * (j0 + j) + lane;
            pages = pg < n_pages ? table[pg] : -1;
            if (pages >= p.n_pages || pages < 0) pages = -1;       // (a box outside of the map arrives as zeros)
          }
          int pg0, pg1, place0 = 0, place1 = 0;
          if (SPARSE) {
            place0 = merge.next(bits[0], bits[2]);
            place1 = merge.next(bits[1], bits[3]);
            const int place = (lane & 1) ? place1 : place0;
            pages = place < NO_PAGE ? table[place] : -1;
            if (pages >= p.n_pages || pages < 0) pages = -1;
            pg0 = __shfl_sync(0xffffffffu, pages, 0);
            pg1 = __shfl_sync(0xffffffffu, pages, 1);
          } else {
            pg0 = __shfl_sync(0xffffffffu, pages, 2 * (j & 15));
            pg1 = __shfl_sync(0xffffffffu, pages, 2 * (j & 15) + 1);
          }
          const uint32_t st = g % KV_STAGES, use = g / KV_STAGES;
          auto load = [&](uint32_t smem, const CUtensorMap* map, uint32_t full) {
            if (!leader) return;
            mbar_expect_tx(full, TILE_BYTES);
#pragma unroll
            for (int ch = 0; ch < NCH; ++ch) {
              tma_load_4d(smem + ch * HALF_COLS_BYTES, map, ch * 64, 0, head, pg0, full);
              tma_load_4d(smem + ch * HALF_COLS_BYTES + SLOT_BYTES, map, ch * 64, 0, head, pg1, full);
            }
          };
          if (use > 0) ok = wait_all(bar(K_EMPTY + st), (use - 1) & 1, abort_flag, p.status, 1 + K_EMPTY);
          if (!ok) break;
          if (SPARSE && lane == 0) {
            volatile int32_t* info = info_base + (g % INFO_RING) * INFO_WORDS;
            info[I_PLACE] = place0;
            info[I_PLACE + 1] = place1;
#pragma unroll
            for (int i = 0; i < 4; ++i) info[I_BITS + i] = (int32_t)bits[i];
          }
          __syncwarp();
          armed_k |= 1u << st;
          par_k = (par_k & ~(1u << st)) | ((use & 1) << st);
          load(sbase + SM_K + st * TILE_BYTES, &maps.k, bar(K_FULL + st));
          if (j == 0) {
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              if (y >= nq || !ok) continue;
              if (iq[y] > 0) ok = wait_all(bar(Q_EMPTY + y), (iq[y] - 1) & 1, abort_flag, p.status, 1 + Q_EMPTY);
              if (!ok) continue;
              armed_q |= 1u << y;
              par_q = (par_q & ~(1u << y)) | ((iq[y] & 1) << y);
              ++iq[y];
              if (leader) {
                mbar_expect_tx(bar(Q_FULL + y), NCH * q_bytes);
                for (int ch = 0; ch < NCH; ++ch)
                  tma_load_4d(sbase + SM_Q + y * TILE_BYTES + ch * HALF_COLS_BYTES, &maps.q, ch * 64, head * p.G, tok0 + y * p.tile_tokens, 0,
                              bar(Q_FULL + y));
              }
            }
            if (!ok) break;
          }
          if (use > 0) ok = wait_all(bar(V_EMPTY + st), (use - 1) & 1, abort_flag, p.status, 1 + V_EMPTY);
          if (!ok) break;
          armed_v |= 1u << st;
          par_v = (par_v & ~(1u << st)) | ((use & 1) << st);
          load(sbase + SM_V + st * TILE_BYTES, &maps.v, bar(V_FULL + st));
          __syncwarp();
        }
        __syncwarp();
        if (ok && leader) mbar_arrive(bar(ITEM_EMPTY + slot));
      }
      if (!ok || *abort_flag) {
        // leaving early: every copy under way lands before the CTA exits
        for (int s = 0; s < KV_STAGES; ++s) {
          if (armed_k & (1u << s))
            settle(bar(K_FULL + s), (par_k >> s) & 1);
          if (armed_v & (1u << s))
            settle(bar(V_FULL + s), (par_v >> s) & 1);
        }
        for (int y = 0; y < 2; ++y)
          if (armed_q & (1u << y))
            settle(bar(Q_FULL + y), (par_q >> y) & 1);
      }
    } else if (warp == 2) {
      // ---------------------------------------------------------------- the CTA's run
      const bool leader = elect_one();
      const int32_t* run = tp.runs + blockIdx.x * RUN_WORDS;
      int64_t left = *reinterpret_cast<const int64_t*>(run + R_UNITS); // what is left of the run
      int seq = 0, head = 0, item = 0, j0 = 0;                         // where it goes on
      if (left > 0) {
        seq = run[R_SEQ];
        head = run[R_HEAD];
        item = run[R_ITEM];
        j0 = run[R_J0];
      }
      for (uint32_t it = 0;; ++it) {
        const uint32_t slot = it & 1;
        volatile int32_t* ring = ring_base + slot * 16;
        if (it >= 2 && !wait_all(bar(ITEM_EMPTY + slot), ((it >> 1) - 1) & 1, abort_flag, p.status, 1 + ITEM_EMPTY)) break;
        if (left <= 0) {
          if (lane == 0) ring[W_KIND] = 0;
          __syncwarp();
          if (leader) mbar_arrive(bar(ITEM_FULL + slot));
          break;
        }
        int q_first;
        const int n_items = tp.item_begin[seq + 1] - tp.item_begin[seq];
        const int n = request_tokens(p, seq, q_first), kv = request_keys(p, seq);
        const int tok = item * 2 * p.tile_tokens, tokens = min(n - tok, 2 * p.tile_tokens);
        const int flat = SPARSE ? (tp.item_begin[seq] + item) * p.Hkv + head : 0;
        const int tiles = SPARSE ? tp.item_prefix[flat + 1] - tp.item_prefix[flat] - ITEM_END : item_tiles(p, tok, n, kv),
                  n_tiles = (int)min((int64_t)(tiles - j0), left);
        int seek = j0 > 0 ? -1 : 0;
        if (SPARSE) {
          uint16_t* list = reinterpret_cast<uint16_t*>(sgen + L::SM_LIST) + slot * LIST_ENTRIES;
          const bool ascend = load_lists(p, list, q_first + tok, tokens, kv - n + tok, head, lane);
          if (j0 > 0 && ascend) {                                  // (the run's first item alone)
            uint32_t* marks = reinterpret_cast<uint32_t*>(sgen + L::SM_LIST + 2 * LIST_ENTRIES * 2);
            const int words = pages_words(p, kv - n + tok + tokens - 1);
            mark_pages(list, tokens * p.n_sel, marks, words, lane);
            seek = page_of_rank(marks, words, 2 * j0, lane);
          }
        }
        if (lane == 0) {
          ring[W_KIND] = 1;
          ring[W_SEQ] = seq;
          ring[W_HEAD] = head;
          ring[W_TOK0] = q_first + tok;
          ring[W_TOKENS] = tokens;
          ring[W_POS0] = kv - n + tok;
          ring[W_KV] = kv;
          ring[W_J0] = j0;
          ring[W_NT] = n_tiles;
          ring[W_TILES] = tiles;
          ring[W_C0] = it == 0 ? run[R_C0_FIRST] : (int)blockIdx.x;
          ring[W_C1] = it == 0 ? run[R_C1_FIRST] : run[R_C1_LAST];
          ring[W_SEEK] = seek;
        }
        __syncwarp();
        if (leader) mbar_arrive(bar(ITEM_FULL + slot));
        left -= n_tiles + (j0 + n_tiles == tiles ? ITEM_END : 0);
        // the next item of the run: the request's next tokens, its next head, the next request with tokens
        // (over selected pages the heads come first: the order of the sums)
        j0 = 0;
        bool request_done;
        if (SPARSE) {
          if (++head == p.Hkv) {
            head = 0;
            ++item;
          }
          request_done = item == n_items;
        } else {
          if (++item == n_items) {
            item = 0;
            ++head;
          }
          request_done = head == p.Hkv;
        }
        if (request_done) {
          item = head = 0;
          do ++seq; while (left > 0 && seq + 1 < p.n_seq && tp.item_begin[seq + 1] == tp.item_begin[seq]);
        }
      }
    } else if (warp == 1) {
      // ---------------------------------------------------------------- products
      constexpr uint32_t TYPE = F16 ? ~((1u << 7) | (1u << 10)) : ~0u;           // operand types: the descriptor's default is bf16
      constexpr uint32_t IDESC_S = instr_desc(BM, BN, 0, 0) & TYPE, IDESC_PV = instr_desc(BM, D, 0, 1) & TYPE;
      bool ok = true;
      auto mma_wait = [&](uint32_t which, uint32_t parity) { return wait_all(bar(which), parity, abort_flag, p.status, 1 + which); };
      const uint32_t q_lo = desc_lo(sbase + SM_Q, 16), k_lo = desc_lo(sbase + SM_K, 16), v_lo = desc_lo(sbase + SM_V, HALF_COLS_BYTES);
      auto issue_s = [&](uint32_t lead, int x, int st) {
        const uint32_t qa = q_lo + x * (TILE_BYTES >> 4), ka = k_lo + st * (TILE_BYTES >> 4);
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
          const uint32_t off = ((ks >> 2) * HALF_COLS_BYTES + (ks & 3) * 32) >> 4;
          mma_ss(lead, tmem + x * 128, qa + off, ka + off, IDESC_S, ks > 0);
        }
      };
      auto issue_pv = [&](uint32_t lead, int x, int st, int h, bool first) {
        const uint32_t va = v_lo + st * (TILE_BYTES >> 4);
#pragma unroll
        for (int ks = 4 * h; ks < 4 * h + 4; ++ks)
          mma_ts(lead, tmem + 256 + x * 128, tmem + x * 128 + ks * 8, va + ks * (2048 >> 4), IDESC_PV, !(first && ks == 0));
      };
      uint32_t g = 0, cx[2] = {0, 0}, iq[2] = {0, 0};
      for (uint32_t it = 0; ok; ++it) {
        const uint32_t slot = it & 1;
        volatile int32_t* ring = ring_base + slot * 16;
        ok = mma_wait(ITEM_FULL + slot, (it >> 1) & 1);
        if (!ok) break;
        if (ring_word(ring, W_KIND) == 0) break;
        const int nq = ring_word(ring, W_TOKENS) > p.tile_tokens ? 2 : 1, n_tiles = ring_word(ring, W_NT);
        const int nt[2] = {tiles_of_a<SPARSE>(p, ring, n_tiles), n_tiles};
        const int kv_len = ring_word(ring, W_KV), kv_left = kv_len - ring_word(ring, W_J0) * BN;      // keys of the request from the item's first on
        // values of the tile: waited for, and rows without a key in the request's last page made zero
        auto values = [&](uint32_t st, uint32_t parity, int j) {
          if (!mma_wait(V_FULL + st, parity)) return false;
          int r0 = 0, r1 = 0;
          if (SPARSE) {
            const volatile int32_t* info = info_base + ((g + j) % INFO_RING) * INFO_WORDS;
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
              const int place = ring_word(info, I_PLACE + hf), rows = place < NO_PAGE ? kv_len - place * PAGE : PAGE;
              if (rows > 0 && rows < PAGE) {
                r0 = hf * PAGE + rows;
                r1 = hf * PAGE + PAGE;
              }
            }
          } else {
            const int left = kv_left - j * BN;
            if (left < BN && left > 0) {
              r0 = left;
              r1 = (left + PAGE - 1) & ~(PAGE - 1);
            }
          }
          if (r0 < r1) {
            for (int i = lane; i < (r1 - r0) * 8 * NCH; i += 32) {
              const int ch = i / ((r1 - r0) * 8), rest = i - ch * (r1 - r0) * 8;
              const uint32_t at = SM_V + st * TILE_BYTES + ch * HALF_COLS_BYTES + (r0 + (rest >> 3)) * 128 + (rest & 7) * 16;
              *reinterpret_cast<int4*>(sgen + at) = make_int4(0, 0, 0, 0);
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
          }
          return true;
        };
        const uint32_t st0 = g % KV_STAGES, par0 = (g / KV_STAGES) & 1;
#pragma unroll
        for (int x = 0; x < 2; ++x)
          if (x < nq && ok) ok = mma_wait(Q_FULL + x, iq[x] & 1);
        if (ok) ok = mma_wait(K_FULL + st0, par0);
        if (ok) {
          const uint32_t lead = elect_one();
          tc_fence_after();
          for (int x = 0; x < nq; ++x) {
            issue_s(lead, x, st0);
            tc_commit(lead, bar(S_FULL + x));
            if (nt[x] == 1) tc_commit(lead, bar(Q_EMPTY + x));
          }
          tc_commit(lead, bar(K_EMPTY + st0));
        }
        if (ok) ok = values(st0, par0, 0);
        for (int j = 0; j < n_tiles && ok; ++j) {
          const uint32_t st = (g + j) % KV_STAGES, stn = (g + j + 1) % KV_STAGES;
          const uint32_t parn = ((g + j + 1) / KV_STAGES) & 1;
          const bool last = j + 1 == n_tiles;
          bool keys = last;                                        // the next tile's keys are there (or not wanted)
          const uint32_t lead = elect_one();
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            if (x >= nq || j >= nt[x] || !ok) continue;
            const bool more = j + 1 < nt[x];
            const uint32_t ph = (cx[x] + j) & 1;
            ok = mma_wait(P_FULL + 2 * x, ph);
            if (!ok) continue;
            tc_fence_after();
            issue_pv(lead, x, st, 0, j == 0);
            if (!keys) ok = mma_wait(K_FULL + stn, parn);
            keys = true;
            if (!ok) continue;
            ok = mma_wait(P_FULL + 2 * x + 1, ph);
            if (!ok) continue;
            tc_fence_after();
            issue_pv(lead, x, st, 1, false);
            if (more) {
              issue_s(lead, x, stn);
              tc_commit(lead, bar(S_FULL + x));
              if (j + 2 == nt[x]) tc_commit(lead, bar(Q_EMPTY + x));
            } else {
              tc_commit(lead, bar(PV_DONE + x));
            }
          }
          if (ok) {
            tc_commit(lead, bar(V_EMPTY + st));
            if (!last) tc_commit(lead, bar(K_EMPTY + stn));
          }
          if (ok && !last) ok = values(stn, parn, j + 1);
        }
        g += n_tiles;
#pragma unroll
        for (int x = 0; x < 2; ++x)
          if (x < nq) {
            cx[x] += nt[x];
            ++iq[x];
          }
        __syncwarp();
        if (ok && elect_one()) mbar_arrive(bar(ITEM_EMPTY + slot));
      }
      if (!ok) {
        // leaving early: products under way end before their operands and the tensor memory are given back
        __syncwarp();
        tc_commit(elect_one(), bar(DRAIN));
        settle(bar(DRAIN), 0);
      }
    }
  } else {
    reg_alloc<REGS_SOFTMAX>();
    // ------------------------------------------------------------------ softmax and results
    const int x = (warp - 4) >> 2;
    const int row = (warp & 3) * 32 + lane;                        // row of the tile == TMEM lane
    const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t t_s = tmem + lane_base + x * 128, t_o = tmem + lane_base + 256 + x * 128;
    unsigned char* stage = sgen + SM_OUT + (warp - 4) * STAGE_BYTES;
    const int row_tok = row / p.G, row_head = row - row_tok * p.G;
    uint32_t cx = 0, items_x = 0, g = 0;                            // key tiles of this tile's rows; its items; key tiles in all
    bool ok = true;
    for (uint32_t it = 0; ok; ++it) {
      const uint32_t slot = it & 1;
      volatile int32_t* ring = ring_base + slot * 16;
      ok = wait_all(bar(ITEM_FULL + slot), (it >> 1) & 1, abort_flag, p.status, 1 + ITEM_FULL);
      if (!ok) break;
      if (ring_word(ring, W_KIND) == 0) break;
      const int all_tiles = ring_word(ring, W_NT), tokens = ring_word(ring, W_TOKENS);
      const int n_tiles = x == 0 && tokens > p.tile_tokens ? tiles_of_a<SPARSE>(p, ring, all_tiles) : all_tiles;      // of this row tile
      if (x == 0 || tokens > p.tile_tokens) {
        const int kv = ring_word(ring, W_KV), pos0 = ring_word(ring, W_POS0), skipped = ring_word(ring, W_J0) * BN;
        const bool valid = row_tok < p.tile_tokens && x * p.tile_tokens + row_tok < tokens;
        // keys that the row sees, counted from the run's first
        const int sees = p.causal && valid ? min(pos0 + x * p.tile_tokens + row_tok + 1, kv) : kv;
        const int lim = SPARSE ? sees : sees - skipped;
        const int least = __reduce_min_sync(0xffffffffu, lim);
        float m_ref = NO_MAX, l_sum = 0.f;
#pragma unroll 1
        for (int j = 0; j < n_tiles && ok; ++j) {
          const uint32_t ph = (cx + j) & 1;
          ok = wait_all(bar(S_FULL + x), ph, abort_flag, p.status, 1 + S_FULL);
          if (!ok) break;
          tc_fence_after();
          uint32_t r0[32], r1[32], r2[32], r3[32];
          tmem_ld32(t_s, r0);
          tmem_ld32(t_s + 32, r1);
          tmem_ld32(t_s + 64, r2);
          tmem_ld32(t_s + 96, r3);
          tmem_wait_ld();
          bool sel0 = true, sel1 = true;                           // does the row see the tile's two pages at all
          // keys of each half that the row sees, where some row of the warp does not see all of them (else more than it has)
          int left0 = BN, left1 = BN;
          if (SPARSE) {
            const volatile int32_t* info = info_base + ((g + j) % INFO_RING) * INFO_WORDS;
            const int place0 = info[I_PLACE], place1 = info[I_PLACE + 1];
            sel0 = valid && ((uint32_t)info[I_BITS + 2 * x] >> row_tok & 1u);
            sel1 = valid && ((uint32_t)info[I_BITS + 2 * x + 1] >> row_tok & 1u);
            // (in pages that no row selected, and in the last one past the row's own position)
            if (place0 * PAGE + PAGE > least) left0 = sees - place0 * PAGE;
            if (place1 * PAGE + PAGE > least) left1 = sees - place1 * PAGE;
          } else if ((j + 1) * BN > least) {
            left0 = lim - j * BN;
            left1 = left0 - PAGE;
          }
          auto mask = [](uint32_t (&a)[32], uint32_t (&b)[32], int left) {
#pragma unroll
            for (int i = 0; i < 32; ++i) {
              if (i >= left) a[i] = 0xff800000u;
              if (i + 32 >= left) b[i] = 0xff800000u;
            }
          };
          if (__any_sync(0xffffffffu, left0 < PAGE)) mask(r0, r1, left0);
          if (__any_sync(0xffffffffu, left1 < PAGE)) mask(r2, r3, left1);
          auto top_of = [](const uint32_t (&a)[32], const uint32_t (&b)[32]) {
            float mq[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) mq[c] = fmaxf(__uint_as_float(a[c]), __uint_as_float(b[c]));
#pragma unroll
            for (int i = 4; i < 32; ++i) mq[i & 3] = fmax3(mq[i & 3], __uint_as_float(a[i]), __uint_as_float(b[i]));
            return fmaxf(fmaxf(mq[0], mq[1]), fmaxf(mq[2], mq[3]));
          };
          const uint64_t scale2 = pack2(p.scale_log2, p.scale_log2);
          // The sum takes the probabilities as 32-bit numbers; for the product with V they are rounded to the 16 bits of the matrix unit's operand in
          // tensor memory: the result's error is then 1.3 times that of its own rounding, and a product for the low halves would be as long again.
          // (a page that the row did not select: every exponent minus infinity)
          const uint64_t none2 = pack2(-INFINITY, -INFINITY);
          uint64_t sum2 = pack2(0.f, 0.f);
          auto exp_chunk = [&](const uint32_t (&rc)[32], uint64_t shift, int c) {
            uint32_t pk[16];
#pragma unroll
            for (int i = 0; i < 32; i += 2) {
              const uint64_t xx = fma2(pack2(__uint_as_float(rc[i]), __uint_as_float(rc[i + 1])), scale2, shift);
              float e0, e1;
              if (POLY && (i >> 1 & 3) == 3) {
                exp2_pair(xx, e0, e1);
              } else {
                float x0, x1;
                unpack2(xx, x0, x1);
                e0 = ex2_approx(x0);
                e1 = ex2_approx(x1);
              }
              sum2 = add2(sum2, pack2(e0, e1));
              pk[i >> 1] = pack16<F16>(e0, e1);
            }
            tmem_st16(t_s + c * 16, pk);
          };
          const float mx0 = sel0 ? top_of(r0, r1) : -INFINITY, mx1 = sel1 ? top_of(r2, r3) : -INFINITY;
          const float m_new = fmaxf(m_ref, fmaxf(mx0, mx1) * p.scale_log2);
          // also on the first tile with a key the row sees; (rows that are none hold anything)
          const bool grow = valid && m_new > m_ref + THRESHOLD;
          if (j > 0 && __any_sync(0xffffffffu, grow)) {
            // O is complete up to tile j - 1: the commit behind S_FULL covers every product issued before it
            const float f = grow ? exp2f(m_ref - m_new) : 1.f;
#pragma unroll
            for (int c = 0; c < D / 32; ++c) {
              uint32_t r[32];
              tmem_ld32(t_o + c * 32, r);
              tmem_wait_ld();
#pragma unroll
              for (int i = 0; i < 32; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) * f);
              tmem_st32(t_o + c * 32, r);
            }
            tmem_wait_st();
            l_sum *= f;
          }
          if (grow) m_ref = m_new;
          const uint64_t shift2 = pack2(-m_ref, -m_ref);
          exp_chunk(r0, sel0 ? shift2 : none2, 0);
          exp_chunk(r1, sel0 ? shift2 : none2, 1);
          tmem_wait_st();
          tc_fence_before();
          mbar_arrive(bar(P_FULL + 2 * x));                        // the product with values 0..63 may start
          exp_chunk(r2, sel1 ? shift2 : none2, 2);
          exp_chunk(r3, sel1 ? shift2 : none2, 3);
          float sa, sb;
          unpack2(sum2, sa, sb);
          l_sum += sa + sb;
          tmem_wait_st();
          tc_fence_before();
          mbar_arrive(bar(P_FULL + 2 * x + 1));
        }
        if (ok) ok = wait_all(bar(PV_DONE + x), items_x & 1, abort_flag, p.status, 1 + PV_DONE);
        ++items_x;
        cx += n_tiles;
        if (ok) {
          tc_fence_after();
          const int tok = ring_word(ring, W_TOK0) + x * p.tile_tokens + row_tok, hd = ring_word(ring, W_HEAD) * p.G + row_head;
          const int64_t o_at = (int64_t)tok * p.o_tok + (int64_t)hd * p.o_head;
          // 32 columns of the warp's rows, through shared memory so that four lanes write 64 bytes of a row
          auto store_rows = [&](const float (&acc)[32], float inv, int c) {
#pragma unroll
            for (int i = 0; i < 32; i += 8) {
              int4 v;
              v.x = (int)pack16<F16>(acc[i] * inv, acc[i + 1] * inv);
              v.y = (int)pack16<F16>(acc[i + 2] * inv, acc[i + 3] * inv);
              v.z = (int)pack16<F16>(acc[i + 4] * inv, acc[i + 5] * inv);
              v.w = (int)pack16<F16>(acc[i + 6] * inv, acc[i + 7] * inv);
              *reinterpret_cast<int4*>(stage + lane * 64 + (((i >> 3) ^ ((lane >> 1) & 3)) << 4)) = v;
            }
            __syncwarp();
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const int r = k * 8 + (lane >> 2), ch = lane & 3;
              const int4 v = *reinterpret_cast<const int4*>(stage + r * 64 + ((ch ^ ((r >> 1) & 3)) << 4));
              const int64_t at = __shfl_sync(0xffffffffu, o_at, r);
              if (__shfl_sync(0xffffffffu, (int)valid, r))
                *reinterpret_cast<int4*>(static_cast<__nv_bfloat16*>(p.out) + at + c * 32 + ch * 8) = v;
            }
            __syncwarp();
          };
          auto finish = [&](float m, float l) {                    // 1 / sum, and the row's logarithm
            // the key that set the reference counts 1, so a sum below that has no key, or none with a weight; one that is NaN stays NaN
            const bool any = !(l <= 0.5f);
            if (p.lse && valid) p.lse[(int64_t)tok * p.H + hd] = any ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
            const float inv = any ? 1.f / l : 0.f;
            __syncwarp();                                          // the loads of tensor memory that follow are the whole warp's
            return inv;
          };
          const int tiles = ring_word(ring, W_TILES);
          if (all_tiles == tiles) {
            const float inv = finish(m_ref, l_sum);
#pragma unroll 1
            for (int c = 0; c < D / 32; ++c) {
              uint32_t r[32];
              tmem_ld32(t_o + c * 32, r);
              tmem_wait_ld();
              float acc[32];
#pragma unroll
              for (int i = 0; i < 32; ++i) acc[i] = __uint_as_float(r[i]);
              store_rows(acc, inv, c);
            }
          } else {
            const int c0 = ring_word(ring, W_C0), c1 = ring_word(ring, W_C1), me = blockIdx.x;
            auto part = [&](int c) { return p.partials + (int64_t)(2 * c + (c == c0 ? 1 : 0)) * L::SLOT_FLOATS; };
            uint32_t* ctr = p.counters + c0 * 8 + (warp - 4);
            // all other parts of these 32 rows there already?  Then this one stays in tensor memory
            uint32_t last = 0;
            if (lane == 0) {
              uint32_t seen;
              asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(seen) : "l"(ctr) : "memory");
              last = seen == (uint32_t)(c1 - c0);
              if (last) *reinterpret_cast<volatile uint32_t*>(ctr) = 0;
            }
            last = __shfl_sync(0xffffffffu, last, 0);
            if (!last) {
              float* own = part(me);
              int4* oc = reinterpret_cast<int4*>(own) + x * BM + row;
#pragma unroll 1
              for (int c = 0; c < D / 32; ++c) {
                uint32_t r[32];
                tmem_ld32(t_o + c * 32, r);
                tmem_wait_ld();
#pragma unroll
                for (int q = 0; q < 8; ++q) oc[(c * 8 + q) * (2 * BM)] = make_int4((int)r[4 * q], (int)r[4 * q + 1], (int)r[4 * q + 2], (int)r[4 * q + 3]);
              }
              own[2 * BM * D + x * BM + row] = m_ref;
              own[2 * BM * D + 2 * BM + x * BM + row] = l_sum;
              __threadfence();
              __syncwarp();
              if (lane == 0) {
                const uint32_t old = atomicAdd(ctr, 1u);
                last = old == (uint32_t)(c1 - c0);
                if (last) *reinterpret_cast<volatile uint32_t*>(ctr) = 0;
              }
              last = __shfl_sync(0xffffffffu, last, 0);
            }
            if (last) {
              __threadfence();
              // in key order, this warp's own part from tensor memory at its place
              auto m_of = [&](int c) { return c == me ? m_ref : __ldcg(part(c) + 2 * BM * D + x * BM + row); };
              auto l_of = [&](int c) { return c == me ? l_sum : __ldcg(part(c) + 2 * BM * D + 2 * BM + x * BM + row); };
              constexpr int FAST = 4;                              // parts whose two words are read once, all on their way together
              float w4[FAST], l4[FAST];
#pragma unroll
              for (int i = 0; i < FAST; ++i) {
                w4[i] = c0 + i <= c1 ? m_of(c0 + i) : NO_MAX;
                l4[i] = c0 + i <= c1 ? l_of(c0 + i) : 0.f;
              }
              float m_all = fmaxf(fmaxf(w4[0], w4[1]), fmaxf(w4[2], w4[3]));
              for (int c = c0 + FAST; c <= c1; ++c) m_all = fmaxf(m_all, m_of(c));
              float l_all = 0.f;
#pragma unroll
              for (int i = 0; i < FAST; ++i) {
                w4[i] = exp2f(w4[i] - m_all);                      // from here on: the part's weight
                l_all = fmaf(l4[i], w4[i], l_all);
              }
              for (int c = c0 + FAST; c <= c1; ++c) l_all = fmaf(l_of(c), exp2f(m_of(c) - m_all), l_all);
              const float inv = finish(m_all, l_all);
#pragma unroll 1
              for (int cc = 0; cc < D / 32; ++cc) {
                uint32_t r[32];
                tmem_ld32(t_o + cc * 32, r);
                tmem_wait_ld();
                float acc[32];
#pragma unroll
                for (int i = 0; i < 32; ++i) acc[i] = 0.f;
#pragma unroll 1
                for (int c = c0; c <= c1; ++c) {
                  const int i4 = c - c0;
                  const float w = i4 == 0 ? w4[0] : i4 == 1 ? w4[1] : i4 == 2 ? w4[2] : i4 == 3 ? w4[3] : exp2f(m_of(c) - m_all);
                  if (c == me) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) acc[i] = fmaf(__uint_as_float(r[i]), w, acc[i]);
                    continue;
                  }
                  const float4* oc = reinterpret_cast<const float4*>(part(c)) + (cc * 8) * (2 * BM) + x * BM + row;
#pragma unroll
                  for (int i = 0; i < 8; ++i) {
                    const float4 v = __ldcg(oc + i * (2 * BM));
                    acc[4 * i] = fmaf(v.x, w, acc[4 * i]);
                    acc[4 * i + 1] = fmaf(v.y, w, acc[4 * i + 1]);
                    acc[4 * i + 2] = fmaf(v.z, w, acc[4 * i + 2]);
                    acc[4 * i + 3] = fmaf(v.w, w, acc[4 * i + 3]);
                  }
                }
                store_rows(acc, inv, cc);
              }
            }
          }
          tc_fence_before();                                       // orders this item's reads of O before the next one's products
        }
      }
      g += all_tiles;
      __syncwarp();
      if (ok && lane == 0) mbar_arrive(bar(ITEM_EMPTY + slot));
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 0) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
  }
}

// room for the plan of a call, in bytes
uint64_t plan_items(int tile_tokens, int n_tokens, int n_seq) { return (uint64_t)n_tokens / (2 * (uint64_t)tile_tokens) + (uint64_t)n_seq; }
// tokens of a row tile over selected pages: a bit each in a word
int sparse_tile_tokens(int G) { return std::min(32, BM / G); }
uint64_t run_bytes(int n_sm) { return ((uint64_t)n_sm * RUN_WORDS * 4 + 255) / 256 * 256; }
uint64_t item_words(int n_seq) { return ((uint64_t)n_seq + 2) & ~1ull; }      // of item_begin: 64-bit numbers follow it
// (room for either kind of call: over selected pages every kv head's items count for themselves, and have at most 32 tokens a tile)
uint64_t plan_bytes(int G, int Hkv, int n_tokens, int n_seq) {
  const uint64_t dense = plan_items(BM / G, n_tokens, n_seq), sparse = plan_items(sparse_tile_tokens(G), n_tokens, n_seq) * Hkv + 1;
  return (4 * item_words(n_seq) + std::max(8 * dense, 4 * sparse) + 255) / 256 * 256;
}

template <int D, bool F16, bool SPARSE>
cudaError_t launch(const TcParams& tp, const TcMaps& maps, int grid, cudaStream_t stream) {
  auto kernel = paged_tc_kernel<D, F16, SPARSE>;
  constexpr int smem = (int)Layout<D>::SM_ALLOC + (SPARSE ? LIST_BYTES + LIST_ENTRIES * 2 : 0);
  cudaError_t rc = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (rc != cudaSuccess) return rc;
  // the register hand-over must fit in what the launch allocates, or it would wait for ever
  cudaFuncAttributes attr;
  rc = cudaFuncGetAttributes(&attr, kernel);
  if (rc != cudaSuccess) return rc;
  if (attr.numRegs * THREADS < 128 * REGS_SMALL + 256 * REGS_SOFTMAX) return cudaErrorLaunchOutOfResources;
  if (SPARSE) {
    const int bytes = ((tp.a.n_seq + 1) * 4 + 15) / 16 * 16 + UNION_WARPS * LIST_BYTES;
    rc = cudaFuncSetAttribute(union_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (PAGED_MAX_SEQ + 4) * 4 + UNION_WARPS * LIST_BYTES);
    if (rc != cudaSuccess) return rc;
    const int64_t warps = (int64_t)tp.items * tp.a.Hkv;
    rc = launch_pdl(union_kernel, dim3((unsigned)((warps + UNION_WARPS - 1) / UNION_WARPS)), dim3(UNION_THREADS), bytes, stream, tp);
  } else {
    constexpr int most = (PAGED_MAX_SEQ + 1) * 20 + PLAN_ITEMS * 8;
    const int bytes = (tp.a.n_seq + 1) * 20 + (tp.items <= PLAN_ITEMS ? tp.items * 8 : 0);
    rc = cudaFuncSetAttribute(plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
    if (rc != cudaSuccess) return rc;
    rc = launch_pdl(plan_kernel, dim3(1), dim3(PT), bytes, stream, tp);
  }
  if (rc != cudaSuccess) return rc;
  return launch_pdl(kernel, dim3(grid), dim3(THREADS), smem, stream, tp, maps);
}
template <int D, bool F16>
cudaError_t launch_either(const TcParams& tp, const TcMaps& maps, int grid, cudaStream_t stream) {
  return tp.a.sel ? launch<D, F16, true>(tp, maps, grid, stream) : launch<D, F16, false>(tp, maps, grid, stream);
}

}  // namespace

uint64_t paged_tc_partial_bytes(int d, int n_sm, int G, int Hkv, int n_tokens, int n_seq) {
  const uint64_t floats = d == 128 ? Layout<128>::SLOT_FLOATS : Layout<64>::SLOT_FLOATS;
  return run_bytes(n_sm) + plan_bytes(G, Hkv, n_tokens, n_seq) + 2 * (uint64_t)n_sm * floats * 4;
}

bool paged_tc_takes_lists(int G, int Hkv, int n_sel, int table_pages, int n_tokens, int n_seq) {
  const int tile_tokens = sparse_tile_tokens(G);
  if (2 * tile_tokens * (int64_t)n_sel > LIST_ENTRIES || table_pages >= 0xffff) return false;
  // the plan sums up key tiles in 32 bits: an item has half as many as its lists have pages, at most one more, and its end
  return ((int64_t)n_tokens * n_sel / 2 + (int64_t)plan_items(tile_tokens, n_tokens, n_seq) * (1 + ITEM_END)) * Hkv <= INT32_MAX;
}

cudaError_t launch_paged_tc(const PagedParams& p, const heatkv_paged_pool& pool, const PagedDevice& dev, cudaStream_t stream) {
  TcParams tp;
  tp.a = p;
  tp.a.tile_tokens = p.sel ? sparse_tile_tokens(p.G) : BM / p.G;
  tp.runs = reinterpret_cast<int32_t*>(p.partials);
  tp.item_begin = reinterpret_cast<int32_t*>(p.partials + run_bytes(dev.n_sm) / 4);
  tp.ticket = p.counters + PAGED_WS_CTRS * 8 - 1;
  tp.item_prefix = tp.item_begin + item_words(p.n_seq);
  tp.item_units = reinterpret_cast<int64_t*>(tp.item_prefix);
  tp.n_cta = dev.n_sm;
  tp.items = (int32_t)plan_items(tp.a.tile_tokens, p.n_tokens, p.n_seq);
  tp.a.partials = p.partials + (run_bytes(dev.n_sm) + plan_bytes(p.G, p.Hkv, p.n_tokens, p.n_seq)) / 4;
  TcMaps maps;
  if (!paged_encode_pool(dev, &maps.k, pool.k, pool) || !paged_encode_pool(dev, &maps.v, pool.v, pool) || !paged_encode_q(dev, &maps.q, tp.a, pool))
    return cudaErrorInvalidValue;
  const bool fp16 = pool.dtype == HEATKV_DTYPE_FP16;
  if (pool.d == 128) return fp16 ? launch_either<128, true>(tp, maps, dev.n_sm, stream) : launch_either<128, false>(tp, maps, dev.n_sm, stream);
  return fp16 ? launch_either<64, true>(tp, maps, dev.n_sm, stream) : launch_either<64, false>(tp, maps, dev.n_sm, stream);
}

}  // namespace heatkv
