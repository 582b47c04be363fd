// Attention of few query rows (decode, drafted tokens) over a paged cache in 4 bits, on warp-level MMA.
//
// A request's new tokens times the G query heads of one kv head are its rows, token by token; a row tile is 8 or 16 of them, a unit a row tile of one
// request and kv head, and its pages come one after another.  The pages of all units, request by request, head by head, are dealt out in equal
// runs, a CTA of eight warps each, and page x of a run belongs to warp x mod 8, whatever unit it is of: a warp takes whole pages by itself, from the
// copy that it sends for (9216 bytes, a ring of its own) to the product with V, and meets the others only where a unit, or the run's part of
// it, ends.  There every warp that had a page of it leaves its unnormalised rows in the stage that the page was in, and the last to come adds
// them up, in page order.  A unit that a run's border cuts leaves the sum in the workspace, which a second small kernel adds up.
//
// The products are transposed, S^T = K Q^T and O^T = V^T P^T, so that the cache is the operand with 16 rows and the queries the one with 8: a group of up to
// eight heads costs half of what it would the other way round.  Which columns a step of a product takes is free as long as both operands take the
// same, so a lane's part of K is what lies next to each other: 32 codes of one key (16 bytes) with their two scales, and of V 16 codes of one
// key with their scale.  Codes become fp16 numbers in registers, exactly (Steps4): bf16 queries are scaled, row by row, to fp16's range by a power of
// two, and probabilities are fp16 for either type.
#include <algorithm>
#include <climits>

#include "paged4.cuh"
#include "paged_wait.cuh"

namespace heatkv {
namespace {

using namespace tc;

constexpr int WARPS = 8, THREADS = WARPS * 32;
constexpr int MAX_STAGES = 6;
constexpr float MOVE = 8.f;                    // a reference moves when a maximum passes it by more than 2^MOVE (P fits fp16)
constexpr int WHOLE = 8;                       // units of up to so many pages, one a warp, are never cut
constexpr int MIN_PART = 4;                    // pages of a part
constexpr int OPEN = 32;                       // parts whose counters are kept: warps meet every other round, so fewer are under way at a time

struct Small4Params {
  Paged4Params q;
  int2* cuts;                                  // [n_tokens][H] {the CTA with the unit's first page, its parts | the row's place in it << 16}; no parts: not cut
  int32_t stages;
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
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
               : "memory");
}

__host__ __device__ constexpr int64_t slot_floats(int rows, int d) { return (int64_t)rows * (d + 2); }

// The runs.  `pre`: pages before each request; request i has `units` units of `pages` pages.
struct Shape {
  int pages, tiles;                            // of a unit; row tiles of the request
};
struct Runs {
  int64_t all;
  int grid;
  __device__ int64_t raw(int c) const { return all * c / grid; }
  // a border inside a unit of `pages` pages from `begin` on: not near its ends, not in a short one
  __device__ static int64_t snap(int64_t y, int64_t begin, int pages) {
    const int at = (int)(y - begin);
    if (pages <= WHOLE) return 2 * at < pages ? begin : begin + pages;
    return at < MIN_PART ? begin : pages - at < MIN_PART ? begin + pages : y;
  }
};

// Where a walk over the pages of a run is.
struct Walk {
  int seq, head, tile, j;                      // the page is number j of the unit
  int unit;                                    // units since the run's first
  Shape s;
  __device__ void next_unit(const Shape* shapes, int Hkv, int n_seq) {
    ++unit;
    if (++tile < s.tiles) return;
    tile = 0;
    if (++head < Hkv) return;
    head = 0;
    do {
      if (++seq >= n_seq) {                    // (behind the last page of all: nothing is read there)
        s.pages = INT_MAX;
        return;
      }
      s = shapes[seq];
    } while (s.pages == 0 || s.tiles == 0);
  }
  __device__ void advance(int by, const Shape* shapes, int Hkv, int n_seq) {
    j += by;
    while (j >= s.pages) {
      j -= s.pages;
      next_unit(shapes, Hkv, n_seq);
    }
  }
};

template <int D, int NT, bool F16>
__global__ void __launch_bounds__(THREADS, 1) paged4_small_kernel(const __grid_constant__ Small4Params sp) {
  using B = Block4<D>;
  constexpr int ROWS = 8 * NT, WORDS = D / 32;                     // words of codes that a lane has of a key
  constexpr int MTILES = D / 16;                                   // 16-row tiles of O^T: two neighbouring columns of a lane each
  const Paged4Params& q4 = sp.q;
  const PagedParams& p = q4.a;
  static_assert(ROWS * (D + 2) * 4 <= B::BYTES, "a warp's rows fit the stage that its page was in");
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ __align__(8) uint64_t bars[2 * WARPS * MAX_STAGES];
  __shared__ uint32_t counters[OPEN];
  __shared__ uint32_t abort_word;
  __shared__ int64_t sums[WARPS];
  volatile uint32_t* abort_flag = &abort_word;
  const int stages = sp.stages;
  int64_t* pre = reinterpret_cast<int64_t*>(smem + WARPS * stages * B::BYTES);      // [n_seq + 1]
  Shape* shapes = reinterpret_cast<Shape*>(pre + p.n_seq + 1);                      // [n_seq]
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  const uint32_t bar0 = smem_u32(bars);
  auto full = [&](int s) { return bar0 + (warp * MAX_STAGES + s) * 8; };
  auto merged = [&](int w, int s) { return bar0 + ((WARPS + w) * MAX_STAGES + s) * 8; };

  pdl_trigger();
  for (int i = threadIdx.x; i < 2 * WARPS * MAX_STAGES; i += THREADS) mbar_init(bar0 + i * 8, 1);
  if (threadIdx.x < OPEN) counters[threadIdx.x] = 0;
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  pdl_wait();
  if (threadIdx.x == 0) *abort_flag = *reinterpret_cast<volatile uint32_t*>(p.status) != 0;
  // ------------------------------------------------------------------ the run
  Runs runs;
  {
    const int per = (p.n_seq + THREADS - 1) / THREADS, i0 = min((int)threadIdx.x * per, p.n_seq), i1 = min(i0 + per, p.n_seq);
    int64_t mine = 0;
    for (int i = i0; i < i1; ++i) {
      const int b = max(p.q_begin[i], 0), n = max(min(p.q_begin[i + 1], p.n_tokens) - b, 0);
      const int kv = min(max(p.kv_len[i], 0), p.table_pages * PAGE);
      shapes[i] = {(kv + PAGE - 1) / PAGE, (n * p.G + ROWS - 1) / ROWS};
      mine += (int64_t)shapes[i].pages * shapes[i].tiles * p.Hkv;
    }
    int64_t inc = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t up = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += up;
    }
    if (lane == 31) sums[warp] = inc;
    __syncthreads();
    int64_t at = inc - mine;
    runs.all = 0;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
      const int64_t x = sums[w];
      if (w < warp) at += x;
      runs.all += x;
    }
    for (int i = i0; i < i1; ++i) {
      pre[i] = at;
      at += (int64_t)shapes[i].pages * shapes[i].tiles * p.Hkv;
    }
    if (threadIdx.x == 0) pre[p.n_seq] = runs.all;
    __syncthreads();
  }
  // rows of requests without keys
  for (int i = blockIdx.x; i < p.n_seq; i += gridDim.x) {
    if (shapes[i].pages > 0) continue;
    const int b = max(p.q_begin[i], 0), e = min(p.q_begin[i + 1], p.n_tokens);
    const int64_t n = (int64_t)max(e - b, 0) * p.H;
    for (int64_t j = threadIdx.x; j < n * D; j += THREADS) {
      const int64_t t = b + j / ((int64_t)p.H * D), hd = j / D % p.H;
      static_cast<uint16_t*>(p.out)[t * p.o_tok + hd * p.o_head + j % D] = 0;
    }
    if (p.lse)
      for (int64_t j = threadIdx.x; j < n; j += THREADS) p.lse[b * (int64_t)p.H + j] = -INFINITY;
    for (int64_t j = threadIdx.x; j < n; j += THREADS) sp.cuts[b * (int64_t)p.H + j] = make_int2(-1, 0);
  }
  runs.grid = (int)min((int64_t)gridDim.x, (runs.all + WHOLE - 1) / WHOLE);
  if ((int)blockIdx.x >= runs.grid) return;
  // the unit that holds page y of all
  auto find = [&](int64_t y, int64_t& begin) {
    int lo = 0, hi = p.n_seq - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (pre[mid] <= y) lo = mid; else hi = mid - 1;
    }
    Walk w;
    w.seq = lo;
    w.s = shapes[lo];
    const int64_t local = y - pre[lo], unit = local / w.s.pages;
    w.head = (int)(unit / w.s.tiles);
    w.tile = (int)(unit - (int64_t)w.head * w.s.tiles);
    w.j = (int)(local - unit * w.s.pages);
    w.unit = 0;
    begin = y - w.j;
    return w;
  };
  auto bound = [&](int c) {
    const int64_t y = runs.raw(c);
    if (c == 0 || c == runs.grid) return y;
    int64_t begin;
    const Walk w = find(y, begin);
    return Runs::snap(y, begin, w.s.pages);
  };
  const int64_t y0 = bound(blockIdx.x), y1 = bound(blockIdx.x + 1);
  if (y0 >= y1) return;
  const int n_run = (int)min(y1 - y0, (int64_t)INT_MAX / 2);
  int64_t first_begin;
  const Walk start = find(y0, first_begin);
  const int j_first = start.j;                                     // where the run's first unit goes on
  const int rounds = (n_run + WARPS - 1) / WARPS;

  // ------------------------------------------------------------------ copies
  unsigned char* ring = smem + warp * stages * B::BYTES;
  Walk ahead = start;                                              // the page to be sent for next, its round
  int ahead_round = 0, ahead_page = -1;
  if (warp > 0 && warp < n_run) ahead.advance(warp, shapes, p.Hkv, p.n_seq);
  // pages of a unit's part that are multiplied: those that some row sees, at least one; run-relative numbers of the part
  struct Part {
    int begin, count;                                              // first page, pages
    int j0, kv, pos0, tok0;                                        // tokens of the request; place and number of its first new one
    int row0, rows;                                                // the tile's
    bool ends;                                                     // the part has the unit's last page
  };
  auto part_of = [&](const Walk& w, int x) {                       // w: at the run's page x
    Part r;
    const int b = max(p.q_begin[w.seq], 0), n = max(min(p.q_begin[w.seq + 1], p.n_tokens) - b, 0);
    r.kv = min(max(p.kv_len[w.seq], 0), p.table_pages * PAGE);
    r.tok0 = b;
    r.pos0 = r.kv - n;
    r.row0 = w.tile * ROWS;
    r.rows = min(ROWS, n * p.G - r.row0);
    r.j0 = w.unit == 0 ? j_first : 0;
    r.begin = x - (w.j - r.j0);
    const int end = min(r.begin + w.s.pages - r.j0, n_run);
    r.ends = end == r.begin + w.s.pages - r.j0;
    const int sees = p.causal ? min(r.pos0 + (r.row0 + r.rows - 1) / p.G + 1, r.kv) : r.kv;
    r.count = max(min(end - r.begin, (max(sees, 0) + PAGE - 1) / PAGE - r.j0), 1);
    return r;
  };
  uint32_t held = 0, phase = 0;                                    // stages with rows that wait to be added up; the parity of their barriers
  auto look_up = [&]() {
    ahead_page = -1;
    if (ahead_round >= rounds || ahead_round * WARPS + warp >= n_run) return;
    ahead_page = __ldg(p.block_table + ahead.seq * p.table_stride + ahead.j);
  };
  auto send = [&]() {                                              // the page looked up, and on to the next
    const int x = ahead_round * WARPS + warp, st = ahead_round % stages;
    if (x < n_run) {
      unsigned char* dst = ring + st * B::BYTES;
      if (ahead_page >= 0 && ahead_page < p.n_pages) {
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");           // (rows or zeros of this warp may have been there)
        __syncwarp();
        if (lane == 0) {
          mbar_expect_tx(full(st), B::BYTES);
          bulk_load(smem_u32(dst), q4.blocks + ahead_page * q4.page_stride + ahead.head * q4.head_stride, B::BYTES, full(st));
        }
      } else {                                                     // no page of the pool: zeros
        for (int i = lane; i < B::BYTES / 16; i += 32) reinterpret_cast<int4*>(dst)[i] = make_int4(0, 0, 0, 0);
        __syncwarp();
        if (lane == 0) mbar_arrive(full(st));
      }
      __syncwarp();
      ahead.advance(WARPS, shapes, p.Hkv, p.n_seq);
    }
    ++ahead_round;
    look_up();
  };
  look_up();
  for (int r = 0; r < stages - 1; ++r) send();

  // ------------------------------------------------------------------ products and softmax
  const int gr = lane >> 2, qd = lane & 3;
  const int key_of = gr ^ ((gr >> 1) & 1);                         // keys of a block of eight in the order in which neither K's nor V's reads meet in a bank
  const int v0 = (2 * qd) ^ (qd & 1), v1 = v0 ^ 1;                 // the keys of the operands' columns 2 qd and 2 qd + 1
  uint32_t qf[NT][4 * WORDS];                                      // this lane's part of the query rows
  float row_scale[NT][2], m_ref[NT][2], l_sum[NT][2], o[MTILES][NT][4];
  int lim[NT][2], least = 0;                                       // keys that a row may see; the fewest
  Walk at = start;
  if (warp > 0 && warp < n_run) at.advance(warp, shapes, p.Hkv, p.n_seq);
  int unit_at_hand = -1;
  Part part = {};
  bool ok = true;
  for (int r = 0; r < rounds; ++r) {
    if (r > 0 && (r & 1) == 0) __syncthreads();
    const int x = r * WARPS + warp, st = r % stages;
    // the stage of the last round gets its next page, at once if nobody waits for rows in it
    const int next_st = (r + stages - 1) % stages;
    bool sent = false;
    if (!(held >> next_st & 1)) {
      send();
      sent = true;
    }
    if (x < n_run) {
      if (at.unit != unit_at_hand) {
        unit_at_hand = at.unit;
        part = part_of(at, x);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const int row = part.row0 + nt * 8 + gr, tok = row / p.G;
          uint4 w[WORDS];
#pragma unroll
          for (int i = 0; i < WORDS; ++i) w[i] = make_uint4(0, 0, 0, 0);
          if (nt * 8 + gr < part.rows) {
            const uint4* src = reinterpret_cast<const uint4*>(static_cast<const __half*>(p.q) + (int64_t)(part.tok0 + tok) * p.q_tok +
                                                              (int64_t)(at.head * p.G + row - tok * p.G) * p.q_head + qd * (D / 4));
#pragma unroll
            for (int i = 0; i < WORDS; ++i) w[i] = __ldg(src + i);
          }
#pragma unroll
          for (int i = 0; i < WORDS; ++i) {
            qf[nt][4 * i] = w[i].x;
            qf[nt][4 * i + 1] = w[i].y;
            qf[nt][4 * i + 2] = w[i].z;
            qf[nt][4 * i + 3] = w[i].w;
          }
          float unit = 1.f;                                        // of row `row`: what it was divided by
          if (!F16) {
            float top = 0.f;
#pragma unroll
            for (int i = 0; i < 4 * WORDS; ++i) top = fmaxf(top, fmaxf(fabsf(__uint_as_float(qf[nt][i] << 16)), fabsf(__uint_as_float(qf[nt][i] & 0xffff0000u))));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
            // 2^14 times the power of two in `top`; rows of infinities, of zeros or below 2^-86 are left as near as fp16 comes to them
            const int e = (int)(__float_as_uint(top) >> 23);
            const int power = top == 0.f || e == 255 ? 0 : min(14 + 127 - e, 100);
            const float up = __uint_as_float((uint32_t)(127 + power) << 23);
            unit = __uint_as_float((uint32_t)(127 - power) << 23);
#pragma unroll
            for (int i = 0; i < 4 * WORDS; ++i)
              qf[nt][i] = pack_half(__uint_as_float(qf[nt][i] << 16) * up, __uint_as_float(qf[nt][i] & 0xffff0000u) * up);
          }
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            row_scale[nt][e] = F16 ? p.scale_log2 : p.scale_log2 * __shfl_sync(0xffffffffu, unit, (2 * qd + e) * 4);
            const int mine = nt * 8 + 2 * qd + e;
            lim[nt][e] = p.causal && mine < part.rows ? min(part.pos0 + (part.row0 + mine) / p.G + 1, part.kv) : part.kv;
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
      }
      ok = wait_all(full(st), (r / stages) & 1, abort_flag, p.status, 1);
      const int rank = x - part.begin;                             // place of the page in the part
      if (ok && rank < part.count) {
        const unsigned char* page = ring + st * B::BYTES;
        const int first = at.j * PAGE;                             // key number of the page's first key
        float s[4][NT][4];
#pragma unroll
        for (int mt = 0; mt < 4; ++mt) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[mt][nt][i] = 0.f;
          uint32_t w[2][WORDS], bytes[2];
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const int key = mt * 16 + u * 8 + key_of;
            if (D == 128) {
              const uint4 y = *reinterpret_cast<const uint4*>(page + B::K + key * B::ROW + qd * 16);
              w[u][0] = y.x, w[u][1] = y.y, w[u][WORDS - 2] = y.z, w[u][WORDS - 1] = y.w;
              bytes[u] = *reinterpret_cast<const uint16_t*>(page + B::KS + key * B::SCALES + qd * 2);
            } else {
              const uint2 y = *reinterpret_cast<const uint2*>(page + B::K + key * B::ROW + qd * 8);
              w[u][0] = y.x, w[u][1] = y.y;
              bytes[u] = page[B::KS + key * B::SCALES + qd];
            }
          }
#pragma unroll
          for (int g = 0; g < WORDS / 2; ++g) {                    // sixteen columns with one scale
            const Steps4 a(__byte_perm(bytes[0], 0, g ? 0x4141 : 0x4040)), b(__byte_perm(bytes[1], 0, g ? 0x4141 : 0x4040));
#pragma unroll
            for (int i = 2 * g; i < 2 * g + 2; ++i) {
              uint32_t ka[4], kb[4];
              values4(w[0][i], a, ka);
              values4(w[1][i], b, kb);
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                mma_half(s[mt][nt], ka[0], kb[0], ka[1], kb[1], qf[nt][4 * i], qf[nt][4 * i + 1]);
                mma_half(s[mt][nt], ka[2], kb[2], ka[3], kb[3], qf[nt][4 * i + 2], qf[nt][4 * i + 3]);
              }
            }
          }
        }
        if (first + PAGE > least) {                                // some row may not see some of the keys (uniform)
#pragma unroll
          for (int mt = 0; mt < 4; ++mt)
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
            for (int mt = 1; mt < 4; ++mt) t = fmax3(t, s[mt][nt][e], s[mt][nt][2 + e]);
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
              const float m_new = fmaxf(m_ref[nt][e], t), f = exp2f(m_ref[nt][e] - m_new);
              m_ref[nt][e] = m_new;
              l_sum[nt][e] *= f;
#pragma unroll
              for (int j = 0; j < MTILES; ++j) {
                o[j][nt][e] *= f;
                o[j][nt][2 + e] *= f;
              }
            }
        }
        // probabilities: their sums take them as 32-bit numbers, the product with V rounded to fp16, as the matrix unit wants its operands
        uint32_t pf[4][NT][2];
#pragma unroll
        for (int mt = 0; mt < 4; ++mt)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              const float e0 = ex2_approx(fmaf(s[mt][nt][2 * u], row_scale[nt][0], -m_ref[nt][0]));
              const float e1 = ex2_approx(fmaf(s[mt][nt][2 * u + 1], row_scale[nt][1], -m_ref[nt][1]));
              l_sum[nt][0] += e0;
              l_sum[nt][1] += e1;
              pf[mt][nt][u] = transpose8(pack_half(e0, e1));
            }
        const int there = part.kv - first;                         // keys of the page that exist
#pragma unroll
        for (int mt = 0; mt < 4; ++mt) {
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
            if (there < PAGE && key >= there) bytes[u] = 0;        // what lies behind the last key may be anything
          }
          const Steps4 a(bytes[0] | bytes[1] << 16), b(bytes[2] | bytes[3] << 16);
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
        // ---------------------------------------------------------------- the last of this warp's pages of the part
        if (rank + WARPS >= part.count) {
          __syncwarp();                                            // everybody has read the page
          float* rows = reinterpret_cast<float*>(ring + st * B::BYTES);
          float2* stats = reinterpret_cast<float2*>(rows + ROWS * D);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int row = nt * 8 + 2 * qd + e;
              float l = l_sum[nt][e];
              l += __shfl_xor_sync(0xffffffffu, l, 4);
              l += __shfl_xor_sync(0xffffffffu, l, 8);
              l += __shfl_xor_sync(0xffffffffu, l, 16);
              if (gr == 0) stats[row] = make_float2(m_ref[nt][e], l);
              // columns gr * D / 8 ..: words of four, their places changed so that the four lanes of a row group do not meet in a bank
#pragma unroll
              for (int c = 0; c < D / 32; ++c)
                reinterpret_cast<float4*>(rows + row * D)[(gr * (D / 32) + c) ^ qd] =
                    make_float4(o[2 * c][nt][e], o[2 * c][nt][2 + e], o[2 * c + 1][nt][e], o[2 * c + 1][nt][2 + e]);
            }
          const int involved = min(part.count, WARPS);
          uint32_t last = 0;
          __syncwarp();
          held |= 1u << st;
          if (lane == 0) {
            __threadfence_block();
            uint32_t* ctr = counters + at.unit % OPEN;
            last = atomicAdd(ctr, 1u) == (uint32_t)involved - 1;
            if (last) *reinterpret_cast<volatile uint32_t*>(ctr) = 0;
            __threadfence_block();
          }
          last = __shfl_sync(0xffffffffu, last, 0);
          if (last) {
            // where warp w's rows are: the stage of its last page of the part
            const int part_end = part.begin + part.count;
            auto stage_of = [&](int i) {                           // i: in the order of the pages
              const int w = (part.begin + i) % WARPS, last_page = part_end - 1 - (part_end - 1 - w) % WARPS;
              return make_int2(w, last_page / WARPS % stages);
            };
            const bool cut = part.j0 > 0 || !part.ends;
            float* slot = p.partials + (2 * (int64_t)blockIdx.x + (part.j0 > 0 ? 0 : 1)) * slot_floats(ROWS, D);
            constexpr int LANES = D / 4, AT_ONCE = 32 / LANES;     // lanes of a row, rows at once
            const int my = lane % LANES, n_rows = part.rows;
            for (int r0 = 0; r0 < n_rows; r0 += AT_ONCE) {
              const int row = r0 + lane / LANES, col = (my ^ ((row >> 1) & 3)) * 4;
              float2 ml[WARPS];
              float4 c[WARPS];
              float m = NO_MAX, l = 0.f;
#pragma unroll
              for (int i = 0; i < WARPS; ++i) {
                ml[i] = make_float2(NO_MAX, 0.f);
                c[i] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (i >= involved) continue;
                const int2 ws = stage_of(i);
                const float* base = reinterpret_cast<const float*>(smem + (ws.x * stages + ws.y) * B::BYTES);
                ml[i] = reinterpret_cast<const float2*>(base + ROWS * D)[row];
                c[i] = reinterpret_cast<const float4*>(base + row * D)[my];
                m = fmaxf(m, ml[i].x);
              }
              float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
              for (int i = 0; i < WARPS; ++i) {
                if (i >= involved) continue;
                const float f = exp2f(ml[i].x - m);
                l = fmaf(ml[i].y, f, l);
                acc.x = fmaf(c[i].x, f, acc.x);
                acc.y = fmaf(c[i].y, f, acc.y);
                acc.z = fmaf(c[i].z, f, acc.z);
                acc.w = fmaf(c[i].w, f, acc.w);
              }
              if (row >= n_rows) continue;
              if (cut) {
                __stcg(reinterpret_cast<float4*>(slot + row * D + col), acc);
                if (my == 0) __stcg(reinterpret_cast<float2*>(slot + ROWS * D) + row, make_float2(m, l));
              } else {
                const int of = part.row0 + row, tok = part.tok0 + of / p.G, hd = at.head * p.G + of % p.G;
                const float inv = l == 0.f ? 0.f : q4.v_unit / l;
                uint32_t* dst = reinterpret_cast<uint32_t*>(static_cast<__half*>(p.out) + (int64_t)tok * p.o_tok + (int64_t)hd * p.o_head + col);
                *reinterpret_cast<uint2*>(dst) = make_uint2(pack_out<F16>(acc.x * inv, acc.y * inv), pack_out<F16>(acc.z * inv, acc.w * inv));
                if (p.lse && my == 0) p.lse[(int64_t)tok * p.H + hd] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
              }
            }
            if (part.j0 == 0) {
              // the part with the unit's first page says how many there are
              int parts = 0;
              if (!part.ends) {
                const int64_t begin = y0 + part.begin, end = begin + at.s.pages;
                int lo = blockIdx.x + 1, hi = runs.grid - 1;       // the last CTA whose run begins inside
                while (lo < hi) {
                  const int mid = (lo + hi + 1) >> 1;
                  const int64_t y = runs.raw(mid);
                  if (y < end && Runs::snap(y, begin, at.s.pages) < end) lo = mid; else hi = mid - 1;
                }
                parts = lo - (int)blockIdx.x + 1;
              }
              const int of = part.row0 + lane;
              if (lane < part.rows) sp.cuts[(int64_t)(part.tok0 + of / p.G) * p.H + at.head * p.G + of % p.G] = make_int2(blockIdx.x, parts | lane << 16);
            }
            __syncwarp();
            if (lane < involved) {
              const int2 ws = stage_of(lane);
              mbar_arrive(merged(ws.x, ws.y));
            }
            __syncwarp();
          }
        }
      }
      at.advance(WARPS, shapes, p.Hkv, p.n_seq);
    }
    if (!sent) {
      ok = wait_all(merged(warp, next_st), (phase >> next_st) & 1, abort_flag, p.status, 2);
      held &= ~(1u << next_st);
      phase ^= 1u << next_st;
      send();
    }
  }
  if (*abort_flag) {
    // leaving early: every copy under way lands before the CTA exits
    for (int r = max(ahead_round - stages, 0); r < min(ahead_round, rounds); ++r)
      if (r * WARPS + warp < n_run) settle(full(r % stages), (r / stages) & 1);
  }
}

// Adds up the parts of the rows whose units were cut, in page order, a warp per row.
constexpr int MERGE_WARPS = 8;
template <int D, bool F16>
__global__ void __launch_bounds__(MERGE_WARPS * 32) paged4_merge_kernel(const __grid_constant__ Small4Params sp, int rows_of_slot, int n_cta) {
  const PagedParams& p = sp.q.a;
  constexpr int N = D / 32, AHEAD = 8;
  pdl_trigger();
  pdl_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int begin_tok = __ldg(p.q_begin), end_tok = __ldg(p.q_begin + p.n_seq);
  const int64_t pitch = slot_floats(rows_of_slot, D), rows = (int64_t)p.n_tokens * p.H;
  for (int64_t x = (int64_t)blockIdx.x * MERGE_WARPS + warp; x < rows; x += (int64_t)gridDim.x * MERGE_WARPS) {
    const int tok = (int)(x / p.H), hd = (int)(x - (int64_t)tok * p.H);
    const int2 cut = __ldcg(sp.cuts + x);
    const int parts = cut.y & 0xffff, row = cut.y >> 16;
    // (rows that are nobody's have an entry of some call before, or none; no entry leads out of the workspace)
    if (tok < begin_tok || tok >= end_tok || parts < 2 || cut.x < 0 || cut.x > n_cta - parts || (uint32_t)row >= (uint32_t)rows_of_slot) continue;
    auto slot = [&](int i) { return p.partials + (2 * (int64_t)(cut.x + i) + (i == 0)) * pitch; };
    float top = NO_MAX;
    for (int i = lane; i < parts; i += 32) top = fmaxf(top, __ldcg(reinterpret_cast<const float2*>(slot(i) + rows_of_slot * D) + row).x);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    float acc[N], l = 0.f;
#pragma unroll
    for (int k = 0; k < N; ++k) acc[k] = 0.f;
    for (int base = 0; base < parts; base += AHEAD) {
      float c[AHEAD][N];
      float2 ml[AHEAD];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        ml[i] = make_float2(NO_MAX, 0.f);
#pragma unroll
        for (int k = 0; k < N; ++k) c[i][k] = 0.f;
        if (base + i >= parts) continue;
        const float* s = slot(base + i);
        ml[i] = __ldcg(reinterpret_cast<const float2*>(s + rows_of_slot * D) + row);
        if (N == 4) {
          const float4 y = __ldcg(reinterpret_cast<const float4*>(s + row * D) + lane);
          c[i][0] = y.x, c[i][1] = y.y, c[i][N - 2] = y.z, c[i][N - 1] = y.w;
        } else {
          const float2 y = __ldcg(reinterpret_cast<const float2*>(s + row * D) + lane);
          c[i][0] = y.x, c[i][1] = y.y;
        }
      }
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        if (base + i >= parts) continue;
        const float f = exp2f(ml[i].x - top);
        l = fmaf(ml[i].y, f, l);
#pragma unroll
        for (int k = 0; k < N; ++k) acc[k] = fmaf(c[i][k], f, acc[k]);
      }
    }
    const float inv = l == 0.f ? 0.f : sp.q.v_unit / l;
    uint32_t* dst = reinterpret_cast<uint32_t*>(static_cast<__half*>(p.out) + (int64_t)tok * p.o_tok + (int64_t)hd * p.o_head + lane * N);
#pragma unroll
    for (int k = 0; k < N; k += 2) dst[k / 2] = pack_out<F16>(acc[k] * inv, acc[k + 1] * inv);
    if (p.lse && lane == 0) p.lse[(int64_t)tok * p.H + hd] = l == 0.f ? -INFINITY : (top + log2f(l)) * 0.6931471805599453f;
  }
}

uint64_t cut_bytes(int n_tokens, int H) { return ((uint64_t)n_tokens * H * 8 + 255) / 256 * 256; }

template <int D, int NT, bool F16>
cudaError_t launch(const Paged4Params& q, int n_sm, cudaStream_t stream) {
  constexpr int stage = WARPS * Block4<D>::BYTES, room = 226 * 1024 - 2048;
  const int fixed = q.a.n_seq * 16 + 8;                            // requests' pages before, and shapes
  Small4Params sp;
  sp.q = q;
  sp.cuts = reinterpret_cast<int2*>(q.a.partials);
  sp.q.a.partials = q.a.partials + cut_bytes(q.a.n_tokens, q.a.H) / 4;
  // as many pages under way as shared memory holds
  sp.stages = std::max(2, std::min(MAX_STAGES, (room - fixed) / stage));
  auto kernel = paged4_small_kernel<D, NT, F16>;
  // (the kernel's limit is the process's: always the most that any call takes, as another thread may set it between this line and the launch)
  cudaError_t rc = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, room);
  if (rc != cudaSuccess) return rc;
  rc = launch_pdl(kernel, dim3(n_sm), dim3(THREADS), fixed + sp.stages * stage, stream, sp);
  // nothing can have been cut where no unit has more pages
  if (rc != cudaSuccess || q.a.table_pages <= WHOLE) return rc;
  const int64_t rows = (int64_t)q.a.n_tokens * q.a.H, ctas = std::min<int64_t>((rows + MERGE_WARPS - 1) / MERGE_WARPS, 8 * n_sm);
  return launch_pdl(paged4_merge_kernel<D, F16>, dim3((unsigned)ctas), dim3(MERGE_WARPS * 32), 0, stream, sp, 8 * NT, n_sm);
}
template <int D>
cudaError_t launch_typed(const Paged4Params& q, int rows, int n_sm, cudaStream_t stream) {
  if (q.fp16) return rows <= 8 ? launch<D, 1, true>(q, n_sm, stream) : launch<D, 2, true>(q, n_sm, stream);
  return rows <= 8 ? launch<D, 1, false>(q, n_sm, stream) : launch<D, 2, false>(q, n_sm, stream);
}

}  // namespace

uint64_t paged4_small_partial_bytes(int d, int n_sm, int H, int n_tokens) { return cut_bytes(n_tokens, H) + (uint64_t)2 * n_sm * slot_floats(16, d) * 4; }

cudaError_t launch_paged4_small(const Paged4Params& p, int d, const PagedDevice& dev, cudaStream_t stream) {
  const int rows = (int64_t)std::max(1, p.a.max_new) * p.a.G <= 8 ? 8 : 16;
  return d == 128 ? launch_typed<128>(p, rows, dev.n_sm, stream) : launch_typed<64>(p, rows, dev.n_sm, stream);
}

}  // namespace heatkv
