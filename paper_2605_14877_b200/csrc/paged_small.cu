// Attention of few query rows over a paged cache (decode, drafted tokens) and over selected pages, on warp-level MMA.
//
// A row tile is tile_tokens consecutive tokens of a request times the G query heads of one kv head, up to 16 MT rows; its keys come
// page by page.  What bounds it is the reading of K and V, so the work is cut by pages, not by requests: the pages of all (request,
// row tile, kv head) units, one after another, are dealt out in equal runs, one per CTA.  A unit that a run's border cuts leaves
// partial results (unnormalised O, maximum, sum) in the workspace, and the CTA that arrives last adds them up in page order, so the
// result does not depend on which was last.
//
// Warp 4 sends for pages (TMA, K and V of one page per stage, as many stages as shared memory holds); warps 0-3 each take 16 keys of
// every page for all rows, with a running maximum and sum of their own, and meet at the end of a unit.  Rows past a request's last key
// in its last page are whatever the pool holds: their logits are masked and their values replaced by zero.
#include <algorithm>

#include <cuda_fp16.h>

#include "paged_wait.cuh"

namespace heatkv {
namespace {

using namespace tc;

constexpr int SM_WARPS = 4;
constexpr int SM_THREADS = (SM_WARPS + 1) * 32;
constexpr int MAX_STAGES = 12;
constexpr float MOVE = 8.f;                    // a reference moves when a maximum passes it by more than 2^MOVE (P fits fp16)

struct SmallParams {
  PagedParams a;
  int32_t stages;
};
struct SmallMaps {
  CUtensorMap k, v;
};

template <int D, int MT>
struct SmallLayout {
  static constexpr int ROWS = 16 * MT;
  static constexpr uint32_t TILE = PAGE * D * 2;                 // K or V of one page
  static constexpr int PITCH = D + 4;                            // floats of a row in the meeting area
  static constexpr uint32_t MEET = SM_WARPS * ROWS * PITCH * 4;
  static constexpr uint32_t ML = SM_WARPS * ROWS * 2 * 4;
  static constexpr int SLOT_FLOATS = ROWS * D + 2 * ROWS;        // one partial result
};

// c += a x b for one 16 x 8 x 16 product of bf16 or fp16
template <bool F16>
__device__ __forceinline__ void mma16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if (F16)
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    mma_bf16(d, a, b0, b1);
}
template <bool F16>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
  if (F16) {
    __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&v);
  }
  return pack_bf16(lo, hi);
}

// One CTA's share of a unit.
struct Run {
  int seq, tok0, rows, head, tile0, tile1, tiles, kv, q_len, pos0;   // pos0: position of the tile's first token
  int64_t begin;                               // the unit's first page among all
};

// The equal runs of all units' pages, walked by every role on its own.
template <bool SPARSE>
struct Walk {
  const PagedParams& p;
  const int64_t* prefix;                       // dense: [n_seq + 1] pages before the request
  int64_t x, end, total;
  int grid;
  __device__ Walk(const PagedParams& p_, const int64_t* prefix_, int64_t total_) : p(p_), prefix(prefix_), total(total_) {
    grid = (int)min((int64_t)gridDim.x, total);    // every run holds a page: all CTAs between a unit's first and last have a part of it
    x = (int)blockIdx.x < grid ? bound(blockIdx.x) : total;
    end = (int)blockIdx.x < grid ? bound(blockIdx.x + 1) : total;
  }
  __device__ int64_t bound(int c) const { return total * c / grid; }
  // the CTA whose run holds page y
  __device__ int owner(int64_t y) const {
    int c = (int)(y * grid / total);
    while (c + 1 < grid && bound(c + 1) <= y) ++c;
    while (c > 0 && bound(c) > y) --c;
    return c;
  }
  __device__ bool next(Run& r) {
    if (x >= end) return false;
    if (SPARSE) {
      const int64_t unit = x / p.n_sel;
      r.begin = unit * p.n_sel;
      r.tiles = p.n_sel;
      r.head = (int)(unit % p.Hkv);
      r.tok0 = (int)(unit / p.Hkv);
      int lo = 0, hi = p.n_seq - 1;
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (p.q_begin[mid] <= r.tok0) lo = mid; else hi = mid - 1;
      }
      r.seq = lo;
      const int b = p.q_begin[lo], e = p.q_begin[lo + 1];
      r.kv = p.kv_len[lo];
      r.q_len = e - b;
      r.pos0 = r.tok0 < e ? r.kv - e + r.tok0 : -1;
      r.rows = p.G;
    } else {
      int lo = 0, hi = p.n_seq - 1;            // last request with prefix <= x (those without pages have none to themselves)
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (prefix[mid] <= x) lo = mid; else hi = mid - 1;
      }
      r.seq = lo;
      r.kv = min(max(p.kv_len[lo], 0), p.table_pages * PAGE);
      r.tiles = (r.kv + PAGE - 1) / PAGE;
      const int b = max(p.q_begin[lo], 0), e = min(p.q_begin[lo + 1], p.n_tokens);
      r.q_len = e - b;
      const int64_t local = x - prefix[lo];
      const int64_t unit = local / r.tiles;
      r.begin = prefix[lo] + unit * r.tiles;
      r.head = (int)(unit % p.Hkv);
      const int first = (int)(unit / p.Hkv) * p.tile_tokens;
      r.tok0 = b + first;
      r.rows = min(p.tile_tokens, r.q_len - first) * p.G;
      r.pos0 = r.kv - r.q_len + first;
    }
    r.tile0 = (int)(x - r.begin);
    r.tile1 = (int)min((int64_t)r.tiles, end - r.begin);
    x = r.begin + r.tile1;
    return true;
  }
};

__device__ __forceinline__ void meet_sync() { asm volatile("bar.sync 1, %0;" ::"n"(SM_WARPS * 32) : "memory"); }

template <int D, int MT, bool F16, bool SPARSE>
__global__ void __launch_bounds__(SM_THREADS, 1) paged_small_kernel(const __grid_constant__ SmallParams sp, const __grid_constant__ SmallMaps maps) {
  using L = SmallLayout<D, MT>;
  constexpr int NCH = D / 64, ROWS = L::ROWS;
  const PagedParams& p = sp.a;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t sbase = (raw + 1023u) & ~1023u;
  unsigned char* sgen = smem_raw + (sbase - raw);
  const int stages = sp.stages;
  const uint32_t meet_off = stages * 2 * L::TILE, ml_off = meet_off + L::MEET, pre_off = ml_off + L::ML;
  float* meet = reinterpret_cast<float*>(sgen + meet_off);
  float2* ml = reinterpret_cast<float2*>(sgen + ml_off);
  int64_t* prefix = reinterpret_cast<int64_t*>(sgen + pre_off);
  __shared__ __align__(8) uint64_t bars[2 * MAX_STAGES];
  __shared__ uint32_t abort_word, last_word, leave_word;
  __shared__ int64_t warp_sums[SM_WARPS + 1];
  volatile uint32_t* abort_flag = &abort_word;
  const uint32_t bar0 = smem_u32(bars);
  auto full = [&](int s) { return bar0 + s * 16; };
  auto empty = [&](int s) { return bar0 + s * 16 + 8; };
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;

  pdl_trigger();
  pdl_wait();
  if (threadIdx.x == 0) {
    *abort_flag = *reinterpret_cast<volatile uint32_t*>(p.status) != 0;
    for (int s = 0; s < stages; ++s) {
      mbar_init(full(s), 1);
      mbar_init(empty(s), SM_WARPS);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  int64_t total;
  if (SPARSE) {
    total = (int64_t)p.n_tokens * p.Hkv * p.n_sel;
  } else {
    // pages of every request, summed up; a request without keys has none, and its rows get their zeros here
    const int per = (p.n_seq + SM_THREADS - 1) / SM_THREADS, i0 = min((int)threadIdx.x * per, p.n_seq), i1 = min(i0 + per, p.n_seq);
    int64_t sum = 0;
    for (int i = i0; i < i1; ++i) {
      const int b = max(p.q_begin[i], 0), e = min(p.q_begin[i + 1], p.n_tokens), n = max(e - b, 0);
      const int kv = min(max(p.kv_len[i], 0), p.table_pages * PAGE);
      const int64_t w = (int64_t)((kv + PAGE - 1) / PAGE) * ((n + p.tile_tokens - 1) / p.tile_tokens) * p.Hkv;
      prefix[i] = w;
      sum += w;
    }
    int64_t inc = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t up = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += up;
    }
    if (lane == 31) warp_sums[warp] = inc;
    __syncthreads();
    int64_t at = inc - sum;
    total = 0;
    for (int w = 0; w <= SM_WARPS; ++w) {
      if (w < warp) at += warp_sums[w];
      total += warp_sums[w];
    }
    for (int i = i0; i < i1; ++i) {
      const int64_t w = prefix[i];
      prefix[i] = at;
      at += w;
    }
    if (threadIdx.x == 0) prefix[p.n_seq] = total;
  }
  __syncthreads();
  if (!SPARSE) {
    for (int i = blockIdx.x; i < p.n_seq; i += gridDim.x) {
      if (prefix[i + 1] != prefix[i]) continue;
      const int b = max(p.q_begin[i], 0), e = min(p.q_begin[i + 1], p.n_tokens);
      const int64_t n = (int64_t)max(e - b, 0) * p.H;
      for (int64_t j = threadIdx.x; j < n * D; j += SM_THREADS) {
        const int64_t t = b + j / ((int64_t)p.H * D), hd = j / D % p.H;
        static_cast<uint16_t*>(p.out)[t * p.o_tok + hd * p.o_head + j % D] = 0;
      }
      if (p.lse)
        for (int64_t j = threadIdx.x; j < n; j += SM_THREADS) p.lse[b * (int64_t)p.H + j] = -INFINITY;
    }
  }
  if (total == 0) return;

  if (warp == SM_WARPS) {
    // ------------------------------------------------------------------ producer
    Walk<SPARSE> walk(p, prefix, total);
    Run r;
    const bool leader = elect_one();
    uint32_t g = 0;
    bool ok = true;
    while (ok && walk.next(r)) {
      int pages = 0;
      for (int j = r.tile0; j < r.tile1; ++j, ++g) {
        const int in = (j - r.tile0) & 31;
        if (in == 0) {                                             // 32 page numbers at a time, one per lane
          const int jj = j + lane;
          pages = -1;
          if (jj < r.tile1) {
            int lp = jj;
            if (SPARSE) {
              lp = p.sel[((int64_t)r.tok0 * p.Hkv + r.head) * p.n_sel + jj];
              if (lp > r.pos0 / PAGE || r.pos0 < 0) lp = -1;       // nothing there that the query may see
            }
            if (lp >= 0 && lp < p.table_pages) pages = p.block_table[r.seq * p.table_stride + lp];
            if (pages >= p.n_pages) pages = -1;                    // (a box outside of the map arrives as zeros)
            if (pages < 0) pages = -1;
          }
        }
        const int page = __shfl_sync(0xffffffffu, pages, in);
        const uint32_t st = g % stages, use = g / stages;
        if (use > 0) ok = wait_all(empty(st), (use - 1) & 1, abort_flag, p.status, 1);
        if (!ok) break;
        if (leader) {
          mbar_expect_tx(full(st), 2 * L::TILE);
          const uint32_t dst = sbase + st * 2 * L::TILE;
#pragma unroll
          for (int ch = 0; ch < NCH; ++ch) {
            tma_load_4d(dst + ch * PAGE * 128, &maps.k, ch * 64, 0, r.head, page, full(st));
            tma_load_4d(dst + L::TILE + ch * PAGE * 128, &maps.v, ch * 64, 0, r.head, page, full(st));
          }
        }
        __syncwarp();
      }
    }
    if (!ok || *abort_flag) {
      // leaving early: every copy under way lands before the CTA exits
      for (uint32_t s = 0; s < (uint32_t)stages; ++s) {
        if (g <= s) break;
        const uint32_t uses = (g - s + stages - 1) / stages;       // copies into this stage so far
        settle(full(s), (uses - 1) & 1);
      }
    }
    return;
  }

  // ------------------------------------------------------------------ products and softmax
  const int gr = lane >> 2, qd = lane & 3;                         // row group and column pair of the fragments
  const int key0 = warp * 16;
  // ldmatrix rows of this lane: K (keys x dims as they lie), V (transposed)
  const int k_row = key0 + (lane & 7) + ((lane >> 4) << 3), k_ch = (lane >> 3) & 1;
  const int v_row = key0 + (lane & 7) + (((lane >> 3) & 1) << 3), v_ch = lane >> 4;
  Walk<SPARSE> walk(p, prefix, total);
  Run r;
  uint32_t g = 0;
  bool ok = true;
  while (walk.next(r)) {
    // the unit's query rows as A fragments; rows past the last are zero
    uint32_t qa[MT][D / 16][4];
    int lim[MT][2];                                                // keys that a row may see
    int least = INT_MAX;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int row = m * 16 + i * 8 + gr;
        const bool valid = row < r.rows;
        const int tok = row / p.G, hd = r.head * p.G + row - tok * p.G;
        const uint32_t* src = reinterpret_cast<const uint32_t*>(static_cast<const __nv_bfloat16*>(p.q) + (int64_t)(r.tok0 + tok) * p.q_tok + (int64_t)hd * p.q_head);
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
          qa[m][ks][i] = valid ? __ldg(src + ks * 8 + qd) : 0u;
          qa[m][ks][2 + i] = valid ? __ldg(src + ks * 8 + qd + 4) : 0u;
        }
        lim[m][i] = p.causal ? min(r.pos0 + tok + 1, r.kv) : r.kv;
        if (SPARSE && r.pos0 < 0) lim[m][i] = 0;
        if (valid) least = min(least, lim[m][i]);
      }
    least = __reduce_min_sync(0xffffffffu, least);
    float o[MT][D / 8][4], m_ref[MT][2], l_sum[MT][2];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
#pragma unroll
      for (int n = 0; n < D / 8; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[m][n][i] = 0.f;
      m_ref[m][0] = m_ref[m][1] = NO_MAX;
      l_sum[m][0] = l_sum[m][1] = 0.f;
    }
    int places = 0;
    for (int j = r.tile0; j < r.tile1; ++j, ++g) {
      int lp = j;                                                  // logical page
      if (SPARSE) {
        const int in = (j - r.tile0) & 31;
        if (in == 0) places = j + lane < r.tile1 ? p.sel[((int64_t)r.tok0 * p.Hkv + r.head) * p.n_sel + j + lane] : -1;
        lp = __shfl_sync(0xffffffffu, places, in);
        if (lp < 0 || lp >= p.table_pages) lp = 1 << 24;           // past every limit
      }
      const uint32_t st = g % stages, use = g / stages;
      ok = wait_all(full(st), use & 1, abort_flag, p.status, 2);
      if (!ok) break;
      const uint32_t kt = sbase + st * 2 * L::TILE, vt = kt + L::TILE;
      const int first = lp * PAGE + key0;                          // key number of this warp's first key
      float s[MT][2][4];
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[m][n][i] = 0.f;
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) {
        uint32_t b[4];
        const int c = (ks * 2 + k_ch) & 7;
        ldmatrix_x4(b, kt + (ks >> 2) * PAGE * 128 + k_row * 128 + ((c ^ (k_row & 7)) << 4));
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          mma16<F16>(s[m][0], qa[m][ks], b[0], b[1]);
          mma16<F16>(s[m][1], qa[m][ks], b[2], b[3]);
        }
      }
      const bool edge = first + 16 > least;                        // some row may not see some of the keys (uniform)
      if (edge) {
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (first + n * 8 + qd * 2 + (i & 1) >= lim[m][i >> 1]) s[m][n][i] = -INFINITY;
      }
      uint32_t pa[MT][4];
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        bool grow = false;
        float top[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          top[i] = fmaxf(fmaxf(s[m][0][2 * i], s[m][0][2 * i + 1]), fmaxf(s[m][1][2 * i], s[m][1][2 * i + 1])) * p.scale_log2;
          top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 1));
          top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 2));
          grow |= top[i] > m_ref[m][i] + MOVE;
        }
        if (__any_sync(0xffffffffu, grow)) {
          float f[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float m_new = fmaxf(m_ref[m][i], top[i]);
            f[i] = exp2f(m_ref[m][i] - m_new);
            m_ref[m][i] = m_new;
            l_sum[m][i] *= f[i];
          }
#pragma unroll
          for (int n = 0; n < D / 8; ++n) {
            o[m][n][0] *= f[0];
            o[m][n][1] *= f[0];
            o[m][n][2] *= f[1];
            o[m][n][3] *= f[1];
          }
        }
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float e0 = ex2_approx(fmaf(s[m][n][2 * i], p.scale_log2, -m_ref[m][i]));
            const float e1 = ex2_approx(fmaf(s[m][n][2 * i + 1], p.scale_log2, -m_ref[m][i]));
            l_sum[m][i] += e0 + e1;
            pa[m][n * 2 + i] = pack16<F16>(e0, e1);
          }
      }
      // values of keys that the request does not have are whatever the pool holds
      uint32_t keep0 = 0xffffffffu, keep1 = 0xffffffffu;
      if (first + 16 > r.kv) {
        const int a = r.kv - first - qd * 2;                       // keys from this lane's first that exist
        keep0 = a >= 2 ? 0xffffffffu : a == 1 ? 0xffffu : 0u;
        keep1 = a >= 10 ? 0xffffffffu : a == 9 ? 0xffffu : 0u;
      }
#pragma unroll
      for (int n = 0; n < D / 16; ++n) {
        uint32_t b[4];
        const int c = (n * 2 + v_ch) & 7;
        ldmatrix_x4_trans(b, vt + (n >> 2) * PAGE * 128 + v_row * 128 + ((c ^ (v_row & 7)) << 4));
        b[0] &= keep0;
        b[1] &= keep1;
        b[2] &= keep0;
        b[3] &= keep1;
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          mma16<F16>(o[m][2 * n], pa[m], b[0], b[1]);
          mma16<F16>(o[m][2 * n + 1], pa[m], b[2], b[3]);
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(empty(st));
    }
    // ------------------------------------------------------------------ the four warps meet
    // (also after a wait that ran out, so that none waits for one that left; one thread's look at the flag is everybody's)
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float l = l_sum[m][i];
        l += __shfl_xor_sync(0xffffffffu, l, 1);
        l += __shfl_xor_sync(0xffffffffu, l, 2);
        const int row = m * 16 + i * 8 + gr;
        if (qd == 0) ml[warp * ROWS + row] = make_float2(m_ref[m][i], l);
        float* dst = meet + (warp * ROWS + row) * L::PITCH + qd * 2;
#pragma unroll
        for (int n = 0; n < D / 8; ++n) *reinterpret_cast<float2*>(dst + n * 8) = make_float2(o[m][n][2 * i], o[m][n][2 * i + 1]);
      }
    if (threadIdx.x == 0) leave_word = *abort_flag;
    meet_sync();
    if (leave_word) break;
    const bool whole = r.tile0 == 0 && r.tile1 == r.tiles;
    const int c0 = whole ? 0 : walk.owner(r.begin);
    // two slots a CTA: its run's first unit, begun by another CTA, and its last one, begun here
    float* slot = p.partials + (int64_t)(2 * blockIdx.x + (r.tile0 == 0 ? 1 : 0)) * L::SLOT_FLOATS;
    constexpr int QUADS = D / 4;
    for (int i = threadIdx.x; i < r.rows * QUADS; i += SM_WARPS * 32) {
      const int row = i / QUADS, cq = i % QUADS;
      float2 w[SM_WARPS];
      float m_all = NO_MAX;
#pragma unroll
      for (int x = 0; x < SM_WARPS; ++x) {
        w[x] = ml[x * ROWS + row];
        m_all = fmaxf(m_all, w[x].x);
      }
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
      float l = 0.f;
#pragma unroll
      for (int x = 0; x < SM_WARPS; ++x) {
        const float f = exp2f(w[x].x - m_all);
        const float4 v = *reinterpret_cast<const float4*>(meet + (x * ROWS + row) * L::PITCH + cq * 4);
        l = fmaf(w[x].y, f, l);
        acc.x = fmaf(v.x, f, acc.x);
        acc.y = fmaf(v.y, f, acc.y);
        acc.z = fmaf(v.z, f, acc.z);
        acc.w = fmaf(v.w, f, acc.w);
      }
      if (whole) {
        const int tok = r.tok0 + row / p.G, hd = r.head * p.G + row % p.G;
        const float inv = l > 0.f ? 1.f / l : 0.f;
        uint2 v;
        v.x = pack16<F16>(acc.x * inv, acc.y * inv);
        v.y = pack16<F16>(acc.z * inv, acc.w * inv);
        *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.out) + (int64_t)tok * p.o_tok + (int64_t)hd * p.o_head + cq * 4) = v;
        if (p.lse && cq == 0) p.lse[(int64_t)tok * p.H + hd] = l > 0.f ? (m_all + log2f(l)) * 0.6931471805599453f : -INFINITY;
      } else {
        __stcg(reinterpret_cast<float4*>(slot) + row * QUADS + cq, acc);
        if (cq == 0) __stcg(reinterpret_cast<float2*>(slot + ROWS * D) + row, make_float2(m_all, l));
      }
    }
    if (!whole) {
      const int c1 = walk.owner(r.begin + r.tiles - 1);
      __threadfence();
      meet_sync();
      if (threadIdx.x == 0) {
        const uint32_t old = atomicAdd(p.counters + c0, 1u);
        last_word = old == (uint32_t)(c1 - c0);
        if (last_word) p.counters[c0] = 0;                         // ready for the next launch
      }
      meet_sync();
      if (last_word) {
        __threadfence();
        for (int i = threadIdx.x; i < r.rows * QUADS; i += SM_WARPS * 32) {
          const int row = i / QUADS, cq = i % QUADS;
          auto part = [&](int c) { return p.partials + (int64_t)(2 * c + (c == c0 ? 1 : 0)) * L::SLOT_FLOATS; };
          float m_all = NO_MAX;
          for (int c = c0; c <= c1; ++c) m_all = fmaxf(m_all, __ldcg(reinterpret_cast<const float2*>(part(c) + ROWS * D) + row).x);
          float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
          float l = 0.f;
#pragma unroll 4
          for (int c = c0; c <= c1; ++c) {
            const float2 w = __ldcg(reinterpret_cast<const float2*>(part(c) + ROWS * D) + row);
            const float4 v = __ldcg(reinterpret_cast<const float4*>(part(c)) + row * QUADS + cq);
            const float f = exp2f(w.x - m_all);
            l = fmaf(w.y, f, l);
            acc.x = fmaf(v.x, f, acc.x);
            acc.y = fmaf(v.y, f, acc.y);
            acc.z = fmaf(v.z, f, acc.z);
            acc.w = fmaf(v.w, f, acc.w);
          }
          const int tok = r.tok0 + row / p.G, hd = r.head * p.G + row % p.G;
          const float inv = l > 0.f ? 1.f / l : 0.f;
          uint2 v;
          v.x = pack16<F16>(acc.x * inv, acc.y * inv);
          v.y = pack16<F16>(acc.z * inv, acc.w * inv);
          *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.out) + (int64_t)tok * p.o_tok + (int64_t)hd * p.o_head + cq * 4) = v;
          if (p.lse && cq == 0) p.lse[(int64_t)tok * p.H + hd] = l > 0.f ? (m_all + log2f(l)) * 0.6931471805599453f : -INFINITY;
        }
      }
    }
    meet_sync();                                                   // the meeting area is free again
  }
}

template <int D, int MT, bool F16, bool SPARSE>
cudaError_t launch(const PagedParams& p, const SmallMaps& maps, int grid, cudaStream_t stream) {
  using L = SmallLayout<D, MT>;
  const uint32_t fixed = L::MEET + L::ML + (SPARSE ? 0 : (p.n_seq + 1) * 8) + 1024;
  SmallParams sp;
  sp.a = p;
  sp.stages = std::min<int>(MAX_STAGES, (226 * 1024 - (int)fixed) / (int)(2 * L::TILE));
  if (sp.stages < 2) return cudaErrorInvalidValue;
  const int smem = (int)fixed + sp.stages * 2 * (int)L::TILE;
  auto kernel = paged_small_kernel<D, MT, F16, SPARSE>;
  const cudaError_t rc = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (rc != cudaSuccess) return rc;
  return launch_pdl(kernel, dim3(grid), dim3(SM_THREADS), smem, stream, sp, maps);
}
template <int D, int MT>
cudaError_t launch_typed(const PagedParams& p, bool fp16, const SmallMaps& maps, int grid, cudaStream_t stream) {
  if (p.sel) return fp16 ? launch<D, MT, true, true>(p, maps, grid, stream) : launch<D, MT, false, true>(p, maps, grid, stream);
  return fp16 ? launch<D, MT, true, false>(p, maps, grid, stream) : launch<D, MT, false, false>(p, maps, grid, stream);
}

}  // namespace

uint64_t paged_small_partial_bytes(int d, int n_sm) {
  const uint64_t floats = d == 128 ? SmallLayout<128, 2>::SLOT_FLOATS : SmallLayout<64, 2>::SLOT_FLOATS;
  return 2 * (uint64_t)n_sm * floats * 4;
}

cudaError_t launch_paged_small(const PagedParams& p, const heatkv_paged_pool& pool, const PagedDevice& dev, cudaStream_t stream) {
  SmallMaps maps;
  if (!paged_encode_pool(dev, &maps.k, pool.k, pool) || !paged_encode_pool(dev, &maps.v, pool.v, pool)) return cudaErrorInvalidValue;
  const bool fp16 = pool.dtype == HEATKV_DTYPE_FP16;
  PagedParams q = p;
  const int tokens = p.sel ? 1 : std::max(1, p.max_new);
  const bool one = tokens * p.G <= 16;                             // rows of a tile: 16, or 32
  q.tile_tokens = p.sel ? 1 : (one ? 16 : 32) / p.G;
  if (pool.d == 128) return one ? launch_typed<128, 1>(q, fp16, maps, dev.n_sm, stream) : launch_typed<128, 2>(q, fp16, maps, dev.n_sm, stream);
  return one ? launch_typed<64, 1>(q, fp16, maps, dev.n_sm, stream) : launch_typed<64, 2>(q, fp16, maps, dev.n_sm, stream);
}

}  // namespace heatkv
