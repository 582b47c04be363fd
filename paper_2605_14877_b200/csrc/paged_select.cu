// Page selection: for every query token and kv head the pages whose mean key scores highest, plus the first and the last ones.
//
// Query summary: the sum of the group's heads in 32 bits, in head order, held as 8-bit codes (largest magnitude / 127; the query's own
// scale is common to its scores and drops out).  Score of a page: the whole-number dot product of the two codes, times the page's
// scale.  |dot| <= 128 * 127^2 < 2^24 is exact in 32 bits whatever the order of its sums, so the choice is the same for every kernel
// and launch shape; equal scores go to the lower page.
//
// Choosing: the pages fall into groups (page number modulo 32, or more of them), and the want-th largest of the groups' maxima is a score
// that at least `want` pages reach and, where large scores are spread over the groups, few more.  Those few are listed and ranked
// against each other.  Where the list would not hold them (many equal or badly spread scores, more pages wanted than groups), the want-th
// largest score is found bit by bit instead: 32 counts of all scores, each behind the last (2047 pages, 13 to 32 wanted: 11 us of 23).
// Scores are compared as unsigned words in the same order.
#include <algorithm>

#include <cuda_fp16.h>

#include "device_common.cuh"
#include "paged.h"

namespace heatkv {
namespace {

constexpr int ROWS_THREADS = 256, ROWS_WARPS = ROWS_THREADS / 32;
constexpr int LIST = 256, ROW_LIST = 128;                     // pages that are ranked: of one token by a CTA, by a warp
constexpr int SEL_ROWS = 16;                                  // tokens of a CTA where requests have many (sixteen_at_once)
constexpr int SEL_ROWS_PAGES = 3200;                          // pages whose scores fit shared memory for all of them

__device__ __forceinline__ float load_half(const void* p, int64_t i, bool fp16) {
  return fp16 ? __half2float(static_cast<const __half*>(p)[i]) : __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
}
// ascending order of floats as unsigned words (-0 counts as +0)
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ int8_t to_code(float x, float scale) {
  return (int8_t)(scale > 0.f ? fminf(fmaxf(rintf(__fdiv_rn(x, scale)), -127.f), 127.f) : 0.f);
}
__device__ __forceinline__ int request_of(const SelectParams& p, int t) {      // last request whose first token is not past t
  int lo = 0, hi = p.n_seq - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (p.q_begin[mid] <= t) lo = mid; else hi = mid - 1;
  }
  return lo;
}
// Which pages of a token's context are always taken, [0, first) and [last, pages), and how many of the others.
struct Range {
  int pages, first, last, want;
  __device__ Range(const SelectParams& p, int pos) {
    pages = pos < 0 ? 0 : min(pos / PAGE + 1, p.table_pages);
    first = min(p.sink, pages);
    last = max(first, pages - p.local);
    want = min(p.n_sel - first - (pages - last), last - first);
  }
};

// ------------------------------------------------------------------------------------------------ one token, one CTA
// What bounds it: the chain of loads before and counts behind the scores, and for few tokens the scores of a whole context by one SM.
// So a cluster's CTAs share a token's pages while that leaves no SM without work, and write the scores into the first one's shared memory,
// which chooses (one token, 8 kv heads, 2047 pages: 9.9 us with 8 CTAs, 14.1 with one; 32 kv heads, 625 pages: 12.3 with 4, 13.1 with one; 3100
// pages, one head: 10.7 and 18.1).  32 requests of 140 to 620 pages, 16 kv heads, a CTA a token: 12.5 us, 14 MB of codes at 1.1 TB/s.
__device__ __forceinline__ int cluster_rank() {
  int r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ int cluster_ctas() {
  int r;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

template <int D, int THREADS, bool CLUSTER>
__global__ void __launch_bounds__(THREADS, THREADS == 256 ? 4 : 1) select_kernel(const __grid_constant__ SelectParams p) {
  constexpr int WARPS = THREADS / 32;
  extern __shared__ __align__(16) uint32_t keys[];            // [pages, up to a multiple of 4] scores; 0: not to be chosen
  __shared__ __align__(16) int8_t code[D];
  __shared__ float tops[WARPS];
  __shared__ int counts[2][WARPS];
  __shared__ int warp_cnt[WARPS][2];
  __shared__ uint32_t tops_of[WARPS][32], list_key[LIST];
  __shared__ int list_page[LIST], n_list;
  __shared__ uint32_t reach;
  pdl_trigger();
  const int rank = CLUSTER ? cluster_rank() : 0, ctas = CLUSTER ? cluster_ctas() : 1, unit = blockIdx.x / ctas;
  if (CLUSTER) cluster_arrive();                              // this CTA's shared memory is there
  pdl_wait();
  const int t = unit / p.Hkv, h = unit % p.Hkv, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  int32_t* sel = p.sel + ((int64_t)t * p.Hkv + h) * p.n_sel;
  // summed query -> codes
  float q = 0.f;
  if (tid < D) {
    const int64_t at = t * p.q_tok + (int64_t)h * p.G * p.q_head + tid;
    q = load_half(p.q, at, p.fp16);
#pragma unroll 4
    for (int g = 1; g < p.G; ++g) q += load_half(p.q, at + g * p.q_head, p.fp16);
  }
  const int seq = request_of(p, t);
  const int b = p.q_begin[seq], e = p.q_begin[seq + 1], kv = p.kv_len[seq];
  const Range r(p, t >= b && t < e ? kv - e + t : -1);                        // its own key is the last that a token sees
  const int32_t* table = p.block_table + seq * p.table_stride;
  // scores: D / 16 lanes a page, 16 bytes of its codes each; the CTA's pages are the j-th STEP of every `stride`
  constexpr int LANES = D / 16, STEP = THREADS / LANES, UNROLL = 8;
  const int stride = STEP * ctas, own = r.first + rank * STEP, rounds = (r.last - own + stride - 1) / stride;
#pragma unroll 4
  for (int j = tid; j < rounds * STEP; j += THREADS) {        // the pages' numbers first, where their scores will be
    const int i = own + j / STEP * stride + j % STEP;
    if (i < r.last) {
      const int page = table[i];
      keys[i] = (uint32_t)(page >= 0 && page < p.n_pages ? page : -1);
    }
  }
  float top = fabsf(q);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  if (lane == 0) tops[warp] = top;
  __syncthreads();
  if (tid < D) code[tid] = to_code(q, fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])) * (1.f / 127.f));
  __syncthreads();
  if (CLUSTER) cluster_wait();
  if (rank == 0) {
    const int taken = r.first + r.want + (r.pages - r.last);
    for (int i = taken + tid; i < p.n_sel; i += THREADS) sel[i] = -1;
    for (int i = tid; i < r.first; i += THREADS) sel[i] = i;
    for (int i = tid; i < r.pages - r.last; i += THREADS) sel[r.first + r.want + i] = r.last + i;
    if (r.want == r.last - r.first)
      for (int i = tid; i < r.want; i += THREADS) sel[r.first + i] = r.first + i;
  }
  if (r.want == r.last - r.first || r.want == 0) return;      // (all CTAs of the cluster)
  const int sub = tid % LANES;
  const int4 mine = reinterpret_cast<const int4*>(code)[sub];
  uint32_t keys_of_first = 0;
  if (CLUSTER) asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(keys_of_first) : "r"(smem_u32(keys)));
  for (int round = 0; round < rounds; round += UNROLL) {
    const int base = own + round * stride + tid / LANES;
    int4 w[UNROLL];
    float scale[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const int i = base + u * stride;
      const int page = i < r.last ? (int)keys[i] : -1;
      w[u] = make_int4(0, 0, 0, 0);
      scale[u] = 0.f;
      if (page >= 0) {
        const int64_t at = (int64_t)page * p.Hkv + h;
        w[u] = __ldg(reinterpret_cast<const int4*>(p.k_code + at * D) + sub);
        if (sub == 0) scale[u] = __ldg(p.k_scale + at);
      }
    }
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      if (CLUSTER && round + u >= rounds) break;
      const int i = base + u * stride;
      int dot = __dp4a(w[u].x, mine.x, 0);
      dot = __dp4a(w[u].y, mine.y, dot);
      dot = __dp4a(w[u].z, mine.z, dot);
      dot = __dp4a(w[u].w, mine.w, dot);
#pragma unroll
      for (int o = LANES / 2; o > 0; o >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, o);
      if (sub == 0 && i < r.last) {
        const uint32_t key = (int)keys[i] >= 0 ? ordered(__fmul_rn((float)dot, scale[u])) : 0u;
        if (CLUSTER) asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(keys_of_first + 4 * i), "r"(key) : "memory");
        else keys[i] = key;
      }
    }
  }
  if (CLUSTER) {
    cluster_arrive();
    cluster_wait();
    if (rank != 0) return;
  } else {
    __syncthreads();
  }
  for (int i = tid; i < ((r.pages + 3) & ~3); i += THREADS)
    if (i < r.first || i >= r.last) keys[i] = 0;
  if (tid == 0) {
    n_list = 0;
    reach = 0;
  }
  __syncthreads();
  // groups: lane by warp modulo `sets`
  const int sets = min(WARPS, (r.want + 31) / 32);
  if (r.want <= 32 * WARPS && r.want <= LIST) {
    uint32_t most = 0;
    for (int i = tid; i < r.last; i += THREADS) most = max(most, keys[i]);
    tops_of[warp][lane] = most;
    __syncthreads();
    if (warp < sets) {
      for (int x = warp + sets; x < WARPS; x += sets) most = max(most, tops_of[x][lane]);
      tops_of[warp][lane] = most;                             // (read by this warp alone until the barrier)
    }
    __syncthreads();
    if (warp < sets) {
      int rank = 0;                                           // among the groups, ties by number
      for (int x = 0; x < sets; ++x)
        for (int y = 0; y < 32; ++y) {
          const uint32_t other = tops_of[x][y];
          rank += other > most || (other == most && x * 32 + y < tid);
        }
      if (rank == r.want - 1) reach = most;
    }
    __syncthreads();
    const uint32_t bound = reach;
    for (int i = r.first + tid; i < r.last; i += THREADS)
      if (keys[i] >= bound) {
        const int at = atomicAdd(&n_list, 1);
        if (at < LIST) {
          list_key[at] = keys[i];
          list_page[at] = i;
        }
      }
    __syncthreads();
    if (n_list <= LIST) {
      const int n = n_list;
      bool chosen = false;
      const uint32_t key = tid < n ? list_key[tid] : 0;
      const int page = tid < n ? list_page[tid] : 0;
      if (tid < n) {
        int rank = 0;
        for (int i = 0; i < n; ++i) rank += list_key[i] > key || (list_key[i] == key && list_page[i] < page);
        chosen = rank < r.want;
      }
      __syncthreads();
      if (tid < n && !chosen) list_page[tid] = INT32_MAX;
      __syncthreads();
      if (chosen) {
        int before = 0;
        for (int i = 0; i < n; ++i) before += list_page[i] < page;
        sel[r.first + before] = page;
      }
      return;
    }
  }
  // the want-th largest score, bit by bit
  const int quads = (r.last + 3) >> 2;
  uint32_t thr = 0;
  int above_wanted = -1;
#pragma unroll 1
  for (int bit = 31; bit >= 0; --bit) {
    const uint32_t cand = thr | (1u << bit);
    int n = 0;
    for (int i = tid; i < quads; i += THREADS) {
      const uint4 k = reinterpret_cast<const uint4*>(keys)[i];
      n += (k.x >= cand) + (k.y >= cand) + (k.z >= cand) + (k.w >= cand);
    }
    n = __reduce_add_sync(0xffffffffu, n);
    if (lane == 0) counts[bit & 1][warp] = n;
    __syncthreads();
    int all = 0;
#pragma unroll
    for (int x = 0; x < WARPS; ++x) all += counts[bit & 1][x];
    if (all >= r.want) thr = cand;
    if (all == r.want) {
      above_wanted = all;
      break;
    }
  }
  // scores above it all go, and the first of those equal to it; written in page order
  const bool exact = above_wanted >= 0;                       // then those that reach it are as many as are wanted
  int above = 0, equal = 0, equal_wanted = r.want;
  if (!exact) {                                               // how many are above it
    int n = 0;
    for (int i = tid; i < quads; i += THREADS) {
      const uint4 k = reinterpret_cast<const uint4*>(keys)[i];
      n += (k.x > thr) + (k.y > thr) + (k.z > thr) + (k.w > thr);
    }
    n = __reduce_add_sync(0xffffffffu, n);
    __syncthreads();
    if (lane == 0) counts[0][warp] = n;
    __syncthreads();
    for (int x = 0; x < WARPS; ++x) equal_wanted -= counts[0][x];
  }
  for (int base = r.first; base < r.last; base += THREADS) {
    const int i = base + tid;
    const uint32_t key = i < r.last ? keys[i] : 0;
    const bool up = i < r.last && (exact ? key >= thr : key > thr), same = i < r.last && !exact && key == thr;
    const uint32_t va = __ballot_sync(0xffffffffu, up), vs = __ballot_sync(0xffffffffu, same);
    if (lane == 0) {
      warp_cnt[warp][0] = __popc(va);
      warp_cnt[warp][1] = __popc(vs);
    }
    __syncthreads();
    int a = above, s = equal;
#pragma unroll
    for (int x = 0; x < WARPS; ++x) {
      if (x < warp) {
        a += warp_cnt[x][0];
        s += warp_cnt[x][1];
      }
      above += warp_cnt[x][0];
      equal += warp_cnt[x][1];
    }
    const uint32_t below = (1u << lane) - 1;
    a += __popc(va & below);
    s += __popc(vs & below);
    if (up) sel[r.first + a + min(s, equal_wanted)] = i;
    if (same && s < equal_wanted) sel[r.first + a + s] = i;
    __syncthreads();
  }
}

// ------------------------------------------------------------------------------------------------ 16 tokens, one CTA
// A request's tokens share its pages: their codes are read once for 16 tokens and multiplied on the matrix units (as fp16, in which the
// codes, and in 32 bits their products' sums, are exact); a warp then chooses for two tokens.  What bounds it is that choice (a
// warp reads a token's scores from shared memory for the groups' maxima and again for the list, and ranks both): issue slots 56 %, the matrix unit
// 6 %, the DRAM 6 %.  2001 tokens, 4 kv heads, 500 pages take 28.5 us with four CTAs on an SM (64 registers), 33.8 with the two that 109 registers allow.
template <int D>
__global__ void __launch_bounds__(ROWS_THREADS, 4) select_rows_kernel(const __grid_constant__ SelectParams p, int pitch) {
  extern __shared__ __align__(16) uint32_t keys[];            // [16][pitch] scores; 0: not to be chosen
  __shared__ __align__(16) int8_t code[SEL_ROWS][D];
  __shared__ uint32_t list_key[ROWS_WARPS][ROW_LIST];
  __shared__ int list_page[ROWS_WARPS][ROW_LIST];
  pdl_trigger();
  pdl_wait();
  const int t0 = blockIdx.x / p.Hkv * SEL_ROWS, h = blockIdx.x % p.Hkv, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  constexpr int PER = D / 32;                                 // columns of a lane
  for (int row = warp; row < SEL_ROWS; row += ROWS_WARPS) {
    const int t = min(t0 + row, p.n_tokens - 1);
    float q[PER];
    float top = 0.f;
#pragma unroll
    for (int c = 0; c < PER; ++c) q[c] = load_half(p.q, t * p.q_tok + (int64_t)h * p.G * p.q_head + c * 32 + lane, p.fp16);
#pragma unroll 4
    for (int g = 1; g < p.G; ++g)
#pragma unroll
      for (int c = 0; c < PER; ++c) q[c] += load_half(p.q, t * p.q_tok + ((int64_t)h * p.G + g) * p.q_head + c * 32 + lane, p.fp16);
#pragma unroll
    for (int c = 0; c < PER; ++c) top = fmaxf(top, fabsf(q[c]));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
#pragma unroll
    for (int c = 0; c < PER; ++c) code[row][c * 32 + lane] = to_code(q[c], top * (1.f / 127.f));
  }
  __syncthreads();
  // codes as fp16 pairs: 1024 + (code + 128) has the byte in its low bits
  auto widen = [](uint32_t four, uint32_t& lo, uint32_t& hi) {
    const uint32_t u = four ^ 0x80808080u;
    const uint32_t a = __byte_perm(u, 0x64646464u, 0x4140), b = __byte_perm(u, 0x64646464u, 0x4342);
    const __half2 off = __float2half2_rn(1152.f);
    const __half2 x = __hsub2(*reinterpret_cast<const __half2*>(&a), off), y = __hsub2(*reinterpret_cast<const __half2*>(&b), off);
    lo = *reinterpret_cast<const uint32_t*>(&x);
    hi = *reinterpret_cast<const uint32_t*>(&y);
  };
  // A lane of a column pair has a quarter of a row, four bytes for every product: the order of the columns is the same on both sides
  const int gr = lane >> 2, qd = lane & 3;
  uint32_t a[D / 16][4];
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks) {
    widen(*reinterpret_cast<const uint32_t*>(&code[gr][qd * (D / 4) + ks * 4]), a[ks][0], a[ks][2]);
    widen(*reinterpret_cast<const uint32_t*>(&code[gr + 8][qd * (D / 4) + ks * 4]), a[ks][1], a[ks][3]);
  }
  const int t_end = min(t0 + SEL_ROWS, p.n_tokens);
  int t = t0;
  int seq = request_of(p, t0);
  while (t < t_end) {                                         // the requests that the 16 tokens belong to
    while (seq + 1 < p.n_seq && p.q_begin[seq + 1] <= t) ++seq;
    const int b = p.q_begin[seq], e = p.q_begin[seq + 1], kv = p.kv_len[seq];
    // tokens in front of the first request and behind the last one are nobody's (all requests between begin where the one before ends)
    const bool before = t < b, nobody = before || t >= e;
    const int t_next = before ? min(b, t_end) : nobody ? t_end : min(e, t_end);
    const Range widest(p, nobody ? -1 : kv - e + t_next - 1);
    const int32_t* table = p.block_table + seq * p.table_stride;
    // scores of all rows against the request's pages, 8 pages a product
    // (page numbers of eight products first: a load behind another would be waited for each time)
    constexpr int AHEAD = 8;
    for (int base8 = warp * 8; base8 < widest.last; base8 += ROWS_WARPS * 8 * AHEAD) {
      int pages[AHEAD];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int i = base8 + u * ROWS_WARPS * 8 + gr;         // this lane's page
        pages[u] = i < widest.last ? __ldg(table + i) : -1;
        if (pages[u] >= p.n_pages) pages[u] = -1;
      }
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int base = base8 + u * ROWS_WARPS * 8, page = pages[u];
        if (base >= widest.last) break;
        uint32_t w[D / 16];
#pragma unroll
        for (int c = 0; c < D / 16; ++c) w[c] = 0;
        float scale = 0.f;
        if (page >= 0) {
          const int64_t at = (int64_t)page * p.Hkv + h;
          const int4* src = reinterpret_cast<const int4*>(p.k_code + at * D + qd * (D / 4));
#pragma unroll
          for (int c = 0; c < D / 64; ++c) {
            const int4 v = __ldg(src + c);
            w[4 * c] = (uint32_t)v.x, w[4 * c + 1] = (uint32_t)v.y, w[4 * c + 2] = (uint32_t)v.z, w[4 * c + 3] = (uint32_t)v.w;
          }
          scale = __ldg(p.k_scale + at);
        }
        float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
          uint32_t b0, b1;
          widen(w[ks], b0, b1);
          asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
              : "+f"(s[0]), "+f"(s[1]), "+f"(s[2]), "+f"(s[3])
              : "r"(a[ks][0]), "r"(a[ks][1]), "r"(a[ks][2]), "r"(a[ks][3]), "r"(b0), "r"(b1));
        }
        // columns 2 qd and 2 qd + 1: the pages of row groups 2 qd and 2 qd + 1
        uint32_t out[4];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const float sc = __shfl_sync(0xffffffffu, scale, (2 * qd + c) * 4);
          const bool there = __shfl_sync(0xffffffffu, (int)(page >= 0), (2 * qd + c) * 4);
          out[c] = there ? ordered(__fmul_rn(s[c], sc)) : 0u;
          out[2 + c] = there ? ordered(__fmul_rn(s[2 + c], sc)) : 0u;
        }
        *reinterpret_cast<uint2*>(keys + gr * pitch + base + 2 * qd) = make_uint2(out[0], out[1]);
        *reinterpret_cast<uint2*>(keys + (gr + 8) * pitch + base + 2 * qd) = make_uint2(out[2], out[3]);
      }
    }
    __syncthreads();
    for (int tt = t + warp; tt < t_next; tt += ROWS_WARPS) {
      uint32_t* k = keys + (tt - t0) * pitch;
      const Range r(p, nobody ? -1 : kv - e + tt);
      int32_t* sel = p.sel + ((int64_t)tt * p.Hkv + h) * p.n_sel;
      const int taken = r.first + r.want + (r.pages - r.last);
      for (int i = taken + lane; i < p.n_sel; i += 32) sel[i] = -1;
      for (int i = lane; i < r.first; i += 32) sel[i] = i;
      for (int i = lane; i < r.pages - r.last; i += 32) sel[r.first + r.want + i] = r.last + i;
      if (r.want == r.last - r.first) {
        for (int i = lane; i < r.want; i += 32) sel[r.first + i] = r.first + i;
        continue;
      }
      if (r.want == 0) continue;
      // what is not to be chosen; (the row's first multiple of 4 past its last page is inside its pitch)
      for (int i = lane; i < r.first; i += 32) k[i] = 0;
      const int quads = (r.last + 3) >> 2;
      if (lane < 4 * quads - r.last) k[r.last + lane] = 0;
      __syncwarp();
      if (r.want <= 64) {
        // groups: lane, and for more than 32 pages odd and even rounds
        const bool two = r.want > 32;
        uint32_t most[2] = {0, 0};
        int round = 0;
#pragma unroll 4
        for (int i = lane; i < r.last; i += 32, ++round) {
          const uint32_t key = k[i];
          if (two && (round & 1)) most[1] = max(most[1], key); else most[0] = max(most[0], key);
        }
        int rank[2] = {0, 0};
#pragma unroll
        for (int y = 0; y < 32; ++y) {
          const uint32_t other = __shfl_sync(0xffffffffu, most[0], y);
          rank[0] += other > most[0] || (other == most[0] && y < lane);
          rank[1] += other >= most[1];
        }
        if (two) {
#pragma unroll
          for (int y = 0; y < 32; ++y) {
            const uint32_t other = __shfl_sync(0xffffffffu, most[1], y);
            rank[0] += other > most[0];
            rank[1] += other > most[1] || (other == most[1] && y < lane);
          }
        }
        uint32_t bound = rank[0] == r.want - 1 ? most[0] : two && rank[1] == r.want - 1 ? most[1] : 0;
        bound = __reduce_max_sync(0xffffffffu, bound);
        int n = 0;                                            // those that reach it, in page order
        for (int base = 0; base < r.last; base += 32) {
          const int i = base + lane;
          const uint32_t key = i < r.last ? k[i] : 0;
          const bool in = i >= r.first && i < r.last && key >= bound;
          const uint32_t vote = __ballot_sync(0xffffffffu, in);
          const int at = n + __popc(vote & ((1u << lane) - 1));
          if (in && at < ROW_LIST) {
            list_key[warp][at] = key;
            list_page[warp][at] = i;
          }
          n += __popc(vote);
        }
        __syncwarp();
        if (n <= ROW_LIST) {
          int out = r.first;
          for (int base = 0; base < n; base += 32) {
            const int c = base + lane;
            const uint32_t key = c < n ? list_key[warp][c] : 0;
            int rank_c = 0;
            for (int i = 0; i < n; ++i) rank_c += list_key[warp][i] > key || (list_key[warp][i] == key && i < c);
            const bool chosen = c < n && rank_c < r.want;
            const uint32_t vote = __ballot_sync(0xffffffffu, chosen);
            if (chosen) sel[out + __popc(vote & ((1u << lane) - 1))] = list_page[warp][c];
            out += __popc(vote);
          }
          __syncwarp();
          continue;
        }
      }
      uint32_t thr = 0;
      bool exact = false;
#pragma unroll 1
      for (int bit = 31; bit >= 0 && !exact; --bit) {
        const uint32_t cand = thr | (1u << bit);
        int n = 0;
#pragma unroll 4
        for (int i = lane; i < quads; i += 32) {
          const uint4 x = reinterpret_cast<const uint4*>(k)[i];
          n += (x.x >= cand) + (x.y >= cand) + (x.z >= cand) + (x.w >= cand);
        }
        n = __reduce_add_sync(0xffffffffu, n);
        if (n >= r.want) thr = cand;
        exact = n == r.want;
      }
      int equal_wanted = r.want, above = 0, equal = 0;
      if (!exact) {
        int n = 0;
        for (int i = lane; i < quads; i += 32) {
          const uint4 x = reinterpret_cast<const uint4*>(k)[i];
          n += (x.x > thr) + (x.y > thr) + (x.z > thr) + (x.w > thr);
        }
        equal_wanted -= __reduce_add_sync(0xffffffffu, n);
      }
      for (int base = r.first; base < r.last; base += 32) {
        const int i = base + lane;
        const uint32_t key = i < r.last ? k[i] : 0;
        const bool up = i < r.last && (exact ? key >= thr : key > thr), same = i < r.last && !exact && key == thr;
        const uint32_t va = __ballot_sync(0xffffffffu, up), vs = __ballot_sync(0xffffffffu, same), below = (1u << lane) - 1;
        const int x = above + __popc(va & below), y = equal + __popc(vs & below);
        if (up) sel[r.first + x + min(y, equal_wanted)] = i;
        if (same && y < equal_wanted) sel[r.first + x + y] = i;
        above += __popc(va);
        equal += __popc(vs);
      }
    }
    t = t_next;
    __syncthreads();                                          // the scores' place is free again
  }
}

}  // namespace

// Whether 16 tokens share a CTA.  That takes 7 us or so for every request among the 16, one behind another, where a CTA or cluster of its own for
// every token and kv head takes 14 ns of the whole device.  How many requests 16 tokens belong to is known to the host on average only: the tokens
// beside the longest request's are taken to be spread evenly over the others.  Contexts of 20 000 tokens, 8 kv heads of 4 heads, us with a
// token a CTA and with 16: 1 request of 16 new tokens 8.1 and 14, 8 of them 19 and 14.5, 64 126 and 25; 64 of 4 36 and 37; a chunk of 8 beside
// 64 single tokens 11 and 108, of 256 43 and 113, of 1024 131 and 132, of 2048 252 and 162; 2048 beside one 231 and 40.  Two kv heads: 64 of 8
// 20 and 18, 2048 beside 8 62 and 58, beside 32 64 and 111.  Of 132 shapes measured two lose more than 5 % (9.0 us for 7.0).
bool sixteen_at_once(const SelectParams& p, int max_new) {
  const int64_t units = (int64_t)p.n_tokens * p.Hkv, others = std::max(p.n_tokens - max_new, 0), n = p.n_seq;
  const int64_t requests = std::min<int64_t>(std::min<int64_t>(n, SEL_ROWS), 1 + (SEL_ROWS - 1) * (n - 1) / std::max<int64_t>(std::max(others, n - 1), 1));
  return p.table_pages <= SEL_ROWS_PAGES && units > 200 + 400 * requests;
}

cudaError_t launch_paged_select(const SelectParams& p, int max_new, int n_sm, cudaStream_t stream) {
  // (a kernel's limit is the process's: always set to the most that any call takes, or another thread's smaller call, between this one's
  // limit and its launch, would have the launch refused)
  auto go = [&](auto kernel, int64_t units, int threads, size_t smem, int most, int ctas, auto... more) {
    if (smem > 24 * 1024) {
      const cudaError_t rc = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
      if (rc != cudaSuccess) return rc;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(units * ctas));
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)ctas;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = ctas > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, p, more...);
  };
  if (sixteen_at_once(p, max_new)) {
    // (eight pages a product may run past the last; odd multiples of 16 bytes spread the rows over the banks)
    auto pitch_of = [](int pages) { return (pages + 7) / 8 * 8 + 4; };
    const int pitch = pitch_of(p.table_pages), most = SEL_ROWS * pitch_of(SEL_ROWS_PAGES) * 4;
    const int64_t units = (int64_t)((p.n_tokens + SEL_ROWS - 1) / SEL_ROWS) * p.Hkv;
    const size_t smem = (size_t)SEL_ROWS * pitch * 4;
    return p.d == 128 ? go(select_rows_kernel<128>, units, ROWS_THREADS, smem, most, 1, pitch) : go(select_rows_kernel<64>, units, ROWS_THREADS, smem, most, 1, pitch);
  }
  const int64_t units = (int64_t)p.n_tokens * p.Hkv;
  const size_t smem = ((size_t)p.table_pages + 3) / 4 * 16;
  constexpr int most = (PAGED_MAX_SELECT_PAGES + 3) / 4 * 16;
  // few tokens: more of a context's codes on their way at once (without a cluster 1024 threads: 16 requests of 8 kv heads 14.9 us, 15.4 with 256)
  int ctas = 8;
  while (ctas > 1 && units * ctas > n_sm) ctas /= 2;
  if (ctas > 1) return p.d == 128 ? go(select_kernel<128, 512, true>, units, 512, smem, most, ctas) : go(select_kernel<64, 512, true>, units, 512, smem, most, ctas);
  if (units <= n_sm) return p.d == 128 ? go(select_kernel<128, 1024, false>, units, 1024, smem, most, 1) : go(select_kernel<64, 1024, false>, units, 1024, smem, most, 1);
  return p.d == 128 ? go(select_kernel<128, 256, false>, units, 256, smem, most, 1) : go(select_kernel<64, 256, false>, units, 256, smem, most, 1);
}

}  // namespace heatkv
