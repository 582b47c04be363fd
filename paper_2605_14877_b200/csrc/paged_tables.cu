// Bookkeeping of the paged cache: block tables and slot maps from request lengths, pages given back, and the store of new rows
// with the summaries that page selection reads.
#include <algorithm>

#include <cuda_fp16.h>

#include "device_common.cuh"
#include "paged.h"

namespace heatkv {
namespace {

constexpr int TT = 256;                        // threads of the two table kernels

// Exclusive sum over the CTA; `total` gets the sum of all.
__device__ __forceinline__ int64_t block_exclusive(int64_t v, int64_t* warp_sums, int64_t& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int64_t inc = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t up = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += up;
  }
  __syncthreads();                             // the last use of warp_sums is over
  if (lane == 31) warp_sums[warp] = inc;
  __syncthreads();
  int64_t before = 0;
  total = 0;
  for (int w = 0; w < TT / 32; ++w) {
    const int64_t s = warp_sums[w];
    if (w < warp) before += s;
    total += s;
  }
  return before + inc - v;
}
__device__ __forceinline__ int saturate(int64_t v) { return (int)min(v, (int64_t)INT32_MAX); }
// last i in [0, n) with a[i] <= x (a ascending, a[0] <= x)
__device__ __forceinline__ int find_last(const int32_t* a, int n, int x) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a[mid] <= x) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// Every CTA takes the sums over all requests for itself (a few hundred lengths, read from L2) and then writes its share of the
// tokens and of the fresh pages, so there is one launch and no CTA waits for another.  A page that this call hands out is looked
// up in the ring, never in the table that another CTA is writing.  What bounds it is the chain of loads and sums before the first write:
// 3.8 us for the 24 new tokens of 24 requests, 5.6 for 141 786 of 300 (1.2 MB; a thread with one token at a time and one sum behind
// another 9.2).
__global__ void __launch_bounds__(TT) tables_kernel(const TablesParams p) {
  extern __shared__ int32_t sm[];
  int32_t* begin = sm;                         // [n_seq + 1] first token
  int32_t* taken = sm + p.n_seq + 1;           // [n_seq + 1] pages handed out before the request
  int32_t* had = taken + p.n_seq + 1;          // [n_seq] pages it had; -1: refused
  int32_t* past = had + p.n_seq;               // [n_seq]
  __shared__ int64_t warp_tokens[TT / 32], warp_pages[TT / 32];
  __shared__ int handed, turned_down;
  pdl_trigger();
  if (threadIdx.x == 0) handed = turned_down = 0;
  pdl_wait();
  const int per = (p.n_seq + TT - 1) / TT, i0 = min((int)threadIdx.x * per, p.n_seq), i1 = min(i0 + per, p.n_seq);
  const int head = (p.state_in[0] % p.n_pages + p.n_pages) % p.n_pages, free = min(max(p.state_in[1], 0), p.n_pages);
  int64_t tokens = 0, pages = 0;
#pragma unroll 2
  for (int i = i0; i < i1; ++i) {
    const int64_t a = max(__ldg(p.past_tokens + i), 0), n = max(__ldg(p.new_tokens + i), 0);
    const int64_t h0 = (a + PAGE - 1) / PAGE, h1 = (a + n + PAGE - 1) / PAGE;
    begin[i] = (int)n;
    past[i] = (int)a;
    had[i] = h1 <= p.table_pages ? (int)h0 : -1;
    taken[i] = h1 <= p.table_pages ? (int)(h1 - h0) : 0;
    tokens += n;
    pages += taken[i];
  }
  // both sums in one go: tokens and pages before this thread's requests
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int64_t t = tokens, r = pages;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t t_up = __shfl_up_sync(0xffffffffu, t, o), r_up = __shfl_up_sync(0xffffffffu, r, o);
    if (lane >= o) {
      t += t_up;
      r += r_up;
    }
  }
  if (lane == 31) {
    warp_tokens[warp] = t;
    warp_pages[warp] = r;
  }
  __syncthreads();
  t -= tokens;
  r -= pages;
  int64_t all_tokens = 0;
#pragma unroll
  for (int w = 0; w < TT / 32; ++w) {
    all_tokens += warp_tokens[w];
    if (w < warp) {
      t += warp_tokens[w];
      r += warp_pages[w];
    }
  }
  int refused = 0;
  int granted = 0;                             // pages handed out up to this thread's last served request
  for (int i = i0; i < i1; ++i) {
    const int n = begin[i], need = taken[i];
    if (had[i] < 0 || (need > 0 && r + need > free)) {
      had[i] = -1;
      ++refused;
    } else if (need > 0) {
      granted = (int)(r + need);
    }
    begin[i] = saturate(t);
    taken[i] = saturate(min(r, (int64_t)free));
    t += n;
    r += need;
  }
  if (threadIdx.x == 0) begin[p.n_seq] = saturate(all_tokens);
  // served requests that take pages are the first ones: the most that any thread saw is what the call hands out
  if (granted > 0) atomicMax(&handed, granted);
  if (refused > 0) atomicAdd(&turned_down, refused);
  __syncthreads();
  const int got = handed;
  auto page_of = [&](int rank) {                 // (rank < free <= n_pages)
    const uint32_t at = (uint32_t)head + (uint32_t)rank;
    return p.free_pages[at < (uint32_t)p.n_pages ? at : at - (uint32_t)p.n_pages];
  };
  const int gid = blockIdx.x * TT + threadIdx.x, step = gridDim.x * TT;
  // fresh pages -> block tables
  for (int x = gid; x < got; x += step) {
    int i = find_last(taken, p.n_seq, x);
    p.block_table[i * p.table_stride + had[i] + (x - taken[i])] = page_of(x);
  }
  // tokens -> positions and slots, four neighbours by a thread: they look up one request and mostly one page
  const int n_tokens = min(begin[p.n_seq], p.n_tokens);
  const bool wide = ((reinterpret_cast<uintptr_t>(p.slot_map) | reinterpret_cast<uintptr_t>(p.positions)) & 15) == 0;
  for (int64_t x0 = (int64_t)gid * 4; x0 < p.n_tokens; x0 += (int64_t)step * 4) {
    int slot[4], at[4], page = -1, page_at = -1;
    int i = x0 < n_tokens ? find_last(begin, p.n_seq, (int)x0) : 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t x = x0 + u;
      slot[u] = -1;
      at[u] = 0;
      if (x >= n_tokens) continue;               // places past the last token
      while (begin[i + 1] <= x) {
        ++i;
        page_at = -1;
      }
      const int pos = past[i] + ((int)x - begin[i]), pg = pos / PAGE;
      at[u] = pos;
      if (had[i] < 0) continue;
      if (pg != page_at) {
        page = pg >= had[i] ? page_of(taken[i] + pg - had[i]) : p.block_table[i * p.table_stride + pg];
        page_at = pg;
      }
      if (page >= 0 && page < p.n_pages) slot[u] = page * PAGE + pos % PAGE;
    }
    if (wide && x0 + 4 <= p.n_tokens) {
      *reinterpret_cast<int4*>(p.slot_map + x0) = make_int4(slot[0], slot[1], slot[2], slot[3]);
      if (p.positions) *reinterpret_cast<int4*>(p.positions + x0) = make_int4(at[0], at[1], at[2], at[3]);
    } else {
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (x0 + u < p.n_tokens) {
          p.slot_map[x0 + u] = slot[u];
          if (p.positions) p.positions[x0 + u] = at[u];
        }
    }
  }
  for (int i = gid; i <= p.n_seq; i += step) {
    p.q_begin[i] = begin[i];
    if (i < p.n_seq) p.kv_len[i] = had[i] >= 0 ? past[i] + (begin[i + 1] - begin[i]) : 0;
  }
  if (gid == 0) {
    p.state_out[0] = (int)(((int64_t)head + got) % p.n_pages);
    p.state_out[1] = free - got;
    p.state_out[2] = turned_down;
    p.state_out[3] = begin[p.n_seq];
  }
}

// Pages past the kept tokens go to the end of the ring, request by request.  One CTA, bound by latency: a chain of loads and one sum, then for every
// 256 pages a search among the requests and two loads, one behind another.  24 requests that give back 43 pages: 2.0 us; 300 and 14 700: 35;
// 64 and 40 100: 75.
__global__ void __launch_bounds__(TT) release_kernel(const ReleaseParams p) {
  extern __shared__ int32_t sm[];
  int32_t* before = sm;                        // [n_seq]
  int32_t* keep = sm + p.n_seq;                // [n_seq]
  __shared__ int64_t warp_sums[TT / 32];
  pdl_trigger();
  pdl_wait();
  const int per = (p.n_seq + TT - 1) / TT, i0 = min((int)threadIdx.x * per, p.n_seq), i1 = min(i0 + per, p.n_seq);
  const int head = (p.state_in[0] % p.n_pages + p.n_pages) % p.n_pages, free = min(max(p.state_in[1], 0), p.n_pages);
  int64_t pages = 0;
  for (int i = i0; i < i1; ++i) {
    const int64_t kv = max(p.kv_len[i], 0), kp = min(max((int64_t)p.keep_len[i], (int64_t)0), kv);
    const int have = (int)min((kv + PAGE - 1) / PAGE, (int64_t)p.table_pages);
    keep[i] = min((int)((kp + PAGE - 1) / PAGE), have);
    before[i] = have - keep[i];
    pages += before[i];
  }
  int64_t all;
  int64_t r = block_exclusive(pages, warp_sums, all);
  for (int i = i0; i < i1; ++i) {
    const int n = before[i];
    before[i] = saturate(r);
    r += n;
  }
  __syncthreads();
  const int room = max(p.n_pages - free, 0), total = (int)min(all, (int64_t)room);
  for (int x = threadIdx.x; x < total; x += TT) {
    const int i = find_last(before, p.n_seq, x);
    p.free_pages[(int)(((int64_t)head + free + x) % p.n_pages)] = p.block_table[i * p.table_stride + keep[i] + (x - before[i])];
  }
  if (threadIdx.x == 0) {
    p.state_out[0] = head;
    p.state_out[1] = free + total;
    p.state_out[2] = 0;
    p.state_out[3] = total;
  }
}

// ---------------------------------------------------------------- store
constexpr int ST = 128;
constexpr int STORE_UNROLL = 4;                // 16-byte words of K and of V that a thread has on their way
constexpr int SUMMARY_TOKENS = 64;             // tokens whose completed pages one CTA summarises, for one head

__device__ __forceinline__ float2 widen(uint32_t w, bool fp16) {
  if (fp16) return __half22float2(*reinterpret_cast<__half2*>(&w));
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}

__device__ __forceinline__ const __nv_bfloat16* pool_row(const StoreParams& p, int page, int row, int h) {
  return static_cast<const __nv_bfloat16*>(p.k) + (int64_t)page * p.page_stride + h * p.head_stride + (int64_t)row * p.row_stride;
}

// Pages whose row 63 is among the slots of 64 tokens, for one head: mean key as 8-bit codes and a scale.  row_at(token, slot, row, head): where row `row` of
// the page lies whose last row is the token's.
template <int D, typename Row>
__device__ __forceinline__ void summaries(const StoreParams& p, int unit, Row row_at) {
  constexpr int CH = D / 8;
  __shared__ float part[8][D];
  __shared__ float tops[ST / 32];
  __shared__ int found[SUMMARY_TOKENS];
  __shared__ int n_found;
  const uint32_t n_slots = (uint32_t)p.n_pages * PAGE;
  const int h = unit % p.Hkv, t0 = unit / p.Hkv * SUMMARY_TOKENS;
  if (threadIdx.x == 0) n_found = 0;
  __syncthreads();
  if (threadIdx.x < SUMMARY_TOKENS && t0 + (int)threadIdx.x < p.n_tokens) {
    const uint32_t slot = (uint32_t)p.slot_map[t0 + threadIdx.x];
    if (slot < n_slots && slot % PAGE == PAGE - 1) found[atomicAdd(&n_found, 1)] = t0 + threadIdx.x;
  }
  __syncthreads();
  for (int f = 0; f < n_found; ++f) {
    const int t = found[f];
    const int slot = p.slot_map[t], page = slot / PAGE;
    const int rg = threadIdx.x / CH, ch = threadIdx.x % CH;
    if (rg < 8) {
      int4 w[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        w[j] = *reinterpret_cast<const int4*>(row_at(t, slot, rg + 8 * j, h) + ch * 8);
      }
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        float2 x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = widen(reinterpret_cast<const uint32_t*>(&w[j])[c], p.fp16);
#pragma unroll
        for (int s = 4; s > 0; s >>= 1)
#pragma unroll
          for (int j = 0; j < s; ++j) {
            x[j].x += x[j + s].x;
            x[j].y += x[j + s].y;
          }
        part[rg][ch * 8 + 2 * c] = x[0].x;
        part[rg][ch * 8 + 2 * c + 1] = x[0].y;
      }
    }
    __syncthreads();
    const int col = threadIdx.x;
    float m = 0.f;
    if (col < D) {
      m = (((part[0][col] + part[4][col]) + (part[2][col] + part[6][col])) + ((part[1][col] + part[5][col]) + (part[3][col] + part[7][col]))) *
          (1.f / PAGE);
    }
    float top = fabsf(m);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    if ((threadIdx.x & 31) == 0) tops[threadIdx.x >> 5] = top;
    __syncthreads();
    top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
    const float scale = top * (1.f / 127.f);
    if (col < D) {
      const float c = scale > 0.f ? fminf(fmaxf(rintf(__fdiv_rn(m, scale)), -127.f), 127.f) : 0.f;
      p.k_code[((int64_t)page * p.Hkv + h) * D + col] = (int8_t)c;
      if (col == 0) p.k_scale[(int64_t)page * p.Hkv + h] = scale;
    }
    __syncthreads();
  }
}

// Blocks 0 .. copy_blocks - 1 copy rows, 16 bytes at a time; the others look for pages whose row 63 is written by this call and
// write the summary of each: mean key as 8-bit codes and a scale.  The mean is a tree (rows i and i + 32, then i and i + 16, ..), so
// its value depends on the page's rows alone.  Rows that this call writes are read from the caller's tensor, since the pool's may not be
// there yet: a request's tokens lie one after another in position order.  6 356 rows of 16 kv heads, 128 columns (104 MB read and written) take
// 21.6 us, 4.8 TB/s, a decode's 64 rows 2.1.  What bounds it is waiting for loads (a word's address stands behind its slot's load and two 64-bit
// divisions; four words of K and of V are on their way per thread): the DRAM is busy 42 % of the time, the issue slots 44 %.
template <int D>
__global__ void __launch_bounds__(ST) store_kernel(const StoreParams p) {
  constexpr int CH = D / 8;
  pdl_trigger();
  pdl_wait();
  const uint32_t n_slots = (uint32_t)p.n_pages * PAGE;
  if ((int)blockIdx.x < p.copy_blocks) {
    const int64_t total = (int64_t)p.n_tokens * p.Hkv * CH;
    const int64_t base = (int64_t)blockIdx.x * (ST * STORE_UNROLL) + threadIdx.x;
    int4 k[STORE_UNROLL], v[STORE_UNROLL];
    int64_t dst[STORE_UNROLL];
#pragma unroll
    for (int u = 0; u < STORE_UNROLL; ++u) {
      const int64_t i = base + u * ST;
      dst[u] = -1;
      if (i >= total) continue;
      const int ch = (int)(i % CH);
      const int64_t th = i / CH;
      const int h = (int)(th % p.Hkv);
      const int64_t t = th / p.Hkv;
      const uint32_t slot = (uint32_t)p.slot_map[t];
      const int64_t src = t * p.tok + h * p.head + ch * 8;
      k[u] = __ldg(reinterpret_cast<const int4*>(static_cast<const __nv_bfloat16*>(p.k_new) + src));
      v[u] = __ldg(reinterpret_cast<const int4*>(static_cast<const __nv_bfloat16*>(p.v_new) + src));
      if (slot < n_slots) dst[u] = (int64_t)(slot / PAGE) * p.page_stride + h * p.head_stride + (int64_t)(slot % PAGE) * p.row_stride + ch * 8;
    }
#pragma unroll
    for (int u = 0; u < STORE_UNROLL; ++u) {
      if (dst[u] < 0) continue;
      *reinterpret_cast<int4*>(static_cast<__nv_bfloat16*>(p.k) + dst[u]) = k[u];
      *reinterpret_cast<int4*>(static_cast<__nv_bfloat16*>(p.v) + dst[u]) = v[u];
    }
    return;
  }
  summaries<D>(p, (int)blockIdx.x - p.copy_blocks, [&](int t, int slot, int row, int h) {
    const int tt = t - (PAGE - 1 - row);
    const bool fresh = tt >= 0 && p.slot_map[tt] == slot - (PAGE - 1 - row);
    return fresh ? static_cast<const __nv_bfloat16*>(p.k_new) + (int64_t)tt * p.tok + h * p.head : pool_row(p, slot / PAGE, row, h);
  });
}

// The summaries alone, of pages whose last row is among the slots: all rows are in the pool.
template <int D>
__global__ void __launch_bounds__(ST) summary_kernel(const StoreParams p) {
  pdl_trigger();
  pdl_wait();
  summaries<D>(p, (int)blockIdx.x, [&](int, int slot, int row, int h) { return pool_row(p, slot / PAGE, row, h); });
}

}  // namespace

cudaError_t launch_paged_tables(const TablesParams& p, cudaStream_t stream) {
  const int64_t work = std::max<int64_t>(p.n_tokens, p.n_seq);
  const int grid = (int)std::min<int64_t>(296, std::max<int64_t>(1, (work + TT * 4 - 1) / (TT * 4)));
  const size_t smem = (4 * (size_t)p.n_seq + 2) * sizeof(int32_t);
  if (smem > 48 * 1024) {
    // (the most that any call takes: the limit is the process's, and another thread may set it before this launch)
    const cudaError_t rc = cudaFuncSetAttribute(tables_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (4 * PAGED_MAX_SEQ + 2) * (int)sizeof(int32_t));
    if (rc != cudaSuccess) return rc;
  }
  return launch_pdl(tables_kernel, dim3(grid), dim3(TT), smem, stream, p);
}

cudaError_t launch_paged_release(const ReleaseParams& p, cudaStream_t stream) {
  return launch_pdl(release_kernel, dim3(1), dim3(TT), 2 * (size_t)p.n_seq * sizeof(int32_t), stream, p);
}

cudaError_t launch_paged_store(StoreParams p, cudaStream_t stream) {
  const int64_t words = (int64_t)p.n_tokens * p.Hkv * (p.d / 8);
  const int64_t copy = (words + ST * STORE_UNROLL - 1) / (ST * STORE_UNROLL);
  const int64_t sums = p.k_code ? (int64_t)((p.n_tokens + SUMMARY_TOKENS - 1) / SUMMARY_TOKENS) * p.Hkv : 0;
  if (copy + sums > INT32_MAX) return cudaErrorInvalidValue;
  p.copy_blocks = (int)copy;
  const dim3 grid((unsigned)(copy + sums));
  return p.d == 128 ? launch_pdl(store_kernel<128>, grid, dim3(ST), 0, stream, p) : launch_pdl(store_kernel<64>, grid, dim3(ST), 0, stream, p);
}

cudaError_t launch_paged_summaries(const StoreParams& p, cudaStream_t stream) {
  const int64_t blocks = (int64_t)((p.n_tokens + SUMMARY_TOKENS - 1) / SUMMARY_TOKENS) * p.Hkv;
  if (blocks > INT32_MAX) return cudaErrorInvalidValue;
  const dim3 grid((unsigned)blocks);
  return p.d == 128 ? launch_pdl(summary_kernel<128>, grid, dim3(ST), 0, stream, p) : launch_pdl(summary_kernel<64>, grid, dim3(ST), 0, stream, p);
}

}  // namespace heatkv
