// Page selection: for every query token and kv head the pages whose mean key scores highest, plus the first and the last ones.
//
// Query summary: the sum of the group's heads in 32 bits, in head order, held as 8-bit codes (largest magnitude / 127; the query's own
// scale is common to its scores and drops out).  Score of a page: the whole-number dot product of the two codes, times the page's
// scale.  |dot| <= 128 * 127^2 < 2^24 is exact in 32 bits whatever the order of its sums, so the choice is the same for every launch
// shape; equal scores go to the lower page.
#include <cuda_fp16.h>

#include "device_common.cuh"
#include "paged.h"

namespace heatkv {
namespace {

constexpr int SEL_THREADS = 256;

__device__ __forceinline__ float load_half(const void* p, int64_t i, bool fp16) {
  return fp16 ? __half2float(static_cast<const __half*>(p)[i]) : __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
}
// ascending order of floats as unsigned words (-0 was made +0 before)
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// One CTA per (token, kv head).
template <int D>
__global__ void __launch_bounds__(SEL_THREADS) select_kernel(const SelectParams p) {
  extern __shared__ __align__(16) uint32_t keys[];          // [middle pages] scores as ordered words
  __shared__ __align__(16) int8_t code[D];
  __shared__ float tops[SEL_THREADS / 32];
  __shared__ uint32_t hist[256];
  __shared__ uint32_t chosen_digit, left;
  __shared__ int seq_of;
  __shared__ int warp_cnt[SEL_THREADS / 32][2];
  pdl_trigger();
  pdl_wait();
  const int t = blockIdx.x / p.Hkv, h = blockIdx.x % p.Hkv, tid = threadIdx.x;
  int32_t* sel = p.sel + ((int64_t)t * p.Hkv + h) * p.n_sel;
  if (tid == 0) {
    int lo = 0, hi = p.n_seq - 1;                           // last request whose first token is not past t
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (p.q_begin[mid] <= t) lo = mid; else hi = mid - 1;
    }
    seq_of = lo;
  }
  // summed query -> codes
  float q = 0.f;
  if (tid < D) {
    const int64_t at = t * p.q_tok + (int64_t)h * p.G * p.q_head + tid;
    q = load_half(p.q, at, p.fp16);
    for (int g = 1; g < p.G; ++g) q += load_half(p.q, at + g * p.q_head, p.fp16);
  }
  float top = fabsf(q);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  if ((tid & 31) == 0) tops[tid >> 5] = top;
  __syncthreads();
  if (tid < D) {
    top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
    const float scale = top * (1.f / 127.f);
    code[tid] = (int8_t)(scale > 0.f ? fminf(fmaxf(rintf(__fdiv_rn(q, scale)), -127.f), 127.f) : 0.f);
  }
  const int seq = seq_of;
  const int kv = p.kv_len[seq], pos = kv - p.q_begin[seq + 1] + t;            // its own key is the last it sees
  const bool none = t < p.q_begin[seq] || t >= p.q_begin[seq + 1] || pos < 0;
  const int pages = none ? 0 : min(pos / PAGE + 1, p.table_pages);
  // pages [0, first) and [last, pages) are always taken, `want` of those between
  const int first = min(p.sink, pages), last = max(first, pages - p.local);
  const int middle = last - first;
  const int want = min(p.n_sel - first - (pages - last), middle);
  __syncthreads();
  const int taken = first + want + (pages - last);
  for (int i = taken + tid; i < p.n_sel; i += SEL_THREADS) sel[i] = -1;
  for (int i = tid; i < first; i += SEL_THREADS) sel[i] = i;
  for (int i = tid; i < pages - last; i += SEL_THREADS) sel[first + want + i] = last + i;
  if (want == middle) {
    for (int i = tid; i < middle; i += SEL_THREADS) sel[first + i] = first + i;
    return;
  }
  if (want == 0) return;
  const int32_t* table = p.block_table + seq * p.table_stride + first;
  int qc[D / 4];
#pragma unroll
  for (int i = 0; i < D / 4; ++i) qc[i] = reinterpret_cast<const int*>(code)[i];
  for (int i = tid; i < middle; i += SEL_THREADS) {
    const int page = table[i];
    uint32_t key = 0;
    if (page >= 0 && page < p.n_pages) {
      const int64_t at = (int64_t)page * p.Hkv + h;
      const int4* kc = reinterpret_cast<const int4*>(p.k_code + at * D);
      int dot = 0;
#pragma unroll
      for (int c = 0; c < D / 16; ++c) {
        const int4 w = __ldg(kc + c);
        dot = __dp4a(w.x, qc[4 * c], dot);
        dot = __dp4a(w.y, qc[4 * c + 1], dot);
        dot = __dp4a(w.z, qc[4 * c + 2], dot);
        dot = __dp4a(w.w, qc[4 * c + 3], dot);
      }
      key = ordered(__fmul_rn((float)dot, p.k_scale[at]) + 0.f);
    }
    keys[i] = key;
  }
  // the want-th largest key, eight bits at a time from the top
  uint32_t prefix = 0, mask = 0;
  if (tid == 0) left = want;
#pragma unroll 1
  for (int shift = 24; shift >= 0; shift -= 8) {
    hist[tid] = 0;
    __syncthreads();
    for (int i = tid; i < middle; i += SEL_THREADS)
      if ((keys[i] & mask) == prefix) atomicAdd(&hist[(keys[i] >> shift) & 255], 1u);
    __syncthreads();
    if (tid < 32) {                                        // digits from the top, eight per lane
      uint32_t c[8], sum = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) sum += c[j] = hist[255 - (tid * 8 + j)];
      uint32_t inc = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t up = __shfl_up_sync(0xffffffffu, inc, o);
        if (tid >= o) inc += up;
      }
      uint32_t before = inc - sum;
      const uint32_t need = left;
      __syncwarp();
      if (before < need && need <= inc) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (before < need && need <= before + c[j]) {
            chosen_digit = 255 - (tid * 8 + j);
            left = need - before;
          }
          before += c[j];
        }
      }
    }
    __syncthreads();
    prefix |= chosen_digit << shift;
    mask |= 255u << shift;
  }
  // keys above it all go, and the first `left` of those equal to it; written in page order
  const uint32_t threshold = prefix;
  const int equal_wanted = (int)left;
  int out = 0, equal = 0;                                   // above / equal ones before this round
  const int lane = tid & 31, warp = tid >> 5;
  for (int base = 0; base < middle; base += SEL_THREADS) {
    const int i = base + tid;
    const uint32_t key = i < middle ? keys[i] : 0;
    const bool above = i < middle && key > threshold, same = i < middle && key == threshold;
    const uint32_t va = __ballot_sync(0xffffffffu, above), vs = __ballot_sync(0xffffffffu, same);
    if (lane == 0) {
      warp_cnt[warp][0] = __popc(va);
      warp_cnt[warp][1] = __popc(vs);
    }
    __syncthreads();
    int a = 0, e = 0, a_all = 0, e_all = 0;
#pragma unroll
    for (int w = 0; w < SEL_THREADS / 32; ++w) {
      if (w < warp) { a += warp_cnt[w][0]; e += warp_cnt[w][1]; }
      a_all += warp_cnt[w][0];
      e_all += warp_cnt[w][1];
    }
    const uint32_t below = (1u << lane) - 1;
    a += out + __popc(va & below);
    e += equal + __popc(vs & below);
    if (above) sel[first + a + min(e, equal_wanted)] = first + i;
    if (same && e < equal_wanted) sel[first + a + e] = first + i;
    out += a_all;
    equal += e_all;
    __syncthreads();
  }
}

}  // namespace

cudaError_t launch_paged_select(const SelectParams& p, int n_sm, cudaStream_t stream) {
  (void)n_sm;
  const size_t smem = (size_t)p.table_pages * 4;
  auto go = [&](auto kernel) {
    if (smem > 40 * 1024) {
      const cudaError_t rc = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
      if (rc != cudaSuccess) return rc;
    }
    return launch_pdl(kernel, dim3((unsigned)p.n_tokens * p.Hkv), dim3(SEL_THREADS), smem, stream, p);
  };
  return p.d == 128 ? go(select_kernel<128>) : go(select_kernel<64>);
}

}  // namespace heatkv
