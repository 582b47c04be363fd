// Attention over a paged cache in 4 bits.
#include "paged4.cuh"
#include "tc_common.cuh"

namespace heatkv {
namespace {

// A warp per query row, a key at a time: lane l holds columns l D / 32 ..
template <int D>
__global__ void __launch_bounds__(128) paged4_plain_kernel(const Paged4Params q4) {
  using B = Block4<D>;
  constexpr int N = D / 32;
  const PagedParams& p = q4.a;
  pdl_trigger();
  pdl_wait();
  const int lane = threadIdx.x & 31;
  const int64_t x = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
  if (x >= (int64_t)p.n_tokens * p.H) return;
  const int tok = (int)(x / p.H), hd = (int)(x - (int64_t)tok * p.H), head = hd / p.G;
  int lo = 0, hi = p.n_seq - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (p.q_begin[mid] <= tok) lo = mid; else hi = mid - 1;
  }
  if (tok < p.q_begin[lo] || tok >= p.q_begin[lo + 1]) return;
  const int kv = min(max(p.kv_len[lo], 0), p.table_pages * PAGE);
  const int sees = p.causal ? kv - (p.q_begin[lo + 1] - 1 - tok) : kv;
  float qv[N], acc[N], m = NO_MAX, l = 0.f;
  auto number = [&](const void* base, int64_t at) {
    return q4.fp16 ? __half2float(static_cast<const __half*>(base)[at]) : __bfloat162float(static_cast<const __nv_bfloat16*>(base)[at]);
  };
#pragma unroll
  for (int i = 0; i < N; ++i) {
    qv[i] = number(p.q, tok * p.q_tok + hd * p.q_head + lane * N + i);
    acc[i] = 0.f;
  }
  for (int j = 0; j < sees; ++j) {
    const int page = p.block_table[lo * p.table_stride + j / PAGE], row = j % PAGE;
    float kx[N], vx[N];
    if (page < 0 || page >= p.n_pages) {
#pragma unroll
      for (int i = 0; i < N; ++i) kx[i] = vx[i] = 0.f;
    } else {
      const unsigned char* b = q4.blocks + page * q4.page_stride + head * q4.head_stride;
      auto value = [&](int codes, int scales, int c) {
        const uint32_t w = *reinterpret_cast<const uint32_t*>(b + codes + row * B::ROW + c / 8 * 4), byte = b[scales + row * B::SCALES + c / 16];
        uint32_t v[4];
        values4(w, Steps4(byte | byte << 16), v);
        const float2 pair = __half22float2(as_half2(v[c % 8 / 2]));
        return c & 1 ? pair.y : pair.x;
      };
#pragma unroll
      for (int i = 0; i < N; ++i) {
        kx[i] = value(B::K, B::KS, lane * N + i);
        vx[i] = value(B::V, B::VS, lane * N + i);
      }
    }
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) s = fmaf(qv[i], kx[i], s);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    s *= p.scale_log2;
    const float top = fmaxf(m, s), f = exp2f(m - top), e = exp2f(s - top);
    m = top;
    l = fmaf(l, f, e);
#pragma unroll
    for (int i = 0; i < N; ++i) acc[i] = fmaf(acc[i], f, e * vx[i]);
  }
  const float inv = l == 0.f ? 0.f : q4.v_unit / l;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int64_t at = tok * p.o_tok + hd * p.o_head + lane * N + i;
    if (q4.fp16) static_cast<__half*>(p.out)[at] = __float2half_rn(acc[i] * inv);
    else static_cast<__nv_bfloat16*>(p.out)[at] = __float2bfloat16_rn(acc[i] * inv);
  }
  if (p.lse && lane == 0) p.lse[(int64_t)tok * p.H + hd] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
}

}  // namespace

uint64_t paged4_small_partial_bytes(int, int, int, int) { return 256; }

cudaError_t launch_paged4_small(const Paged4Params& p, int d, const PagedDevice&, cudaStream_t stream) {
  const dim3 grid((unsigned)(((int64_t)p.a.n_tokens * p.a.H + 3) / 4));
  return d == 128 ? launch_pdl(paged4_plain_kernel<128>, grid, dim3(128), 0, stream, p) : launch_pdl(paged4_plain_kernel<64>, grid, dim3(128), 0, stream, p);
}

}  // namespace heatkv
