// Rows of the 4-bit cache: quantised to their slots, read back, moved.
#include <cuda_fp8.h>

#include "paged4.cuh"

namespace heatkv {
namespace {

constexpr int T4 = 256;
constexpr float SEVENTH = 1.f / 7.f;

__device__ __forceinline__ float2 widen2(uint32_t w, bool fp16) {
  if (fp16) return __half22float2(*reinterpret_cast<__half2*>(&w));
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}

// 2^e as a 32-bit number, |e| <= 64
__host__ __device__ inline float power_of_two(int e) { return ldexpf(1.f, e); }

// Eight columns as 4-byte words of pairs -> their codes + 8.  A code is the nearest whole number to x / s, ties to even: x r with r = 1 / s in 32 bits is off by
// less than 2^-19, a quotient of an 11-bit and a 4-bit number that is no tie is 2^-11 away from the nearest one, so the step of 2^-16 to which
// adding 192 rounds x r makes ties ties again and moves nothing across one; 192 is even.
__device__ __forceinline__ uint32_t codes_of(const uint32_t (&x)[4], float r, bool fp16) {
  float half[2] = {0.f, 0.f};                                    // fields of the even columns, of the odd ones, as one number each
#pragma unroll
  for (int i = 3; i >= 0; --i) {
    const float2 v = widen2(x[i], fp16);
    const float pair[2] = {v.x, v.y};
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const float w = fminf(fmaxf(fmaf(pair[k], r, 192.f), 185.f), 199.f);
      const float field = (w + 12582912.f) - 12583096.f;         // the nearest whole number to w, less 184
      half[k] = fmaf(half[k], 16.f, field);
    }
  }
  return (uint32_t)half[0] | (uint32_t)half[1] << 16;
}

// A thread takes sixteen columns of K or V of a token and head: 32 bytes in, 8 bytes and a scale out.
template <int D>
__global__ void __launch_bounds__(T4) store4_kernel(const Store4Params p) {
  using B = Block4<D>;
  constexpr int GROUPS = D / 16;
  pdl_trigger();
  pdl_wait();
  const uint32_t n_slots = (uint32_t)p.n_pages * PAGE;
  const int64_t i = (int64_t)blockIdx.x * T4 + threadIdx.x;
  const int g = (int)(i % GROUPS), v = (int)(i / GROUPS % 2);
  const int64_t th = i / (2 * GROUPS), t = th / p.Hkv;
  const int h = (int)(th - t * p.Hkv);
  if (t >= p.n_tokens) return;
  const uint32_t slot = (uint32_t)p.slot_map[t];
  if (slot >= n_slots) return;
  const uint4* src = reinterpret_cast<const uint4*>(static_cast<const __half*>(v ? p.v_new : p.k_new) + t * p.tok + h * p.head + g * 16);
  const uint4 a = __ldg(src), b = __ldg(src + 1);
  const uint32_t x0[4] = {a.x, a.y, a.z, a.w}, x1[4] = {b.x, b.y, b.z, b.w};
  float top = 0.f;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float2 y0 = widen2(x0[k], p.fp16), y1 = widen2(x1[k], p.fp16);
    top = fmaxf(fmaxf(top, fmaxf(fabsf(y0.x), fabsf(y0.y))), fmaxf(fabsf(y1.x), fabsf(y1.y)));
  }
  const float unit = power_of_two(-(v ? p.v_exp : p.k_exp));
  const uint8_t byte = __nv_cvt_float_to_fp8(top * unit * SEVENTH, __NV_SATFINITE, __NV_E4M3);
  const float s = __half2float(__half(__nv_cvt_fp8_to_halfraw(byte, __NV_E4M3)));
  const float r = s > 0.f ? __frcp_rn(s) * unit : 0.f;
  unsigned char* block = p.blocks + (int64_t)(slot / PAGE) * p.page_stride + h * p.head_stride;
  const int row = (int)(slot % PAGE);
  *reinterpret_cast<uint2*>(block + (v ? B::V : B::K) + row * B::ROW + g * 8) = make_uint2(codes_of(x0, r, p.fp16), codes_of(x1, r, p.fp16));
  block[(v ? B::VS : B::KS) + row * B::SCALES + g] = byte;
}

// The reverse; rows without a slot in the pool are zero.
template <int D>
__global__ void __launch_bounds__(T4) load4_kernel(const Store4Params p) {
  using B = Block4<D>;
  constexpr int GROUPS = D / 16;
  pdl_trigger();
  pdl_wait();
  const uint32_t n_slots = (uint32_t)p.n_pages * PAGE;
  const int64_t i = (int64_t)blockIdx.x * T4 + threadIdx.x;
  const int g = (int)(i % GROUPS), v = (int)(i / GROUPS % 2);
  const int64_t th = i / (2 * GROUPS), t = th / p.Hkv;
  const int h = (int)(th - t * p.Hkv);
  if (t >= p.n_tokens) return;
  const uint32_t slot = (uint32_t)p.slot_map[t];
  uint32_t out[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  if (slot < n_slots) {
    const unsigned char* block = p.blocks + (int64_t)(slot / PAGE) * p.page_stride + h * p.head_stride;
    const int row = (int)(slot % PAGE);
    const uint2 w = *reinterpret_cast<const uint2*>(block + (v ? B::V : B::K) + row * B::ROW + g * 8);
    const uint32_t byte = block[(v ? B::VS : B::KS) + row * B::SCALES + g];
    const Steps4 steps(byte | byte << 16);
    const float unit = VALUES4_UNIT * power_of_two(v ? p.v_exp : p.k_exp);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      uint32_t x[4];
      values4(k ? w.y : w.x, steps, x);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 y = __half22float2(as_half2(x[j]));
        if (p.fp16) {
          const __half2 z = __floats2half2_rn(y.x * unit, y.y * unit);
          out[4 * k + j] = *reinterpret_cast<const uint32_t*>(&z);
        } else {
          out[4 * k + j] = pack_bf16(y.x * unit, y.y * unit);
        }
      }
    }
  }
  uint4* dst = reinterpret_cast<uint4*>(static_cast<__half*>(const_cast<void*>(v ? p.v_new : p.k_new)) + t * p.tok + h * p.head + g * 16);
  dst[0] = make_uint4(out[0], out[1], out[2], out[3]);
  dst[1] = make_uint4(out[4], out[5], out[6], out[7]);
}

}  // namespace

cudaError_t launch_paged4_rows(const Store4Params& p, bool load, int d, cudaStream_t stream) {
  const int64_t items = (int64_t)p.n_tokens * p.Hkv * 2 * (d / 16), blocks = (items + T4 - 1) / T4;
  if (blocks > INT32_MAX) return cudaErrorInvalidValue;
  const dim3 grid((unsigned)blocks), block(T4);
  if (load) return d == 128 ? launch_pdl(load4_kernel<128>, grid, block, 0, stream, p) : launch_pdl(load4_kernel<64>, grid, block, 0, stream, p);
  return d == 128 ? launch_pdl(store4_kernel<128>, grid, block, 0, stream, p) : launch_pdl(store4_kernel<64>, grid, block, 0, stream, p);
}

}  // namespace heatkv
