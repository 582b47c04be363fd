// Rows of the 4-bit cache: quantised to their slots, and read back.
#include <cuda_fp8.h>

#include <type_traits>

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
// less than 2^-20, a quotient of an 11-bit and a 4-bit number that is no tie is 2^-12 away from the nearest one, so the step of 2^-16 to which
// adding 192 rounds x r makes ties ties again and moves nothing across one; 192 is even.  Adding 1.5 * 2^23 then rounds to a whole number, whose low bits
// are 192 + code: its lowest four, one of them turned round, are the field.  CLAMP: quotients may exceed 7 (where the scale is the largest there is,
// or so small that it has fewer bits).
template <bool F16, bool CLAMP>
__device__ __forceinline__ uint32_t codes_of(const uint32_t (&x)[4], float r) {
  uint32_t z[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 v = widen2(x[i], F16);
    float w0 = fmaf(v.x, r, 192.f), w1 = fmaf(v.y, r, 192.f);
    if (CLAMP) {
      w0 = fminf(fmaxf(w0, 185.f), 199.f);
      w1 = fminf(fmaxf(w1, 185.f), 199.f);
    }
    z[2 * i] = __float_as_uint(w0 + 12582912.f);
    z[2 * i + 1] = __float_as_uint(w1 + 12582912.f);
  }
  // bytes of the word: columns 0 and 2, 4 and 6, 1 and 3, 5 and 7
  const uint32_t lo = __byte_perm(__byte_perm(z[0], z[4], 0x0040), __byte_perm(z[1], z[5], 0x0040), 0x5410);
  const uint32_t hi = __byte_perm(__byte_perm(z[2], z[6], 0x0040), __byte_perm(z[3], z[7], 0x0040), 0x5410);
  return ((lo & 0x0f0f0f0fu) | (hi << 4 & 0xf0f0f0f0u)) ^ 0x88888888u;
}
// the largest magnitude of a thread's sixteen columns (NaN counts for nothing)
template <bool F16>
__device__ __forceinline__ float largest(const uint4& a, const uint4& b) {
  const uint32_t x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t y = x[i] & 0x7fff7fffu;
    if (F16) {
      const __half2 m = __hmax2(as_half2(top), as_half2(y));
      top = as_word(m);
    } else {
      const __nv_bfloat162 m = __hmax2(*reinterpret_cast<const __nv_bfloat162*>(&top), *reinterpret_cast<const __nv_bfloat162*>(&y));
      top = *reinterpret_cast<const uint32_t*>(&m);
    }
  }
  const float2 m = widen2(top, F16);
  return fmaxf(m.x, m.y);
}

// A thread takes sixteen columns of K or V of a token and head, 32 bytes on one side and 8 and a scale on the other, of UNROLL rows (a row: K
// and V of a token and head, by D / 8 threads) whose loads are all on their way at once (a row at a time: 62 us for both kernels instead of 56; two or eight rows are no
// better than four).  What bounds it are instructions as much as bytes: 199 700 rows of 128, 131 MB either way, take 26.4 us to store (5.0 TB/s, three of four issue slots) and 29.2 to load (4.5).
constexpr int UNROLL = 4;
template <int D>
struct Piece {
  static constexpr int GROUPS = D / 16, ROWS = T4 / (2 * GROUPS);  // rows at a time by a CTA
  int64_t tok[UNROLL];                                             // < 0: no row
  int head[UNROLL];
  uint32_t slot[UNROLL];
  int g, v;
  __device__ __forceinline__ explicit Piece(const Store4Params& p) {
    const int i = threadIdx.x, local = i / (2 * GROUPS);
    g = i % GROUPS;
    v = i / GROUPS % 2;
    const int64_t first = (int64_t)blockIdx.x * (ROWS * UNROLL), t0 = first / p.Hkv;
    const int h0 = (int)(first - t0 * p.Hkv);
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const uint32_t h = h0 + local + u * ROWS, t = h / (uint32_t)p.Hkv;
      head[u] = h - t * p.Hkv;
      tok[u] = t0 + t < p.n_tokens ? t0 + t : -1;
      slot[u] = tok[u] < 0 ? 0xffffffffu : (uint32_t)p.slot_map[tok[u]];
    }
  }
};

template <int D, bool F16>
__global__ void __launch_bounds__(T4) store4_kernel(const Store4Params p) {
  using B = Block4<D>;
  pdl_trigger();
  pdl_wait();
  const uint32_t n_slots = (uint32_t)p.n_pages * PAGE;
  const Piece<D> x(p);
  uint4 a[UNROLL], b[UNROLL];
#pragma unroll
  for (int u = 0; u < UNROLL; ++u) {
    a[u] = b[u] = make_uint4(0, 0, 0, 0);
    if (x.slot[u] >= n_slots) continue;
    const uint4* src = reinterpret_cast<const uint4*>(static_cast<const __half*>(x.v ? p.v_new : p.k_new) + x.tok[u] * p.tok + x.head[u] * p.head + x.g * 16);
    a[u] = __ldg(src);
    b[u] = __ldg(src + 1);
  }
  const float unit = power_of_two(-(x.v ? p.v_exp : p.k_exp));
#pragma unroll
  for (int u = 0; u < UNROLL; ++u) {
    if (x.slot[u] >= n_slots) continue;
    const uint32_t x0[4] = {a[u].x, a[u].y, a[u].z, a[u].w}, x1[4] = {b[u].x, b[u].y, b[u].z, b[u].w};
    const float top = largest<F16>(a[u], b[u]);
    const uint8_t byte = __nv_cvt_float_to_fp8(top * unit * SEVENTH, __NV_SATFINITE, __NV_E4M3);
    const float s = __half2float(__half(__nv_cvt_fp8_to_halfraw(byte, __NV_E4M3)));
    const float r = s > 0.f ? __frcp_rn(s) * unit : 0.f;
    unsigned char* block = p.blocks + (int64_t)(x.slot[u] / PAGE) * p.page_stride + x.head[u] * p.head_stride;
    const int row = (int)(x.slot[u] % PAGE);
    uint2 codes;
    if (top * r <= 7.49f) codes = make_uint2(codes_of<F16, false>(x0, r), codes_of<F16, false>(x1, r));
    else codes = make_uint2(codes_of<F16, true>(x0, r), codes_of<F16, true>(x1, r));
    *reinterpret_cast<uint2*>(block + (x.v ? B::V : B::K) + row * B::ROW + x.g * 8) = codes;
    block[(x.v ? B::VS : B::KS) + row * B::SCALES + x.g] = byte;
  }
}

// The reverse; rows without a slot in the pool are zero.
template <int D, bool F16>
__global__ void __launch_bounds__(T4) load4_kernel(const Store4Params p) {
  using B = Block4<D>;
  pdl_trigger();
  pdl_wait();
  const uint32_t n_slots = (uint32_t)p.n_pages * PAGE;
  const Piece<D> x(p);
  uint2 w[UNROLL];
  uint32_t byte[UNROLL];
#pragma unroll
  for (int u = 0; u < UNROLL; ++u) {
    w[u] = make_uint2(0, 0);
    byte[u] = 0;
    if (x.slot[u] >= n_slots) continue;
    const unsigned char* block = p.blocks + (int64_t)(x.slot[u] / PAGE) * p.page_stride + x.head[u] * p.head_stride;
    const int row = (int)(x.slot[u] % PAGE);
    w[u] = *reinterpret_cast<const uint2*>(block + (x.v ? B::V : B::K) + row * B::ROW + x.g * 8);
    byte[u] = block[(x.v ? B::VS : B::KS) + row * B::SCALES + x.g];
  }
  const float unit = VALUES4_UNIT * power_of_two(x.v ? p.v_exp : p.k_exp);
#pragma unroll
  for (int u = 0; u < UNROLL; ++u) {
    if (x.tok[u] < 0) continue;
    uint32_t out[8];
    typename std::conditional<F16, Steps4, Steps4Bf16>::type steps(byte[u] | byte[u] << 16);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      uint32_t y[4];
      values4(k ? w[u].y : w[u].x, steps, y);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (unit == VALUES4_UNIT) {                                // (the pool's power of two is 1: the numbers are exact in 16 bits)
          if (F16) {
            out[4 * k + j] = as_word(__hmul2(as_half2(y[j]), __float2half2_rn(VALUES4_UNIT)));
          } else {
            const __nv_bfloat162 z = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&y[j]), __float2bfloat162_rn(VALUES4_UNIT));
            out[4 * k + j] = *reinterpret_cast<const uint32_t*>(&z);
          }
        } else {
          const float2 z = widen2(y[j], F16);
          if (F16) {
            const __half2 q = __floats2half2_rn(z.x * unit, z.y * unit);
            out[4 * k + j] = *reinterpret_cast<const uint32_t*>(&q);
          } else {
            out[4 * k + j] = pack_bf16(z.x * unit, z.y * unit);
          }
        }
      }
    }
    uint4* dst = reinterpret_cast<uint4*>(static_cast<__half*>(const_cast<void*>(x.v ? p.v_new : p.k_new)) + x.tok[u] * p.tok + x.head[u] * p.head + x.g * 16);
    dst[0] = make_uint4(out[0], out[1], out[2], out[3]);
    dst[1] = make_uint4(out[4], out[5], out[6], out[7]);
  }
}

template <int D, bool F16>
cudaError_t launch(const Store4Params& p, bool load, cudaStream_t stream) {
  constexpr int rows = Piece<D>::ROWS * UNROLL;
  const int64_t blocks = ((int64_t)p.n_tokens * p.Hkv + rows - 1) / rows;
  if (blocks > INT32_MAX) return cudaErrorInvalidValue;
  return launch_pdl(load ? load4_kernel<D, F16> : store4_kernel<D, F16>, dim3((unsigned)blocks), dim3(T4), 0, stream, p);
}

}  // namespace

cudaError_t launch_paged4_rows(const Store4Params& p, bool load, int d, cudaStream_t stream) {
  if (d == 128) return p.fp16 ? launch<128, true>(p, load, stream) : launch<128, false>(p, load, stream);
  return p.fp16 ? launch<64, true>(p, load, stream) : launch<64, false>(p, load, stream);
}

}  // namespace heatkv
