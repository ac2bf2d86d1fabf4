// GELU whose input is kept in 8 bits for the backward pass.
//
// The checkpoint of a row of F values is F codes (int8) and one exponent (uint8, biased by 127) for every 32 columns:
// x = code 2^(e - 127), e the least for which the block's largest value fits into 127 steps, so that a value is off by at most
// half a step, between 1/508 and 1/254 of the block's largest value.  Steps are powers of two: encoding rounds once (to nearest
// even), decoding not at all, and x fits into bf16.  A block that holds a NaN or an infinity gets exponent 255 and decodes to NaN.
//
//   forward   g = h Phi(h) from h itself; codes and exponents of h
//   backward  dh = dg (Phi(x) + x phi(x)), and g = x Phi(x) again for the weight gradient that reads it
//
// Both are one pass; a thread holds 16 bytes of a row (8 bytes where rows of bf16 are an odd multiple of 4 values long), a block
// of 32 is 4 or 8 neighbouring lanes.
#include "common.h"
#include "kernels.h"

namespace pt {
namespace {

template <typename T, int V> struct Piece;
template <> struct Piece<bf16, 8> { typedef uint4 raw; };
template <> struct Piece<bf16, 4> { typedef uint2 raw; };
template <> struct Piece<float, 4> { typedef float4 raw; };

template <typename T, int V>
__device__ __forceinline__ void get(const T* p, float (&x)[V]) {
  union { typename Piece<T, V>::raw r; T t[V]; } u;
  u.r = *reinterpret_cast<const typename Piece<T, V>::raw*>(p);
#pragma unroll
  for (int i = 0; i < V; ++i) x[i] = to_f32(u.t[i]);
}
template <typename T, int V>
__device__ __forceinline__ void put(T* p, const float (&x)[V]) {
  union { typename Piece<T, V>::raw r; T t[V]; } u;
#pragma unroll
  for (int i = 0; i < V; ++i) u.t[i] = from_f32<T>(x[i]);
  *reinterpret_cast<typename Piece<T, V>::raw*>(p) = u.r;
}
template <int V>
__device__ __forceinline__ void get_codes(const int8_t* p, float (&x)[V]) {
  union { uint32_t w[V / 4]; int8_t c[V]; } u;
#pragma unroll
  for (int i = 0; i < V / 4; ++i) u.w[i] = reinterpret_cast<const uint32_t*>(p)[i];
#pragma unroll
  for (int i = 0; i < V; ++i) x[i] = (float)u.c[i];
}

// Phi and phi.  bf16 results: the framework's rational approximation (4e-7); fp32 results: the library's erfc and exp.
template <typename T> __device__ __forceinline__ float cdf_of(float x, float* pdf);
template <> __device__ __forceinline__ float cdf_of<bf16>(float x, float* pdf) {
  float e;
  const float c = gelu_cdf(x, &e);
  *pdf = e * 0.39894228040143268f;
  return c;
}
template <> __device__ __forceinline__ float cdf_of<float>(float x, float* pdf) {
  *pdf = expf(-0.5f * x * x) * 0.39894228040143268f;
  return 0.5f * erfcf(x * -0.70710678118654752f);
}

// pieces per row are padded to whole blocks of 32, so that a block never crosses rows; `per` = pieces of V in a padded row
template <typename T, int V>
__global__ __launch_bounds__(256) void gelu8_fwd_kernel(const T* __restrict__ h, T* __restrict__ g, int8_t* __restrict__ codes,
                                                        uint8_t* __restrict__ exps, int64_t pieces, int per, int F) {
  const int64_t p = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (p >= pieces) return;   // whole blocks of 32 leave together
  const int64_t row = p / per;
  const int c = (int)(p - row * per) * V;
  const bool in = c < F;
  const int64_t at = row * F + c;
  float x[V];
#pragma unroll
  for (int i = 0; i < V; ++i) x[i] = 0.f;
  if (in) get<T, V>(h + at, x);
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const uint32_t b = __float_as_uint(x[i]) & 0x7fffffffu;
    top = b > top ? b : top;
  }
#pragma unroll
  for (int o = 1; o < 32 / V; o <<= 1) {
    const uint32_t b = __shfl_xor(top, o, 64);
    top = b > top ? b : top;
  }
  // top = 1.f 2^(E - 127) fits into 127 steps of 2^(E - 133) if 1.f <= 127 / 64, else into steps twice as large
  int e = (int)(top >> 23) - 6 + ((top & 0x7fffffu) > 0x7e0000u ? 1 : 0);
  e = e < 1 ? 1 : e;
  const bool finite = top < 0x7f800000u;
  const float inv = finite ? __uint_as_float((uint32_t)(254 - e) << 23) : 0.f;
  if (in) {
    union { uint32_t w[V / 4]; int8_t c[V]; } q;
#pragma unroll
    for (int i = 0; i < V; ++i) q.c[i] = finite ? (int8_t)__float2int_rn(x[i] * inv) : (int8_t)0;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      float pdf;
      x[i] *= cdf_of<T>(x[i], &pdf);
    }
    put<T, V>(g + at, x);
#pragma unroll
    for (int i = 0; i < V / 4; ++i) reinterpret_cast<uint32_t*>(codes + at)[i] = q.w[i];
    if (c % 32 == 0) exps[row * (per * V / 32) + c / 32] = (uint8_t)(finite ? e : 255);
  }
}

template <typename T, int V>
__global__ __launch_bounds__(256) void gelu8_bwd_kernel(const int8_t* __restrict__ codes, const uint8_t* __restrict__ exps, const T* dg,
                                                        T* dh, T* __restrict__ g, int64_t pieces, int per, int F) {
  const int64_t p = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (p >= pieces) return;
  const int64_t row = p / per;
  const int c = (int)(p - row * per) * V;
  if (c >= F) return;
  const int64_t at = row * F + c;
  const float step = __uint_as_float((uint32_t)exps[row * ((F + 31) / 32) + c / 32] << 23);   // 255: infinity, times code 0 a NaN
  float x[V], d[V];
  get_codes<V>(codes + at, x);
  get<T, V>(dg + at, d);
#pragma unroll
  for (int i = 0; i < V; ++i) {
    float pdf;
    x[i] *= step;
    const float cdf = cdf_of<T>(x[i], &pdf);
    d[i] *= fmaf(x[i], pdf, cdf);
    x[i] *= cdf;
  }
  put<T, V>(dh + at, d);
  if (g) put<T, V>(g + at, x);
}

template <typename T, int V>
hipError_t fwd(const void* h, void* g, int8_t* codes, uint8_t* exps, int64_t T_, int F, hipStream_t st) {
  const int per = (F + 31) / 32 * (32 / V);
  const int64_t pieces = T_ * per;
  hipLaunchKernelGGL((gelu8_fwd_kernel<T, V>), dim3((unsigned)cdiv64(pieces, 256)), dim3(256), 0, st, (const T*)h, (T*)g, codes, exps, pieces, per, F);
  return hipGetLastError();
}
template <typename T, int V>
hipError_t bwd(const int8_t* codes, const uint8_t* exps, const void* dg, void* dh, void* g, int64_t T_, int F, hipStream_t st) {
  const int per = (F + V - 1) / V;
  const int64_t pieces = T_ * per;
  hipLaunchKernelGGL((gelu8_bwd_kernel<T, V>), dim3((unsigned)cdiv64(pieces, 256)), dim3(256), 0, st, codes, exps, (const T*)dg, (T*)dh, (T*)g, pieces, per, F);
  return hipGetLastError();
}

}  // namespace

hipError_t gelu8_fwd(int dt, const void* h, void* g, int8_t* codes, uint8_t* exps, int64_t rows, int F, hipStream_t st) {
  if (dt == 0) return fwd<float, 4>(h, g, codes, exps, rows, F, st);
  return F % 8 == 0 ? fwd<bf16, 8>(h, g, codes, exps, rows, F, st) : fwd<bf16, 4>(h, g, codes, exps, rows, F, st);
}
hipError_t gelu8_bwd(int dt, const int8_t* codes, const uint8_t* exps, const void* dg, void* dh, void* g, int64_t rows, int F, hipStream_t st) {
  if (dt == 0) return bwd<float, 4>(codes, exps, dg, dh, g, rows, F, st);
  return F % 8 == 0 ? bwd<bf16, 8>(codes, exps, dg, dh, g, rows, F, st) : bwd<bf16, 4>(codes, exps, dg, dh, g, rows, F, st);
}

}  // namespace pt
