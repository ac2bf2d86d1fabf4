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
// of 32 is 4 or 8 neighbouring lanes.  Memory bounds both: in bf16 a value moves 5 bytes forward (2 in, 2 + 1 out) and 7 back.
// 32768 x 4096 values take 114 us forward (5.9 TB/s) and 160 back (5.9 TB/s), where a large copy reaches 5.1 TB/s (its reads and
// writes are equal, these read more or less than they write); 12608 x 1540, in pieces of 8 bytes, 25 us back (5.5 TB/s); 231 x 1024
// 3 us each, a launch.
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
// four codes in a word.  Adding 1.5 2^23 to a number of at most 127 leaves it, rounded to nearest even, in the last byte.
__device__ __forceinline__ uint32_t encode4(const float* x, float inv) {
  constexpr float kRound = 12582912.f;
  const uint32_t a = __float_as_uint(fmaf(x[0], inv, kRound)), b = __float_as_uint(fmaf(x[1], inv, kRound));
  const uint32_t c = __float_as_uint(fmaf(x[2], inv, kRound)), d = __float_as_uint(fmaf(x[3], inv, kRound));
  return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0c0c0400), __builtin_amdgcn_perm(b, a, 0x0c0c0400), 0x05040100);
}
// code step; the code as an unsigned byte 128 larger, which converts in one instruction (step infinite: 0 times it, a NaN)
__device__ __forceinline__ void decode4(uint32_t w, float step, float* x) {
  w ^= 0x80808080u;
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = ((float)(w >> (8 * i) & 0xffu) - 128.f) * step;
}

// Phi, and phi.  bf16 results: the rational approximation of erfc of gelu_cdf() (4e-7 absolute: 0.2 % of Phi at -5 and 1 % at -8, where x
// Phi(x) is 1e-6 and 5e-15), with the factors folded into its coefficients; fp32 results: the library's erfc and exp.
template <typename T> __device__ __forceinline__ float cdf_of(float x, float* pdf);
template <> __device__ __forceinline__ float cdf_of<bf16>(float x, float* pdf) {
  const float t = __builtin_amdgcn_rcpf(fmaf(0.23164189f, fabsf(x), 1.0f));
  const float e = __builtin_amdgcn_exp2f(x * (x * -0.72134752044448170f));   // exp(-x*x/2)
  const float q = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 0.5307027145f, -0.7265760135f), 0.7107068705f), -0.142248368f), 0.127414796f) * e;
  *pdf = e * 0.39894228040143268f;
  return x < 0.f ? q : 1.0f - q;
}
template <> __device__ __forceinline__ float cdf_of<float>(float x, float* pdf) {
  *pdf = expf(-0.5f * x * x) * 0.39894228040143268f;
  return 0.5f * erfcf(x * -0.70710678118654752f);
}

// the largest magnitude of a block of 32: of the thread's values, then of its 32 / V neighbours (a quad, or two)
template <int V>
__device__ __forceinline__ uint32_t block_top(uint32_t top) {
  auto with = [&](uint32_t o) { top = o > top ? o : top; };
  with(__builtin_amdgcn_update_dpp(0, top, 0xb1, 0xf, 0xf, true));                  // lane ^ 1
  with(__builtin_amdgcn_update_dpp(0, top, 0x4e, 0xf, 0xf, true));                  // lane ^ 2
  if (V == 4) with(__builtin_amdgcn_update_dpp(0, top, 0x141, 0xf, 0xf, true));     // the other quad of eight
  return top;
}

// Where a thread's piece of V values lies.  A row has `per` pieces; where F is no multiple of 32 the forward pass pads rows to whole
// blocks, so that a block is always the same neighbouring lanes.  Division by `per` is a multiplication (p < 2^31).
struct Pieces {
  uint32_t n, per, mul, shift;
  Pieces(int64_t rows, uint32_t per_) : n((uint32_t)(rows * per_)), per(per_) {
    shift = 0;
    while ((1ull << shift) < per) ++shift;
    mul = (uint32_t)(((1ull << 32) * ((1ull << shift) - per)) / per + 1);
  }
  __device__ __forceinline__ uint32_t row(uint32_t p) const {
    const uint32_t t = __umulhi(mul, p);
    return shift == 0 ? p : (t + ((p - t) >> 1)) >> (shift - 1);
  }
};

template <typename T, int V>
__global__ __launch_bounds__(256) void gelu8_fwd_kernel(const T* __restrict__ h, T* __restrict__ g, int8_t* __restrict__ codes,
                                                        uint8_t* __restrict__ exps, Pieces ps, int F) {
  const uint32_t p = blockIdx.x * 256 + threadIdx.x;
  if (p >= ps.n) return;   // whole blocks of 32 leave together
  const uint32_t row = ps.row(p);
  const int c = (int)(p - row * ps.per) * V;
  const bool in = c < F;
  const int64_t at = (int64_t)row * F + c;
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
  top = block_top<V>(top);
  // top = 1.f 2^(E - 127) fits into 127 steps of 2^(E - 133) if 1.f <= 127 / 64, else into steps twice as large
  int e = (int)(top >> 23) - 6 + ((top & 0x7fffffu) > 0x7e0000u ? 1 : 0);
  e = e < 1 ? 1 : e;
  const bool finite = top < 0x7f800000u;
  if (!in) return;
  const float inv = __uint_as_float((uint32_t)(254 - e) << 23);
  uint32_t q[V / 4];
#pragma unroll
  for (int i = 0; i < V / 4; ++i) q[i] = finite ? encode4(x + 4 * i, inv) : 0u;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    float pdf;
    x[i] *= cdf_of<T>(x[i], &pdf);
  }
  put<T, V>(g + at, x);
  if (V == 8) *reinterpret_cast<uint2*>(codes + at) = make_uint2(q[0], q[V / 4 - 1]);
  else *reinterpret_cast<uint32_t*>(codes + at) = q[0];
  if (c % 32 == 0) exps[(int64_t)row * ((F + 31) / 32) + c / 32] = (uint8_t)(finite ? e : 255);
}

template <typename T, int V>
__global__ __launch_bounds__(256) void gelu8_bwd_kernel(const int8_t* __restrict__ codes, const uint8_t* __restrict__ exps, const T* dg,
                                                        T* dh, T* __restrict__ g, Pieces ps, int F) {
  const uint32_t p = blockIdx.x * 256 + threadIdx.x;
  if (p >= ps.n) return;
  const uint32_t row = ps.row(p);
  const int c = (int)(p - row * ps.per) * V;
  const int64_t at = (int64_t)row * F + c;
  uint32_t q[V / 4];
  if (V == 8) {
    const uint2 w = *reinterpret_cast<const uint2*>(codes + at);
    q[0] = w.x; q[V / 4 - 1] = w.y;
  } else {
    q[0] = *reinterpret_cast<const uint32_t*>(codes + at);
  }
  const float step = __uint_as_float((uint32_t)exps[(int64_t)row * ((F + 31) / 32) + c / 32] << 23);   // 255: infinity
  float x[V], d[V];
  get<T, V>(dg + at, d);
#pragma unroll
  for (int i = 0; i < V / 4; ++i) decode4(q[i], step, x + 4 * i);
#pragma unroll
  for (int i = 0; i < V; ++i) {
    float pdf;
    const float cdf = cdf_of<T>(x[i], &pdf);
    d[i] *= fmaf(x[i], pdf, cdf);
    x[i] *= cdf;
  }
  put<T, V>(dh + at, d);
  if (g) put<T, V>(g + at, x);
}

template <typename T, int V>
hipError_t fwd(const void* h, void* g, int8_t* codes, uint8_t* exps, int64_t rows, int F, hipStream_t st) {
  const Pieces ps(rows, (uint32_t)((F + 31) / 32 * (32 / V)));
  hipLaunchKernelGGL((gelu8_fwd_kernel<T, V>), dim3((ps.n + 255) / 256), dim3(256), 0, st, (const T*)h, (T*)g, codes, exps, ps, F);
  return hipGetLastError();
}
template <typename T, int V>
hipError_t bwd(const int8_t* codes, const uint8_t* exps, const void* dg, void* dh, void* g, int64_t rows, int F, hipStream_t st) {
  const Pieces ps(rows, (uint32_t)(F / V));
  hipLaunchKernelGGL((gelu8_bwd_kernel<T, V>), dim3((ps.n + 255) / 256), dim3(256), 0, st, codes, exps, (const T*)dg, (T*)dh, (T*)g, ps, F);
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
