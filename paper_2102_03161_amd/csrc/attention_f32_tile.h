// Tiles and fragments of the attention kernels on the fp32 matrix instructions (v_mfma_f32_16x16x4_f32), shared by the kernels
// without a mask (attention.hip) and those under a rule (attention_rules_f32.hip).
#pragma once
#include "common.h"

namespace pt {

typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x4 load4(const float* p) { return *reinterpret_cast<const f32x4*>(p); }
__device__ __forceinline__ f32x4 load4(const bf16* p) {
  union { uint2 u; bf16 h[4]; } t;
  t.u = *reinterpret_cast<const uint2*>(p);
  return f32x4{to_f32(t.h[0]), to_f32(t.h[1]), to_f32(t.h[2]), to_f32(t.h[3])};
}
__device__ __forceinline__ void store4(float* p, f32x4 v) { *reinterpret_cast<f32x4*>(p) = v; }
__device__ __forceinline__ void store4(bf16* p, f32x4 v) {
  union { uint2 u; bf16 h[4]; } t;
#pragma unroll
  for (int i = 0; i < 4; ++i) t.h[i] = from_f32<bf16>(v[i]);
  *reinterpret_cast<uint2*>(p) = t.u;
}

constexpr int kAttnRows = 64;   // rows of a streamed tile, and rows owned by a workgroup of four waves

// DP: the head size rounded up to 16, 32, 64 or 128; columns from dh on are zeros
template <typename T, int DP>
struct AttnTile {
  static constexpr int LD = DP + 4;          // conflict-free for 16-byte reads of 16 rows and for single floats of 4 x 16
  static constexpr int FLOATS = kAttnRows * LD;
  static constexpr int N4 = DP / 16;         // pieces of four elements per thread
  static constexpr int NF = DP / 16;         // fragments of 16 columns
  static __device__ __forceinline__ void place(int tid, int i, int* row, int* d) {
    const int c = tid + 256 * i;
    *row = c / (DP / 4);
    *d = (c % (DP / 4)) * 4;
  }
  static __device__ __forceinline__ void load(const T* p, int64_t ld, int r0, int S, int dh, int tid, f32x4 (&reg)[N4]) {
#pragma unroll
    for (int i = 0; i < N4; ++i) {
      int row, d;
      place(tid, i, &row, &d);
      reg[i] = r0 + row < S && d < dh ? load4(p + (int64_t)(r0 + row) * ld + d) : f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }
  static __device__ __forceinline__ void store(float* s, int tid, const f32x4 (&reg)[N4]) {
#pragma unroll
    for (int i = 0; i < N4; ++i) {
      int row, d;
      place(tid, i, &row, &d);
      *reinterpret_cast<f32x4*>(s + row * LD + d) = reg[i];
    }
  }
  // an owned row's operand: lane group g holds columns 16 q + 4 g .. + 3 of row lane % 16
  static __device__ __forceinline__ void own(const T* p, int64_t ld, int row, int S, int dh, int g, float f, f32x4 (&reg)[NF]) {
#pragma unroll
    for (int q = 0; q < NF; ++q) {
      const int d = 16 * q + 4 * g;
      reg[q] = row < S && d < dh ? load4(p + (int64_t)row * ld + d) * f : f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }
  // rows r0 + 0..15 of the tile times the owned rows, over the columns
  static __device__ __forceinline__ f32x4 dot(const float* s, int r0, int l, int g, const f32x4 (&own_)[NF]) {
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int q = 0; q < NF; ++q) {
      const f32x4 a = *reinterpret_cast<const f32x4*>(s + (r0 + l) * LD + 16 * q + 4 * g);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], own_[q][e], acc, 0, 0, 0);
    }
    return acc;
  }
  // acc (columns 16 n + 4 g + v of the owned rows) += sum over rows r0 + 0..15 of tile row x weight
  static __device__ __forceinline__ void add(const float* s, int r0, int l, int g, f32x4 w, f32x4 (&acc)[NF]) {
#pragma unroll
    for (int v = 0; v < 4; ++v)
#pragma unroll
      for (int n = 0; n < NF; ++n)
        acc[n] = __builtin_amdgcn_mfma_f32_16x16x4f32(s[(r0 + 4 * g + v) * LD + 16 * n + l], w[v], acc[n], 0, 0, 0);
  }
  static __device__ __forceinline__ void put(T* p, int dh, int g, float f, const f32x4 (&acc)[NF]) {
#pragma unroll
    for (int n = 0; n < NF; ++n)
      if (16 * n + 4 * g < dh) store4(p + 16 * n + 4 * g, acc[n] * f);
  }
};

__device__ __forceinline__ float group_sum(float v) {   // over the four lane groups
  v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}

}  // namespace pt
