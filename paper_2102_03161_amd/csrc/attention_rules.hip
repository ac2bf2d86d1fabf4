// Softmax attention under a rule, forward and backward, bf16 (the fp32 kernels are in attention_rules_f32.hip).
//
//   t_ij = scale q_i . k_j      s_ij = cap tanh(t_ij / cap) - slope_h |q0 + i - j|      (cap and slopes optional)
//   p_i  = softmax over the keys that query i sees          o_i = sum_j p_ij v_j
//   dS = p (dP - delta), dP_ij = dO_i . v_j, delta_i = dO_i . o_i;   dT = dS (1 - tanh^2);   dq = scale dT k, dk = scale dT^T q
//
// What a query sees: keys up to lim_i (its own position, the end of the sample's prefix, or the last key) of its own document.
//
// One wave owns 32 rows (queries in the forward pass and for dq, keys for dk / dv); a workgroup of four waves streams the other
// side through LDS in tiles of 64 rows.  Scores are computed with the owned row as the MFMA's column, so that softmax statistics
// are one value per lane and the probabilities, rounded to bf16, are the next MFMA's operand as they stand in registers.
//
// Work that a mask leaves out is not done: before anything else a workgroup writes the list of the tiles that any of its waves
// needs, each with four bits "this wave needs it" and four bits "all 32 x 64 pairs of this wave are visible".  Only tiles without
// the latter bit are masked pair by pair.  The list is built from the documents' ids as they are, in any order.
#include <algorithm>

#include "attention_rules.h"

namespace pt {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef __attribute__((__vector_size__(4 * sizeof(__bf16)))) __bf16 bf16x4;
typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16;

namespace {

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float half_swap(float x) { return __shfl_xor(x, 32, 64); }

// accumulator register v of a 32x32 tile holds tile row 8*(v/4) + 4*half + v%4 (column = lane%32)
__device__ __forceinline__ int acc_row(int v, int half) { return 8 * (v >> 2) + 4 * half + (v & 3); }
__device__ __forceinline__ f32x16 zero16() {
  f32x16 z;
#pragma unroll
  for (int v = 0; v < 16; ++v) z[v] = 0.f;
  return z;
}
__device__ __forceinline__ bf16x8 pack8(const f32x16& a, int first) {
  bf16x8 r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = from_f32<bf16>(a[first + i]);
  return r;
}

// DP: the head size rounded up to 64 or 128; columns from dh on are zeros
template <int DP>
struct Tile {
  static constexpr int LD = DP + 8;                   // 16-byte row reads without conflicts
  static constexpr int ELEMS = kRuleTile * LD;
  static constexpr int N = kRuleTile * DP / 8 / 256;  // 16-byte pieces per thread
  static constexpr int KS = DP / 16;                  // k steps of a product over the head size
  static constexpr int DT = DP / 32;                  // 32-column tiles of the head size
  static __device__ __forceinline__ int row_of(int tid, int u) { return (tid + 256 * u) / (DP / 8); }
  static __device__ __forceinline__ int col_of(int tid) { return (tid % (DP / 8)) * 8; }
  static __device__ __forceinline__ uint4 load(const bf16* p, int64_t ld, int row, int n, int col, int dh) {
    return row < n && col < dh ? *reinterpret_cast<const uint4*>(p + row * ld + col) : make_uint4(0, 0, 0, 0);
  }
  static __device__ __forceinline__ void store(bf16* s, int tid, int u, uint4 x, bool keep) {
    *reinterpret_cast<uint4*>(s + row_of(tid, u) * LD + col_of(tid)) = keep ? x : make_uint4(0, 0, 0, 0);
  }
  // the wave's own row as an operand: columns 16 ks + 8 half .. + 7
  static __device__ __forceinline__ void own(const bf16* row, bool ok, int dh, int half, bf16x8 (&f)[KS]) {
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      union { uint4 u; bf16x8 v; } t;
      const int col = 16 * ks + 8 * half;
      t.u = ok && col < dh ? *reinterpret_cast<const uint4*>(row + col) : make_uint4(0, 0, 0, 0);
      f[ks] = t.v;
    }
  }
  // rows r0 .. r0 + 31 of the tile times the owned rows
  static __device__ __forceinline__ f32x16 dot(const bf16* s, int r0, int lane, const bf16x8 (&f)[KS]) {
    f32x16 acc = zero16();
    const bf16* p = s + (r0 + (lane & 31)) * LD + (lane >> 5) * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
      acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(p + 16 * ks), f[ks], acc, 0, 0, 0);
    return acc;
  }
  // acc[dt] (columns 32 dt + .. of the owned rows) += sum over rows r0 .. r0 + 31 of tile row x weight; the transposing LDS read
  // hands a lane four consecutive rows of one column, in the order in which the weights stand in the accumulator
  static __device__ __forceinline__ void add(const bf16* s, int r0, int lane, const f32x16& w, f32x16 (&acc)[DT]) {
    const int l16 = lane & 15, grp = lane >> 4;
    const bf16* p = s + (r0 + 4 * (grp >> 1) + (l16 >> 2)) * LD + 16 * (grp & 1) + 4 * (l16 & 3);
#pragma unroll
    for (int ks2 = 0; ks2 < 2; ++ks2) {
      const bf16x8 b = pack8(w, 8 * ks2);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        typedef __attribute__((address_space(3))) bf16x4 lds4;
        const bf16* q = p + 16 * ks2 * LD + 32 * dt;
        union { bf16x4 h[2]; bf16x8 v; } t;
        t.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds4*)(q));
        t.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds4*)(q + 8 * LD));
        acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(t.v, b, acc[dt], 0, 0, 0);
      }
    }
  }
  static __device__ __forceinline__ void put(bf16* row, int dh, int half, float f, const f32x16 (&acc)[DT]) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int col = 32 * dt + 8 * g + 4 * half;
        union { bf16 h[4]; uint2 u; } t;
#pragma unroll
        for (int e = 0; e < 4; ++e) t.h[e] = from_f32<bf16>(acc[dt][4 * g + e] * f);
        if (col < dh) *reinterpret_cast<uint2*>(row + col) = t.u;
      }
  }
};

// Scores in the log2 domain.  tanh(x) = 1 - 2 r with r = 1 / (1 + e^2x), which needs no case for large |x|; its derivative
// 4 r (1 - r) has no cancellation.  The absolute error of 1e-7 cap that this form has near zero is far below a bf16 score's.
struct Score {
  float c, e1, a, sl;
  __device__ __forceinline__ Score(const AttnRuleArgs& g, int h) {
    constexpr float kLog2e = 1.44269504088896f;
    c = g.scale * kLog2e;
    e1 = g.cap > 0.f ? 2.f * c / g.cap : 0.f;
    a = g.cap * kLog2e;
    sl = g.slopes ? -g.slopes[h] * kLog2e : 0.f;
  }
  __device__ __forceinline__ float bend(float s) const { return __builtin_amdgcn_rcpf(1.f + fast_exp2(s * e1)); }   // r
  // dist: |position of the query - position of the key|
  template <int MOD>
  __device__ __forceinline__ float at(float s, float dist) const {
    float x = (MOD & 1) ? fmaf(-2.f * a, bend(s), a) : s * c;
    return (MOD & 2) ? fmaf(sl, dist, x) : x;
  }
};

// ---------------------------------------------------------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------------------------------------------------------
template <int DP, int MOD>
__global__ __launch_bounds__(256) void rule_fwd_kernel(AttnRuleArgs g) {
  typedef Tile<DP> T;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  bf16* buf = reinterpret_cast<bf16*>(smem);                                  // [2][K tile, V tile]
  int* kdoc = reinterpret_cast<int*>(buf + 4 * T::ELEMS);                     // [2][64]
  RuleList list(reinterpret_cast<int*>(kdoc + 2 * kRuleTile));
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5;
  const int nqb = (g.Sq + 127) / 128;
  const RuleUnit u(g, nqb, g.H);
  const int b = u.b, h = u.h, hk = h / (g.H / g.Hkv);
  const int i = u.blk * 128 + wave * 32 + (lane & 31);
  const RuleRows rows(g, b);
  const int lim = rows.lim(g, i), qd = rows.qdoc(g, i);
  const bool ok = i < g.Sq;
  const int n = list.keys(g, rows, wave, lane, ok, lim, qd);
  bf16x8 qf[T::KS];
  T::own(static_cast<const bf16*>(g.q.p) + b * g.q.b + (int64_t)i * g.q.t + h * g.q.h, ok && qd >= 0, g.dh, half, qf);
  const bf16* kp = static_cast<const bf16*>(g.k.p) + b * g.k.b + hk * g.k.h;
  const bf16* vp = static_cast<const bf16*>(g.v.p) + b * g.v.b + hk * g.v.h;
  const Score sc(g, h);
  f32x16 o[T::DT];
#pragma unroll
  for (int dt = 0; dt < T::DT; ++dt) o[dt] = zero16();
  float m = -1e30f, lsum = 0.f;
  uint4 rk[T::N], rv[T::N];
  int rd[T::N];
  auto load = [&](int it) {
    const int j0 = list.tile(it) * kRuleTile;
#pragma unroll
    for (int x = 0; x < T::N; ++x) {
      const int j = j0 + T::row_of(tid, x);
      rk[x] = T::load(kp, g.k.t, j, g.Sk, T::col_of(tid), g.dh);
      rv[x] = T::load(vp, g.v.t, j, g.Sk, T::col_of(tid), g.dh);
      rd[x] = rows.kdoc(g, j);
    }
  };
  auto store = [&](int it) {
    bf16* kb = buf + (it & 1) * 2 * T::ELEMS;
#pragma unroll
    for (int x = 0; x < T::N; ++x) {
      T::store(kb, tid, x, rk[x], rd[x] >= 0);
      T::store(kb + T::ELEMS, tid, x, rv[x], rd[x] >= 0);
      if (T::col_of(tid) == 0) kdoc[(it & 1) * kRuleTile + T::row_of(tid, x)] = rd[x];
    }
  };
  if (n > 0) { load(0); store(0); }
  for (int it = 0; it < n; ++it) {
    __syncthreads();
    if (it + 1 < n) load(it + 1);
    if (list.needed(it, wave)) {
      const bf16* kb = buf + (it & 1) * 2 * T::ELEMS;
      const int j0 = list.tile(it) * kRuleTile;
      const bool full = list.full(it, wave);
      f32x16 s[2];
#pragma unroll
      for (int st = 0; st < 2; ++st) s[st] = T::dot(kb, 32 * st, lane, qf);
      const float at = (float)(g.q0 + i - j0);
#pragma unroll
      for (int st = 0; st < 2; ++st)
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (MOD) s[st][v] = sc.at<MOD>(s[st][v], fabsf(at - (float)(32 * st + acc_row(v, half))));
      if (!full) {
#pragma unroll
        for (int st = 0; st < 2; ++st)
#pragma unroll
          for (int g4 = 0; g4 < 4; ++g4) {
            const int r0 = 32 * st + 8 * g4 + 4 * half;
            const int4 kd = *reinterpret_cast<const int4*>(kdoc + (it & 1) * kRuleTile + r0);
            const int kds[4] = {kd.x, kd.y, kd.z, kd.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) s[st][4 * g4 + e] = kds[e] == qd && j0 + r0 + e <= lim ? s[st][4 * g4 + e] : -INFINITY;
          }
      }
      float mx = fmaxf(s[0][0], s[1][0]);
#pragma unroll
      for (int v = 1; v < 16; ++v) mx = fmaxf(mx, fmaxf(s[0][v], s[1][v]));
      mx = fmaxf(mx, half_swap(mx));
      if (!MOD) mx *= sc.c;
      // the reference maximum only has to keep exp2 in range: it moves when a row's maximum has grown by more than 2^8
      if (__any(mx > m + 8.f)) {
        const float mn = mx > m + 8.f ? mx : m;
        const float alpha = fast_exp2(m - mn);
        lsum *= alpha;
        m = mn;
#pragma unroll
        for (int dt = 0; dt < T::DT; ++dt)
#pragma unroll
          for (int v = 0; v < 16; ++v) o[dt][v] *= alpha;
      }
#pragma unroll
      for (int st = 0; st < 2; ++st) {
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          s[st][v] = fast_exp2(MOD ? s[st][v] - m : fmaf(s[st][v], sc.c, -m));
          lsum += s[st][v];
        }
        T::add(kb + T::ELEMS, 32 * st, lane, s[st], o);
      }
    }
    if (it + 1 < n) store(it + 1);
  }
  lsum += half_swap(lsum);
  if (!ok) return;
  T::put(static_cast<bf16*>(const_cast<void*>(g.o.p)) + b * g.o.b + (int64_t)i * g.o.t + h * g.o.h, g.dh, half, lsum > 0.f ? 1.f / lsum : 0.f, o);
  if (g.lse && half == 0) g.lse[(int64_t)b * g.lse_b + (int64_t)h * g.lse_h + i] = lsum > 0.f ? (m + __log2f(lsum)) * 0.693147180559945f : -INFINITY;
}

// ---------------------------------------------------------------------------------------------------------------------------
// backward: delta, then one launch whose workgroups take dk / dv of 128 keys (first) or dq of 128 queries
// ---------------------------------------------------------------------------------------------------------------------------
// p of 1 means a query that sees one key: dS is exactly 0 then, where dP - delta would leave the rounding of two different sums
constexpr float kOneKey = 1.f - 1.f / 65536.f;

template <int DP, int MOD>
__device__ __forceinline__ void rule_dq(const AttnRuleArgs& g, int unit, unsigned char* smem) {
  typedef Tile<DP> T;
  bf16* buf = reinterpret_cast<bf16*>(smem);
  int* kdoc = reinterpret_cast<int*>(buf + 4 * T::ELEMS);
  RuleList list(reinterpret_cast<int*>(kdoc + 2 * kRuleTile));
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5;
  const int nqb = (g.Sq + 127) / 128;
  const RuleUnit u(g, nqb, g.H, unit);
  const int b = u.b, h = u.h, hk = h / (g.H / g.Hkv);
  const int i = u.blk * 128 + wave * 32 + (lane & 31);
  const RuleRows rows(g, b);
  const int lim = rows.lim(g, i), qd = rows.qdoc(g, i);
  const bool ok = i < g.Sq, on = ok && qd >= 0;
  const int n = list.keys(g, rows, wave, lane, ok, lim, qd);
  bf16x8 qf[T::KS], dof[T::KS];
  T::own(static_cast<const bf16*>(g.q.p) + b * g.q.b + (int64_t)i * g.q.t + h * g.q.h, on, g.dh, half, qf);
  T::own(static_cast<const bf16*>(g.d_o.p) + b * g.d_o.b + (int64_t)i * g.d_o.t + h * g.d_o.h, on, g.dh, half, dof);
  const bf16* kp = static_cast<const bf16*>(g.k.p) + b * g.k.b + hk * g.k.h;
  const bf16* vp = static_cast<const bf16*>(g.v.p) + b * g.v.b + hk * g.v.h;
  const Score sc(g, h);
  const float lse2 = on ? rule_lse2(g.lse[(int64_t)b * g.lse_b + (int64_t)h * g.lse_h + i]) : INFINITY;
  const float dl = on ? g.delta[((int64_t)b * g.H + h) * g.Sq + i] : 0.f;
  f32x16 dq[T::DT];
#pragma unroll
  for (int dt = 0; dt < T::DT; ++dt) dq[dt] = zero16();
  uint4 rk[T::N], rv[T::N];
  int rd[T::N];
  auto load = [&](int it) {
    const int j0 = list.tile(it) * kRuleTile;
#pragma unroll
    for (int x = 0; x < T::N; ++x) {
      const int j = j0 + T::row_of(tid, x);
      rk[x] = T::load(kp, g.k.t, j, g.Sk, T::col_of(tid), g.dh);
      rv[x] = T::load(vp, g.v.t, j, g.Sk, T::col_of(tid), g.dh);
      rd[x] = rows.kdoc(g, j);
    }
  };
  auto store = [&](int it) {
    bf16* kb = buf + (it & 1) * 2 * T::ELEMS;
#pragma unroll
    for (int x = 0; x < T::N; ++x) {
      T::store(kb, tid, x, rk[x], rd[x] >= 0);
      T::store(kb + T::ELEMS, tid, x, rv[x], rd[x] >= 0);
      if (T::col_of(tid) == 0) kdoc[(it & 1) * kRuleTile + T::row_of(tid, x)] = rd[x];
    }
  };
  if (n > 0) { load(0); store(0); }
  for (int it = 0; it < n; ++it) {
    __syncthreads();
    if (it + 1 < n) load(it + 1);
    if (list.needed(it, wave)) {
      const bf16* kb = buf + (it & 1) * 2 * T::ELEMS;
      const int j0 = list.tile(it) * kRuleTile;
      const bool full = list.full(it, wave);
      const float at = (float)(g.q0 + i - j0);
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        f32x16 s = T::dot(kb, 32 * st, lane, qf);
        const f32x16 dp = T::dot(kb + T::ELEMS, 32 * st, lane, dof);
        float ds[16];
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const float x = sc.at<MOD>(s[v], fabsf(at - (float)(32 * st + acc_row(v, half))));
          const float p = fast_exp2(x - lse2);
          ds[v] = p * (dp[v] - dl);
          if (!full) ds[v] = p < kOneKey ? ds[v] : 0.f;
          if (MOD & 1) { const float r = sc.bend(s[v]); ds[v] *= 4.f * r * (1.f - r); }
        }
        if (!full) {
#pragma unroll
          for (int g4 = 0; g4 < 4; ++g4) {
            const int r0 = 32 * st + 8 * g4 + 4 * half;
            const int4 kd = *reinterpret_cast<const int4*>(kdoc + (it & 1) * kRuleTile + r0);
            const int kds[4] = {kd.x, kd.y, kd.z, kd.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) ds[4 * g4 + e] = kds[e] == qd && j0 + r0 + e <= lim ? ds[4 * g4 + e] : 0.f;
          }
        }
#pragma unroll
        for (int v = 0; v < 16; ++v) s[v] = ds[v];
        T::add(kb, 32 * st, lane, s, dq);
      }
    }
    if (it + 1 < n) store(it + 1);
  }
  if (ok) T::put(static_cast<bf16*>(const_cast<void*>(g.dq.p)) + b * g.dq.b + (int64_t)i * g.dq.t + h * g.dq.h, g.dh, half, g.scale, dq);
}

template <int DP, int MOD>
__device__ __forceinline__ void rule_dkv(const AttnRuleArgs& g, int unit, unsigned char* smem) {
  typedef Tile<DP> T;
  bf16* buf = reinterpret_cast<bf16*>(smem);                                  // [2][Q tile, dO tile]
  float* stat = reinterpret_cast<float*>(buf + 4 * T::ELEMS);                 // [2][lse, delta][64]
  int* info = reinterpret_cast<int*>(stat + 4 * kRuleTile);                   // [2][document, lim][64]
  RuleList list(info + 4 * kRuleTile);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5;
  const int nkb = (g.Sk + 127) / 128, G = g.H / g.Hkv;
  const RuleUnit u(g, nkb, g.Hkv, unit);
  const int b = u.b, hk = u.h;
  const int j = u.blk * 128 + wave * 32 + (lane & 31);
  const RuleRows rows(g, b);
  const int kd = rows.kdoc(g, j);
  const bool ok = j < g.Sk, on = ok && kd >= 0;
  const int n = list.queries(g, rows, wave, lane, ok, j, kd);
  bf16x8 kf[T::KS], vf[T::KS];
  T::own(static_cast<const bf16*>(g.k.p) + b * g.k.b + (int64_t)j * g.k.t + hk * g.k.h, on, g.dh, half, kf);
  T::own(static_cast<const bf16*>(g.v.p) + b * g.v.b + (int64_t)j * g.v.t + hk * g.v.h, on, g.dh, half, vf);
  f32x16 dk[T::DT], dv[T::DT];
#pragma unroll
  for (int dt = 0; dt < T::DT; ++dt) { dk[dt] = zero16(); dv[dt] = zero16(); }
  uint4 rq[T::N], ro[T::N];
  int rd[T::N];
  float rl = 0.f, rdl = 0.f;
  int rid = 0, rlim = 0;
  auto load = [&](int it) {
    const int h = hk * G + it / n, i0 = list.tile(it % n) * kRuleTile;
    const bf16* qp = static_cast<const bf16*>(g.q.p) + b * g.q.b + h * g.q.h;
    const bf16* op = static_cast<const bf16*>(g.d_o.p) + b * g.d_o.b + h * g.d_o.h;
#pragma unroll
    for (int x = 0; x < T::N; ++x) {
      const int i = i0 + T::row_of(tid, x);
      rq[x] = T::load(qp, g.q.t, i, g.Sq, T::col_of(tid), g.dh);
      ro[x] = T::load(op, g.d_o.t, i, g.Sq, T::col_of(tid), g.dh);
      rd[x] = rows.qdoc(g, i);
    }
    if (tid < kRuleTile) {
      const int i = i0 + tid;
      const bool in = i < g.Sq;
      rid = rows.qdoc(g, i);
      rlim = rows.lim(g, i);
      rl = in ? rule_lse2(g.lse[(int64_t)b * g.lse_b + (int64_t)h * g.lse_h + i]) : INFINITY;
      rdl = in ? g.delta[((int64_t)b * g.H + h) * g.Sq + i] : 0.f;
    }
  };
  auto store = [&](int it) {
    bf16* qb = buf + (it & 1) * 2 * T::ELEMS;
#pragma unroll
    for (int x = 0; x < T::N; ++x) {
      T::store(qb, tid, x, rq[x], rd[x] >= 0);
      T::store(qb + T::ELEMS, tid, x, ro[x], rd[x] >= 0);
    }
    if (tid < kRuleTile) {
      const int at = (it & 1) * 2 * kRuleTile + tid;
      stat[at] = rid >= 0 ? rl : INFINITY;
      stat[at + kRuleTile] = rdl;
      info[at] = rid;
      info[at + kRuleTile] = rlim;
    }
  };
  const int total = n * G;
  if (total > 0) { load(0); store(0); }
  for (int it = 0; it < total; ++it) {
    __syncthreads();
    if (it + 1 < total) load(it + 1);
    const int item = it % n;
    if (list.needed(item, wave)) {
      const bf16* qb = buf + (it & 1) * 2 * T::ELEMS;
      const float* st2 = stat + (it & 1) * 2 * kRuleTile;
      const int* inf = info + (it & 1) * 2 * kRuleTile;
      const Score sc(g, hk * G + it / n);
      const bool full = list.full(item, wave);
      const float at = (float)(g.q0 + list.tile(item) * kRuleTile - j);
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        f32x16 s = T::dot(qb, 32 * st, lane, kf);
        f32x16 ds = T::dot(qb + T::ELEMS, 32 * st, lane, vf);
#pragma unroll
        for (int g4 = 0; g4 < 4; ++g4) {
          const int r0 = 32 * st + 8 * g4 + 4 * half;
          const float4 l4 = *reinterpret_cast<const float4*>(st2 + r0);
          const float4 d4 = *reinterpret_cast<const float4*>(st2 + kRuleTile + r0);
          const float ls[4] = {l4.x, l4.y, l4.z, l4.w}, dl[4] = {d4.x, d4.y, d4.z, d4.w};
          float p[4], d[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int v = 4 * g4 + e;
            p[e] = fast_exp2(sc.at<MOD>(s[v], fabsf(at + (float)(r0 + e))) - ls[e]);
            d[e] = p[e] * (ds[v] - dl[e]);
            if (MOD & 1) { const float r = sc.bend(s[v]); d[e] *= 4.f * r * (1.f - r); }
          }
          if (!full) {
            const int4 qd4 = *reinterpret_cast<const int4*>(inf + r0);
            const int4 lm4 = *reinterpret_cast<const int4*>(inf + kRuleTile + r0);
            const int qds[4] = {qd4.x, qd4.y, qd4.z, qd4.w}, lms[4] = {lm4.x, lm4.y, lm4.z, lm4.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const bool see = qds[e] == kd && j <= lms[e];
              d[e] = see && p[e] < kOneKey ? d[e] : 0.f;
              p[e] = see ? p[e] : 0.f;
            }
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) { s[4 * g4 + e] = p[e]; ds[4 * g4 + e] = d[e]; }
        }
        T::add(qb + T::ELEMS, 32 * st, lane, s, dv);
        T::add(qb, 32 * st, lane, ds, dk);
      }
    }
    if (it + 1 < total) store(it + 1);
  }
  if (ok) {
    T::put(static_cast<bf16*>(const_cast<void*>(g.dk.p)) + b * g.dk.b + (int64_t)j * g.dk.t + hk * g.dk.h, g.dh, half, g.scale, dk);
    T::put(static_cast<bf16*>(const_cast<void*>(g.dv.p)) + b * g.dv.b + (int64_t)j * g.dv.t + hk * g.dv.h, g.dh, half, 1.f, dv);
  }
}

template <int DP, int MOD>
__global__ __launch_bounds__(256) void rule_bwd_kernel(AttnRuleArgs g, int ndkv) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  if ((int)blockIdx.x < ndkv) rule_dkv<DP, MOD>(g, blockIdx.x, smem);
  else rule_dq<DP, MOD>(g, blockIdx.x - ndkv, smem);
}

template <int DP>
size_t lds_bytes(int Sq, int Sk, bool bwd) {
  const int nt = (std::max(bwd ? Sq : 0, Sk) + kRuleTile - 1) / kRuleTile;
  return (size_t)4 * Tile<DP>::ELEMS * 2 + (bwd ? 8 : 2) * kRuleTile * 4 + RuleList::ints(nt) * 4;
}

template <int DP, int MOD>
hipError_t launch_fwd(const AttnRuleArgs& g, hipStream_t st) {
  const size_t lds = lds_bytes<DP>(g.Sq, g.Sk, false);
  const int blocks = g.nb * g.H * ((g.Sq + 127) / 128);
  PT_RULE_LDS((rule_fwd_kernel<DP, MOD>), lds);
  hipLaunchKernelGGL((rule_fwd_kernel<DP, MOD>), dim3(blocks), dim3(256), lds, st, g);
  return hipGetLastError();
}
template <int DP, int MOD>
hipError_t launch_bwd(const AttnRuleArgs& g, hipStream_t st) {
  const size_t lds = lds_bytes<DP>(g.Sq, g.Sk, true);
  const int ndkv = g.nb * g.Hkv * ((g.Sk + 127) / 128), ndq = g.nb * g.H * ((g.Sq + 127) / 128);
  if (ndkv + ndq == 0) return hipSuccess;
  PT_RULE_LDS((rule_bwd_kernel<DP, MOD>), lds);
  hipLaunchKernelGGL((rule_bwd_kernel<DP, MOD>), dim3(ndkv + ndq), dim3(256), lds, st, g, ndkv);
  return hipGetLastError();
}
template <int DP>
hipError_t by_mod(const AttnRuleArgs& g, bool bwd, hipStream_t st) {
  switch ((g.cap > 0.f ? 1 : 0) | (g.slopes ? 2 : 0)) {
    case 0: return bwd ? launch_bwd<DP, 0>(g, st) : launch_fwd<DP, 0>(g, st);
    case 1: return bwd ? launch_bwd<DP, 1>(g, st) : launch_fwd<DP, 1>(g, st);
    case 2: return bwd ? launch_bwd<DP, 2>(g, st) : launch_fwd<DP, 2>(g, st);
    default: return bwd ? launch_bwd<DP, 3>(g, st) : launch_fwd<DP, 3>(g, st);
  }
}

}  // namespace

hipError_t attention_rule_fwd(int dt, const AttnRuleArgs& g, hipStream_t st) {
  return dt ? attention_rule_bf16(g, false, st) : attention_rule_f32(g, false, st);
}
hipError_t attention_rule_bwd(int dt, const AttnRuleArgs& g, hipStream_t st) {
  if (g.Sq > 0) {   // (without queries the launch below writes zeros)
    const hipError_t e = attention_rule_delta(dt, g, st);
    if (e != hipSuccess) return e;
  }
  return dt ? attention_rule_bf16(g, true, st) : attention_rule_f32(g, true, st);
}

hipError_t attention_rule_bf16(const AttnRuleArgs& g, bool bwd, hipStream_t st) {
  return g.dh <= 64 ? by_mod<64>(g, bwd, st) : by_mod<128>(g, bwd, st);
}

}  // namespace pt
