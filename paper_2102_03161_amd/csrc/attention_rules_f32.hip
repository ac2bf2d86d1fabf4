// Attention under a rule in fp32 on the fp32 matrix instructions (the formulas, the masks and the list of tiles are those of
// attention_rules.hip; the tiles and fragments those of attention_f32_tile.h).
//
// A wave owns 16 rows, a workgroup 64; the other side streams through LDS in tiles of 64 rows.  Where such workgroups are fewer than
// the CUs, two waves share 16 rows, each with one half of every tile (SHARE = 2), and what they summed is joined through LDS at the
// end: a tile then takes half the time on twice as many CUs.
//
// The matrix instructions bound it (153 TFLOP/s in a large product); at a few hundred rows it is the chain of one workgroup's
// tiles: 4 x 203 rows x 6 heads of 64, packed, 13.8 us forward and 26.8 backward with two waves a row, 18.4 and 34.5 with one.
// One launch does the backward pass: its first workgroups own keys, the others queries, and each takes delta from the dO and o that it
// has loaded anyway.
#include "attention_rules.h"
#include "attention_f32_tile.h"

namespace pt {
namespace {

// scores in the log2 domain, with the library's tanh (scores are held to fp32's rounding here)
struct ScoreF {
  float c, scale, cap, inv_cap, a, sl;
  __device__ __forceinline__ ScoreF(const AttnRuleArgs& g, int h) {
    constexpr float kLog2e = 1.44269504088896f;
    scale = g.scale;
    c = g.scale * kLog2e;
    cap = g.cap;
    inv_cap = g.cap > 0.f ? g.scale / g.cap : 0.f;
    a = g.cap * kLog2e;
    sl = g.slopes ? -g.slopes[h] * kLog2e : 0.f;
  }
  // *bent: tanh, 0 without a cap
  __device__ __forceinline__ float at(float s, float dist, float* bent) const {
    *bent = cap > 0.f ? tanhf(s * inv_cap) : 0.f;
    const float x = cap > 0.f ? a * *bent : s * c;
    return fmaf(sl, dist, x);
  }
};

// Two staged tiles, and the barrier behind which they are read.  Rows that are padding (which may hold anything) or behind the last
// become zeros: those of a tile that has any wait for the documents, which one wave has just written.
template <typename A>
__device__ __forceinline__ void rule_stage(bool plain, float* xs, const f32x4 (&x)[A::N4], float* ys, const f32x4 (&y)[A::N4], int tid, const int* docs) {
  if (plain) {
    A::store(xs, tid, x);
    A::store(ys, tid, y);
  } else {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < A::N4; ++i) {
      int row, d;
      A::place(tid, i, &row, &d);
      const bool keep = docs[row] >= 0;
      *reinterpret_cast<f32x4*>(xs + row * A::LD + d) = keep ? x[i] : f32x4{0.f, 0.f, 0.f, 0.f};
      *reinterpret_cast<f32x4*>(ys + row * A::LD + d) = keep ? y[i] : f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }
  __syncthreads();
}

template <int DP, int SHARE>
__global__ __launch_bounds__(256, DP > 64 ? 1 : 2) void rule_fwd_f32_kernel(AttnRuleArgs g) {
  typedef AttnTile<float, DP> A;
  constexpr int kRows = 64 / SHARE, NX = 4 / SHARE;   // rows of a workgroup; 16-row parts of a tile that a wave takes
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  float* xs = reinterpret_cast<float*>(smem);
  float* ys = xs + A::FLOATS;
  int* kdoc = reinterpret_cast<int*>(ys + A::FLOATS);
  const RuleList<16, SHARE> list(kdoc + kRuleTile, g.Sk);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), gr = lane >> 4, l = lane & 15;
  const int group = wave / SHARE, part = wave % SHARE, x0 = part * NX;
  const RuleUnit u(g, (g.Sq + kRows - 1) / kRows, g.H, blockIdx.x, gridDim.x, g.order != 0);
  const int b = u.b, h = u.h, hk = h / (g.H / g.Hkv);
  const int i = u.blk * kRows + group * 16 + l;
  const RuleRows rows(g, b);
  const int lim = rows.lim(g, i), qd = rows.qdoc(g, i);
  const bool ok = i < g.Sq, on = ok && qd >= 0;
  const int n = list.template build<true>(g, rows, wave, lane, u.blk, qd, ok);
  const float* kp = static_cast<const float*>(g.k.p) + b * g.k.b + hk * g.k.h;
  const float* vp = static_cast<const float*>(g.v.p) + b * g.v.b + hk * g.v.h;
  const ScoreF sc(g, h);
  f32x4 q[A::NF], o[A::NF], rk[A::N4], rv[A::N4];
  A::own(static_cast<const float*>(g.q.p) + b * g.q.b + h * g.q.h, g.q.t, on ? i : g.Sq, g.Sq, g.dh, gr, 1.f, q);
#pragma unroll
  for (int x = 0; x < A::NF; ++x) o[x] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -1e30f, sum = 0.f;
  int rd = 0;
  auto load = [&](int it) {
    const int j0 = list.tile(list.entry(it)) * kRuleTile;
    A::load(kp, g.k.t, j0, g.Sk, g.dh, tid, rk);
    A::load(vp, g.v.t, j0, g.Sk, g.dh, tid, rv);
    if (tid < kRuleTile) rd = rows.k_raw(g, j0 + tid);
  };
  if (n > 0) load(0);
  for (int it = 0; it < n; ++it) {
    __syncthreads();
    if (tid < kRuleTile) kdoc[tid] = RuleRows::k_id(rd);
    rule_stage<A>(list.plain(list.entry(it)), xs, rk, ys, rv, tid, kdoc);
    if (it + 1 < n) load(it + 1);
    if (!list.needed(list.entry(it), wave)) continue;
    const int j0 = list.tile(list.entry(it)) * kRuleTile;
    const float at = (float)(g.q0 + i - j0);
    f32x4 s[NX];
    float mx = m;
#pragma unroll
    for (int x = 0; x < NX; ++x) {
      s[x] = A::dot(xs, 16 * (x0 + x), l, gr, q);
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const int r = 16 * (x0 + x) + 4 * gr + v;
        float bent;
        s[x][v] = sc.at(s[x][v], fabsf(at - (float)r), &bent);
        if (kdoc[r] != qd || j0 + r > lim) s[x][v] = -INFINITY;
        mx = fmaxf(mx, s[x][v]);
      }
    }
    mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    const float alpha = __builtin_amdgcn_exp2f(m - mx);
    m = mx;
    sum *= alpha;
#pragma unroll
    for (int x = 0; x < A::NF; ++x) o[x] *= alpha;
#pragma unroll
    for (int x = 0; x < NX; ++x) {
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        s[x][v] = __builtin_amdgcn_exp2f(s[x][v] - mx);
        sum += s[x][v];
      }
      A::add(ys, 16 * (x0 + x), l, gr, s[x], o);
    }
  }
  sum += __shfl_xor(sum, 16, 64);
  sum += __shfl_xor(sum, 32, 64);
  if (SHARE == 2) {   // the second half's part, with a reference of its own
    float* at = xs + (group * 64 + lane) * (4 * A::NF + 4);
    __syncthreads();
    if (part == 1) {
#pragma unroll
      for (int x = 0; x < A::NF; ++x) *reinterpret_cast<f32x4*>(at + 4 * x) = o[x];
      at[4 * A::NF] = m;
      at[4 * A::NF + 1] = sum;
    }
    __syncthreads();
    if (part == 1) return;
    const float m2 = at[4 * A::NF], sum2 = at[4 * A::NF + 1], top = fmaxf(m, m2);
    const float f = __builtin_amdgcn_exp2f(m - top), f2 = __builtin_amdgcn_exp2f(m2 - top);
#pragma unroll
    for (int x = 0; x < A::NF; ++x) o[x] = o[x] * f + *reinterpret_cast<const f32x4*>(at + 4 * x) * f2;
    sum = sum * f + sum2 * f2;
    m = top;
  }
  if (!ok) return;
  A::put(static_cast<float*>(const_cast<void*>(g.o.p)) + b * g.o.b + (int64_t)i * g.o.t + h * g.o.h, g.dh, gr, sum > 0.f ? 1.f / sum : 0.f, o);
  if (g.lse && gr == 0) g.lse[(int64_t)b * g.lse_b + (int64_t)h * g.lse_h + i] = sum > 0.f ? (m + log2f(sum)) * 0.693147180559945f : -INFINITY;
}

// a += a of the second wave that shares the rows, and b likewise unless it is a; false in that second wave, which has no more to do
template <typename A>
__device__ __forceinline__ bool join(float* xs, int group, int part, int lane, f32x4 (&a)[A::NF], f32x4 (&b)[A::NF]) {
  float* at = xs + (group * 64 + lane) * (8 * A::NF + 4);
  const bool two = &a != &b;
  __syncthreads();
  if (part == 1) {
#pragma unroll
    for (int x = 0; x < A::NF; ++x) {
      *reinterpret_cast<f32x4*>(at + 4 * x) = a[x];
      if (two) *reinterpret_cast<f32x4*>(at + 4 * (A::NF + x)) = b[x];
    }
  }
  __syncthreads();
  if (part == 1) return false;
#pragma unroll
  for (int x = 0; x < A::NF; ++x) {
    a[x] += *reinterpret_cast<const f32x4*>(at + 4 * x);
    if (two) b[x] += *reinterpret_cast<const f32x4*>(at + 4 * (A::NF + x));
  }
  return true;
}

// a probability this near 1 means a query that sees one key: dS is exactly 0 then (see attention_rules.hip)
constexpr float kOneKeyF = 1.f - 1.f / 262144.f;

template <int DP, int SHARE>
__global__ __launch_bounds__(256, DP > 64 ? 1 : 2) void rule_bwd_f32_kernel(AttnRuleArgs g, int ndkv) {
  typedef AttnTile<float, DP> A;
  constexpr int kRows = 64 / SHARE, NX = 4 / SHARE;   // rows of a workgroup; 16-row parts of a tile that a wave takes
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  float* xs = reinterpret_cast<float*>(smem);
  float* ys = xs + A::FLOATS;
  float* ls = ys + A::FLOATS;                            // [lse][delta]
  int* docs = reinterpret_cast<int*>(ls + 2 * kRuleTile);   // [document][lim]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), gr = lane >> 4, l = lane & 15;
  const int group = wave / SHARE, part = wave % SHARE, x0 = part * NX;
  f32x4 rx[A::N4], ry[A::N4], a0[A::NF], a1[A::NF], ax[A::NF];
#pragma unroll
  for (int x = 0; x < A::NF; ++x) ax[x] = f32x4{0.f, 0.f, 0.f, 0.f};
  if ((int)blockIdx.x >= ndkv) {   // dq of 64 queries
    const RuleList<16, SHARE> list(docs + 2 * kRuleTile, g.Sk);
    const RuleUnit u(g, (g.Sq + kRows - 1) / kRows, g.H, blockIdx.x - ndkv, gridDim.x - ndkv, g.order != 0);
    const int b = u.b, h = u.h, hk = h / (g.H / g.Hkv);
    const int i = u.blk * kRows + group * 16 + l;
    const RuleRows rows(g, b);
    const int lim = rows.lim(g, i), qd = rows.qdoc(g, i);
    const bool ok = i < g.Sq, on = ok && qd >= 0;
    const int n = list.template build<true>(g, rows, wave, lane, u.blk, qd, ok);
    A::own(static_cast<const float*>(g.q.p) + b * g.q.b + h * g.q.h, g.q.t, on ? i : g.Sq, g.Sq, g.dh, gr, 1.f, a0);
    A::own(static_cast<const float*>(g.d_o.p) + b * g.d_o.b + h * g.d_o.h, g.d_o.t, on ? i : g.Sq, g.Sq, g.dh, gr, 1.f, a1);
    const float* kp = static_cast<const float*>(g.k.p) + b * g.k.b + hk * g.k.h;
    const float* vp = static_cast<const float*>(g.v.p) + b * g.v.b + hk * g.v.h;
    const ScoreF sc(g, h);
    const float lw = on ? rule_lse2(g.lse[(int64_t)b * g.lse_b + (int64_t)h * g.lse_h + i]) : INFINITY;
    float dl = 0.f;   // delta = dO . o
    {
      f32x4 o[A::NF];
      A::own(static_cast<const float*>(g.o.p) + b * g.o.b + h * g.o.h, g.o.t, on ? i : g.Sq, g.Sq, g.dh, gr, 1.f, o);
#pragma unroll
      for (int x = 0; x < A::NF; ++x)
#pragma unroll
        for (int e = 0; e < 4; ++e) dl = fmaf(a1[x][e], o[x][e], dl);
      dl += __shfl_xor(dl, 16, 64);
      dl += __shfl_xor(dl, 32, 64);
    }
    int rd = 0;
    auto load = [&](int it) {
      const int j0 = list.tile(list.entry(it)) * kRuleTile;
      A::load(kp, g.k.t, j0, g.Sk, g.dh, tid, rx);
      A::load(vp, g.v.t, j0, g.Sk, g.dh, tid, ry);
      if (tid < kRuleTile) rd = rows.k_raw(g, j0 + tid);
    };
    if (n > 0) load(0);
    for (int it = 0; it < n; ++it) {
      __syncthreads();
      if (tid < kRuleTile) docs[tid] = RuleRows::k_id(rd);
      rule_stage<A>(list.plain(list.entry(it)), xs, rx, ys, ry, tid, docs);
      if (it + 1 < n) load(it + 1);
      if (!list.needed(list.entry(it), wave)) continue;
      const int j0 = list.tile(list.entry(it)) * kRuleTile;
      const float at = (float)(g.q0 + i - j0);
#pragma unroll
      for (int x = x0; x < x0 + NX; ++x) {
        f32x4 s = A::dot(xs, 16 * x, l, gr, a0);
        const f32x4 dp = A::dot(ys, 16 * x, l, gr, a1);
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const int r = 16 * x + 4 * gr + v;
          float bent;
          const float p = __builtin_amdgcn_exp2f(sc.at(s[v], fabsf(at - (float)r), &bent) - lw);
          const bool see = docs[r] == qd && j0 + r <= lim && !(p >= kOneKeyF);
          s[v] = see ? p * (dp[v] - dl) * (1.f - bent * bent) : 0.f;
        }
        A::add(xs, 16 * x, l, gr, s, ax);
      }
    }
    if (SHARE == 2 && !join<A>(xs, group, part, lane, ax, ax)) return;
    if (ok) A::put(static_cast<float*>(const_cast<void*>(g.dq.p)) + b * g.dq.b + (int64_t)i * g.dq.t + h * g.dq.h, g.dh, gr, g.scale, ax);
    return;
  }
  // dk and dv of 64 keys
  const int G = g.H / g.Hkv;
  const RuleList<16, SHARE> list(docs + 2 * kRuleTile, g.Sq);
  const RuleUnit u(g, (g.Sk + kRows - 1) / kRows, g.Hkv, blockIdx.x, ndkv, false);
  const int b = u.b, hk = u.h;
  const int j = u.blk * kRows + group * 16 + l;
  const RuleRows rows(g, b);
  const int kd = rows.kdoc(g, j);
  const bool ok = j < g.Sk, on = ok && kd >= 0;
  const int n = list.template build<false>(g, rows, wave, lane, u.blk, kd, ok);
  A::own(static_cast<const float*>(g.k.p) + b * g.k.b + hk * g.k.h, g.k.t, on ? j : g.Sk, g.Sk, g.dh, gr, 1.f, a0);
  A::own(static_cast<const float*>(g.v.p) + b * g.v.b + hk * g.v.h, g.v.t, on ? j : g.Sk, g.Sk, g.dh, gr, 1.f, a1);
  f32x4 ay[A::NF], ro[A::N4];
#pragma unroll
  for (int x = 0; x < A::NF; ++x) ay[x] = f32x4{0.f, 0.f, 0.f, 0.f};
  int rd = 0, rlim = 0;
  float rl = 0.f;
  auto load = [&](int it) {
    const int h = hk * G + it / n, i0 = list.tile(list.entry(it % n)) * kRuleTile;
    A::load(static_cast<const float*>(g.q.p) + b * g.q.b + h * g.q.h, g.q.t, i0, g.Sq, g.dh, tid, rx);
    A::load(static_cast<const float*>(g.d_o.p) + b * g.d_o.b + h * g.d_o.h, g.d_o.t, i0, g.Sq, g.dh, tid, ry);
    A::load(static_cast<const float*>(g.o.p) + b * g.o.b + h * g.o.h, g.o.t, i0, g.Sq, g.dh, tid, ro);
    if (tid < kRuleTile) {
      const int i = i0 + tid;
      rd = rows.q_raw(g, i);
      rlim = rows.lim(g, i);
      rl = i < g.Sq ? g.lse[(int64_t)b * g.lse_b + (int64_t)h * g.lse_h + i] : -INFINITY;
    }
  };
  const int total = n * G;
  if (total > 0) load(0);
  for (int it = 0; it < total; ++it) {
    __syncthreads();
    if (tid < kRuleTile) { docs[tid] = RuleRows::q_id(rd); docs[kRuleTile + tid] = rlim; ls[tid] = rd >= 0 ? rule_lse2(rl) : INFINITY; }
#pragma unroll
    for (int x = 0; x < A::N4; ++x) {   // delta of the tile's rows: DP / 4 neighbouring lanes hold a row
      int r, d;
      A::place(tid, x, &r, &d);
      float part = 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) part = fmaf(ry[x][e], ro[x][e], part);
#pragma unroll
      for (int o = 1; o < DP / 4; o <<= 1) part += __shfl_xor(part, o, 64);
      if (d == 0) ls[kRuleTile + r] = part;
    }
    rule_stage<A>(list.plain(list.entry(it % n)), xs, rx, ys, ry, tid, docs);
    if (it + 1 < total) load(it + 1);
    const int item = it % n;
    if (!list.needed(list.entry(item), wave)) continue;
    const ScoreF sc(g, hk * G + it / n);
    const float at = (float)(g.q0 + list.tile(list.entry(item)) * kRuleTile - j);
#pragma unroll
    for (int x = x0; x < x0 + NX; ++x) {
      f32x4 p = A::dot(xs, 16 * x, l, gr, a0);
      f32x4 ds = A::dot(ys, 16 * x, l, gr, a1);
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const int r = 16 * x + 4 * gr + v;
        float bent;
        const float e = __builtin_amdgcn_exp2f(sc.at(p[v], fabsf(at + (float)r), &bent) - ls[r]);
        const bool see = docs[r] == kd && j <= docs[kRuleTile + r];
        p[v] = see ? e : 0.f;
        ds[v] = see && !(e >= kOneKeyF) ? e * (ds[v] - ls[kRuleTile + r]) * (1.f - bent * bent) : 0.f;
      }
      A::add(ys, 16 * x, l, gr, p, ay);
      A::add(xs, 16 * x, l, gr, ds, ax);
    }
  }
  if (SHARE == 2 && !join<A>(xs, group, part, lane, ax, ay)) return;
  if (ok) {
    A::put(static_cast<float*>(const_cast<void*>(g.dk.p)) + b * g.dk.b + (int64_t)j * g.dk.t + hk * g.dk.h, g.dh, gr, g.scale, ax);
    A::put(static_cast<float*>(const_cast<void*>(g.dv.p)) + b * g.dv.b + (int64_t)j * g.dv.t + hk * g.dv.h, g.dh, gr, 1.f, ay);
  }
}

template <int DP, int SHARE>
hipError_t launch_shared(const AttnRuleArgs& g, bool bwd, hipStream_t st) {
  constexpr int kRows = 64 / SHARE;
  const int nt = ((bwd && g.Sq > g.Sk ? g.Sq : g.Sk) + kRuleTile - 1) / kRuleTile;
  const size_t lds = (size_t)2 * AttnTile<float, DP>::FLOATS * 4 + (bwd ? 4 : 1) * kRuleTile * 4 + RuleList<16, SHARE>::ints(nt) * 4;
  const int nq = g.nb * g.H * ((g.Sq + kRows - 1) / kRows), nk = g.nb * g.Hkv * ((g.Sk + kRows - 1) / kRows);
  if ((bwd ? nk + nq : nq) == 0) return hipSuccess;
  if (bwd) PT_RULE_LDS((rule_bwd_f32_kernel<DP, SHARE>), lds);
  else PT_RULE_LDS((rule_fwd_f32_kernel<DP, SHARE>), lds);
  if (bwd) hipLaunchKernelGGL((rule_bwd_f32_kernel<DP, SHARE>), dim3(nk + nq), dim3(256), lds, st, g, nk);
  else hipLaunchKernelGGL((rule_fwd_f32_kernel<DP, SHARE>), dim3(nq), dim3(256), lds, st, g);
  return hipGetLastError();
}
template <int DP>
hipError_t launch_f32(const AttnRuleArgs& g, bool bwd, hipStream_t st) {
  return rule_share_f32(rule_shape(g), bwd) == 2 ? launch_shared<DP, 2>(g, bwd, st) : launch_shared<DP, 1>(g, bwd, st);
}

}  // namespace

hipError_t attention_rule_f32(const AttnRuleArgs& g, bool bwd, hipStream_t st) {
  if (g.dh <= 16) return launch_f32<16>(g, bwd, st);
  if (g.dh <= 32) return launch_f32<32>(g, bwd, st);
  if (g.dh <= 64) return launch_f32<64>(g, bwd, st);
  return launch_f32<128>(g, bwd, st);
}

}  // namespace pt
