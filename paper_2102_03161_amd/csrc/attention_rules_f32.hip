// Attention under a rule in fp32 on the fp32 matrix instructions (the formulas, the masks and the list of tiles are those of
// attention_rules.hip; the tiles and fragments those of attention_f32_tile.h).
//
// A wave owns 16 rows, a workgroup 64; the other side streams through LDS in tiles of 64 rows.  Where such workgroups are fewer than
// the CUs, two waves share 16 rows, each with one half of every tile (SHARE = 2), and what they summed is joined through LDS at the
// end: a tile then takes half the time on twice as many CUs.
//
// The matrix instructions bound it (153 TFLOP/s in a large product); at a few hundred rows it is the chain of one workgroup's
// tiles: 4 x 203 rows x 6 heads of 64, packed, 12 us forward and 35 backward; 16 x 197 x 12 41 and 149.  The backward pass is two
// launches: dq, which leaves what the other needs of each query, then dk and dv.
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
  float m = -INFINITY, sum = 0.f;   // the largest score of a visible pair so far
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
    const float ref = mx == -INFINITY ? 0.f : mx;   // nothing visible yet: any finite reference will do
    const float alpha = __builtin_amdgcn_exp2f(m - ref);
    m = mx;
    sum *= alpha;
#pragma unroll
    for (int x = 0; x < A::NF; ++x) o[x] *= alpha;
#pragma unroll
    for (int x = 0; x < NX; ++x) {
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        s[x][v] = __builtin_amdgcn_exp2f(s[x][v] - ref);
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
    const float ref = top == -INFINITY ? 0.f : top;
    const float f = __builtin_amdgcn_exp2f(m - ref), f2 = __builtin_amdgcn_exp2f(m2 - ref);
#pragma unroll
    for (int x = 0; x < A::NF; ++x) o[x] = o[x] * f + *reinterpret_cast<const f32x4*>(at + 4 * x) * f2;
    sum = sum * f + sum2 * f2;
    m = top;
  }
  if (!ok) return;
  A::put(static_cast<float*>(const_cast<void*>(g.o.p)) + b * g.o.b + (int64_t)i * g.o.t + h * g.o.h, g.dh, gr, sum == 0.f ? 0.f : 1.f / sum, o);
  if (g.lse && gr == 0) g.lse[(int64_t)b * g.lse_b + (int64_t)h * g.lse_h + i] = sum == 0.f ? -INFINITY : (m + log2f(sum)) * 0.693147180559945f;
}

// a += a of the second wave that shares the rows; false in that second wave, which has no more to do
template <typename A>
__device__ __forceinline__ bool join(float* room, int group, int part, int lane, f32x4 (&a)[A::NF]) {
  float* at = room + (group * 64 + lane) * (4 * A::NF + 4);
  if (part == 1)
#pragma unroll
    for (int x = 0; x < A::NF; ++x) *reinterpret_cast<f32x4*>(at + 4 * x) = a[x];
  __syncthreads();
  if (part == 1) return false;
#pragma unroll
  for (int x = 0; x < A::NF; ++x) a[x] += *reinterpret_cast<const f32x4*>(at + 4 * x);
  return true;
}

// A key with nearly all of a query's weight (p above 3/4: there is at most one) has dS_m = p_m (dP_m - delta), which is as small as the
// weight that the others have, while dP_m and delta = dO . o are two sums that are rounded apart: at 1 - p = 3e-6 rounding is as large as
// dS_m.  But the dS of a query sum to 0 in front of the cap's slope, so dS_m is minus the sum of the others', which have no such
// cancellation: dq's pass leaves that sum, times the key's slope, out of its products and adds it with the key's row at the end, and
// hands it to the keys' pass, which takes it for every pair of that query with more than half of the weight.  For a query that
// sees one key the sum has no term, and its gradients are exactly 0.
constexpr float kMost = 0.75f, kHalf = 0.5f;
constexpr float kNoTop = INFINITY;   // in place of that sum: the query has no such key

// dq of 64 queries; what it leaves for the keys' pass: delta and that sum
template <int DP, int SHARE>
__global__ __launch_bounds__(256, DP > 64 ? 1 : 2) void rule_dq_f32_kernel(AttnRuleArgs g) {
  typedef AttnTile<float, DP> A;
  constexpr int kRows = 64 / SHARE, NX = 4 / SHARE;   // rows of a workgroup; 16-row parts of a tile that a wave takes
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  float* xs = reinterpret_cast<float*>(smem);
  float* ys = xs + A::FLOATS;
  int* docs = reinterpret_cast<int*>(ys + A::FLOATS);
  const RuleList<16, SHARE> list(docs + kRuleTile, g.Sk);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), gr = lane >> 4, l = lane & 15;
  const int group = wave / SHARE, part = wave % SHARE, x0 = part * NX;
  f32x4 rx[A::N4], ry[A::N4], a0[A::NF], a1[A::NF], ax[A::NF];
#pragma unroll
  for (int x = 0; x < A::NF; ++x) ax[x] = f32x4{0.f, 0.f, 0.f, 0.f};
  const RuleUnit u(g, (g.Sq + kRows - 1) / kRows, g.H, blockIdx.x, gridDim.x, g.order != 0);
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
  float others = 0.f, bend = 0.f;   // sum of the other keys' p (dP - delta); slope of the cap at the dominant one
  int top = -1;                     // the dominant key
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
        const bool see = docs[r] == qd && j0 + r <= lim, most = see && p > kMost;
        const float ds = see && !most ? p * (dp[v] - dl) : 0.f, f = 1.f - bent * bent;
        others += ds;
        s[v] = ds * f;
        top = most ? j0 + r : top;
        bend = most ? f : bend;
      }
      A::add(xs, 16 * x, l, gr, s, ax);
    }
  }
  // one lane of the row, of one wave, has met the dominant key
  others += __shfl_xor(others, 16, 64);
  others += __shfl_xor(others, 32, 64);
  bend += __shfl_xor(bend, 16, 64);
  bend += __shfl_xor(bend, 32, 64);
  top = max(top, __shfl_xor(top, 16, 64));
  top = max(top, __shfl_xor(top, 32, 64));
  if (SHARE == 2) {
    __syncthreads();   // the last tile is read
    float* at = xs + (group * 64 + lane) * (4 * A::NF + 4) + 4 * A::NF;
    if (part == 1) { at[0] = others; at[1] = bend; at[2] = __int_as_float(top); }
    if (!join<A>(xs, group, part, lane, ax)) return;
    others += at[0];
    bend += at[1];
    top = max(top, __float_as_int(at[2]));
  }
  if (!ok) return;
  const int64_t row = ((int64_t)b * g.H + h) * g.Sq + i;
  if (gr == 0) {
    g.delta[row] = dl;
    g.delta[(int64_t)g.nb * g.H * g.Sq + row] = top >= 0 ? -others : kNoTop;
  }
  f32x4 kt[A::NF];
  A::own(kp, g.k.t, top >= 0 ? top : g.Sk, g.Sk, g.dh, gr, 1.f, kt);
  if (top >= 0)
#pragma unroll
    for (int x = 0; x < A::NF; ++x) ax[x] -= kt[x] * (others * bend);
  A::put(static_cast<float*>(const_cast<void*>(g.dq.p)) + b * g.dq.b + (int64_t)i * g.dq.t + h * g.dq.h, g.dh, gr, g.scale, ax);
}

// dk and dv of 64 keys, the heads that share them one after the other
template <int DP, int SHARE>
__global__ __launch_bounds__(256, DP > 64 ? 1 : 2) void rule_dkv_f32_kernel(AttnRuleArgs g) {
  typedef AttnTile<float, DP> A;
  constexpr int kRows = 64 / SHARE, NX = 4 / SHARE;   // rows of a workgroup; 16-row parts of a tile that a wave takes
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  float* xs = reinterpret_cast<float*>(smem);
  float* ys = xs + A::FLOATS;
  float* ls = ys + A::FLOATS;                               // [lse][delta][sum for the dominant key]
  int* docs = reinterpret_cast<int*>(ls + 3 * kRuleTile);   // [document][lim]
  const RuleList<16, SHARE> list(docs + 2 * kRuleTile, g.Sq);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), gr = lane >> 4, l = lane & 15;
  const int group = wave / SHARE, part = wave % SHARE, x0 = part * NX;
  const int G = g.H / g.Hkv;
  const RuleUnit u(g, (g.Sk + kRows - 1) / kRows, g.Hkv, blockIdx.x, gridDim.x, false);
  const int b = u.b, hk = u.h;
  const int j = u.blk * kRows + group * 16 + l;
  const RuleRows rows(g, b);
  const int kd = rows.kdoc(g, j);
  const bool ok = j < g.Sk, on = ok && kd >= 0;
  const int n = list.template build<false>(g, rows, wave, lane, u.blk, kd, ok);
  f32x4 rx[A::N4], ry[A::N4], a0[A::NF], a1[A::NF], ax[A::NF], ay[A::NF];
  A::own(static_cast<const float*>(g.k.p) + b * g.k.b + hk * g.k.h, g.k.t, on ? j : g.Sk, g.Sk, g.dh, gr, 1.f, a0);
  A::own(static_cast<const float*>(g.v.p) + b * g.v.b + hk * g.v.h, g.v.t, on ? j : g.Sk, g.Sk, g.dh, gr, 1.f, a1);
#pragma unroll
  for (int x = 0; x < A::NF; ++x) { ax[x] = f32x4{0.f, 0.f, 0.f, 0.f}; ay[x] = f32x4{0.f, 0.f, 0.f, 0.f}; }
  int rd = 0, rlim = 0;
  float rl = 0.f, rdl = 0.f, rtop = 0.f;
  auto load = [&](int it) {
    const int h = hk * G + it / n, i0 = list.tile(list.entry(it % n)) * kRuleTile;
    A::load(static_cast<const float*>(g.q.p) + b * g.q.b + h * g.q.h, g.q.t, i0, g.Sq, g.dh, tid, rx);
    A::load(static_cast<const float*>(g.d_o.p) + b * g.d_o.b + h * g.d_o.h, g.d_o.t, i0, g.Sq, g.dh, tid, ry);
    if (tid < kRuleTile) {
      const int i = i0 + tid;
      const int64_t row = ((int64_t)b * g.H + h) * g.Sq + i;
      rd = rows.q_raw(g, i);
      rlim = rows.lim(g, i);
      rl = i < g.Sq ? g.lse[(int64_t)b * g.lse_b + (int64_t)h * g.lse_h + i] : -INFINITY;
      rdl = i < g.Sq ? g.delta[row] : 0.f;
      rtop = i < g.Sq ? g.delta[(int64_t)g.nb * g.H * g.Sq + row] : kNoTop;
    }
  };
  const int total = n * G;
  if (total > 0) load(0);
  for (int it = 0; it < total; ++it) {
    __syncthreads();
    if (tid < kRuleTile) {
      docs[tid] = RuleRows::q_id(rd);
      docs[kRuleTile + tid] = rlim;
      ls[tid] = rd >= 0 ? rule_lse2(rl) : INFINITY;
      ls[kRuleTile + tid] = rdl;
      ls[2 * kRuleTile + tid] = rtop;
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
        const float top = ls[2 * kRuleTile + r];
        const float raw = e > kHalf && top != kNoTop ? top : e * (ds[v] - ls[kRuleTile + r]);
        p[v] = see ? e : 0.f;
        ds[v] = see ? raw * (1.f - bent * bent) : 0.f;
      }
      A::add(ys, 16 * x, l, gr, p, ay);
      A::add(xs, 16 * x, l, gr, ds, ax);
    }
  }
  if (SHARE == 2) {
    __syncthreads();   // the last tile is read
    join<A>(xs, group, part, lane, ax);
    if (!join<A>(ys, group, part, lane, ay)) return;
  }
  if (ok) {
    A::put(static_cast<float*>(const_cast<void*>(g.dk.p)) + b * g.dk.b + (int64_t)j * g.dk.t + hk * g.dk.h, g.dh, gr, g.scale, ax);
    A::put(static_cast<float*>(const_cast<void*>(g.dv.p)) + b * g.dv.b + (int64_t)j * g.dv.t + hk * g.dv.h, g.dh, gr, 1.f, ay);
  }
}

template <typename K>
hipError_t launch(K kernel, int64_t blocks, size_t lds, const AttnRuleArgs& g, hipStream_t st) {
  if (blocks == 0) return hipSuccess;
  PT_RULE_LDS(kernel, lds);
  hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), lds, st, g);
  return hipGetLastError();
}
template <int DP>
hipError_t launch_f32(const AttnRuleArgs& g, bool bwd, hipStream_t st) {
  const RuleShape s = rule_shape(g);
  const int64_t heads = (int64_t)g.nb * g.H, key_heads = (int64_t)g.nb * g.Hkv;
  auto lds = [](int streamed, int stats) {
    return (size_t)2 * AttnTile<float, DP>::FLOATS * 4 + stats * kRuleTile * 4 + RuleList<16>::ints((streamed + kRuleTile - 1) / kRuleTile) * 4;
  };
  if (!bwd)
    return rule_share_f32_fwd(s) == 2 ? launch(rule_fwd_f32_kernel<DP, 2>, rule_blocks(heads, g.Sq, 32), lds(g.Sk, 1), g, st)
                                      : launch(rule_fwd_f32_kernel<DP, 1>, rule_blocks(heads, g.Sq, 64), lds(g.Sk, 1), g, st);
  const hipError_t e = rule_share_f32_dq(s) == 2 ? launch(rule_dq_f32_kernel<DP, 2>, rule_blocks(heads, g.Sq, 32), lds(g.Sk, 1), g, st)
                                                 : launch(rule_dq_f32_kernel<DP, 1>, rule_blocks(heads, g.Sq, 64), lds(g.Sk, 1), g, st);
  if (e != hipSuccess) return e;
  return rule_share_f32_dkv(s) == 2 ? launch(rule_dkv_f32_kernel<DP, 2>, rule_blocks(key_heads, g.Sk, 32), lds(g.Sq, 5), g, st)
                                    : launch(rule_dkv_f32_kernel<DP, 1>, rule_blocks(key_heads, g.Sk, 64), lds(g.Sq, 5), g, st);
}

}  // namespace

hipError_t attention_rule_f32(const AttnRuleArgs& g, bool bwd, hipStream_t st) {
  if (g.dh <= 16) return launch_f32<16>(g, bwd, st);
  if (g.dh <= 32) return launch_f32<32>(g, bwd, st);
  if (g.dh <= 64) return launch_f32<64>(g, bwd, st);
  return launch_f32<128>(g, bwd, st);
}

}  // namespace pt
