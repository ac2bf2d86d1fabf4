// Softmax attention under a rule, forward and backward, bf16 (the fp32 kernels are in attention_rules_f32.hip).
//
//   t_ij = scale q_i . k_j      s_ij = cap tanh(t_ij / cap) - slope_h |q0 + i - j|      (cap and slopes optional)
//   p_i  = softmax over the keys that query i sees          o_i = sum_j p_ij v_j
//   dS = p (dP - delta), dP_ij = dO_i . v_j, delta_i = dO_i . o_i;   dT = dS (1 - tanh^2);   dq = scale dT k, dk = scale dT^T q
//
// What a query sees: keys up to lim_i (its own position, the end of the sample's prefix, or the last key) of its own document.
//
// One wave owns 32 rows (queries in the forward pass and for dq, keys for dk / dv), or, where that makes too few workgroups
// (attention_choice.h), half of the streamed rows of 32 rows, joined at the end; a workgroup of four waves streams the other side
// through LDS in tiles of 64 rows.  Scores are computed with the owned row as the MFMA's column, so that softmax statistics are one value per lane and the
// probabilities, rounded to bf16, are the next MFMA's operand as they stand in registers.
//
// Work that a mask leaves out is not done: before anything else a workgroup writes the list of the tiles that any of its waves
// needs, each with four bits "this wave needs it" and four bits "all 32 x 64 pairs of this wave are visible".  Only tiles without
// the latter bit are masked pair by pair.  The list is built from the documents' ids as they are, in any order.
//
// What bounds it: per pair and head the forward pass takes 4 dh flops of MFMA and about 2.5 VALU instructions (exp2 is a quarter
// rate one), dq 8 dh (two products for the score and dP, two for dq and its correction), dk / dv 8 dh; at a head size of 64 the
// VALU work takes about as long as the MFMAs, and of the four waves of a SIMD only some overlap the two: 740 - 830 TFLOP/s forward in
// the steady state, 840 - 920 at 128 (a large product reaches 1444).  Measured (medians of a trace): 32 x 384 rows x 12 heads of 64,
// padded, 38 us forward, 59 dq, 60 dk / dv; 4 x 2048 x 16 packed, prefix, cap 57 / 103 / 83; 1 x 8192 x 16 of 128, causal, 4 key heads,
// forward 357, and 321 a call with pauses in between (856 TFLOP/s of the visible pairs).  Tiles of 64 rows: two buffers of two take 32 KB
// at a head size of 64, so four workgroups fit a CU and hide each other's barriers, first loads and lists.
#include "attention_rules.h"

namespace pt {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;
typedef __attribute__((__vector_size__(4 * sizeof(__bf16)))) __bf16 bf16x4;
typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16;

namespace {

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ uint64_t swapped(uint64_t lanes) { return lanes >> 32 | lanes << 32; }   // the mask of the lanes 32 away
// the value of the lane 32 away
__device__ __forceinline__ float half_swap(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float((threadIdx.x & 32) ? r[0] : r[1]);
}

// accumulator register v of a 32x32 tile holds tile row 8*(v/4) + v%4 + 4*half (column = lane%32)
constexpr int acc_row(int v) { return 8 * (v >> 2) + (v & 3); }
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

__device__ __forceinline__ unsigned lds_addr(const void* p) {
  return (unsigned)(size_t)((__attribute__((address_space(3))) const void*)(p));
}
typedef __attribute__((address_space(3))) const bf16x8 lds8;
typedef __attribute__((address_space(3))) bf16x4 lds4;

// DP: the head size rounded up to 64 or 128; columns from dh on are zeros.
// A tile in LDS is 64 rows of DP values without padding, as the direct loads from global memory leave it; the 16-byte pieces of a row
// are permuted, piece c lies at c ^ swizzle(row), so that neither eight rows' 16-byte reads of one piece nor the four rows of a
// transposing read share a bank.
template <int DP>
struct Tile {
  static constexpr int RB = DP * 2;                   // bytes of a row
  static constexpr int BYTES = kRuleTile * RB;
  static constexpr int N = kRuleTile * DP / 8 / 256;  // 16-byte pieces per thread
  static constexpr int PR = DP / 8;                   // pieces of a row
  static constexpr int KS = DP / 16;                  // k steps of a product over the head size
  static constexpr int DT = DP / 32;                  // 32-column tiles of the head size
  static __device__ __forceinline__ int swizzle(int row) { return DP == 64 ? row & 7 : (row & 7) * 2; }
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
  // a lane's address in a tile at LDS address s for dot() and for add()
  static __device__ __forceinline__ unsigned row_addr(unsigned s, int lane) {
    return s + (lane & 31) * RB + (((lane >> 5) ^ swizzle(lane)) << 4);
  }
  static __device__ __forceinline__ unsigned col_addr(unsigned s, int lane) {
    const int l16 = lane & 15, grp = lane >> 4, row = 4 * (grp >> 1) + (l16 >> 2), piece = 2 * (grp & 1) + ((l16 & 3) >> 1);
    return s + row * RB + ((piece ^ swizzle(row)) << 4) + 8 * (l16 & 1);
  }
  // rows r0 .. r0 + 31 of the tile times the owned rows; at: row_addr()
  static __device__ __forceinline__ f32x16 dot(unsigned at, int r0, const bf16x8 (&f)[KS]) {
    f32x16 acc = zero16();
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
      acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*(lds8*)(size_t)((at ^ (32 * ks)) + r0 * RB), f[ks], acc, 0, 0, 0);
    return acc;
  }
  // the transposing LDS read hands a lane four consecutive rows of one column, in the order in which the weights of add() stand in
  // the accumulator
  static __device__ __forceinline__ bf16x8 column(unsigned at, int r0, int dt) {
    const unsigned p = at ^ (64 * dt);
    union { bf16x4 h[2]; bf16x8 v; } t;
    t.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds4*)(size_t)(p + r0 * RB));
    t.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds4*)(size_t)(p + (r0 + 8) * RB));
    return t.v;
  }
  // acc[dt] (columns 32 dt + .. of the owned rows) += sum over rows r0 .. r0 + 31 of tile row x weight; at: col_addr()
  static __device__ __forceinline__ void add(unsigned at, int r0, const f32x16& w, f32x16 (&acc)[DT]) {
#pragma unroll
    for (int ks2 = 0; ks2 < 2; ++ks2) {
      const bf16x8 b = pack8(w, 8 * ks2);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(column(at, r0 + 16 * ks2, dt), b, acc[dt], 0, 0, 0);
    }
  }
  // the same for two weights and two results; *sum += the first weights as they were rounded, unless null
  static __device__ __forceinline__ void add2(unsigned at, int r0, const f32x16& w, f32x16 (&acc)[DT], const f32x16& w2, f32x16 (&acc2)[DT], float* sum) {
#pragma unroll
    for (int ks2 = 0; ks2 < 2; ++ks2) {
      const bf16x8 b = pack8(w, 8 * ks2), b2 = pack8(w2, 8 * ks2);
      if (sum) {
        const bf16x2 one = {static_cast<bf16>(1.f), static_cast<bf16>(1.f)};
#pragma unroll
        for (int e = 0; e < 4; ++e) *sum = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{b[2 * e], b[2 * e + 1]}, one, *sum, false);
      }
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const bf16x8 t = column(at, r0 + 16 * ks2, dt);
        acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(t, b, acc[dt], 0, 0, 0);
        acc2[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(t, b2, acc2[dt], 0, 0, 0);
      }
    }
  }
  // the wave's own row of another matrix times its operand f, summed over the head size; the same in both halves
  static __device__ __forceinline__ float own_dot(const bf16* row, bool ok, int dh, int half, const bf16x8 (&f)[KS]) {
    bf16x8 x[KS];
    own(row, ok, dh, half, x);
    float d = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int e = 0; e < 8; ++e) d = fmaf(to_f32(x[ks][e]), to_f32(f[ks][e]), d);
    return d + half_swap(d);
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

// 16 bytes a lane from global memory to LDS, lanes next to each other from `to` on, without a register in between.  Written as
// assembly because the compiler, for the builtin, waits for such loads in front of every LDS read.  loads_done() waits for all of them, in
// front of the barrier behind which the tile is read.  Where registers are spilled inside the loop (below), the compiler's wait for a
// reload is one for the loads in front of it too, these among them.
__device__ __forceinline__ void load_to_lds(unsigned to, const void* from) {
  unsigned kept;   // m0 as it was: the compiler may hold something in it
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, off\n\ts_mov_b32 m0, %0"
               : "=&s"(kept) : "s"(to), "v"(from) : "memory");
}
__device__ __forceinline__ void loads_done() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// Two streamed matrices (K and V, or Q and dO): a thread's N pieces of a tile of each, tiles in LDS next to each other.  Rows behind
// the last are read as the last one; clear() zeroes them, and padding, once they have arrived.  Columns behind the head size are
// never loaded: the buffers start as zeros where there are any.
template <int DP>
struct Streams {
  typedef Tile<DP> T;
  static constexpr int RI = 64 / T::PR;   // rows of one load of a wave
  const bf16* base[2];
  int64_t ld[2];
  int row, piece;    // of the first load
  __device__ __forceinline__ Streams(const HeadView& x, int hx, const HeadView& y, int hy, int b, int wave, int lane) {
    base[0] = static_cast<const bf16*>(x.p) + b * x.b + hx * x.h;
    base[1] = static_cast<const bf16*>(y.p) + b * y.b + hy * y.h;
    ld[0] = x.t;
    ld[1] = y.t;
    row = wave * T::N * RI + lane / T::PR;
    piece = lane % T::PR;
  }
  __device__ __forceinline__ int col(int i) const { return 8 * (piece ^ T::swizzle(row + i * RI)); }
  // to: LDS address of the first tile plus the wave's share, wave * N KB
  __device__ __forceinline__ void load(unsigned to, int r0, int n, int dh) const {
    const bool all = r0 + kRuleTile <= n;
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const bf16* p = base[m] + r0 * ld[m];
#pragma unroll
      for (int i = 0; i < T::N; ++i) {
        int r = row + i * RI;
        if (!all) r = r < n - 1 - r0 ? r : n - 1 - r0;
        const bf16* from = p + r * ld[m] + col(i);
        if (dh == DP || col(i) < dh) load_to_lds(to + m * T::BYTES + i * 1024, from);
      }
    }
  }
  __device__ __forceinline__ void clear(unsigned to, int lane, const bool (&keep)[T::N]) const {
    typedef __attribute__((ext_vector_type(4))) unsigned u32x4;
    typedef __attribute__((address_space(3))) u32x4 lds16;
#pragma unroll
    for (int i = 0; i < T::N; ++i)
      if (!keep[i])
#pragma unroll
        for (int m = 0; m < 2; ++m) *(lds16*)(size_t)(to + m * T::BYTES + i * 1024 + lane * 16) = u32x4{0, 0, 0, 0};
  }
};
template <int DP>
__device__ __forceinline__ void zero_tiles(unsigned char* smem, int dh) {   // both buffers' two tiles; a barrier follows
  if (dh == DP) return;
  for (int i = threadIdx.x; i < 4 * Tile<DP>::BYTES / 16; i += 256) reinterpret_cast<uint4*>(smem)[i] = make_uint4(0, 0, 0, 0);
  __syncthreads();
}
// the documents of the same pieces' rows
template <int DP>
struct StreamDocs {
  typedef Tile<DP> T;
  const int32_t* d;
  int n, row;
  int raw[T::N];
  __device__ __forceinline__ StreamDocs(const int32_t* docs, int n_, int row_) : d(docs), n(n_), row(row_) {}
  __device__ __forceinline__ void load(int r0) {
    if (d) {
#pragma unroll
      for (int x = 0; x < T::N; ++x) {
        const int i = r0 + row + x * Streams<DP>::RI;
        raw[x] = d[i < n ? i : n - 1];
      }
    }
  }
  // keep: the row exists and is no padding; first: this thread writes the row's document (as the owned side compares it)
  __device__ __forceinline__ void finish(int r0, int none, int* docs, bool first, bool (&keep)[T::N]) const {
#pragma unroll
    for (int x = 0; x < T::N; ++x) {
      const int i = row + x * Streams<DP>::RI, v = d ? raw[x] : 0;
      keep[x] = r0 + i < n && v >= 0;
      if (first) docs[i] = keep[x] ? v : none;
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
  // score + nm; raw: the product, or with a cap bend() of it; dist: position of the query - position of the key, of any sign
  template <int MOD>
  __device__ __forceinline__ float at(float raw, float dist, float nm) const {
    const float y = (MOD & 2) ? fmaf(sl, fabsf(dist), nm) : nm;
    return (MOD & 1) ? fmaf(-2.f * a, raw, y + a) : fmaf(raw, c, y);
  }
};

// visible pairs of a tile that is not whole, 4 streamed rows at a time
__device__ __forceinline__ void four(const int* p, int (&x)[4]) {
  const int4 v = *reinterpret_cast<const int4*>(p);
  x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
}

// ---------------------------------------------------------------------------------------------------------------------------
// forward: one pass over the tiles with the running reference and sum of a softmax; four workgroups a CU at a head size of 64 (128
// registers, where a wave owns its rows alone 2 to 16 values more are spilled, none with a cap and without slopes), two at 128.  At short
// rows it is bound by starting up: of 38 us for 32 x 384 x 12, padded, the visible pairs' products take 5.
// ---------------------------------------------------------------------------------------------------------------------------
// Two waves that share their rows: the second one's accumulators through LDS (both buffers' tiles, which nothing reads any more),
// 16 bytes a lane next to each other.
template <int N>
__device__ __forceinline__ void leave(float* room, int group, int lane, const f32x16 (&acc)[N]) {
#pragma unroll
  for (int i = 0; i < 4 * N; ++i) {
    const f32x16& a = acc[i >> 2];
    const int v = 4 * (i & 3);
    *reinterpret_cast<float4*>(room + ((group * 4 * N + i) * 64 + lane) * 4) = make_float4(a[v], a[v + 1], a[v + 2], a[v + 3]);
  }
}
template <int N>
__device__ __forceinline__ void take(const float* room, int group, int lane, f32x16 (&acc)[N], float f, float f2) {
#pragma unroll
  for (int i = 0; i < 4 * N; ++i) {
    const float4 x = *reinterpret_cast<const float4*>(room + ((group * 4 * N + i) * 64 + lane) * 4);
    const float e[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      acc[i >> 2][4 * (i & 3) + v] = acc[i >> 2][4 * (i & 3) + v] * f + e[v] * f2;
    }
  }
}

// FEW (attention_choice.h): what a weight's rounding to bf16 leaves out.  3 x 64 rows x 4 heads take 5.8 / 14.7 us forward / backward with
// that product, 5.7 / 13.9 without.
__device__ __forceinline__ f32x16 left_out(const f32x16& w) {
  f32x16 r;
#pragma unroll
  for (int v = 0; v < 16; ++v) r[v] = w[v] - to_f32(from_f32<bf16>(w[v]));
  return r;
}

// A row's reference m (log2 domain) only has to keep exp2 in range: it is the maximum of the first tile in which the row sees
// anything, and moves only when a tile's sum passes 2^40.  So a tile whose rows all have one needs no maximum at all.
constexpr float kGrown = 1099511627776.f;   // 2^40

template <int DP, int MOD, int SHARE, bool FEW>
__global__ __launch_bounds__(256, DP == 64 ? 4 : 2) void rule_fwd_kernel(AttnRuleArgs g) {
  typedef Tile<DP> T;
  constexpr int kRows = 128 / SHARE, NX = 2 / SHARE;   // rows of a workgroup; parts of 32 rows of a tile that a wave takes
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  int* kdoc = reinterpret_cast<int*>(smem + 4 * T::BYTES);                    // [2][64], behind [2][K tile, V tile]
  const RuleList<32, SHARE> list(kdoc + 2 * kRuleTile, g.Sk);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5;
  const int group = wave / SHARE, x0 = wave % SHARE * NX;   // rows of the wave; its first part of a tile
  const int nqb = (g.Sq + kRows - 1) / kRows;
  const RuleUnit u(g, nqb, g.H, blockIdx.x, gridDim.x, g.order != 0);
  const int b = u.b, h = u.h, hk = h / (g.H / g.Hkv);
  const int i = u.blk * kRows + group * 32 + (lane & 31);
  const RuleRows rows(g, b);
  const bool ok = i < g.Sq;
  const int lim = rows.lim(g, i), qd = rows.qdoc(g, i);
  const bool on = ok && qd >= 0;
  bf16x8 qf[T::KS];
  T::own(static_cast<const bf16*>(g.q.p) + b * g.q.b + (int64_t)i * g.q.t + h * g.q.h, on, g.dh, half, qf);
  const int n = list.template build<true>(g, rows, wave, lane, u.blk, qd, ok);
  const Streams<DP> kv(g.k, hk, g.v, hk, b, wave, lane);
  StreamDocs<DP> sd(rows.k, g.Sk, kv.row);
  const unsigned lds = lds_addr(smem), mine = lds + wave * T::N * 1024;
  const Score sc(g, h);
  f32x16 o[T::DT];
#pragma unroll
  for (int dt = 0; dt < T::DT; ++dt) o[dt] = zero16();
  float m = 0.f, lsum = 0.f;
  auto load = [&](int e, int at) {
    const int j0 = list.tile(e) * kRuleTile;
    sd.load(j0);
    kv.load(mine + at * 2 * T::BYTES, j0, g.Sk, g.dh);
  };
  auto finish = [&](int e, int at) {
    bool keep[T::N];
    sd.finish(list.tile(e) * kRuleTile, -1, kdoc + at * kRuleTile, kv.piece == 0, keep);
    loads_done();
    if (!list.plain(e)) kv.clear(mine + at * 2 * T::BYTES, lane, keep);
  };
  int e = list.entry(0), next = list.entry(1);
  zero_tiles<DP>(smem, g.dh);
  if (n > 0) { load(e, 0); finish(e, 0); }
  for (int it = 0; it < n; ++it) {
    __syncthreads();
    if (it + 1 < n) load(next, (it + 1) & 1);
    if (list.needed(e, wave)) {
      const unsigned kb = lds + (it & 1) * 2 * T::BYTES;
      const int j0 = list.tile(e) * kRuleTile;
      const float at = (float)(g.q0 + i - j0 - 32 * x0 - 4 * half);
      f32x16 s[NX];
      // scores less the reference, of the visible pairs; -infinity of the others
      auto scores = [&]() {
#pragma unroll
        for (int st = 0; st < NX; ++st) {
          s[st] = T::dot(T::row_addr(kb, lane) + 32 * x0 * T::RB, 32 * st, qf);
#pragma unroll
          for (int v = 0; v < 16; ++v) s[st][v] = sc.at<MOD>((MOD & 1) ? sc.bend(s[st][v]) : s[st][v], at - (float)(32 * st + acc_row(v)), -m);
        }
        if (!list.whole(e, wave)) {
          const int far = lim - j0 - 32 * x0 - 4 * half;
#pragma unroll
          for (int st = 0; st < NX; ++st)
#pragma unroll
            for (int g4 = 0; g4 < 4; ++g4) {
              int kd[4];
              four(kdoc + (it & 1) * kRuleTile + 32 * (x0 + st) + 8 * g4 + 4 * half, kd);
#pragma unroll
              for (int x = 0; x < 4; ++x) s[st][4 * g4 + x] = kd[x] == qd ? s[st][4 * g4 + x] : -INFINITY;
              if (g.order != 0) {   // (rows behind the last have no document)
#pragma unroll
                for (int x = 0; x < 4; ++x) s[st][4 * g4 + x] = 32 * st + 8 * g4 + x <= far ? s[st][4 * g4 + x] : -INFINITY;
              }
            }
        }
      };
      auto weights = [&](float shift) {
        float sum = 0.f;
#pragma unroll
        for (int st = 0; st < NX; ++st)
#pragma unroll
          for (int v = 0; v < 16; ++v) {
            s[st][v] = fast_exp2(s[st][v] - shift);
            sum += s[st][v];
          }
        return sum;
      };
      bool found = !__any(on && lsum == 0.f);
      float sum = 0.f;
      if (found) {
        scores();
        sum = weights(0.f);
        found = !__any(sum > kGrown);
      }
      if (!found) {   // some row has no reference yet, or one that is too low
        scores();
        float mx = s[0][0];
#pragma unroll
        for (int v = 1; v < 16 * NX; ++v) mx = fmaxf(mx, s[v >> 4][v & 15]);
        mx = fmaxf(mx, half_swap(mx));
        const bool move = mx > -INFINITY && (lsum == 0.f || mx > 0.f);
        const float up = move ? mx : 0.f, alpha = fast_exp2(-up);
        m += up;
        lsum *= lsum == 0.f ? 1.f : alpha;
#pragma unroll
        for (int dt = 0; dt < T::DT; ++dt)
#pragma unroll
          for (int v = 0; v < 16; ++v) o[dt][v] *= lsum == 0.f ? 0.f : alpha;
        sum = weights(up);
      }
      lsum += sum + half_swap(sum);
#pragma unroll
      for (int st = 0; st < NX; ++st) {
        T::add(T::col_addr(kb + T::BYTES, lane) + 32 * x0 * T::RB, 32 * st, s[st], o);
        if (FEW) T::add(T::col_addr(kb + T::BYTES, lane) + 32 * x0 * T::RB, 32 * st, left_out(s[st]), o);
      }
    }
    if (it + 1 < n) finish(next, (it + 1) & 1);
    e = next;
    next = list.entry(it + 2 <= list.tiles ? it + 2 : list.tiles);
  }
  if (SHARE == 2) {   // the second wave of a group leaves its sums, and the reference that they go by
    float* room = reinterpret_cast<float*>(smem);
    float* stat = room + 128 * 16 * T::DT + group * 128;
    __syncthreads();
    if (x0) {
      leave(room, group, lane, o);
      stat[lane] = m;
      stat[64 + lane] = lsum;
    }
    __syncthreads();
    if (x0) return;
    const float m2 = stat[lane], sum2 = stat[64 + lane];
    const float top = lsum == 0.f ? m2 : sum2 == 0.f ? m : fmaxf(m, m2);
    const float f = lsum == 0.f ? 0.f : fast_exp2(m - top), f2 = sum2 == 0.f ? 0.f : fast_exp2(m2 - top);
    take(room, group, lane, o, f, f2);
    lsum = lsum * f + sum2 * f2;
    m = top;
  }
  if (!ok) return;
  T::put(static_cast<bf16*>(const_cast<void*>(g.o.p)) + b * g.o.b + (int64_t)i * g.o.t + h * g.o.h, g.dh, half, lsum == 0.f ? 0.f : 1.f / lsum, o);
  if (g.lse && half == 0) g.lse[(int64_t)b * g.lse_b + (int64_t)h * g.lse_h + i] = lsum == 0.f ? -INFINITY : (m + __log2f(lsum)) * 0.693147180559945f;
}

// ---------------------------------------------------------------------------------------------------------------------------
// backward: dq (128 queries a workgroup), which also leaves each query's delta, then dk and dv (128 keys a workgroup, the heads that
// share them one after the other).  Two launches, because no workgroup sees all of a row and a column, and sums by atomics would
// depend on their order.  Three workgroups a CU at a head size of 64 where a wave owns its rows alone (168 registers, and 3 to 26 values
// spilled), two where two share them; 272 - 357 registers at 128, one wave a SIMD, which then waits for its own LDS reads: 12 x 384
// rows x 10 heads of 128 take 108 us, of 64 49.
// ---------------------------------------------------------------------------------------------------------------------------
// delta_i = dO_i . o_i with o rounded to bf16 is off by 2^-9 of |dO||o|, which for a query with few keys, or one that takes most
// of the weight, is as large as dS itself.  So the pass uses that value d only to centre dP, and takes out what is left of it:
// with r_i = sum_j p_ij (dP_ij - d_i), the true delta is d_i + r_i, and dq_i = scale (sum_j w_ij (dP_ij - d_i) k_j - r_i sum_j
// w_ij k_j), w = p (1 - tanh^2): one more product with the keys' fragments that the pass has in registers anyway.  Without a cap
// the r of that product is summed from dS as it was rounded to bf16 for the other (two to an instruction): the part of those
// roundings that all keys share, which dS itself, summing to 0, does not have, then cancels.
// A query that sees one key has dS = 0, where dP - delta would leave the rounding of two different sums.  The pass counts the keys that
// have some weight, in masked tiles (a whole one has several) and only until each of the wave's queries has met two, as lane masks in
// scalar registers: the kernel has no vector register left.  The keys' pass finds a mark in place of such a query's delta, and looks
// for it in masked tiles only: a query whose weights vanish beside one must not be marked where it sees 32 keys that one wave owns
// there, so seeing the first and the last of those counts as two, whatever their weights.  (Counting by the masks throughout
// makes the compiler keep them all: 193 us back against 155 at 4 x 2048 x 16.)
constexpr uint32_t kOneKey = 0x7fc0a11eu;   // a NaN that no operation makes

template <int DP, int MOD, int SHARE, bool FEW>
__global__ __launch_bounds__(256, DP == 64 ? 4 - SHARE : 1) void rule_dq_kernel(AttnRuleArgs g) {
  typedef Tile<DP> T;
  constexpr int kRows = 128 / SHARE, NX = 2 / SHARE;   // rows of a workgroup; parts of 32 rows of a tile that a wave takes
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  int* kdoc = reinterpret_cast<int*>(smem + 4 * T::BYTES);
  const RuleList<32, SHARE> list(kdoc + 2 * kRuleTile, g.Sk);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5;
  const int group = wave / SHARE, x0 = wave % SHARE * NX;   // rows of the wave; its first part of a tile
  const int nqb = (g.Sq + kRows - 1) / kRows;
  const RuleUnit u(g, nqb, g.H, blockIdx.x, gridDim.x, g.order != 0);
  const int b = u.b, h = u.h, hk = h / (g.H / g.Hkv);
  const int i = u.blk * kRows + group * 32 + (lane & 31);
  const RuleRows rows(g, b);
  const int lim = rows.lim(g, i), qd = rows.qdoc(g, i);
  const bool ok = i < g.Sq, on = ok && qd >= 0;
  bf16x8 qf[T::KS], dof[T::KS];
  T::own(static_cast<const bf16*>(g.q.p) + b * g.q.b + (int64_t)i * g.q.t + h * g.q.h, on, g.dh, half, qf);
  T::own(static_cast<const bf16*>(g.d_o.p) + b * g.d_o.b + (int64_t)i * g.d_o.t + h * g.d_o.h, on, g.dh, half, dof);
  const float nlse = on ? -rule_lse2(g.lse[(int64_t)b * g.lse_b + (int64_t)h * g.lse_h + i]) : -INFINITY;
  const float dl = T::own_dot(static_cast<const bf16*>(g.o.p) + b * g.o.b + (int64_t)i * g.o.t + h * g.o.h, on, g.dh, half, dof);
  const int n = list.template build<true>(g, rows, wave, lane, u.blk, qd, ok);
  const Streams<DP> kv(g.k, hk, g.v, hk, b, wave, lane);
  StreamDocs<DP> sd(rows.k, g.Sk, kv.row);
  const unsigned lds = lds_addr(smem), mine = lds + wave * T::N * 1024;
  const Score sc(g, h);
  f32x16 dq[T::DT], wk[T::DT];
#pragma unroll
  for (int dt = 0; dt < T::DT; ++dt) { dq[dt] = zero16(); wk[dt] = zero16(); }
  float rest = 0.f, rounded = 0.f;   // r, and r from dS as it was rounded
  uint64_t one = 0, two = __ballot(!on);   // lanes that have met a key of some weight, and another
  auto load = [&](int e, int at) {
    const int j0 = list.tile(e) * kRuleTile;
    sd.load(j0);
    kv.load(mine + at * 2 * T::BYTES, j0, g.Sk, g.dh);
  };
  auto finish = [&](int e, int at) {
    bool keep[T::N];
    sd.finish(list.tile(e) * kRuleTile, -1, kdoc + at * kRuleTile, kv.piece == 0, keep);
    loads_done();
    if (!list.plain(e)) kv.clear(mine + at * 2 * T::BYTES, lane, keep);
  };
  int e = list.entry(0), next = list.entry(1);
  zero_tiles<DP>(smem, g.dh);
  if (n > 0) { load(e, 0); finish(e, 0); }
  for (int it = 0; it < n; ++it) {
    __syncthreads();
    if (it + 1 < n) load(next, (it + 1) & 1);
    if (list.needed(e, wave)) {
      const unsigned kb = lds + (it & 1) * 2 * T::BYTES;
      const int j0 = list.tile(e) * kRuleTile;
      const bool whole = list.whole(e, wave);
      const float at = (float)(g.q0 + i - j0 - 32 * x0 - 4 * half);
      const int far = lim - j0 - 32 * x0 - 4 * half;
#pragma unroll 1
      for (int st = 0; st < NX; ++st) {
        f32x16 s = T::dot(T::row_addr(kb, lane) + 32 * x0 * T::RB, 32 * st, qf);
        f32x16 dp = T::dot(T::row_addr(kb + T::BYTES, lane) + 32 * x0 * T::RB, 32 * st, dof);
        f32x16 w;
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const float r = (MOD & 1) ? sc.bend(s[v]) : s[v];
          w[v] = fast_exp2(sc.at<MOD>(r, at - (float)(32 * st + acc_row(v)), nlse));
          dp[v] -= dl;
          s[v] = r;
        }
        if (!whole) {
#pragma unroll
          for (int g4 = 0; g4 < 4; ++g4) {
            int kd[4];
            four(kdoc + (it & 1) * kRuleTile + 32 * (x0 + st) + 8 * g4 + 4 * half, kd);
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const int v = 4 * g4 + x;
              w[v] = kd[x] == qd ? w[v] : 0.f;
              if (g.order != 0) w[v] = 32 * st + 8 * g4 + x <= far ? w[v] : 0.f;
            }
          }
          if (~(two | swapped(two) | (one & swapped(one)))) {   // some query has not met two keys yet
#pragma unroll
            for (int v = 0; v < 16; ++v) {
              const uint64_t here = __ballot(w[v] != 0.f);
              two |= one & here;
              one |= here;
            }
            const int* ends = kdoc + (it & 1) * kRuleTile + 32 * (x0 + st) + 4 * half;
            two |= __ballot(ends[0] == qd && ends[27] == qd && (g.order == 0 || 32 * st + 27 <= far));
          }
        } else {
          two = ~0ull;
        }
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          dp[v] *= w[v];
          rest += dp[v];
          if (MOD & 1) {
            const float f = 4.f * s[v] * (1.f - s[v]);
            dp[v] *= f;
            w[v] *= f;
          }
        }
        T::add2(T::col_addr(kb, lane) + 32 * x0 * T::RB, 32 * st, dp, dq, w, wk, (MOD & 1) ? nullptr : &rounded);
        if (FEW)
          T::add2(T::col_addr(kb, lane) + 32 * x0 * T::RB, 32 * st, left_out(dp), dq, left_out(w), wk, (MOD & 1) ? nullptr : &rounded);
      }
    }
    if (it + 1 < n) finish(next, (it + 1) & 1);
    e = next;
    next = list.entry(it + 2 <= list.tiles ? it + 2 : list.tiles);
  }
  rest += half_swap(rest);
  rounded = (MOD & 1) ? rest : rounded + half_swap(rounded);
  int seen = (int)(one >> lane & 1) + 2 * (int)(two >> lane & 1);
  seen += __float_as_int(half_swap(__int_as_float(seen)));
  float* room = reinterpret_cast<float*>(smem);
  if (SHARE == 2) {   // r is the sum over both waves' keys, and each takes its own part of the product out with it
    float* stat = room + group * 384;
    __syncthreads();
    stat[192 * x0 + lane] = rest;
    stat[192 * x0 + 64 + lane] = rounded;
    stat[192 * x0 + 128 + lane] = __int_as_float(seen);
    __syncthreads();
    const float rest2 = stat[192 * (1 - x0) + lane], rounded2 = stat[192 * (1 - x0) + 64 + lane];
    seen += __float_as_int(stat[192 * (1 - x0) + 128 + lane]);
    rest = x0 ? rest2 + rest : rest + rest2;
    rounded = x0 ? rounded2 + rounded : rounded + rounded2;
  }
  if (SHARE == 1 && !ok) return;
  if (ok && x0 == 0 && half == 0) g.delta[((int64_t)b * g.H + h) * g.Sq + i] = seen == 1 ? __uint_as_float(kOneKey) : on ? dl + rest : 0.f;
#pragma unroll
  for (int dt = 0; dt < T::DT; ++dt)
#pragma unroll
    for (int v = 0; v < 16; ++v) dq[dt][v] = seen == 1 ? 0.f : fmaf(-rounded, wk[dt][v], dq[dt][v]);
  if (SHARE == 2) {
    __syncthreads();
    if (x0) leave(room, group, lane, dq);
    __syncthreads();
    if (x0 || !ok) return;
    take(room, group, lane, dq, 1.f, 1.f);
  }
  T::put(static_cast<bf16*>(const_cast<void*>(g.dq.p)) + b * g.dq.b + (int64_t)i * g.dq.t + h * g.dq.h, g.dh, half, g.scale, dq);
}

template <int DP, int MOD, int SHARE, bool FEW>
__global__ __launch_bounds__(256, DP == 64 ? 4 - SHARE : 1) void rule_dkv_kernel(AttnRuleArgs g) {
  typedef Tile<DP> T;
  constexpr int kRows = 128 / SHARE, NX = 2 / SHARE;   // rows of a workgroup; parts of 32 rows of a tile that a wave takes
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  float* stat = reinterpret_cast<float*>(smem + 4 * T::BYTES);                // [2][-lse, delta][64], behind [2][Q tile, dO tile]
  int* info = reinterpret_cast<int*>(stat + 4 * kRuleTile);                   // [2][document, lim][64]
  const RuleList<32, SHARE> list(info + 4 * kRuleTile, g.Sq);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5;
  const int group = wave / SHARE, x0 = wave % SHARE * NX;   // rows of the wave; its first part of a tile
  const int nkb = (g.Sk + kRows - 1) / kRows, G = g.H / g.Hkv;
  const RuleUnit u(g, nkb, g.Hkv, blockIdx.x, gridDim.x, false);
  const int b = u.b, hk = u.h;
  const int j = u.blk * kRows + group * 32 + (lane & 31);
  const RuleRows rows(g, b);
  const int kd = rows.kdoc(g, j);
  const bool ok = j < g.Sk, on = ok && kd >= 0;
  bf16x8 kf[T::KS], vf[T::KS];
  T::own(static_cast<const bf16*>(g.k.p) + b * g.k.b + (int64_t)j * g.k.t + hk * g.k.h, on, g.dh, half, kf);
  T::own(static_cast<const bf16*>(g.v.p) + b * g.v.b + (int64_t)j * g.v.t + hk * g.v.h, on, g.dh, half, vf);
  const int n = list.template build<false>(g, rows, wave, lane, u.blk, kd, ok);
  f32x16 dk[T::DT], dv[T::DT];
#pragma unroll
  for (int dt = 0; dt < T::DT; ++dt) { dk[dt] = zero16(); dv[dt] = zero16(); }
  const int first = list.entry(0);
  const unsigned lds = lds_addr(smem), mine = lds + wave * T::N * 1024;
  zero_tiles<DP>(smem, g.dh);
  // the heads that share these keys, one after the other
  for (int h = hk * G; h < hk * G + G; ++h) {
    const Streams<DP> qo(g.q, h, g.d_o, h, b, wave, lane);
    StreamDocs<DP> sd(rows.q, g.Sq, qo.row);
    const Score sc(g, h);
    const float* lse = g.lse + (int64_t)b * g.lse_b + (int64_t)h * g.lse_h;
    const float* delta = g.delta + ((int64_t)b * g.H + h) * g.Sq;
    float rl = 0.f, rdl = 0.f;
    auto load = [&](int e, int at) {
      const int i0 = list.tile(e) * kRuleTile;
      sd.load(i0);
      if (tid < kRuleTile) {
        const int r = i0 + tid < g.Sq ? i0 + tid : g.Sq - 1;
        rl = lse[r];
        rdl = delta[r];
      }
      qo.load(mine + at * 2 * T::BYTES, i0, g.Sq, g.dh);
    };
    auto finish = [&](int e, int at) {
      const int i0 = list.tile(e) * kRuleTile;
      bool keep[T::N];
      sd.finish(i0, -2, info + at * 2 * kRuleTile, qo.piece == 0, keep);
      if (tid < kRuleTile) {
        // a row behind the last has probability 0; so has one that sees nothing (padding among them)
        stat[at * 2 * kRuleTile + tid] = i0 + tid < g.Sq ? -rule_lse2(rl) : -INFINITY;
        stat[at * 2 * kRuleTile + kRuleTile + tid] = rdl;
        info[at * 2 * kRuleTile + kRuleTile + tid] = rows.lim(g, i0 + tid);
      }
      loads_done();
      if (!list.plain(e)) qo.clear(mine + at * 2 * T::BYTES, lane, keep);
    };
    int e = first, next = list.entry(1);
    if (n > 0) {
      if (h > hk * G) __syncthreads();   // the last tile of the head before may still be read
      load(e, 0);
      finish(e, 0);
    }
    for (int it = 0; it < n; ++it) {
      __syncthreads();
      if (it + 1 < n) load(next, (it + 1) & 1);
      if (list.needed(e, wave)) {
        const unsigned qb = lds + (it & 1) * 2 * T::BYTES;
        const float* st2 = stat + (it & 1) * 2 * kRuleTile;
        const int* inf = info + (it & 1) * 2 * kRuleTile;
        const bool whole = list.whole(e, wave);
        const float at = (float)(g.q0 + list.tile(e) * kRuleTile + 32 * x0 - j + 4 * half);
#pragma unroll 1
        for (int st = 0; st < NX; ++st) {
          f32x16 s = T::dot(T::row_addr(qb, lane) + 32 * x0 * T::RB, 32 * st, kf);
          f32x16 ds = T::dot(T::row_addr(qb + T::BYTES, lane) + 32 * x0 * T::RB, 32 * st, vf);
#pragma unroll
          for (int g4 = 0; g4 < 4; ++g4) {
            const int r0 = 32 * (x0 + st) + 8 * g4 + 4 * half;
            const float4 l4 = *reinterpret_cast<const float4*>(st2 + r0);
            const float4 d4 = *reinterpret_cast<const float4*>(st2 + kRuleTile + r0);
            const float nl[4] = {l4.x, l4.y, l4.z, l4.w}, dl[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const int v = 4 * g4 + x;
              const float r = (MOD & 1) ? sc.bend(s[v]) : s[v];
              s[v] = fast_exp2(sc.at<MOD>(r, at + (float)(32 * st + acc_row(v)), nl[x]));
              ds[v] -= dl[x];
              if (MOD & 1) ds[v] *= 4.f * r * (1.f - r);
            }
            if (!whole) {
              int qd[4];
              four(inf + r0, qd);
#pragma unroll
              for (int x = 0; x < 4; ++x) s[4 * g4 + x] = qd[x] == kd ? s[4 * g4 + x] : 0.f;
              if (g.order != 0) {
                int lm[4];
                four(inf + kRuleTile + r0, lm);
#pragma unroll
                for (int x = 0; x < 4; ++x) s[4 * g4 + x] = j <= lm[x] ? s[4 * g4 + x] : 0.f;
              }
#pragma unroll
              for (int x = 0; x < 4; ++x) ds[4 * g4 + x] = __float_as_uint(dl[x]) == kOneKey ? 0.f : ds[4 * g4 + x];
            }
#pragma unroll
            for (int x = 0; x < 4; ++x) ds[4 * g4 + x] *= s[4 * g4 + x];
          }
          T::add(T::col_addr(qb + T::BYTES, lane) + 32 * x0 * T::RB, 32 * st, s, dv);
          if (FEW) T::add(T::col_addr(qb + T::BYTES, lane) + 32 * x0 * T::RB, 32 * st, left_out(s), dv);
          T::add(T::col_addr(qb, lane) + 32 * x0 * T::RB, 32 * st, ds, dk);
          if (FEW) T::add(T::col_addr(qb, lane) + 32 * x0 * T::RB, 32 * st, left_out(ds), dk);
        }
      }
      if (it + 1 < n) finish(next, (it + 1) & 1);
      e = next;
      next = list.entry(it + 2 <= list.tiles ? it + 2 : list.tiles);
    }
  }
  if (SHARE == 2) {
    float* room = reinterpret_cast<float*>(smem);
    __syncthreads();
    if (x0) {
      leave(room, group, lane, dk);
      leave(room + 128 * 16 * T::DT, group, lane, dv);
    }
    __syncthreads();
    if (x0) return;
    take(room, group, lane, dk, 1.f, 1.f);
    take(room + 128 * 16 * T::DT, group, lane, dv, 1.f, 1.f);
  }
  if (ok) {
    T::put(static_cast<bf16*>(const_cast<void*>(g.dk.p)) + b * g.dk.b + (int64_t)j * g.dk.t + hk * g.dk.h, g.dh, half, g.scale, dk);
    T::put(static_cast<bf16*>(const_cast<void*>(g.dv.p)) + b * g.dv.b + (int64_t)j * g.dv.t + hk * g.dv.h, g.dh, half, 1.f, dv);
  }
}

template <int DP>
size_t lds_bytes(int streamed, bool dkv) {
  return (size_t)4 * Tile<DP>::BYTES + (dkv ? 8 : 2) * kRuleTile * 4 + RuleList<32>::ints((streamed + kRuleTile - 1) / kRuleTile) * 4;
}
template <typename K>
hipError_t launch(K kernel, int blocks, size_t lds, const AttnRuleArgs& g, hipStream_t st) {
  if (blocks == 0) return hipSuccess;
  PT_RULE_LDS(kernel, lds);
  hipLaunchKernelGGL(kernel, dim3(blocks), dim3(256), lds, st, g);
  return hipGetLastError();
}
int blocks_of(int heads, int rows, int share) { return (int)rule_blocks(heads, rows, 128 / share); }

template <int DP, int MOD, int SHARE, bool FEW>
hipError_t launch_fwd(const AttnRuleArgs& g, hipStream_t st) {
  return launch(rule_fwd_kernel<DP, MOD, SHARE, FEW>, blocks_of(g.nb * g.H, g.Sq, SHARE), lds_bytes<DP>(g.Sk, false), g, st);
}
template <int DP, int MOD, int SHARE, bool FEW>
hipError_t launch_dq(const AttnRuleArgs& g, hipStream_t st) {
  return launch(rule_dq_kernel<DP, MOD, SHARE, FEW>, blocks_of(g.nb * g.H, g.Sq, SHARE), lds_bytes<DP>(g.Sk, false), g, st);
}
template <int DP, int MOD, int SHARE, bool FEW>
hipError_t launch_dkv(const AttnRuleArgs& g, hipStream_t st) {
  return launch(rule_dkv_kernel<DP, MOD, SHARE, FEW>, blocks_of(g.nb * g.Hkv, g.Sk, SHARE), lds_bytes<DP>(g.Sq, true), g, st);
}
template <int DP, int MOD>
hipError_t launch_all(const AttnRuleArgs& g, bool bwd, hipStream_t st) {
  const RuleShape s = rule_shape(g);
  const bool few = rule_few_pairs(s);
  if (!bwd) return few ? launch_fwd<DP, MOD, 2, true>(g, st) : rule_share_fwd(s) == 2 ? launch_fwd<DP, MOD, 2, false>(g, st) : launch_fwd<DP, MOD, 1, false>(g, st);
  const hipError_t e = few ? launch_dq<DP, MOD, 2, true>(g, st) : rule_share_dq(s) == 2 ? launch_dq<DP, MOD, 2, false>(g, st) : launch_dq<DP, MOD, 1, false>(g, st);
  if (e != hipSuccess) return e;
  return few ? launch_dkv<DP, MOD, 2, true>(g, st) : rule_share_dkv(s) == 2 ? launch_dkv<DP, MOD, 2, false>(g, st) : launch_dkv<DP, MOD, 1, false>(g, st);
}
template <int DP>
hipError_t by_mod(const AttnRuleArgs& g, bool bwd, hipStream_t st) {
  switch ((g.cap > 0.f ? 1 : 0) | (g.slopes ? 2 : 0)) {
    case 0: return launch_all<DP, 0>(g, bwd, st);
    case 1: return launch_all<DP, 1>(g, bwd, st);
    case 2: return launch_all<DP, 2>(g, bwd, st);
    default: return launch_all<DP, 3>(g, bwd, st);
  }
}

}  // namespace

hipError_t attention_rule_fwd(int dt, const AttnRuleArgs& g, hipStream_t st) {
  return dt ? attention_rule_bf16(g, false, st) : attention_rule_f32(g, false, st);
}
hipError_t attention_rule_bwd(int dt, const AttnRuleArgs& g, hipStream_t st) {
  return dt ? attention_rule_bf16(g, true, st) : attention_rule_f32(g, true, st);
}

hipError_t attention_rule_bf16(const AttnRuleArgs& g, bool bwd, hipStream_t st) {
  return g.dh <= 64 ? by_mod<64>(g, bwd, st) : by_mod<128>(g, bwd, st);
}

}  // namespace pt
