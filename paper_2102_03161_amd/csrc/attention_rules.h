// What the kernels of attention under a rule share: their arguments, what a query sees, and the list of the tiles that a
// workgroup has to visit.
#pragma once
#include "common.h"
#include "kernels.h"

namespace pt {

constexpr int kRuleTile = 64;            // rows of a streamed tile

// more than 64 KB of dynamic LDS has to be asked for, kernel by kernel
#define PT_RULE_LDS(kernel, bytes)                                                                                          \
  do {                                                                                                                      \
    if ((bytes) > 64 * 1024) {                                                                                              \
      const hipError_t e_ = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)(bytes)); \
      if (e_ != hipSuccess) return e_;                                                                                      \
    }                                                                                                                       \
  } while (0)

// natural log-sum-exp -> log2 domain; a row that sees nothing has -inf and gets +inf, hence probability 0 everywhere
__device__ __forceinline__ float rule_lse2(float lse) { return lse == -INFINITY ? INFINITY : lse * 1.44269504088896f; }

// What queries and keys of one sample see.  lim: the last key that a query's position allows; documents below 0 are padding,
// reported as -2 for queries and -1 for keys, so that two of them never match.
struct RuleRows {
  const int32_t* q;
  const int32_t* k;
  int prefix;
  __device__ __forceinline__ RuleRows(const AttnRuleArgs& g, int b) {
    const int64_t r = g.bmap ? g.bmap[b] : b;
    q = g.qdoc ? g.qdoc + r * g.Sq : nullptr;
    k = g.kdoc ? g.kdoc + r * g.Sk : nullptr;
    prefix = g.order == 2 ? g.prefix[r] : 0;
  }
  __device__ __forceinline__ int lim(const AttnRuleArgs& g, int i) const {
    if (g.order == 0) return g.Sk - 1;
    const int at = g.q0 + i, to = at > prefix - 1 ? at : prefix - 1;
    return to < g.Sk - 1 ? to : g.Sk - 1;
  }
  __device__ __forceinline__ int qdoc(const AttnRuleArgs& g, int i) const {
    if (i >= g.Sq) return -2;
    const int d = q ? q[i] : 0;
    return d < 0 ? -2 : d;
  }
  __device__ __forceinline__ int kdoc(const AttnRuleArgs& g, int j) const {
    if (j >= g.Sk) return -1;
    const int d = k ? k[j] : 0;
    return d < 0 ? -1 : d;
  }
};

// Which (sample, head, block of owned rows) a workgroup takes.  Workgroups go to the eight XCDs in turn; the units are dealt so
// that one XCD gets consecutive ones: the blocks of a head, and the heads that share keys, find them in the same L2.
struct RuleUnit {
  int b, h, blk;
  __device__ __forceinline__ RuleUnit(const AttnRuleArgs& g, int nblk, int heads, int id, int total) {
    const int q = total / 8, r = total % 8, x = id % 8;
    const int u = x * q + (x < r ? x : r) + id / 8;
    blk = u % nblk;
    h = u / nblk % heads;
    b = u / nblk / heads;
  }
  __device__ __forceinline__ RuleUnit(const AttnRuleArgs& g, int nblk, int heads) : RuleUnit(g, nblk, heads, blockIdx.x, g.nb * heads * nblk) {}
  __device__ __forceinline__ RuleUnit(const AttnRuleArgs& g, int nblk, int heads, int id) : RuleUnit(g, nblk, heads, id, g.nb * heads * nblk) {}
};

// The tiles that a workgroup of four waves visits: entries tile << 8 | full bits << 4 | needed bits.  It lives in LDS behind four
// waves' ranges and the count.
struct RuleList {
  int* base;
  __device__ __forceinline__ explicit RuleList(int* p) : base(p) {}
  static size_t ints(int tiles) { return (size_t)16 + 4 + tiles; }
  __device__ __forceinline__ int* entries() const { return base + 20; }
  __device__ __forceinline__ int entry(int it) const { return __builtin_amdgcn_readfirstlane(entries()[it]); }
  __device__ __forceinline__ int tile(int it) const { return entry(it) >> 8; }
  __device__ __forceinline__ bool needed(int it, int wave) const { return entry(it) >> wave & 1; }
  __device__ __forceinline__ bool full(int it, int wave) const { return entry(it) >> (4 + wave) & 1; }

  static __device__ __forceinline__ int wave_min(int v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) { const int x = __shfl_xor(v, o, 64); v = x < v ? x : v; }
    return v;
  }
  static __device__ __forceinline__ int wave_max(int v) { return ~wave_min(~v); }

  // need / full of one tile for the four waves; d: the lane's row's document (below 0: none), lo / hi: the tile's position bounds
  template <bool KEYS>
  __device__ __forceinline__ int classify(int d, bool in, int lo, int hi) const {
    int e = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const int dmin = base[4 * w], dmax = base[4 * w + 1], far = base[4 * w + 2], near = base[4 * w + 3];
      const bool any = __ballot(in && d >= dmin && d <= dmax) != 0;
      const bool all = __ballot(in ? d != dmin : KEYS) == 0;
      const bool need = any && (KEYS ? lo <= far : hi >= far);
      const bool full = need && all && (KEYS ? hi <= near : lo >= near);
      e |= (need ? 1 : 0) << w | (full ? 1 : 0) << (4 + w);
    }
    return e;
  }
  __device__ __forceinline__ int compact(int nt, int wave, int lane) const {
    __syncthreads();
    if (wave == 0) {
      int n = 0;
      for (int t0 = 0; t0 < nt; t0 += 64) {
        const int t = t0 + lane;
        const int e = t < nt ? entries()[t] : 0;
        const uint64_t bits = __ballot(e != 0);
        if (e) entries()[n + __popcll(bits & ((1ull << lane) - 1))] = t << 8 | e;
        n += __popcll(bits);
      }
      if (lane == 0) base[16] = n;
    }
    __syncthreads();
    return __builtin_amdgcn_readfirstlane(base[16]);
  }
  // tiles of keys for the wave's queries (owned by lane; halves hold the same rows).  Ranges: documents of the rows that see
  // anything, the largest lim (tiles behind it are skipped), and the smallest (tiles in front of it may be whole), the latter -1
  // where the rows are not all of one document.
  __device__ __forceinline__ int keys(const AttnRuleArgs& g, const RuleRows& rows, int wave, int lane, bool ok, int lim, int d) const {
    const bool on = ok && d >= 0;
    const int dmin = wave_min(on ? d : 0x7fffffff), dmax = wave_max(on ? d : -1);
    const int far = wave_max(on ? lim : -1);
    int near = wave_min(on ? lim : 0x7fffffff);
    if (dmin != dmax || __any(ok && !on)) near = -1;
    if (lane == 0) { base[4 * wave] = dmin; base[4 * wave + 1] = dmax; base[4 * wave + 2] = far; base[4 * wave + 3] = near; }
    __syncthreads();
    const int nt = (g.Sk + kRuleTile - 1) / kRuleTile;
    for (int t0 = wave * 8; t0 < nt; t0 += 32) {
      int kd[8];
#pragma unroll
      for (int x = 0; x < 8; ++x) kd[x] = rows.kdoc(g, (t0 + x) * kRuleTile + lane);
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const int j0 = (t0 + x) * kRuleTile;
        const int e = classify<true>(kd[x], j0 + lane < g.Sk, j0, j0 + kRuleTile - 1);
        if (lane == 0 && t0 + x < nt) entries()[t0 + x] = e;
      }
    }
    return compact(nt, wave, lane);
  }
  // tiles of queries for the wave's keys: documents, the first key's position (a tile whose last query does not reach it is
  // skipped) and the last one's (a tile whose first query reaches it may be whole)
  __device__ __forceinline__ int queries(const AttnRuleArgs& g, const RuleRows& rows, int wave, int lane, bool ok, int j, int d) const {
    const bool on = ok && d >= 0;
    const int dmin = wave_min(on ? d : 0x7fffffff), dmax = wave_max(on ? d : -1);
    const int far = wave_min(on ? j : 0x7fffffff);
    int near = wave_max(on ? j : -1);
    if (dmin != dmax || __any(ok && !on)) near = 0x7fffffff;
    if (lane == 0) { base[4 * wave] = dmin; base[4 * wave + 1] = dmax; base[4 * wave + 2] = far; base[4 * wave + 3] = near; }
    __syncthreads();
    const int nt = (g.Sq + kRuleTile - 1) / kRuleTile;
    for (int t0 = wave * 8; t0 < nt; t0 += 32) {
      int qd[8];
#pragma unroll
      for (int x = 0; x < 8; ++x) qd[x] = rows.qdoc(g, (t0 + x) * kRuleTile + lane);
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const int i0 = (t0 + x) * kRuleTile, i1 = i0 + kRuleTile - 1;
        const int e = classify<false>(qd[x], i0 + lane < g.Sq, rows.lim(g, i0), rows.lim(g, i1 < g.Sq ? i1 : g.Sq - 1));
        if (lane == 0 && t0 + x < nt) entries()[t0 + x] = e;
      }
    }
    return compact(nt, wave, lane);
  }
};

}  // namespace pt
