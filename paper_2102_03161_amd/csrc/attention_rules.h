// What the kernels of attention under a rule share: their arguments, what a query sees, and the list of the tiles that a
// workgroup has to visit.
#pragma once
#include "attention_choice.h"
#include "common.h"
#include "kernels.h"

namespace pt {

constexpr int kRuleTile = 64;            // rows of a streamed tile

inline RuleShape rule_shape(const AttnRuleArgs& g) { return RuleShape{g.nb, g.Sq, g.Sk, g.H, g.Hkv, g.dh, g.order != 0, g.qdoc != nullptr}; }

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
    q = g.qdoc ? g.qdoc + r * g.qdoc_ld : nullptr;
    k = g.kdoc ? g.kdoc + r * g.kdoc_ld : nullptr;
    prefix = g.order == 2 ? g.prefix[r] : 0;
  }
  __device__ __forceinline__ int lim(const AttnRuleArgs& g, int i) const {
    if (g.order == 0) return g.Sk - 1;
    const int at = g.q0 + i, to = at >= prefix ? at : prefix - 1;   // (the prefix may be any int)
    return to < g.Sk - 1 ? to : g.Sk - 1;
  }
  // as they stand in memory (below 0 behind the last row): nothing looks at the value, so that a load for a later tile is not
  // waited for where it is issued; q_id / k_id turn it into the above
  __device__ __forceinline__ int q_raw(const AttnRuleArgs& g, int i) const { return i < g.Sq ? (q ? q[i] : 0) : -1; }
  __device__ __forceinline__ int k_raw(const AttnRuleArgs& g, int j) const { return j < g.Sk ? (k ? k[j] : 0) : -1; }
  static __device__ __forceinline__ int q_id(int raw) { return raw < 0 ? -2 : raw; }
  static __device__ __forceinline__ int k_id(int raw) { return raw < 0 ? -1 : raw; }
  __device__ __forceinline__ int qdoc(const AttnRuleArgs& g, int i) const { return q_id(q_raw(g, i)); }
  __device__ __forceinline__ int kdoc(const AttnRuleArgs& g, int j) const { return k_id(k_raw(g, j)); }
};

// Which (sample, head, block of owned rows) a workgroup takes.  Workgroups go to the eight XCDs in turn; the units are dealt so
// that one XCD gets consecutive ones: the blocks of a head, and the heads that share keys, find them in the same L2.  Under an order
// or with documents blocks differ in length: there an XCD takes the longest blocks of all its heads first (last_first: the last
// queries, where the order hides later keys; with documents alone the first, as padding comes last), so that the short ones fill the
// end; unless the heads divide by eight, of all heads, as an XCD that gets half a head gets its long or its short half.  Measured,
// forward / backward, against head after head: causal 4 x 2048 rows x 8 heads of 64 37 / 122 us against 55 / 153, 1 x 8192 x 16 194 /
// 645 against 234 / 745, 4 x 1024 x 9 20 / 55 against 26 / 72; both together 4 x 2048 x 16 with a prefix in documents 234 against
// 281, 32 x 512 x 16 in documents 231 against 245; 4 x 2048 x 9 padded, the worst, 308 against 298.
struct RuleUnit {
  int b, h, blk;
  __device__ __forceinline__ RuleUnit(const AttnRuleArgs& g, int nblk, int heads, int id, int total, bool last_first) {
    const int all = g.nb * heads;   // heads of all samples
    int head;
    if (g.order != 0 || g.qdoc) {
      blk = id / all;
      head = all % 8 ? id % all : id % 8 * (all / 8) + id / 8 % (all / 8);
    } else {
      const int q = total / 8, r = total % 8, x = id % 8;
      const int u = x * q + (x < r ? x : r) + id / 8;
      blk = u % nblk;
      head = u / nblk;
    }
    if (last_first) blk = nblk - 1 - blk;
    h = head % heads;
    b = head / heads;
  }
};

// wave-wide minimum of an int, in every lane: DPP row shifts and broadcasts (a chain of LDS permutes takes ten times as long)
__device__ __forceinline__ int rule_wave_min(int v) {
#define PT_STEP(ctrl, rows)                                                        \
  {                                                                               \
    const int o_ = __builtin_amdgcn_update_dpp(v, v, ctrl, rows, 0xf, false);     \
    v = o_ < v ? o_ : v;                                                          \
  }
  PT_STEP(0x111, 0xf) PT_STEP(0x112, 0xf) PT_STEP(0x114, 0xf) PT_STEP(0x118, 0xf) PT_STEP(0x142, 0xa) PT_STEP(0x143, 0xc)
#undef PT_STEP
  return __builtin_amdgcn_readlane(v, 63);
}
__device__ __forceinline__ int rule_wave_max(int v) { return ~rule_wave_min(~v); }

// The tiles that a workgroup of four waves visits, SHARE waves owning ROWS rows together: entries tile << 9 | plain << 8 |
// whole bits << 4 | needed bits.  plain: all its rows exist and none is padding.
// In LDS: the least and the largest document of each wave's rows and of each tile (the sign of the least says that padding is among
// them, that of the largest that padding or several documents are), then, in place of the tiles' least, the entries.  A tile is
// needed by a wave whose range of documents meets its own and whose positions reach it; it is whole if both are one and the same
// document and all positions of the wave see all of the tile.
template <int ROWS, int SHARE = 1>
struct RuleList {
  int* base;
  int tiles;
  __device__ __forceinline__ RuleList(int* p, int rows) : base(p), tiles((rows + kRuleTile - 1) / kRuleTile) {}
  static size_t ints(int tiles) { return (size_t)12 + 2 * tiles + 2; }
  __device__ __forceinline__ int* lo() const { return base + 12; }              // [tiles + 2]: the loop reads one entry ahead
  __device__ __forceinline__ int* hi() const { return base + 12 + tiles + 2; }
  __device__ __forceinline__ int entry(int it) const { return __builtin_amdgcn_readfirstlane(lo()[it]); }
  static __device__ __forceinline__ int tile(int e) { return e >> 9; }
  static __device__ __forceinline__ bool needed(int e, int wave) { return e >> wave & 1; }
  static __device__ __forceinline__ bool whole(int e, int wave) { return e >> (4 + wave) & 1; }
  static __device__ __forceinline__ bool plain(int e) { return e >> 8 & 1; }

  // raw: the lane's document (below 0: padding); in: it is of a row that exists.  Rows of which none has a document get a range that
  // ends before it begins, and meet no other (but one from 0 to the largest id, and there pair by pair nothing is visible).
  __device__ __forceinline__ void range(int* lo_, int* hi_, int raw, bool in, int lane) const {
    const bool on = in && raw >= 0;
    const int least = rule_wave_min(on ? raw : 0x7fffffff), most = rule_wave_max(on ? raw : -1);
    const bool pad = __any(in && !on), mixed = least != most || pad;
    if (lane == 0) {
      *lo_ = pad ? least | (int)0x80000000 : least;
      *hi_ = mixed ? (most < 0 ? 0 : most) | (int)0x80000000 : most;
    }
  }
  // KEYS: tiles of keys for a block of queries, else tiles of queries for a block of keys; own: the lane's row's document.
  // Returns the number of entries.
  template <bool KEYS>
  __device__ __forceinline__ int build(const AttnRuleArgs& g, const RuleRows& rows, int wave, int lane, int blk, int own, bool own_in) const {
    const bool docs = rows.q != nullptr;
    const int n = KEYS ? g.Sk : g.Sq, m = KEYS ? g.Sq : g.Sk;
    if (docs) {
      for (int t0 = wave; t0 < tiles; t0 += 32) {       // eight tiles' loads in flight
        int d[8];
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          const int r = (t0 + 4 * x) * kRuleTile + lane;
          d[x] = (KEYS ? rows.k : rows.q)[r < n ? r : n - 1];
        }
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          const int t = t0 + 4 * x;
          if (t < tiles) range(lo() + t, hi() + t, d[x], t * kRuleTile + lane < n, lane);
        }
      }
      range(base + 2 * wave, base + 2 * wave + 1, own, own_in, lane);
      __syncthreads();
    }
    if (wave == 0) {
      int count = 0;
      for (int t0 = 0; t0 < tiles; t0 += 64) {
        const int t = t0 + lane, r0 = t * kRuleTile, r1 = r0 + kRuleTile - 1;
        const int tlo_ = docs && t < tiles ? lo()[t] : 0, thi_ = docs && t < tiles ? hi()[t] : 0;
        const int tlo = tlo_ & 0x7fffffff, thi = thi_ & 0x7fffffff;
        const int lim0 = KEYS ? 0 : rows.lim(g, r0), lim1 = KEYS ? 0 : rows.lim(g, r1 < n ? r1 : n - 1);
        int e = 0;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const int o0 = (blk * (4 / SHARE) + w / SHARE) * ROWS, o1 = o0 + ROWS - 1 < m ? o0 + ROWS - 1 : m - 1;
          const int wlo = docs ? base[2 * w] & 0x7fffffff : 0, whi_ = docs ? base[2 * w + 1] : 0, whi = whi_ & 0x7fffffff;
          bool need = t < tiles && o0 < m && tlo <= whi && wlo <= thi;
          bool all = thi_ >= 0 && whi_ >= 0 && tlo == wlo;
          if (KEYS) {
            need = need && r0 <= rows.lim(g, o1);
            all = all && r1 <= rows.lim(g, o0);
          } else {
            need = need && lim1 >= o0;
            all = all && lim0 >= o1 && o0 + ROWS <= m;   // (fewer keys: a query may see one only, which whole tiles rule out)
          }
          e |= (need ? 1 : 0) << w | (need && all ? 1 : 0) << (4 + w);
        }
        const uint64_t bits = __ballot(e != 0);
        if (e) lo()[count + __popcll(bits & ((1ull << lane) - 1))] = t << 9 | (r1 < n && tlo_ >= 0 ? 1 : 0) << 8 | e;
        count += __popcll(bits);
      }
      if (lane == 0) base[8] = count;
    }
    __syncthreads();
    return __builtin_amdgcn_readfirstlane(base[8]);
  }
};

}  // namespace pt
