// Which kernels a call of attention under a rule takes: how many waves share the rows that a wave owns alone otherwise.  Plain C++,
// so that the choice can be looked at without a GPU.
#pragma once
#include <cstdint>

namespace pt {

constexpr int kRuleCUs = 256;

struct RuleShape {
  int nb, Sq, Sk, H, Hkv, dh;
  bool ordered, documents;   // an order hides keys; there are documents
};
inline int64_t rule_blocks(int64_t heads, int rows, int each) { return heads * ((rows + each - 1) / each); }

// bf16: weights are rounded for the second products, which adds as much error again as the results' own rounding (1.4 times in all), on
// average over many weights.  With at most 64 queries and 64 keys little averages, and what the rounding left out goes through one more
// product (the kernels' FEW).  It is a property of the two lengths alone: a sample's results do not depend on its batch.
inline bool rule_few_pairs(const RuleShape& s) { return s.Sq <= 64 && s.Sk <= 64; }

// bf16: blocks of 128 rows, or blocks of 64 with two waves for 32 rows where those of 128 would leave CUs without one.  Measured,
// blocks of 64 against 128, forward / backward: 1 x 384 rows x 8 heads of 64 9.9 / 24 us against 11.5 / 34; 8 x 663 x 2 heads of 128
// 20 / 59 against 26 / 81.  Ordered rows without documents differ in length by their place, and up to two blocks a CU the smaller
// blocks even that out: 3 x 2048 x 8 38 / 107 against 45 / 143, 1 x 4096 x 16 69 / 214 against 78 / 264.  So they do for every rule in the
// forward pass at a head size of 64, whose registers leave room for them (12 x 384 x 10 15 against 16, 2 x 2048 x 12 in documents 22
// against 24), but not back: 55 against 49, 72 against 66.  Heads of 128 take them forward for ordered rows (1 x 3441 x 12 81 against
// 112, but 2 x 2048 x 12 in documents 38 against 33); backward only up to one block a CU, where the longest is all that counts (1 x 8192
// x 16 on 4 key heads 1760 against 2360, but 1 x 4096 x 16 555 against 430).  Few pairs
// are one such block by one tile whatever the batch, and always take it (64 x 64 rows x 16 heads 10.8 / 41 against 12.4 / 47, with the
// extra product in both; 11.1 / 37 without it.  256 x 20 x 12 23 / 101, without it in blocks of 128 25 / 74: the backward kernels' registers
// then leave room for two workgroups a CU instead of three).
inline bool rule_two_waves(const RuleShape& s, int64_t blocks_of_128, bool bwd) {
  if (rule_few_pairs(s)) return true;
  const bool uneven = s.ordered && !s.documents, wide = s.dh > 64;
  const bool twice = bwd ? uneven && !wide : uneven || !wide;
  return twice ? blocks_of_128 <= 2 * kRuleCUs : uneven ? blocks_of_128 <= kRuleCUs : blocks_of_128 < kRuleCUs;
}
// waves that share 32 rows in the forward pass, for dq, and for dk and dv
inline int rule_share_fwd(const RuleShape& s) { return rule_two_waves(s, rule_blocks((int64_t)s.nb * s.H, s.Sq, 128), false) ? 2 : 1; }
inline int rule_share_dq(const RuleShape& s) { return rule_two_waves(s, rule_blocks((int64_t)s.nb * s.H, s.Sq, 128), true) ? 2 : 1; }
inline int rule_share_dkv(const RuleShape& s) { return rule_two_waves(s, rule_blocks((int64_t)s.nb * s.Hkv, s.Sk, 128), true) ? 2 : 1; }

// fp32: waves that share 16 rows, two where workgroups of 64 rows would not be one for each CU, and in the backward launches, which
// take turns, up to two a CU (2 x 1024 rows x 8 heads of 64, causal, 163 us back against 249; 32 x 1 query of 197 keys x 12 72 against 76)
inline int rule_share_f32_fwd(const RuleShape& s) { return rule_blocks((int64_t)s.nb * s.H, s.Sq, 64) < kRuleCUs ? 2 : 1; }
inline int rule_share_f32_dq(const RuleShape& s) { return rule_blocks((int64_t)s.nb * s.H, s.Sq, 64) < 2 * kRuleCUs ? 2 : 1; }
inline int rule_share_f32_dkv(const RuleShape& s) { return rule_blocks((int64_t)s.nb * s.Hkv, s.Sk, 64) < 2 * kRuleCUs ? 2 : 1; }

}  // namespace pt
