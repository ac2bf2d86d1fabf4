// C entry points of the operators that stand by themselves (no context): attention under a rule and the GELU with an 8-bit
// checkpoint.  Arguments are checked here, before anything is enqueued; kernels are in attention_rules*.hip and gelu8.hip.
#include "../../include/pt.h"

#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "kernels.h"
#include "ops.h"

using namespace pt;

namespace {

thread_local char g_message[256] = "no error";

__attribute__((format(printf, 2, 3))) pt_status fail(pt_status s, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_message, sizeof g_message, fmt, ap);
  va_end(ap);
  return s;
}
pt_status launched(hipError_t e) { return e == hipSuccess ? PT_OK : fail(PT_EDEVICE, "%s", hipGetErrorString(e)); }

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// a view of n0 samples, n1 rows, n2 heads; rows are moved in pieces of 16 bytes.  written: the dh values of a row and head are its own
pt_status check_view(const char* name, const pt_heads* v, int64_t n0, int64_t n1, int64_t n2, const pt_attention* a, bool written) {
  if (!v) return fail(PT_EINVAL, "%s is NULL", name);
  if (n0 == 0 || n1 == 0 || n2 == 0) return PT_OK;
  if (!v->data) return fail(PT_EINVAL, "%s: data is NULL", name);
  if (!aligned16(v->data)) return fail(PT_EINVAL, "%s: data must be 16-byte aligned", name);
  const int64_t m = a->dtype == PT_BF16 ? 8 : 4, st[3] = {v->sample, v->row, v->head}, n[3] = {n0, n1, n2};
  for (int i = 0; i < 3; ++i) {
    if (n[i] > 1 && st[i] % m) return fail(PT_EINVAL, "%s: strides must be multiples of %d elements", name, (int)m);
    if (written && n[i] > 1 && st[i] > -a->dh && st[i] < a->dh) return fail(PT_EINVAL, "%s is written: its strides must be at least the head size", name);
  }
  return PT_OK;
}
HeadView view(const pt_heads* v) { return HeadView{v->data, v->sample, v->row, v->head}; }

pt_status check_attention(const pt_attention* a) {
  if (!a) return fail(PT_EINVAL, "the attention description is NULL");
  if (a->dtype != PT_F32 && a->dtype != PT_BF16) return fail(PT_EINVAL, "dtype");
  if (a->nb < 0 || a->Sq < 0 || a->Sk < 0 || a->H < 1 || a->Hkv < 1) return fail(PT_EINVAL, "sizes: nb, Sq, Sk >= 0 and H, Hkv >= 1");
  if (a->H % a->Hkv) return fail(PT_EINVAL, "H must be a multiple of Hkv");
  if (a->dh < 8 || a->dh > 128 || a->dh % 8) return fail(PT_EINVAL, "the head size must be a multiple of 8 and at most 128");
  if (a->Sq > kRuleMaxRows || a->Sk > kRuleMaxRows) return fail(PT_EINVAL, "at most %d queries and keys", kRuleMaxRows);
  if (a->q0 < 0 || (int64_t)a->q0 + a->Sq > (1 << 24)) return fail(PT_EINVAL, "q0 outside 0 .. 2^24 - Sq");
  if (a->order != PT_ATTN_FULL && a->order != PT_ATTN_CAUSAL && a->order != PT_ATTN_PREFIX) return fail(PT_EINVAL, "order");
  if (a->order == PT_ATTN_PREFIX && !a->prefix && a->nb > 0) return fail(PT_EINVAL, "PT_ATTN_PREFIX needs prefix lengths");
  if ((a->q_documents == nullptr) != (a->k_documents == nullptr) && a->nb > 0 && a->Sq > 0 && a->Sk > 0)
    return fail(PT_EINVAL, "documents of the queries and of the keys go together");
  if (!(a->scale > 0.f) || !std::isfinite(a->scale * 3.f)) return fail(PT_EINVAL, "scale must be positive and finite");
  if (!(a->cap >= 0.f) || !std::isfinite(a->cap * 3.f) || (a->cap > 0.f && !std::isfinite(a->scale * 3.f / a->cap))) return fail(PT_EINVAL, "cap must be 0 or a positive finite number");
  const int64_t heads = (int64_t)a->nb * a->H;
  if (heads >= kRuleMaxBlocks || heads * ((a->Sq + 63) / 64) + (int64_t)a->nb * a->Hkv * ((a->Sk + 63) / 64) >= kRuleMaxBlocks)
    return fail(PT_EINVAL, "nb * H * Sq or nb * Hkv * Sk too large");
  return PT_OK;
}
AttnRuleArgs rule_args(const pt_attention* a) {
  AttnRuleArgs g{};
  g.nb = a->nb; g.Sq = a->Sq; g.Sk = a->Sk; g.H = a->H; g.Hkv = a->Hkv; g.dh = a->dh;
  g.order = a->order; g.q0 = a->q0; g.scale = a->scale; g.cap = a->cap; g.slopes = a->slopes;
  g.qdoc = a->q_documents; g.kdoc = a->k_documents; g.prefix = a->prefix;
  g.qdoc_ld = a->Sq; g.kdoc_ld = a->Sk;
  g.lse_h = a->Sq; g.lse_b = (int64_t)a->H * a->Sq;
  return g;
}

pt_status check_gelu8(int32_t dtype, int64_t rows, int32_t F) {
  if (dtype != PT_F32 && dtype != PT_BF16) return fail(PT_EINVAL, "dtype");
  if (rows < 0 || F < 4 || F % 4) return fail(PT_EINVAL, "rows >= 0, F a positive multiple of 4");
  if (rows > gelu8_max_rows(F)) return fail(PT_EINVAL, "more than 2^27 blocks of 32 values");
  return PT_OK;
}

}  // namespace

namespace pt {
const char* ops_last_error() { return g_message; }
}  // namespace pt

pt_status pt_attention_workspace(const pt_attention* a, size_t* bwd_bytes) {
  const pt_status s = check_attention(a);
  if (s != PT_OK) return s;
  if (!bwd_bytes) return fail(PT_EINVAL, "bwd_bytes is NULL");
  // what dq's pass leaves for the keys': delta, and in fp32 another value for each query
  *bwd_bytes = (size_t)a->nb * a->H * a->Sq * sizeof(float) * (a->dtype == PT_BF16 ? 1 : 2);
  return PT_OK;
}

pt_status pt_attention_fwd(const pt_attention* a, const pt_heads* q, const pt_heads* k, const pt_heads* v, const pt_heads* o, float* lse,
                           void* hip_stream) {
  pt_status s = check_attention(a);
  if (s == PT_OK) s = check_view("q", q, a->nb, a->Sq, a->H, a, false);
  if (s == PT_OK) s = check_view("k", k, a->nb, a->Sk, a->Hkv, a, false);
  if (s == PT_OK) s = check_view("v", v, a->nb, a->Sk, a->Hkv, a, false);
  if (s == PT_OK) s = check_view("o", o, a->nb, a->Sq, a->H, a, true);
  if (s != PT_OK) return s;
  if (a->nb == 0 || a->Sq == 0) return PT_OK;
  AttnRuleArgs g = rule_args(a);
  g.q = view(q); g.k = view(k); g.v = view(v); g.o = view(o); g.lse = lse;
  return launched(attention_rule_fwd(a->dtype == PT_BF16, g, reinterpret_cast<hipStream_t>(hip_stream)));
}

pt_status pt_attention_bwd(const pt_attention* a, const pt_heads* q, const pt_heads* k, const pt_heads* v, const pt_heads* o,
                           const float* lse, const pt_heads* d_o, const pt_heads* dq, const pt_heads* dk, const pt_heads* dv, void* ws,
                           size_t ws_bytes, void* hip_stream) {
  size_t need = 0;
  pt_status s = pt_attention_workspace(a, &need);
  if (s == PT_OK) s = check_view("q", q, a->nb, a->Sq, a->H, a, false);
  if (s == PT_OK) s = check_view("k", k, a->nb, a->Sk, a->Hkv, a, false);
  if (s == PT_OK) s = check_view("v", v, a->nb, a->Sk, a->Hkv, a, false);
  if (s == PT_OK) s = check_view("o", o, a->nb, a->Sq, a->H, a, false);
  if (s == PT_OK) s = check_view("d_o", d_o, a->nb, a->Sq, a->H, a, false);
  if (s == PT_OK) s = check_view("dq", dq, a->nb, a->Sq, a->H, a, true);
  if (s == PT_OK) s = check_view("dk", dk, a->nb, a->Sk, a->Hkv, a, true);
  if (s == PT_OK) s = check_view("dv", dv, a->nb, a->Sk, a->Hkv, a, true);
  if (s != PT_OK) return s;
  if (a->nb == 0) return PT_OK;
  if (!lse && a->Sq > 0) return fail(PT_EINVAL, "lse is NULL");
  if (need > 0) {
    if (!ws || ws_bytes < need) return fail(PT_ENOMEM, "the workspace needs %zu bytes", need);
    if (!aligned16(ws)) return fail(PT_EINVAL, "the workspace must be 16-byte aligned");
  }
  AttnRuleArgs g = rule_args(a);
  g.q = view(q); g.k = view(k); g.v = view(v); g.o = view(o); g.d_o = view(d_o);
  g.dq = view(dq); g.dk = view(dk); g.dv = view(dv);
  g.lse = const_cast<float*>(lse); g.delta = static_cast<float*>(ws);
  return launched(attention_rule_bwd(a->dtype == PT_BF16, g, reinterpret_cast<hipStream_t>(hip_stream)));
}

pt_status pt_gelu8_fwd(int32_t dtype, const void* h, void* g, int8_t* codes, uint8_t* exps, int64_t rows, int32_t F, void* hip_stream) {
  const pt_status s = check_gelu8(dtype, rows, F);
  if (s != PT_OK) return s;
  if (rows == 0) return PT_OK;
  if (!h || !g || !codes || !exps) return fail(PT_EINVAL, "h, g, codes or exps is NULL");
  if (!aligned16(h) || !aligned16(g) || !aligned16(codes)) return fail(PT_EINVAL, "h, g and codes must be 16-byte aligned");
  return launched(gelu8_fwd(dtype == PT_BF16, h, g, codes, exps, rows, F, reinterpret_cast<hipStream_t>(hip_stream)));
}

pt_status pt_gelu8_bwd(int32_t dtype, const int8_t* codes, const uint8_t* exps, const void* dg, void* dh, void* g, int64_t rows, int32_t F,
                       void* hip_stream) {
  const pt_status s = check_gelu8(dtype, rows, F);
  if (s != PT_OK) return s;
  if (rows == 0) return PT_OK;
  if (!codes || !exps || !dg || !dh) return fail(PT_EINVAL, "codes, exps, dg or dh is NULL");
  if (!aligned16(codes) || !aligned16(dg) || !aligned16(dh) || !aligned16(g)) return fail(PT_EINVAL, "codes, dg, dh and g must be 16-byte aligned");
  return launched(gelu8_bwd(dtype == PT_BF16, codes, exps, dg, dh, g, rows, F, reinterpret_cast<hipStream_t>(hip_stream)));
}
