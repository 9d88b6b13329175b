// C ABI of the prompt side (adsa_rotate, adsa_append, adsa_prefill, adsa_attend_shared): host-side argument checks and launch order.
#include <algorithm>
#include <cmath>

#include "adsa_internal.h"

namespace adsa {
namespace {

constexpr long long kMaxBlocks = 1ll << 24;      // of 256 threads: a launch has less than 2^32 threads

bool f32_rows(const adsa_params& p, uint32_t flags) { return (flags & ADSA_FLAG_NEW_F32) != 0 && p.dtype == ADSA_BF16; }
int query_heads(const adsa_params& p) { return p.n_heads * (p.q_per_kv > 1 ? p.q_per_kv : 1); }

// Every (sequence, head) a record of its own (sel_groups == n_heads) is no form of these calls.
int resolve(const adsa_params* p, adsa_params* eff) {
  if (!p) return ADSA_ERR_NULL;
  if (p->sel_groups != 1) return ADSA_ERR_UNSUPPORTED;
  return resolve_params(p, eff);
}

int check_rope(const adsa_rope* r) {
  if (!r->freq) return ADSA_ERR_NULL;
  if (!aligned16(r->freq)) return ADSA_ERR_ALIGN;
  if (r->n_axes < 1 || r->n_axes > ADSA_MAX_AXES) return ADSA_ERR_SHAPE;
  if (r->pairing != ADSA_PAIR_HALVES && r->pairing != ADSA_PAIR_NEIGHBOURS) return ADSA_ERR_DTYPE;
  return ADSA_OK;
}

int check_row_stride(long long stride, int heads, const adsa_params& p, bool in_f32) {
  if (stride == 0) return ADSA_OK;
  if (stride < (long long)heads * p.head_dim) return ADSA_ERR_SHAPE;
  return stride * (in_f32 ? 4 : elem_bytes(p)) % 16 ? ADSA_ERR_ALIGN : ADSA_OK;
}

int check_tokens(const adsa_params& p, const adsa_tokens* t) {
  if (!t || !t->begin || !t->slot0) return ADSA_ERR_NULL;
  if (t->n_tokens < 1 || t->n_tokens > (1 << 24)) return ADSA_ERR_SHAPE;
  if (t->max_len < 1 || t->max_len > p.cap || t->max_len > t->n_tokens) return ADSA_ERR_SHAPE;
  return ADSA_OK;
}

int check_mods(const adsa_params& p, const adsa_mods& m, bool prompt) {
  if (!(m.softcap >= 0.0f) || std::isinf(m.softcap)) return ADSA_ERR_SHAPE;
  if (m.softcap > 0.0f) {                            // the kernels' constants are fp32, too
    const float scale = p.softmax_scale > 0.0f ? p.softmax_scale : 1.0f / std::sqrt((float)p.head_dim);
    if (!std::isnormal(scale / m.softcap) || !std::isnormal(m.softcap * 1.4426950408889634f)) return ADSA_ERR_SHAPE;
  }
  if (!prompt) return ADSA_OK;
  if (m.mask != ADSA_MASK_CAUSAL && m.mask != ADSA_MASK_PREFIX) return ADSA_ERR_DTYPE;
  if (m.doc && m.doc_stride < p.cap) return ADSA_ERR_SHAPE;
  return ADSA_OK;
}

int check_shared(const adsa_params& p, const adsa_shared* s) {
  if (!s || !s->prompts || !s->members) return ADSA_ERR_NULL;
  if (s->n_groups < 1 || s->n_groups > p.n_seq || s->max_members < 1 || s->max_members > p.n_seq) return ADSA_ERR_SHAPE;
  if (s->max_prompt < 1 || s->max_prompt > ADSA_MAX_CAP) return ADSA_ERR_CAPACITY;
  const long long eb = elem_bytes(p), slot = s->kv_slot_stride, head = s->kv_head_stride;
  if (slot < 1 || head < 1) return ADSA_ERR_SHAPE;
  if (slot * eb % 16 || head * eb % 16) return ADSA_ERR_ALIGN;
  const bool slot_major = head >= p.head_dim && slot >= (long long)p.n_heads * head;
  const bool head_major = slot >= p.head_dim && head >= (long long)s->max_prompt * slot;
  return slot_major || head_major ? ADSA_OK : ADSA_ERR_SHAPE;
}

int check_space(const void* ws, size_t bytes, size_t need) {
  if (!ws) return ADSA_ERR_WORKSPACE;
  if ((reinterpret_cast<uintptr_t>(ws) & 255u) != 0) return ADSA_ERR_ALIGN;
  return bytes < need ? ADSA_ERR_WORKSPACE : ADSA_OK;
}

int plan_prompt(const adsa_params& p, const adsa_tokens* t, PromptPlan* plan, PromptWorkspace* w) {
  const int rc = check_tokens(p, t);
  if (rc) return rc;
  *plan = make_prompt_plan(p, *t);
  *w = make_prompt_workspace(p, *t, *plan);
  const long long pairs = ((long long)p.n_seq * p.n_heads + 7) / 8 * 8;
  const long long units = std::max((long long)plan->tiles * plan->chunks, (long long)(p.cap + 127) / 128);
  if (pairs * units > kMaxBlocks || (long long)t->n_tokens * query_heads(p) / 4 >= kMaxBlocks) return ADSA_ERR_UNSUPPORTED;
  return ADSA_OK;
}

int plan_shared(const adsa_params& p, const adsa_shared* s, SharedPlan* plan, SharedWorkspace* w) {
  if (p.score_mode == ADSA_SCORE_VCOS_FUSED) return ADSA_ERR_UNSUPPORTED;
  const int rc = check_shared(p, s);
  if (rc) return rc;
  *plan = make_shared_plan(p, *s);
  *w = make_shared_workspace(p, *plan);
  const long long prompts = ((long long)s->n_groups * p.n_heads * plan->prompt_chunks + 7) / 8 * 8 * plan->prompt_tiles;
  if (prompts + (long long)p.n_seq * p.n_heads * plan->own_chunks > kMaxBlocks) return ADSA_ERR_UNSUPPORTED;
  return ADSA_OK;
}

}  // namespace
}  // namespace adsa

using namespace adsa;

extern "C" {

int adsa_rotate(const adsa_params* p, const adsa_rope* rope, const adsa_seq* seqs, const int32_t* coords, const void* q, const void* k,
                int64_t q_stride, int64_t k_stride, void* q_out, void* k_out, uint32_t flags, void* stream) {
  adsa_params eff;
  int rc = resolve(p, &eff);
  if (rc) return rc;
  if (!rope || !seqs || !q || !k || !q_out || !k_out) return ADSA_ERR_NULL;
  rc = check_rope(rope);
  if (rc) return rc;
  if (!aligned16(q) || !aligned16(k) || !aligned16(q_out) || !aligned16(k_out)) return ADSA_ERR_ALIGN;
  const bool in_f32 = f32_rows(eff, flags);
  if ((rc = check_row_stride(q_stride, query_heads(eff), eff, in_f32)) || (rc = check_row_stride(k_stride, eff.n_heads, eff, in_f32))) return rc;
  if (launch_rotate(eff, *rope, seqs, coords, q, k, q_stride, k_stride, q_out, k_out, in_f32, reinterpret_cast<hipStream_t>(stream)) != hipSuccess)
    return ADSA_ERR_LAUNCH;
  return ADSA_OK;
}

int adsa_append(const adsa_params* p, const adsa_tokens* tokens, const adsa_rope* rope, adsa_seq* seqs, const void* q, const void* k, const void* v,
                void* q_out, uint32_t flags, void* stream) {
  adsa_params eff;
  int rc = resolve(p, &eff);
  if (rc) return rc;
  if (!seqs || !k || !v || (q == nullptr) != (q_out == nullptr)) return ADSA_ERR_NULL;
  rc = check_tokens(eff, tokens);
  if (rc) return rc;
  if (rope && (rc = check_rope(rope))) return rc;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(q_out)) return ADSA_ERR_ALIGN;
  const bool in_f32 = f32_rows(eff, flags);
  if ((rc = check_row_stride(tokens->q_stride, query_heads(eff), eff, in_f32)) || (rc = check_row_stride(tokens->k_stride, eff.n_heads, eff, in_f32)) ||
      (rc = check_row_stride(tokens->v_stride, eff.n_heads, eff, in_f32)))
    return rc;
  if (launch_append(eff, *tokens, rope, seqs, q, k, v, q_out, in_f32, (flags & ADSA_FLAG_ADVANCE) != 0, reinterpret_cast<hipStream_t>(stream)) != hipSuccess)
    return ADSA_ERR_LAUNCH;
  return ADSA_OK;
}

size_t adsa_prefill_workspace_bytes(const adsa_params* p, const adsa_tokens* tokens) {
  adsa_params eff;
  PromptPlan plan;
  PromptWorkspace w;
  return resolve(p, &eff) == ADSA_OK && plan_prompt(eff, tokens, &plan, &w) == ADSA_OK ? w.total : 0;
}

int adsa_prefill(const adsa_params* p, const adsa_tokens* tokens, const adsa_mods* mods, adsa_seq* seqs, const void* q, void* out, float* lse,
                 uint32_t flags, void* workspace, size_t workspace_bytes, void* stream) {
  adsa_params eff;
  int rc = resolve(p, &eff);
  if (rc) return rc;
  if (!seqs || !q || !out || !lse) return ADSA_ERR_NULL;
  PromptPlan plan;
  PromptWorkspace w;
  rc = plan_prompt(eff, tokens, &plan, &w);
  if (rc) return rc;
  const adsa_mods none = {};
  const adsa_mods& m = mods ? *mods : none;
  rc = check_mods(eff, m, true);
  if (rc) return rc;
  if (!aligned16(q) || !aligned16(out)) return ADSA_ERR_ALIGN;
  rc = check_space(workspace, workspace_bytes, w.total);
  if (rc) return rc;
  rc = ensure_device_ready();
  if (rc) return rc;
  const bool accumulate = eff.score_mode == ADSA_SCORE_ATTN_MASS && !(flags & ADSA_FLAG_NO_ACCUMULATE);
  if (launch_prefill(eff, *tokens, m, plan, seqs, q, out, lse, (char*)workspace, w, accumulate, (flags & ADSA_FLAG_ADVANCE) != 0,
                     (flags & ADSA_FLAG_SPLIT_P) != 0, reinterpret_cast<hipStream_t>(stream)) != hipSuccess)
    return ADSA_ERR_LAUNCH;
  return ADSA_OK;
}

size_t adsa_shared_workspace_bytes(const adsa_params* p, const adsa_shared* shared) {
  adsa_params eff;
  SharedPlan plan;
  SharedWorkspace w;
  return resolve(p, &eff) == ADSA_OK && plan_shared(eff, shared, &plan, &w) == ADSA_OK ? w.total : 0;
}

int adsa_attend_shared(const adsa_params* p, const adsa_shared* shared, const adsa_mods* mods, adsa_seq* seqs, const void* q, const void* k_new,
                       const void* v_new, const int32_t* sel_idx, const int32_t* sel_cnt, void* out, float* lse, uint32_t flags, void* workspace,
                       size_t workspace_bytes, void* stream) {
  adsa_params eff;
  int rc = resolve(p, &eff);
  if (rc) return rc;
  if (!seqs || !q || !sel_idx || !sel_cnt || !out || !lse) return ADSA_ERR_NULL;
  const bool append = (flags & ADSA_FLAG_APPEND) != 0;
  if (append && (!k_new || !v_new)) return ADSA_ERR_NULL;
  SharedPlan plan;
  SharedWorkspace w;
  rc = plan_shared(eff, shared, &plan, &w);
  if (rc) return rc;
  const adsa_mods none = {};
  const adsa_mods& m = mods ? *mods : none;
  rc = check_mods(eff, m, false);
  if (rc) return rc;
  if (!aligned16(q) || !aligned16(out) || (append && (!aligned16(k_new) || !aligned16(v_new)))) return ADSA_ERR_ALIGN;
  rc = check_space(workspace, workspace_bytes, w.total);
  if (rc) return rc;
  rc = ensure_device_ready();
  if (rc) return rc;
  const bool accumulate = eff.score_mode == ADSA_SCORE_ATTN_MASS && !(flags & ADSA_FLAG_NO_ACCUMULATE);
  if (launch_attend_shared(eff, *shared, m, plan, seqs, q, k_new, v_new, sel_idx, sel_cnt, out, lse, (char*)workspace, w, accumulate, append,
                           (flags & ADSA_FLAG_ADVANCE) != 0, f32_rows(eff, flags), reinterpret_cast<hipStream_t>(stream)) != hipSuccess)
    return ADSA_ERR_LAUNCH;
  return ADSA_OK;
}

}  // extern "C"
