// C ABI of caches in pages (adsa_attend_paged, adsa_compact_paged; the prompt side's two calls are beside their dense forms) and of adsa_sample: host-side
// argument checks and launch order.
#include <cmath>

#include "adsa_internal.h"

namespace adsa {

int resolve_paged(const adsa_params* p, const adsa_pages* g, adsa_params* eff, PageArgs* a) {
  if (!p || !g) return ADSA_ERR_NULL;
  if (p->sel_groups != 1) return ADSA_ERR_UNSUPPORTED;
  adsa_params dense = *p;                            // (a record's own rows are not used: the strides of a dense cache stand in)
  dense.kv_slot_stride = p->head_dim;
  dense.kv_head_stride = (int64_t)p->cap * p->head_dim;
  const int rc = resolve_params(&dense, eff);
  if (rc) return rc;
  if (is_vcos(*eff)) return ADSA_ERR_UNSUPPORTED;
  if (!g->k || !g->v || !g->table) return ADSA_ERR_NULL;
  if (!aligned16(g->k) || !aligned16(g->v) || (reinterpret_cast<uintptr_t>(g->table) & 3u) != 0) return ADSA_ERR_ALIGN;
  const int size = g->page_size;
  if (size < ADSA_MIN_PAGE || size > ADSA_MAX_CAP || (size & (size - 1)) != 0 || g->n_pages < 1) return ADSA_ERR_SHAPE;
  if (g->table_stride < (p->cap + size - 1) / size || g->table_stride > 65535) return ADSA_ERR_SHAPE;
  constexpr int64_t kMost = 1ll << 40;               // (elements; products below stay far from the end of 64 bits)
  const int64_t page = g->page_stride, slot = g->slot_stride, head = g->head_stride, eb = elem_bytes(*eff);
  if (page < 1 || slot < 1 || head < 1 || page > kMost || slot > kMost || head > kMost) return ADSA_ERR_SHAPE;
  if (page * eb % 16 || slot * eb % 16 || head * eb % 16) return ADSA_ERR_ALIGN;
  // rows of different (page, slot, head) must not overlap: one of the two nestings
  const bool head_major = slot >= p->head_dim && head >= size * slot && page >= p->n_heads * head;
  const bool slot_major = head >= p->head_dim && slot >= p->n_heads * head && page >= size * slot;
  if (!head_major && !slot_major) return ADSA_ERR_SHAPE;
  *a = {};
  a->unit_shift = __builtin_ctzll((unsigned long long)((page | slot | head) * eb));
  const int64_t page_units = (page * eb) >> a->unit_shift;
  if (page * eb >= (1ll << 32) || page_units >= (1ll << 31) || page_units * g->n_pages >= (1ll << 31)) return ADSA_ERR_UNSUPPORTED;
  a->slot_units = (uint32_t)((slot * eb) >> a->unit_shift);
  if (slot * eb >= (1ll << 24)) return ADSA_ERR_UNSUPPORTED;             // (products of 24 bits)
  a->table = g->table;
  a->k = (char*)g->k;
  a->v = (char*)g->v;
  a->page_stride_b = page * eb;
  a->slot_stride_b = slot * eb;
  a->head_stride_b = head * eb;
  a->n_pages = g->n_pages;
  a->shift = __builtin_ctz((unsigned)size);
  a->table_stride = g->table_stride;
  a->page_units = (uint32_t)page_units;
  return ADSA_OK;
}

namespace {

int check_space(const void* ws, size_t bytes, size_t need) {
  if (!ws) return ADSA_ERR_WORKSPACE;
  if ((reinterpret_cast<uintptr_t>(ws) & 255u) != 0) return ADSA_ERR_ALIGN;
  return bytes < need ? ADSA_ERR_WORKSPACE : ADSA_OK;
}

}  // namespace
}  // namespace adsa

using namespace adsa;

extern "C" {

size_t adsa_paged_workspace_bytes(const adsa_params* p) {
  if (!p || p->sel_groups != 1) return 0;
  adsa_params dense = *p, eff;
  dense.kv_slot_stride = p->head_dim;
  dense.kv_head_stride = (int64_t)p->cap * p->head_dim;
  if (resolve_params(&dense, &eff) != ADSA_OK || is_vcos(eff)) return 0;
  return make_workspace(eff, make_attend_plan(eff, true)).total;
}

int adsa_attend_paged(const adsa_params* p, const adsa_pages* pages, adsa_seq* seqs, const void* q, const void* k_new, const void* v_new,
                      const int32_t* sel_idx, const int32_t* sel_cnt, void* out, float* lse, uint32_t flags, void* workspace, size_t workspace_bytes,
                      void* stream) {
  adsa_params eff;
  PageArgs args;
  int rc = resolve_paged(p, pages, &eff, &args);
  if (rc) return rc;
  if (!seqs || !q || !sel_idx || !sel_cnt || !out || !lse) return ADSA_ERR_NULL;
  const bool append = (flags & ADSA_FLAG_APPEND) != 0;
  if (append && (!k_new || !v_new)) return ADSA_ERR_NULL;
  if (!aligned16(q) || !aligned16(out) || (append && (!aligned16(k_new) || !aligned16(v_new)))) return ADSA_ERR_ALIGN;
  const AttendPlan plan = make_attend_plan(eff, true);
  const Workspace w = make_workspace(eff, plan);
  if ((rc = check_space(workspace, workspace_bytes, w.total)) || (rc = ensure_device_ready())) return rc;
  const bool accumulate = eff.score_mode == ADSA_SCORE_ATTN_MASS && !(flags & ADSA_FLAG_NO_ACCUMULATE);
  if (launch_attend_paged(eff, args, plan, seqs, q, k_new, v_new, sel_idx, sel_cnt, out, lse, (char*)workspace, w, accumulate, append,
                          (flags & ADSA_FLAG_ADVANCE) ? kAdvance : kAdvanceNone, (flags & ADSA_FLAG_NEW_F32) != 0 && eff.dtype == ADSA_BF16,
                          reinterpret_cast<hipStream_t>(stream)) != hipSuccess)
    return ADSA_ERR_LAUNCH;
  return ADSA_OK;
}

int adsa_compact_paged(const adsa_params* p, const adsa_pages* pages, adsa_seq* seqs, int32_t* keep_map, uint32_t flags, void* workspace,
                       size_t workspace_bytes, void* stream) {
  adsa_params eff;
  PageArgs args;
  int rc = resolve_paged(p, pages, &eff, &args);
  if (rc) return rc;
  if (!seqs || !keep_map) return ADSA_ERR_NULL;
  const AttendPlan plan = make_attend_plan(eff, true);
  const Workspace w = make_workspace(eff, plan);
  if ((rc = check_space(workspace, workspace_bytes, w.total)) || (rc = ensure_device_ready())) return rc;
  if (launch_compact_paged(eff, args, seqs, keep_map, (char*)workspace, w, (flags & ADSA_FLAG_ADVANCE) != 0, reinterpret_cast<hipStream_t>(stream)) != hipSuccess)
    return ADSA_ERR_LAUNCH;
  return ADSA_OK;
}

int adsa_sample(const adsa_sampling* s, const adsa_seq* seqs, const void* logits, const float* uniform, int32_t* token, float* logprob, void* stream) {
  if (!s || !logits || !uniform || !token) return ADSA_ERR_NULL;
  if (s->dtype != ADSA_F32 && s->dtype != ADSA_BF16) return ADSA_ERR_DTYPE;
  if (s->n_rows < 1 || s->n_rows > (1 << 20) || s->vocab < 1 || s->vocab > ADSA_MAX_VOCAB) return ADSA_ERR_SHAPE;
  if (s->guided != 0 && s->guided != 1) return ADSA_ERR_SHAPE;
  if (s->row_stride != 0 && (s->row_stride < s->vocab || s->row_stride > (1ll << 40))) return ADSA_ERR_SHAPE;
  if (s->guided && !std::isfinite(s->guidance)) return ADSA_ERR_SHAPE;
  if (!s->temperatures && !(s->temperature >= 0.0f && std::isfinite(s->temperature))) return ADSA_ERR_SHAPE;
  if ((!s->top_ps && std::isnan(s->top_p)) || (!s->min_ps && std::isnan(s->min_p))) return ADSA_ERR_SHAPE;
  if (reinterpret_cast<uintptr_t>(logits) % (s->dtype == ADSA_F32 ? 4 : 2) != 0) return ADSA_ERR_ALIGN;
  for (const void* x : {(const void*)uniform, (const void*)token, (const void*)logprob, (const void*)s->temperatures, (const void*)s->top_ks, (const void*)s->top_ps,
                        (const void*)s->min_ps})
    if ((reinterpret_cast<uintptr_t>(x) & 3u) != 0) return ADSA_ERR_ALIGN;
  const int rc = ensure_device_ready();
  if (rc) return rc;
  return launch_sample(*s, seqs, logits, uniform, token, logprob, reinterpret_cast<hipStream_t>(stream)) == hipSuccess ? ADSA_OK : ADSA_ERR_LAUNCH;
}

}  // extern "C"
