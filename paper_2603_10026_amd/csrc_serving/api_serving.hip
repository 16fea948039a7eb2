// C-ABI layer of the serving operators: argument validation on the host, then dispatch to the kernel launchers.
#include <math.h>

#include "../../include/rf.h"
#include "../csrc/rf_check.h"
#include "../csrc/rf_device.h"
#include "serving_launch.h"

namespace {

using namespace rf::check;

bool rows_contiguous(const rf_tensor* t) { return t->shape[t->ndim - 1] <= 1 || t->stride[t->ndim - 1] == 1; }
bool aligned4(const rf_tensor* t) { return reinterpret_cast<uintptr_t>(t->data) % 4 == 0; }

// A contiguous vector of n values of one 4-byte type.
rf_status check_vector(const rf_tensor* t, rf_dtype dtype, int64_t n) {
  rf_status st;
  if ((st = check_tensor(t, 1, 1, RF_I32)) != RF_OK) return st;
  if (t->dtype != dtype) return RF_ERR_UNSUPPORTED;
  if (t->shape[0] != n) return RF_ERR_INVALID_ARG;
  if (!rows_contiguous(t)) return RF_ERR_UNSUPPORTED;
  if (n > 0 && t->data == nullptr) return RF_ERR_INVALID_ARG;
  return aligned4(t) ? RF_OK : RF_ERR_ALIGNMENT;
}

// [T, heads, d] bf16
rf_status check_tokens(const rf_tensor* t, int64_t T, int64_t heads, int64_t d) {
  rf_status st;
  if ((st = check_tensor(t, 3, 3)) != RF_OK) return st;
  if (t->dtype != RF_BF16) return RF_ERR_UNSUPPORTED;
  if (t->shape[0] != T || t->shape[1] != heads || t->shape[2] != d) return RF_ERR_INVALID_ARG;
  if (!rows_contiguous(t)) return RF_ERR_UNSUPPORTED;
  if (numel(t) > 0 && t->data == nullptr) return RF_ERR_INVALID_ARG;
  return numel(t) == 0 || aligned16(t) ? RF_OK : RF_ERR_ALIGNMENT;
}

rf::Strides2 strides2(const rf_tensor* t) { return {t->stride[0], t->stride[1]}; }

// What q, a cache and the page table say about a batch, by shapes, strides and types alone.
rf_status paged_shape(const rf_tensor* q, const rf_tensor* cache, const rf_tensor* pages, rf::Paged* p) {
  rf_status st;
  if ((st = check_tensor(q, 3, 3)) != RF_OK) return st;
  if ((st = check_tensor(cache, 4, 4, RF_FP8_E4M3)) != RF_OK) return st;
  if ((st = check_tensor(pages, 2, 2, RF_I32)) != RF_OK) return st;
  if (q->dtype != RF_BF16 || cache->dtype == RF_F32 || pages->dtype != RF_I32) return RF_ERR_UNSUPPORTED;
  const int64_t T = q->shape[0], Hq = q->shape[1], d = q->shape[2], page = cache->shape[1], Hkv = cache->shape[2];
  if (cache->shape[3] != d || Hkv < 1 || Hq < 1 || Hq % Hkv != 0) return RF_ERR_INVALID_ARG;
  if ((d != 64 && d != 128) || page < 16 || page % 16 != 0) return RF_ERR_UNSUPPORTED;
  if (!rows_contiguous(cache) || !rows_contiguous(pages)) return RF_ERR_UNSUPPORTED;
  if (cache->stride[1] > ((int64_t)1 << 26)) return RF_ERR_UNSUPPORTED;  // 32-bit offsets inside 16 slots
  for (int64_t n : {T, Hq, Hkv, page, cache->shape[0], pages->shape[0], pages->shape[1]})
    if (n >= INT32_MAX) return RF_ERR_UNSUPPORTED;
  if (T * Hq > INT32_MAX) return RF_ERR_UNSUPPORTED;
  p->T = (int)T;
  p->B = (int)pages->shape[0];
  p->Hq = (int)Hq;
  p->Hkv = (int)Hkv;
  p->group = (int)(Hq / Hkv);
  p->d = (int)d;
  p->page = (int)page;
  p->n_pages = (int)cache->shape[0];
  p->table_len = p->n_pages > 0 ? (int)pages->shape[1] : 0;  // (without pages no key has a place)
  p->table_pitch = pages->stride[0];
  p->page_stride = cache->stride[0];
  p->slot_stride = cache->stride[1];
  p->head_stride = cache->stride[2];
  return RF_OK;
}

bool scale_ok(float s, bool fp8) { return fp8 ? s > 0.f && isfinite(s) : s == 1.f; }

// Everything that the two paged entry points share.
rf_status check_paged(const rf_tensor* q, const rf_tensor* k_cache, const rf_tensor* v_cache, const rf_tensor* seq_start,
                      const rf_tensor* kv_len, const rf_tensor* pages, float k_scale, float v_scale, rf::Paged* p) {
  rf_status st;
  if ((st = check_tensor(v_cache, 4, 4, RF_FP8_E4M3)) != RF_OK) return st;
  if ((st = paged_shape(q, k_cache, pages, p)) != RF_OK) return st;
  if ((st = check_tokens(q, p->T, p->Hq, p->d)) != RF_OK) return st;
  if (v_cache->dtype != k_cache->dtype) return RF_ERR_UNSUPPORTED;
  if (!same_shape(k_cache, v_cache)) return RF_ERR_INVALID_ARG;
  for (int i = 0; i < 4; ++i)
    if (k_cache->shape[i] > 1 && k_cache->stride[i] != v_cache->stride[i]) return RF_ERR_UNSUPPORTED;
  const bool fp8 = k_cache->dtype == RF_FP8_E4M3;
  if (!scale_ok(k_scale, fp8) || !scale_ok(v_scale, fp8)) return RF_ERR_INVALID_ARG;
  if ((st = check_vector(seq_start, RF_I32, (int64_t)p->B + 1)) != RF_OK) return st;
  if ((st = check_vector(kv_len, RF_I32, p->B)) != RF_OK) return st;
  if (numel(k_cache) > 0) {
    if (k_cache->data == nullptr || v_cache->data == nullptr) return RF_ERR_INVALID_ARG;
    if (!aligned16(k_cache) || !aligned16(v_cache)) return RF_ERR_ALIGNMENT;
  }
  if (numel(pages) > 0 && pages->data == nullptr) return RF_ERR_INVALID_ARG;
  if (!aligned4(pages)) return RF_ERR_ALIGNMENT;
  p->seq_start = (const int32_t*)seq_start->data;
  p->kv_len = (const int32_t*)kv_len->data;
  p->pages = (const int32_t*)pages->data;
  return RF_OK;
}

rf_status check_paged_attention(const rf_tensor* q, const rf_tensor* k_cache, const rf_tensor* v_cache,
                                const rf_tensor* seq_start, const rf_tensor* kv_len, const rf_tensor* pages,
                                int64_t max_q, float scale, int causal, float k_scale, float v_scale, const rf_tensor* o,
                                rf::PagedAttention* a) {
  rf_status st;
  if ((st = check_paged(q, k_cache, v_cache, seq_start, kv_len, pages, k_scale, v_scale, &a->p)) != RF_OK) return st;
  if ((st = check_tokens(o, a->p.T, a->p.Hq, a->p.d)) != RF_OK) return st;
  if (max_q < 0) return RF_ERR_INVALID_ARG;
  if (!rf::paged_attention_fits(a->p, max_q)) return RF_ERR_UNSUPPORTED;
  a->q = q->data;
  a->k_cache = k_cache->data;
  a->v_cache = v_cache->data;
  a->o = o->data;
  a->sq = strides2(q);
  a->so = strides2(o);
  a->scale_log2e = scale * k_scale * rf::kLog2e;
  a->v_scale = v_scale;
  a->causal = causal != 0;
  a->fp8 = k_cache->dtype == RF_FP8_E4M3;
  a->max_q = max_q;
  return RF_OK;
}

bool empty(const rf::Paged& p) { return p.T == 0 || p.B == 0 || p.Hq == 0; }

rf_status check_verify(const rf_tensor* target, const rf_tensor* draft, const rf_tensor* tokens, const rf_tensor* u_accept,
                       const rf_tensor* u_sample, const rf_tensor* seq_start, const rf_tensor* out,
                       const rf_tensor* accepted, rf::VerifyDrafts* a) {
  rf_status st;
  if ((st = check_tensor(target, 2, 2)) != RF_OK) return st;
  if (draft != nullptr) {
    if ((st = check_tensor(draft, 2, 2)) != RF_OK) return st;
    if (draft->dtype != target->dtype) return RF_ERR_UNSUPPORTED;
    if (!same_shape(draft, target)) return RF_ERR_INVALID_ARG;
    if (!rows_contiguous(draft)) return RF_ERR_UNSUPPORTED;
  }
  if (!rows_contiguous(target)) return RF_ERR_UNSUPPORTED;
  if ((st = check_tensor(u_sample, 1, 1)) != RF_OK) return st;
  const int64_t R = target->shape[0], V = target->shape[1], B = u_sample->shape[0];
  if (V < 1) return RF_ERR_INVALID_ARG;
  if (R >= INT32_MAX || V >= INT32_MAX || !rf::verify_drafts_fits(B)) return RF_ERR_UNSUPPORTED;
  if ((st = check_vector(tokens, RF_I32, R)) != RF_OK) return st;
  if ((st = check_vector(u_accept, RF_F32, R)) != RF_OK) return st;
  if ((st = check_vector(u_sample, RF_F32, B)) != RF_OK) return st;
  if ((st = check_vector(seq_start, RF_I32, B + 1)) != RF_OK) return st;
  if ((st = check_vector(out, RF_I32, R)) != RF_OK) return st;
  if ((st = check_vector(accepted, RF_I32, B)) != RF_OK) return st;
  if (R > 0 && (target->data == nullptr || (draft != nullptr && draft->data == nullptr))) return RF_ERR_INVALID_ARG;
  for (const rf_tensor* t : {target, draft})
    if (t != nullptr && reinterpret_cast<uintptr_t>(t->data) % esize(t->dtype) != 0) return RF_ERR_ALIGNMENT;
  a->target = target->data;
  a->draft = draft != nullptr ? draft->data : nullptr;
  a->target_pitch = target->stride[0];
  a->draft_pitch = draft != nullptr ? draft->stride[0] : 0;
  a->tokens = (const int32_t*)tokens->data;
  a->seq_start = (const int32_t*)seq_start->data;
  a->u_accept = (const float*)u_accept->data;
  a->u_sample = (const float*)u_sample->data;
  a->out = (int32_t*)out->data;
  a->accepted = (int32_t*)accepted->data;
  a->V = V;
  a->R = (int)R;
  a->B = (int)B;
  a->bf16 = target->dtype == RF_BF16;
  return RF_OK;
}

rf_status status_of(hipError_t e) { return e == hipSuccess ? RF_OK : RF_ERR_LAUNCH; }

}  // namespace

extern "C" {

rf_status rf_paged_append(const rf_tensor* q, const rf_tensor* k, const rf_tensor* v, const rf_tensor* q_norm,
                          const rf_tensor* k_norm, float eps, const rf_tensor* cos, const rf_tensor* sin, int interleaved,
                          const rf_tensor* seq_start, const rf_tensor* kv_len, const rf_tensor* pages, rf_tensor* k_cache,
                          rf_tensor* v_cache, float k_scale, float v_scale, rf_tensor* q_out, rf_stream stream) {
  rf::PagedAppend a{};
  rf_status st;
  if ((st = check_paged(q, k_cache, v_cache, seq_start, kv_len, pages, k_scale, v_scale, &a.p)) != RF_OK) return st;
  const rf::Paged& p = a.p;
  if ((st = check_tokens(k, p.T, p.Hkv, p.d)) != RF_OK) return st;
  if ((st = check_tokens(v, p.T, p.Hkv, p.d)) != RF_OK) return st;
  if ((st = check_tokens(q_out, p.T, p.Hq, p.d)) != RF_OK) return st;
  for (const rf_tensor* g : {q_norm, k_norm}) {
    if (g == nullptr) continue;
    if ((st = check_tensor(g, 1, 1)) != RF_OK) return st;
    if (g->dtype != RF_BF16) return RF_ERR_UNSUPPORTED;
    if (g->shape[0] != p.d || g->data == nullptr) return RF_ERR_INVALID_ARG;
    if (!rows_contiguous(g)) return RF_ERR_UNSUPPORTED;
    if (!aligned16(g)) return RF_ERR_ALIGNMENT;
  }
  if (!(eps >= 0.f)) return RF_ERR_INVALID_ARG;
  if ((cos == nullptr) != (sin == nullptr)) return RF_ERR_INVALID_ARG;
  if (cos != nullptr) {
    for (const rf_tensor* t : {cos, sin}) {
      if ((st = check_tensor(t, 2, 2)) != RF_OK) return st;
      if (t->dtype != RF_F32 || !rows_contiguous(t)) return RF_ERR_UNSUPPORTED;
    }
    if (!same_shape(cos, sin)) return RF_ERR_INVALID_ARG;
    const int64_t half = cos->shape[1];
    if (half < 1 || 2 * half > p.d) return RF_ERR_INVALID_ARG;
    if (half % 8 != 0) return RF_ERR_UNSUPPORTED;
    if (cos->shape[0] < 1 || cos->data == nullptr || sin->data == nullptr) return RF_ERR_INVALID_ARG;
    if (!aligned4(cos) || !aligned4(sin)) return RF_ERR_ALIGNMENT;
    a.rot = (int)(2 * half);
    a.cos = (const float*)cos->data;
    a.sin = (const float*)sin->data;
    a.cos_pitch = cos->stride[0];
    a.sin_pitch = sin->stride[0];
    a.table_rows = cos->shape[0];
  }
  if (!rf::paged_append_fits(p)) return RF_ERR_UNSUPPORTED;
  if (empty(p)) return RF_OK;
  a.q = q->data;
  a.k = k->data;
  a.v = v->data;
  a.q_norm = q_norm != nullptr ? q_norm->data : nullptr;
  a.k_norm = k_norm != nullptr ? k_norm->data : nullptr;
  a.k_cache = k_cache->data;
  a.v_cache = v_cache->data;
  a.q_out = q_out->data;
  a.sq = strides2(q);
  a.sk = strides2(k);
  a.sv = strides2(v);
  a.so = strides2(q_out);
  a.eps = eps;
  a.k_scale = k_scale;
  a.v_scale = v_scale;
  a.interleaved = interleaved != 0;
  a.fp8 = k_cache->dtype == RF_FP8_E4M3;
  return status_of(rf::launch_paged_append(a, (hipStream_t)stream));
}

rf_status rf_paged_attention(const rf_tensor* q, const rf_tensor* k_cache, const rf_tensor* v_cache,
                             const rf_tensor* seq_start, const rf_tensor* kv_len, const rf_tensor* pages, int64_t max_q,
                             float scale, int causal, float k_scale, float v_scale, rf_tensor* o, rf_stream stream) {
  rf::PagedAttention a{};
  const rf_status st = check_paged_attention(q, k_cache, v_cache, seq_start, kv_len, pages, max_q, scale, causal, k_scale,
                                             v_scale, o, &a);
  if (st != RF_OK || empty(a.p)) return st;
  return status_of(rf::launch_paged_attention(a, nullptr, (hipStream_t)stream));
}

size_t rf_paged_attention_workspace_bytes(const rf_tensor* q, const rf_tensor* k_cache, const rf_tensor* pages,
                                          int64_t max_q) {
  rf::Paged p{};
  if (paged_shape(q, k_cache, pages, &p) != RF_OK || empty(p) || max_q < 0 || !rf::paged_attention_fits(p, max_q)) return 0;
  return rf::paged_attention_bytes(p, max_q);
}

rf_status rf_paged_attention_ws(const rf_tensor* q, const rf_tensor* k_cache, const rf_tensor* v_cache,
                                const rf_tensor* seq_start, const rf_tensor* kv_len, const rf_tensor* pages, int64_t max_q,
                                float scale, int causal, float k_scale, float v_scale, rf_tensor* o, void* workspace,
                                size_t workspace_bytes, rf_stream stream) {
  rf::PagedAttention a{};
  const rf_status st = check_paged_attention(q, k_cache, v_cache, seq_start, kv_len, pages, max_q, scale, causal, k_scale,
                                             v_scale, o, &a);
  if (st != RF_OK || empty(a.p)) return st;
  const size_t need = rf::paged_attention_bytes(a.p, max_q);
  if (need > 0 && (workspace == nullptr || reinterpret_cast<uintptr_t>(workspace) % 16 != 0 || workspace_bytes < need))
    return RF_ERR_WORKSPACE;
  return status_of(rf::launch_paged_attention(a, need > 0 ? workspace : nullptr, (hipStream_t)stream));
}

rf_status rf_verify_drafts(const rf_tensor* target, const rf_tensor* draft, const rf_tensor* tokens,
                           const rf_tensor* u_accept, const rf_tensor* u_sample, const rf_tensor* seq_start, rf_tensor* out,
                           rf_tensor* accepted, rf_stream stream) {
  rf::VerifyDrafts a{};
  const rf_status st = check_verify(target, draft, tokens, u_accept, u_sample, seq_start, out, accepted, &a);
  if (st != RF_OK || a.B == 0) return st;
  return status_of(rf::launch_verify_drafts(a, nullptr, (hipStream_t)stream));
}

size_t rf_verify_drafts_workspace_bytes(int64_t B, int64_t V) {
  if (B < 1 || V < 1 || V >= INT32_MAX || !rf::verify_drafts_fits(B)) return 0;
  return rf::verify_drafts_bytes(B, V);
}

rf_status rf_verify_drafts_ws(const rf_tensor* target, const rf_tensor* draft, const rf_tensor* tokens,
                              const rf_tensor* u_accept, const rf_tensor* u_sample, const rf_tensor* seq_start,
                              rf_tensor* out, rf_tensor* accepted, void* workspace, size_t workspace_bytes,
                              rf_stream stream) {
  rf::VerifyDrafts a{};
  const rf_status st = check_verify(target, draft, tokens, u_accept, u_sample, seq_start, out, accepted, &a);
  if (st != RF_OK || a.B == 0) return st;
  const size_t need = rf::verify_drafts_bytes(a.B, a.V);
  if (need > 0 && (workspace == nullptr || reinterpret_cast<uintptr_t>(workspace) % 16 != 0 || workspace_bytes < need))
    return RF_ERR_WORKSPACE;
  return status_of(rf::launch_verify_drafts(a, need > 0 ? workspace : nullptr, (hipStream_t)stream));
}

}  // extern "C"
