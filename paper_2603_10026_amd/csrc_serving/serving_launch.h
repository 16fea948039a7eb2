// Internal launch interface of the serving operators, between their part of the C-ABI layer and the kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace rf {

// A batch of packed sequences and the paged cache that it meets.  What the three arrays on the device say is not
// known to the host: the kernels keep every access inside the tensors whatever it is.
struct Paged {
  const int32_t* seq_start;  // [B + 1]: sequence b owns the tokens seq_start[b] .. seq_start[b + 1] - 1
  const int32_t* kv_len;     // [B]: its keys, the new ones among them
  const int32_t* pages;      // [B, table_len]: page numbers, rows table_pitch apart
  int64_t table_pitch;
  int64_t page_stride, slot_stride, head_stride;  // of both caches, in elements
  int B, T, table_len, n_pages, page;             // page: slots of one
  int Hq, Hkv, group, d;                          // group: Hq / Hkv; T * Hq < 2^31
};

struct Strides2 {
  int64_t t, h;  // of a [tokens, heads, d] tensor, in elements
};

struct PagedAppend {
  Paged p;
  const void *q, *k, *v, *q_norm, *k_norm;  // bf16; the norms' weights [d] or null
  const float *cos, *sin;                   // [table_rows, rot / 2] with row pitches, or null (rot 0)
  void *k_cache, *v_cache, *q_out;
  Strides2 sq, sk, sv, so;
  int64_t cos_pitch, sin_pitch, table_rows;
  float eps, k_scale, v_scale;
  int rot, interleaved, fp8;
};
bool paged_append_fits(const Paged& p);  // whether its launch can be that large
hipError_t launch_paged_append(const PagedAppend& a, hipStream_t s);

struct PagedAttention {
  Paged p;
  const void *q, *k_cache, *v_cache;
  void* o;
  Strides2 sq, so;
  float scale_log2e, v_scale;  // scale_log2e: with the keys' scale in it
  int causal, fp8;
  int64_t max_q;               // tokens of the longest sequence, for the choice of kernels
};
bool paged_attention_fits(const Paged& p, int64_t max_q);  // whether its launches can be that large
// Device memory that launch_paged_attention takes for the states of split sequences; 0 where no sequence is split.
size_t paged_attention_bytes(const Paged& p, int64_t max_q);
// workspace: that many bytes, 16-byte aligned, or null: no sequence is split then.
hipError_t launch_paged_attention(const PagedAttention& a, void* workspace, hipStream_t s);

struct VerifyDrafts {
  const void *target, *draft;  // [R, V]; draft: null for drafts without probabilities
  int64_t target_pitch, draft_pitch;
  const int32_t *tokens, *seq_start;
  const float *u_accept, *u_sample;
  int32_t *out, *accepted;
  int64_t V;
  int R, B, bf16;
};
bool verify_drafts_fits(int64_t B);                // whether its launches can be that large
size_t verify_drafts_bytes(int64_t B, int64_t V);  // 0 where one launch serves the call
hipError_t launch_verify_drafts(const VerifyDrafts& a, void* workspace, hipStream_t s);

}  // namespace rf
