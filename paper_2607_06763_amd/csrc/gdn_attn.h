// gdn_attn.h -- private declarations of the softmax-attention and sampling
// kernels: arguments, the paged cache's addresses, per-sequence checks.
#pragma once

#include "gdn_internal.h"

namespace gdn {

// ---------------------------------------------------------------------------
// Paged cache (layout documented in gdn_tree.h)
// ---------------------------------------------------------------------------
template <typename T>
struct Pack {
  static constexpr int kN = 16 / int(sizeof(T));  // values of a 16-byte pack
};

struct CacheDims {
  int Hkv, d, page_shift, n_pages, max_pages;
};

// Page of position p of a sequence whose page-table row is given; -1 for an
// entry that must not be followed.  p has a place in the row.
__device__ __forceinline__ int page_of(const CacheDims& c, const int32_t* row, int p) {
  const int id = row[p >> c.page_shift];
  return unsigned(id) < unsigned(c.n_pages) ? id : -1;
}

// First element of a (page, head) block of either cache; a cache may hold
// more than 2^31 elements.
__device__ __forceinline__ size_t block_of(const CacheDims& c, int id, int h) {
  return ((size_t(id) * c.Hkv + h) * c.d) << c.page_shift;
}

// ---------------------------------------------------------------------------
// Arguments
// ---------------------------------------------------------------------------
struct AttnArgs {
  int B, T, Hq, dtype, rot, n_pos;
  float scale;
  CacheDims c;
  const void* meta;      // or NULL: a chain
  const int32_t* n_new;  // chain only, or NULL: T
  const int32_t *ctx_len, *page_table;
  void *k_cache, *v_cache;
  const void *q, *k, *v;
  const float* rope;
  void* out;  // append: rotated queries, attend: outputs
  const int32_t* accepted;
  int32_t *new_len, *status;
};

struct SampleArgs {
  int B, T, V, dtype;
  long long ld;
  const void* meta;
  const void* logits;
  const float *temperature, *top_p, *min_p, *u;
  const int32_t* top_k;
  int32_t* token;
};

int launch_kv_append(const AttnArgs& a, hipStream_t stream);
int launch_kv_commit(const AttnArgs& a, hipStream_t stream);
int launch_attend(const AttnArgs& a, hipStream_t stream);
int launch_sample(const SampleArgs& a, hipStream_t stream);
int launch_accept(int B, int T, const void* meta, const int32_t* draft, const int32_t* token, int32_t* accepted,
                  int32_t* n_emitted, int32_t* emitted, hipStream_t stream);

// ---------------------------------------------------------------------------
// Per-sequence checks
// ---------------------------------------------------------------------------
// Slots of sequence b that the page table must have room for.
__device__ __forceinline__ int span_of(const AttnArgs& a, int b) {
  return a.meta || !a.n_new ? a.T : a.n_new[b];
}

// GDN_KV_BAD_LEN of a sequence (0 otherwise): span outside [0, T], a negative
// length or one that leaves no room.
__device__ __forceinline__ int len_status(const AttnArgs& a, int ctx, int span) {
  const long long room = (long long)(a.c.max_pages) << a.c.page_shift;
  return (span < 0 || span > a.T || ctx < 0 || (long long)(ctx) + span > room) ? GDN_KV_BAD_LEN : 0;
}

// fp32 -> bf16, round to nearest even (NaN stays NaN)
__device__ __forceinline__ void st(float* p, float x) { *p = x; }
__device__ __forceinline__ void st(BF16* p, float x) { *reinterpret_cast<__bf16*>(p) = (__bf16)x; }

}  // namespace gdn
