// gdn_attn_abi.hip -- the extern "C" boundary of the softmax-attention and
// sampling operators (declared in include/gdn_tree.h): argument validation on
// the host and dispatch to the launchers.
#include <math.h>

#include "gdn_attn.h"

namespace gdn {

static int check_attn(const gdn_attn_dims* d, const void* meta, const int32_t* n_new, const char* who) {
  if (!d) return set_error(GDN_EINVAL, "%s: dims is NULL", who);
  if (d->B < 0 || d->T < 0 || d->Hq < 1 || d->Hkv < 1)
    return set_error(GDN_EINVAL, "%s: bad sizes B=%d T=%d Hq=%d Hkv=%d", who, d->B, d->T, d->Hq, d->Hkv);
  if (d->Hq % d->Hkv != 0)
    return set_error(GDN_EINVAL, "%s: Hq=%d is not a multiple of Hkv=%d", who, d->Hq, d->Hkv);
  if (d->dtype != GDN_F32 && d->dtype != GDN_BF16) return set_error(GDN_EINVAL, "%s: dtype=%d", who, d->dtype);
  if (!(d->scale >= 0.0f) || isinf(d->scale))
    return set_error(GDN_EINVAL, "%s: scale must be finite and >= 0", who);
  if (d->n_pages < 1 || d->max_pages < 1)
    return set_error(GDN_EINVAL, "%s: n_pages=%d max_pages=%d", who, d->n_pages, d->max_pages);
  if (d->rot < 0 || d->rot > d->d || d->rot % 2 != 0 || d->n_pos < 0)
    return set_error(GDN_EINVAL, "%s: rot=%d of d=%d, n_pos=%d", who, d->rot, d->d, d->n_pos);
  if (meta && n_new) return set_error(GDN_EINVAL, "%s: n_new together with tree metadata", who);
  if (d->d != 32 && d->d != 64 && d->d != 128 && d->d != 256)
    return set_error(GDN_EUNSUPPORTED, "%s: d=%d (supported 32, 64, 128, 256)", who, d->d);
  if (d->page != 16 && d->page != 32 && d->page != 64 && d->page != 128 && d->page != 256)
    return set_error(GDN_EUNSUPPORTED, "%s: page=%d (supported 16, 32, 64, 128, 256)", who, d->page);
  if (d->T > GDN_MAX_T) return set_error(GDN_EUNSUPPORTED, "%s: T=%d > %d", who, d->T, GDN_MAX_T);
  // a grid's y and z; positions and row offsets inside a sequence are 32-bit
  if (d->B > 65535 || d->Hq > 65535 / 4 || (long long)(d->T) * (d->Hq / d->Hkv) > GDN_MAX_KV_ROWS ||
      (long long)(d->max_pages) * d->page > 0x40000000LL)
    return set_error(GDN_EUNSUPPORTED, "%s: B=%d T=%d Hq=%d Hkv=%d max_pages=%d", who, d->B, d->T, d->Hq, d->Hkv,
                     d->max_pages);
  return GDN_OK;
}

static AttnArgs make_args(const gdn_attn_dims* d, const void* meta, const int32_t* n_new, const int32_t* ctx_len,
                          const int32_t* page_table) {
  AttnArgs a = {};
  a.B = d->B;
  a.T = d->T;
  a.Hq = d->Hq;
  a.dtype = d->dtype;
  a.rot = d->rot;
  a.n_pos = d->n_pos;
  a.scale = d->scale > 0.0f ? d->scale : 1.0f / sqrtf(float(d->d));
  a.c.Hkv = d->Hkv;
  a.c.d = d->d;
  a.c.page_shift = __builtin_ctz(unsigned(d->page));
  a.c.n_pages = d->n_pages;
  a.c.max_pages = d->max_pages;
  a.meta = meta;
  a.n_new = n_new;
  a.ctx_len = ctx_len;
  a.page_table = page_table;
  return a;
}

static bool overlap(const void* p, size_t np, const void* q, size_t nq) {
  const char *x = static_cast<const char*>(p), *y = static_cast<const char*>(q);
  return x < y + nq && y < x + np;
}

}  // namespace gdn

using namespace gdn;

extern "C" {

int gdn_kv_append(const gdn_attn_dims* dims, const void* meta, const int32_t* n_new, const void* q, const void* k,
                  const void* v, const float* rope, const int32_t* ctx_len, const int32_t* page_table, void* k_cache,
                  void* v_cache, void* q_out, int32_t* kv_status, hipStream_t stream) {
  int rc = check_attn(dims, meta, n_new, "kv_append");
  if (rc != GDN_OK) return rc;
  if (dims->B == 0 || dims->T == 0) return GDN_OK;
  if (!q || !k || !v || !ctx_len || !page_table || !k_cache || !v_cache || !q_out || (dims->rot && !rope))
    return set_error(GDN_EINVAL, "kv_append: NULL tensor pointer");
  const size_t qb = size_t(dims->B) * dims->T * dims->Hq * dims->d * (dims->dtype == GDN_BF16 ? 2 : 4);
  if (q != q_out && overlap(q, qb, q_out, qb))
    return set_error(GDN_EINVAL, "kv_append: q and q_out overlap in part");
  const size_t kb = qb / dims->Hq * dims->Hkv;
  if (overlap(k, kb, q_out, qb) || overlap(v, kb, q_out, qb))
    return set_error(GDN_EINVAL, "kv_append: q_out overlaps k or v");
  AttnArgs a = make_args(dims, meta, n_new, ctx_len, page_table);
  a.q = q;
  a.k = k;
  a.v = v;
  a.rope = rope;
  a.k_cache = k_cache;
  a.v_cache = v_cache;
  a.out = q_out;
  a.status = kv_status;
  return launch_kv_append(a, stream);
}

int gdn_tree_attend(const gdn_attn_dims* dims, const void* meta, const int32_t* n_new, const void* q,
                    const void* k_cache, const void* v_cache, const int32_t* page_table, const int32_t* ctx_len,
                    void* out, hipStream_t stream) {
  int rc = check_attn(dims, meta, n_new, "attend");
  if (rc != GDN_OK) return rc;
  if (dims->B == 0 || dims->T == 0) return GDN_OK;
  if (!q || !k_cache || !v_cache || !ctx_len || !page_table || !out)
    return set_error(GDN_EINVAL, "attend: NULL tensor pointer");
  const size_t qb = size_t(dims->B) * dims->T * dims->Hq * dims->d * (dims->dtype == GDN_BF16 ? 2 : 4);
  if (overlap(q, qb, out, qb)) return set_error(GDN_EINVAL, "attend: q and out overlap");
  AttnArgs a = make_args(dims, meta, n_new, ctx_len, page_table);
  a.q = q;
  a.k_cache = const_cast<void*>(k_cache);
  a.v_cache = const_cast<void*>(v_cache);
  a.out = out;
  return launch_attend(a, stream);
}

int gdn_kv_commit(const gdn_attn_dims* dims, const void* meta, const int32_t* accepted, const int32_t* page_table,
                  const int32_t* ctx_len, void* k_cache, void* v_cache, int32_t* new_len, int32_t* kv_status,
                  hipStream_t stream) {
  int rc = check_attn(dims, meta, nullptr, "kv_commit");
  if (rc != GDN_OK) return rc;
  if (dims->B == 0 || dims->T == 0) return GDN_OK;
  if (!accepted || !ctx_len || !page_table || !k_cache || !v_cache || !new_len)
    return set_error(GDN_EINVAL, "kv_commit: NULL tensor pointer");
  const size_t lb = size_t(dims->B) * 4;
  if (overlap(ctx_len, lb, new_len, lb) || overlap(accepted, lb, new_len, lb))
    return set_error(GDN_EINVAL, "kv_commit: new_len overlaps ctx_len or accepted");
  AttnArgs a = make_args(dims, meta, nullptr, ctx_len, page_table);
  a.accepted = accepted;
  a.k_cache = k_cache;
  a.v_cache = v_cache;
  a.new_len = new_len;
  a.status = kv_status;
  return launch_kv_commit(a, stream);
}

int gdn_tree_sample(const gdn_sample_dims* dims, const void* meta, const void* logits, const float* temperature,
                    const int32_t* top_k, const float* top_p, const float* min_p, const float* u, int32_t* token,
                    hipStream_t stream) {
  if (!dims) return set_error(GDN_EINVAL, "sample: dims is NULL");
  if (dims->B < 0 || dims->T < 0 || dims->V < 1)
    return set_error(GDN_EINVAL, "sample: bad sizes B=%d T=%d V=%d", dims->B, dims->T, dims->V);
  if (dims->dtype != GDN_F32 && dims->dtype != GDN_BF16)
    return set_error(GDN_EINVAL, "sample: dtype=%d", dims->dtype);
  if (dims->ld != 0 && dims->ld < dims->V)
    return set_error(GDN_EINVAL, "sample: ld=%lld < V=%d", (long long)(dims->ld), dims->V);
  if (dims->V > GDN_MAX_V) return set_error(GDN_EUNSUPPORTED, "sample: V=%d > %d", dims->V, GDN_MAX_V);
  if (dims->T > GDN_MAX_T) return set_error(GDN_EUNSUPPORTED, "sample: T=%d > %d", dims->T, GDN_MAX_T);
  if ((long long)(dims->B) * dims->T > 0x7fffffffLL)
    return set_error(GDN_EUNSUPPORTED, "sample: B=%d T=%d", dims->B, dims->T);
  if (dims->B == 0 || dims->T == 0) return GDN_OK;
  if (!logits || !u || !token) return set_error(GDN_EINVAL, "sample: NULL tensor pointer");
  SampleArgs a;
  a.B = dims->B;
  a.T = dims->T;
  a.V = dims->V;
  a.dtype = dims->dtype;
  a.ld = dims->ld ? dims->ld : dims->V;
  a.meta = meta;
  a.logits = logits;
  a.temperature = temperature;
  a.top_p = top_p;
  a.min_p = min_p;
  a.u = u;
  a.top_k = top_k;
  a.token = token;
  return launch_sample(a, stream);
}

int gdn_tree_accept(const gdn_dims* dims, const void* meta, const int32_t* draft, const int32_t* token,
                    int32_t* accepted, int32_t* n_emitted, int32_t* emitted, hipStream_t stream) {
  if (!dims) return set_error(GDN_EINVAL, "accept: dims is NULL");
  if (dims->B < 0 || dims->T < 0) return set_error(GDN_EINVAL, "accept: bad sizes B=%d T=%d", dims->B, dims->T);
  if (dims->T > GDN_MAX_T) return set_error(GDN_EUNSUPPORTED, "accept: T=%d > %d", dims->T, GDN_MAX_T);
  if (dims->B == 0 || dims->T == 0) return GDN_OK;
  if (!draft || !token || !accepted || !n_emitted || !emitted)
    return set_error(GDN_EINVAL, "accept: NULL tensor pointer");
  const size_t nb = size_t(dims->B) * dims->T * 4;
  if (overlap(draft, nb, emitted, nb) || overlap(token, nb, emitted, nb))
    return set_error(GDN_EINVAL, "accept: emitted overlaps draft or token");
  return launch_accept(dims->B, dims->T, meta, draft, token, accepted, n_emitted, emitted, stream);
}

}  // extern "C"
