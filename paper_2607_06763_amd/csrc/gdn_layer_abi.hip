// gdn_layer_abi.hip -- the extern "C" boundary of the chain form and of the
// norms around a block (declared in include/gdn_tree.h): argument validation on
// the host and dispatch to the launchers.
#include <float.h>
#include <math.h>

#include <utility>

#include "gdn_layer.h"

namespace gdn {

static bool dtype_ok(int t) { return t == GDN_F32 || t == GDN_BF16; }
static size_t width(int t) { return t == GDN_BF16 ? 2 : 4; }
static bool aligned(const void* p, int t) { return reinterpret_cast<uintptr_t>(p) % width(t) == 0; }

static bool overlap(const void* p, size_t np, const void* q, size_t nq) {
  const char *x = static_cast<const char*>(p), *y = static_cast<const char*>(q);
  return p && q && x < y + nq && y < x + np;
}

static int check_chain(const gdn_chain_dims* d, const int32_t* start, const int32_t* n_new) {
  if (!d) return set_error(GDN_EINVAL, "chain: dims is NULL");
  if (d->B < 0 || d->T < 0 || d->Hk < 1 || d->Hv < 1)
    return set_error(GDN_EINVAL, "chain: bad sizes B=%d T=%d Hk=%d Hv=%d", d->B, d->T, d->Hk, d->Hv);
  if (d->Hv % d->Hk != 0) return set_error(GDN_EINVAL, "chain: Hv=%d is not a multiple of Hk=%d", d->Hv, d->Hk);
  if (!dtype_ok(d->in_dtype) || !dtype_ok(d->out_dtype))
    return set_error(GDN_EINVAL, "chain: in_dtype=%d out_dtype=%d", d->in_dtype, d->out_dtype);
  if (!(d->scale >= 0.0f) || isinf(d->scale)) return set_error(GDN_EINVAL, "chain: scale must be finite and >= 0");
  if (start && n_new) return set_error(GDN_EINVAL, "chain: n_new together with start");
  if (start && d->rows < 0) return set_error(GDN_EINVAL, "chain: rows=%lld", (long long)(d->rows));
  auto dim = [](int x) { return x == 16 || x == 32 || x == 64 || x == 128; };
  if (!dim(d->dk) || !dim(d->dv))
    return set_error(GDN_EUNSUPPORTED, "chain: dk=%d dv=%d (supported 16, 32, 64, 128)", d->dk, d->dv);
  // a grid's y and z; first rows are 32-bit
  if (d->T > GDN_MAX_CHAIN_T || d->B > 65535 || d->Hv > 65535 || (start ? d->rows : (long long)(d->B) * d->T) > 0x7fffffffLL)
    return set_error(GDN_EUNSUPPORTED, "chain: B=%d T=%d Hv=%d rows=%lld", d->B, d->T, d->Hv, (long long)(d->rows));
  return GDN_OK;
}

static bool eps_ok(float e) { return e >= FLT_MIN && e <= FLT_MAX; }

}  // namespace gdn

using namespace gdn;

extern "C" {

int gdn_chain(const gdn_chain_dims* dims, const int32_t* start, const int32_t* n_new, const void* q, const void* k,
              const void* v, const void* alpha, const void* beta, const float* conv_w, const float* conv_state,
              float* conv_state_out, float* S, void* out, int32_t* status, hipStream_t stream) {
  int rc = check_chain(dims, start, n_new);
  if (rc != GDN_OK) return rc;
  if (dims->B == 0) return GDN_OK;
  const size_t rows = start ? size_t(dims->rows) : size_t(dims->B) * dims->T;
  if (!conv_w || !conv_state || !conv_state_out || !S || (rows && (!q || !k || !v || !alpha || !beta || !out)))
    return set_error(GDN_EINVAL, "chain: NULL tensor pointer");
  const size_t C = 2 * size_t(dims->Hk) * dims->dk + size_t(dims->Hv) * dims->dv, cs = size_t(dims->B) * 3 * C * 4;
  if (overlap(conv_state, cs, conv_state_out, cs))
    return set_error(GDN_EINVAL, "chain: conv_state and conv_state_out overlap");
  const size_t e = width(dims->in_dtype), ob = rows * dims->Hv * dims->dv * width(dims->out_dtype);
  const size_t kb = rows * dims->Hk * dims->dk * e, vb = rows * dims->Hv * dims->dv * e, gb = rows * dims->Hv * e;
  const size_t sb = size_t(dims->B) * dims->Hv * dims->dv * dims->dk * 4;
  const size_t ib = size_t(dims->B) * 4;
  const std::pair<const void*, size_t> inputs[] = {{q, kb},    {k, kb},          {v, vb},           {alpha, gb},
                                                   {beta, gb}, {conv_w, 16 * C}, {conv_state, cs}, {start, ib + 4},
                                                   {n_new, ib}};
  const std::pair<const void*, size_t> outputs[] = {{S, sb}, {conv_state_out, cs}, {out, ob}, {status, ib}};
  for (const auto& o : outputs) {
    bool bad = false;
    for (const auto& i : inputs) bad = bad || overlap(o.first, o.second, i.first, i.second);
    for (const auto& i : outputs) bad = bad || (&i != &o && overlap(o.first, o.second, i.first, i.second));
    if (bad) return set_error(GDN_EINVAL, "chain: S, conv_state_out, out or status overlaps another tensor");
  }
  ChainArgs a;
  a.B = dims->B;
  a.T = dims->T;
  a.Hk = dims->Hk;
  a.Hv = dims->Hv;
  a.dk = dims->dk;
  a.dv = dims->dv;
  a.in_dtype = dims->in_dtype;
  a.out_dtype = dims->out_dtype;
  a.rows = (long long)(rows);
  a.scale = dims->scale > 0.0f ? dims->scale : 1.0f / sqrtf(float(dims->dk));
  a.start = start;
  a.n_new = n_new;
  a.q = q;
  a.k = k;
  a.v = v;
  a.alpha = alpha;
  a.beta = beta;
  a.conv_w = conv_w;
  a.conv_state = conv_state;
  a.conv_state_out = conv_state_out;
  a.S = S;
  a.out = out;
  a.status = status;
  // A token costs the steps about the same each, the chunked form 64 of them.
  // us for 16 and 24 tokens (steps, chunks; chunks take the same up to 64), 16 / 48
  // heads of 128: one sequence 18, 24 and 25, 24; 8 of them 49, 50 and 72, 51; 32 of
  // them 95, 119 and 131, 121; 16 of 4 / 8 heads of 64: 13, 21 and 18, 21.  They cross at
  // 23, 17, 22 and 29 tokens; the one limit costs the second 61 for 50 at 20 tokens, the
  // last 21 for 18 at 24.
  return a.T <= GDN_CHAIN_STEP_T ? launch_chain_steps(a, stream) : launch_chain_chunks(a, stream);
}

int gdn_gate_norm(const gdn_gate_norm_dims* dims, const void* x, const void* gate, const float* weight, void* out,
                  hipStream_t stream) {
  if (!dims) return set_error(GDN_EINVAL, "gate_norm: dims is NULL");
  if (dims->N < 0 || dims->H < 1 || dims->d < 1)
    return set_error(GDN_EINVAL, "gate_norm: bad sizes N=%lld H=%d d=%d", (long long)(dims->N), dims->H, dims->d);
  if (!dtype_ok(dims->x_dtype) || !dtype_ok(dims->gate_dtype) || !dtype_ok(dims->out_dtype))
    return set_error(GDN_EINVAL, "gate_norm: dtypes %d %d %d", dims->x_dtype, dims->gate_dtype, dims->out_dtype);
  if (dims->act != GDN_SILU && dims->act != GDN_SIGMOID) return set_error(GDN_EINVAL, "gate_norm: act=%d", dims->act);
  if (!eps_ok(dims->eps)) return set_error(GDN_EINVAL, "gate_norm: eps must be positive, finite and not subnormal");
  const long long row = (long long)(dims->H) * dims->d;
  if ((dims->ldx && dims->ldx < row) || (dims->ldg && dims->ldg < row))
    return set_error(GDN_EINVAL, "gate_norm: ldx=%lld ldg=%lld < %lld", (long long)(dims->ldx), (long long)(dims->ldg), row);
  if (dims->d > GDN_MAX_NORM_D || row > GDN_MAX_ROW || dims->N > 0x7fffffffLL / dims->H || dims->ldx > (1LL << 40) ||
      dims->ldg > (1LL << 40))
    return set_error(GDN_EUNSUPPORTED, "gate_norm: N=%lld H=%d d=%d", (long long)(dims->N), dims->H, dims->d);
  if (dims->N == 0) return GDN_OK;
  if (!x || !out) return set_error(GDN_EINVAL, "gate_norm: NULL tensor pointer");
  if (!aligned(x, dims->x_dtype) || !aligned(gate, dims->gate_dtype) || !aligned(out, dims->out_dtype) ||
      !aligned(weight, GDN_F32))
    return set_error(GDN_EINVAL, "gate_norm: a pointer is not aligned to its elements");
  GateNormArgs a;
  a.N = dims->N;
  a.H = dims->H;
  a.d = dims->d;
  a.act = dims->act;
  a.eps = dims->eps;
  a.ldx = dims->ldx ? dims->ldx : row;
  a.ldg = dims->ldg ? dims->ldg : row;
  a.x = x;
  a.gate = gate;
  a.weight = weight;
  a.out = out;
  const size_t n = size_t(dims->N), ob = n * row * width(dims->out_dtype);
  const size_t xb = ((n - 1) * a.ldx + row) * width(dims->x_dtype), gb = ((n - 1) * a.ldg + row) * width(dims->gate_dtype);
  const bool in_place = x == out && dims->x_dtype == dims->out_dtype && (a.ldx == row || n == 1);
  if ((!in_place && overlap(x, xb, out, ob)) || overlap(gate, gb, out, ob) || overlap(weight, size_t(dims->d) * 4, out, ob))
    return set_error(GDN_EINVAL, "gate_norm: out overlaps an input");
  return launch_gate_norm(a, dims->x_dtype, dims->gate_dtype, dims->out_dtype, stream);
}

int gdn_add_norm(const gdn_add_norm_dims* dims, const void* x, const void* residual, const float* weight,
                 const float* post_weight, const float* scale, void* res_out, void* out, hipStream_t stream) {
  if (!dims) return set_error(GDN_EINVAL, "add_norm: dims is NULL");
  if (dims->N < 0 || dims->D < 1)
    return set_error(GDN_EINVAL, "add_norm: bad sizes N=%lld D=%d", (long long)(dims->N), dims->D);
  if (!dtype_ok(dims->x_dtype) || !dtype_ok(dims->res_dtype) || !dtype_ok(dims->out_dtype))
    return set_error(GDN_EINVAL, "add_norm: dtypes %d %d %d", dims->x_dtype, dims->res_dtype, dims->out_dtype);
  if (!eps_ok(dims->eps)) return set_error(GDN_EINVAL, "add_norm: eps must be positive, finite and not subnormal");
  if (post_weight && !dims->post) return set_error(GDN_EINVAL, "add_norm: post_weight without post");
  if (dims->D > GDN_MAX_NORM_D || dims->N > 0x7fffffffLL)
    return set_error(GDN_EUNSUPPORTED, "add_norm: N=%lld D=%d", (long long)(dims->N), dims->D);
  if (dims->N == 0) return GDN_OK;
  if (!x || (!res_out && !out)) return set_error(GDN_EINVAL, "add_norm: NULL tensor pointer");
  if (!aligned(x, dims->x_dtype) || !aligned(residual, dims->res_dtype) || !aligned(res_out, dims->res_dtype) ||
      !aligned(out, dims->out_dtype) || !aligned(weight, GDN_F32) || !aligned(post_weight, GDN_F32) || !aligned(scale, GDN_F32))
    return set_error(GDN_EINVAL, "add_norm: a pointer is not aligned to its elements");
  const size_t n = size_t(dims->N) * dims->D, xb = n * width(dims->x_dtype), rb = n * width(dims->res_dtype),
               ob = n * width(dims->out_dtype), wb = size_t(dims->D) * 4;
  const bool own_x = x == out && dims->x_dtype == dims->out_dtype;
  if (overlap(res_out, rb, x, xb) || (residual != res_out && overlap(res_out, rb, residual, rb)) || overlap(res_out, rb, out, ob) ||
      (!own_x && overlap(out, ob, x, xb)) || overlap(out, ob, residual, rb))
    return set_error(GDN_EINVAL, "add_norm: an output overlaps another tensor");
  for (const float* p : {weight, post_weight, scale})
    if (overlap(p, wb, res_out, rb) || overlap(p, wb, out, ob))
      return set_error(GDN_EINVAL, "add_norm: an output overlaps a parameter");
  AddNormArgs a;
  a.N = dims->N;
  a.D = dims->D;
  a.post = dims->post;
  a.eps = dims->eps;
  a.x = x;
  a.residual = residual;
  a.weight = weight;
  a.post_weight = post_weight;
  a.scale = scale;
  a.res_out = res_out;
  a.out = out;
  return launch_add_norm(a, dims->x_dtype, dims->res_dtype, dims->out_dtype, stream);
}

}  // extern "C"
