// gdn_layer.h -- private declarations of the chain form of the gated delta rule
// and of the norms around a block: arguments, rows of a sequence.
#pragma once

#include "gdn_internal.h"

namespace gdn {

struct ChainArgs {
  int B, T, Hk, Hv, dk, dv, in_dtype, out_dtype;
  long long rows;
  float scale;
  const int32_t *start, *n_new;
  const void *q, *k, *v, *alpha, *beta;
  const float *conv_w, *conv_state;
  float *conv_state_out, *S;
  void* out;
  int32_t* status;
};

// Tokens of sequence b: rows first .. first + n - 1.
struct Tokens {
  long long first;
  int n, status;
};

__device__ __forceinline__ Tokens tokens_of(const ChainArgs& a, int b) {
  long long first, n;
  if (a.start) {
    const int s0 = a.start[b], s1 = a.start[b + 1];
    first = s0;
    n = (long long)(s1) - s0;
    if (s0 < 0 || s1 > a.rows) n = -1;
  } else {
    first = (long long)(b) * a.T;
    n = a.n_new ? a.n_new[b] : a.T;
  }
  const bool bad = n < 0 || n > a.T;
  return {first, bad ? 0 : int(n), bad ? GDN_CHAIN_BAD_LEN : 0};
}

struct GateNormArgs {
  long long N, ldx, ldg;
  int H, d, act;
  float eps;
  const void *x, *gate;
  const float* weight;
  void* out;
};

struct AddNormArgs {
  long long N;
  int D, post;
  float eps;
  const void *x, *residual;
  const float *weight, *post_weight, *scale;
  void *res_out, *out;
};

// token by token, any length
int launch_chain_steps(const ChainArgs& a, hipStream_t stream);
// in chunks of 64 tokens
int launch_chain_chunks(const ChainArgs& a, hipStream_t stream);
int launch_gate_norm(const GateNormArgs& a, int x_dtype, int gate_dtype, int out_dtype, hipStream_t stream);
int launch_add_norm(const AddNormArgs& a, int x_dtype, int res_dtype, int out_dtype, hipStream_t stream);

// fp32 -> bf16, round to nearest even (NaN stays NaN)
__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(BF16* p, float x) { *reinterpret_cast<__bf16*>(p) = (__bf16)x; }

}  // namespace gdn
