// gdn_layer.h -- private declarations of the chain form of the gated delta rule
// and of the norms around a block: arguments, rows of a sequence.
#pragma once

#include <type_traits>

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

// Packed: whether the table goes backwards anywhere up to sequence b (or behind
// it); one that does not has no row twice.  Read 4 entries a lane without branches,
// by every wave for itself, or far into a long table by all waves of the workgroup.
__device__ __forceinline__ bool goes_back(const ChainArgs& a, int b) {
  const int lane = threadIdx.x % kWave;
  if (a.B < 4) return __any(lane < a.B && a.start[min(lane, a.B - 1) + 1] < a.start[min(lane, a.B - 1)]);
  typedef int i32x4 __attribute__((ext_vector_type(4), aligned(4)));
  bool back = false;
  auto look = [&](auto groups, int i, int first, int step) {
    constexpr int kGroups = decltype(groups)::value;
    i32x4 x[kGroups];
    int next[kGroups];
#pragma unroll
    for (int k = 0; k < kGroups; ++k) {  // the last whole group instead of what is behind the table
      const int32_t* s = a.start + min(i + k * step + first, a.B - 4);
      x[k] = *reinterpret_cast<const i32x4*>(s);
      next[k] = s[4];
    }
#pragma unroll
    for (int k = 0; k < kGroups; ++k) back |= x[k].y < x[k].x || x[k].z < x[k].y || x[k].w < x[k].z || next[k] < x[k].w;
  };
  if (b < 4 * kWave) {
    look(std::integral_constant<int, 1>{}, 0, 4 * lane, 4 * kWave);
    return __any(back);
  }
  const bool split = b >= 1024;
  const int first = 4 * (split ? threadIdx.x : lane), step = 4 * (split ? blockDim.x : kWave);
  for (int i = 0; i < b; i += 4 * step) look(std::integral_constant<int, 4>{}, i, first, step);
  return split ? __syncthreads_or(back) : __any(back);
}
// Whether rows first .. end - 1 of sequence b are also those of a sequence before
// it that is valid by its own two entries: both would write them.
__device__ __forceinline__ bool shares_rows(const ChainArgs& a, int b, int first, int end) {
  bool found = false;
  for (int i = threadIdx.x % kWave; i < b; i += kWave) {
    const int s0 = a.start[i], s1 = a.start[i + 1];
    found |= s0 >= 0 && s1 > s0 && s1 <= a.rows && s1 - s0 <= a.T && s0 < end && s1 > first;
  }
  return __any(found && first < end);
}

// By all threads of a workgroup, for one b.  kAlone: also whether its rows are its
// own, for kernels that write them.  us of packed calls without that and with it:
// one token of 32 sequences of 16 / 48 heads of 128 32.6 and 32.9, of 1024 of 2 / 4
// heads of 64 26.8 and 28.7, 16384 of one head of 16 25 and 63; 15 to 30 tokens of
// 4096 of 1 / 2 heads of 32 284 and 304.
template <bool kAlone = true>
__device__ __forceinline__ Tokens tokens_of(const ChainArgs& a, int b) {
  long long first, n;
  if (a.start) {
    const int s0 = a.start[b], s1 = a.start[b + 1];
    first = s0;
    n = (long long)(s1) - s0;
    if (s0 < 0 || s1 > a.rows) n = -1;
    if constexpr (kAlone)
      if (goes_back(a, b) && shares_rows(a, b, s0, s1)) n = -1;
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
