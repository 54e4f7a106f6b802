// gdn_norm.hip -- norms around a block: every head's norm times a gate, and the
// residual stream with the norms before and after the block.
//
// A team of threads holds a row (a head) in registers: K packs of V values a
// thread, so that a row is read once however many sums it takes.  Element types
// are uniform branches, not template arguments: they cost a scalar compare a
// pack.  Rows of no alignment go value by value (V = 1).
#include <algorithm>

#include "gdn_layer.h"

namespace gdn {
namespace {

constexpr int kThreads = 256;

template <int V>
__device__ __forceinline__ void fetch(const void* p, size_t i, int dtype, float (&x)[V]) {
  if constexpr (V == 1) {
    x[0] = dtype == GDN_BF16 ? to_f32(static_cast<const BF16*>(p)[i]) : static_cast<const float*>(p)[i];
  } else {
    float4 y, z;
    if (dtype == GDN_BF16) {
      const u32x4 u = *reinterpret_cast<const u32x4*>(static_cast<const BF16*>(p) + i);
      y = make_float4(__uint_as_float(u[0] << 16), __uint_as_float(u[0] & 0xffff0000u), __uint_as_float(u[1] << 16),
                      __uint_as_float(u[1] & 0xffff0000u));
      z = make_float4(__uint_as_float(u[2] << 16), __uint_as_float(u[2] & 0xffff0000u), __uint_as_float(u[3] << 16),
                      __uint_as_float(u[3] & 0xffff0000u));
    } else {
      y = *reinterpret_cast<const float4*>(static_cast<const float*>(p) + i);
      z = *reinterpret_cast<const float4*>(static_cast<const float*>(p) + i + 4);
    }
    x[0] = y.x, x[1] = y.y, x[2] = y.z, x[3] = y.w, x[4] = z.x, x[5] = z.y, x[6] = z.z, x[7] = z.w;
  }
}

template <int V>
__device__ __forceinline__ void store(void* p, size_t i, int dtype, const float (&x)[V]) {
  if constexpr (V == 1) {
    if (dtype == GDN_BF16) put(static_cast<BF16*>(p) + i, x[0]);
    else static_cast<float*>(p)[i] = x[0];
  } else if (dtype == GDN_BF16) {
    bf16x8 y;
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = (__bf16)x[e];
    *reinterpret_cast<bf16x8*>(static_cast<BF16*>(p) + i) = y;
  } else {
    float* q = static_cast<float*>(p) + i;
    *reinterpret_cast<float4*>(q) = make_float4(x[0], x[1], x[2], x[3]);
    *reinterpret_cast<float4*>(q + 4) = make_float4(x[4], x[5], x[6], x[7]);
  }
}

// fp32 parameters, 16-byte aligned where V is 8
template <int V>
__device__ __forceinline__ void param(const float* p, int i, float (&x)[V]) {
  if (p) {
    fetch<V>(p, size_t(i), GDN_F32, x);
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) x[e] = 1.0f;
  }
}

// Sum over a team of G consecutive threads.  s: 4 values that no other sum of
// the workgroup uses before the next barrier.
template <int G>
__device__ __forceinline__ float team_sum(float v, float* s) {
  if constexpr (G <= 64) {
    return group_sum<G>(v);
  } else {
    static_assert(G == kThreads, "a team is part of a wave or the workgroup");
    v = wave_sum(v);
    if (threadIdx.x % kWave == 0) s[threadIdx.x / kWave] = v;
    __syncthreads();
    return (s[0] + s[1]) + (s[2] + s[3]);
  }
}

struct Types {
  int x, other, out;  // other: gate or residual
};

template <int V, int K, int G>
__global__ __launch_bounds__(kThreads) void gate_norm_kernel(GateNormArgs a, Types ty) {
  __shared__ float s_sum[2][4];
  const int at = threadIdx.x % G, teams = kThreads / G, d = a.d;
  const float inv = 1.0f / float(d);
  const unsigned rows = unsigned(a.N) * unsigned(a.H), step = gridDim.x * teams;
  int turn = 0;
  for (unsigned r = blockIdx.x * teams + threadIdx.x / G; r < rows; r += step, turn ^= 1) {
    const unsigned n = r / unsigned(a.H), h = r - n * unsigned(a.H);
    const size_t ix = size_t(n) * a.ldx + size_t(h) * d, ig = size_t(n) * a.ldg + size_t(h) * d, io = size_t(r) * d;
    float x[K][V], g[K][V], sum = 0.0f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = (k * G + at) * V;
#pragma unroll
      for (int e = 0; e < V; ++e) x[k][e] = 0.0f;
      if (c >= d) continue;
      fetch<V>(a.x, ix + c, ty.x, x[k]);
      if (a.gate) fetch<V>(a.gate, ig + c, ty.other, g[k]);
    }
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int e = 0; e < V; ++e) sum += x[k][e] * x[k][e];
    const float f = rsqrt_hw(team_sum<G>(sum, s_sum[turn]) * inv + a.eps);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = (k * G + at) * V;
      if (c >= d) continue;
      float w[V];
      param<V>(a.weight, c, w);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        float y = x[k][e] * f * w[e];
        if (a.gate) {
          const float s = __builtin_amdgcn_rcpf(1.0f + __expf(-g[k][e]));
          y *= a.act == GDN_SILU ? g[k][e] * s : s;
        }
        x[k][e] = y;
      }
      store<V>(a.out, io + c, ty.out, x[k]);
    }
  }
}

template <int V, int K, int G>
__global__ __launch_bounds__(kThreads) void add_norm_kernel(AddNormArgs a, Types ty) {
  __shared__ float s_sum[4][4];
  const int at = threadIdx.x % G, teams = kThreads / G, D = a.D;
  const float inv = 1.0f / float(D);
  const unsigned rows = unsigned(a.N), step = gridDim.x * teams;
  int turn = 0;
  for (unsigned r = blockIdx.x * teams + threadIdx.x / G; r < rows; r += step, turn ^= 2) {
    const size_t i = size_t(r) * D;
    float x[K][V], y[K][V];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = (k * G + at) * V;
#pragma unroll
      for (int e = 0; e < V; ++e) x[k][e] = y[k][e] = 0.0f;
      if (c >= D) continue;
      fetch<V>(a.x, i + c, ty.x, x[k]);
      if (a.residual) fetch<V>(a.residual, i + c, ty.other, y[k]);
    }
    float f = 1.0f;
    if (a.post) {
      float sum = 0.0f;
#pragma unroll
      for (int k = 0; k < K; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) sum += x[k][e] * x[k][e];
      f = rsqrt_hw(team_sum<G>(sum, s_sum[turn]) * inv + a.eps);
    }
    float sum = 0.0f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = (k * G + at) * V;
      if (c >= D) continue;
      float w[V], s[V];
      param<V>(a.post ? a.post_weight : nullptr, c, w);
      param<V>(a.scale, c, s);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        y[k][e] += x[k][e] * f * w[e] * s[e];
        sum += y[k][e] * y[k][e];
      }
      if (a.res_out) store<V>(a.res_out, i + c, ty.other, y[k]);
    }
    if (!a.out) continue;
    f = rsqrt_hw(team_sum<G>(sum, s_sum[turn + 1]) * inv + a.eps);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = (k * G + at) * V;
      if (c >= D) continue;
      float w[V];
      param<V>(a.weight, c, w);
#pragma unroll
      for (int e = 0; e < V; ++e) y[k][e] *= f * w[e];
      store<V>(a.out, i + c, ty.out, y[k]);
    }
  }
}

// Runs launch.template go<V, K, G>() for rows of d values.
template <typename F>
int for_rows(int d, bool packs, const F& f) {
  if (packs) {
    const int p = d / 8;
    if (p <= 1) return f.template go<8, 1, 1>();
    if (p <= 2) return f.template go<8, 1, 2>();
    if (p <= 4) return f.template go<8, 1, 4>();
    if (p <= 8) return f.template go<8, 1, 8>();
    if (p <= 16) return f.template go<8, 1, 16>();
    if (p <= 32) return f.template go<8, 1, 32>();
    if (p <= 64) return f.template go<8, 1, 64>();
    if (p <= 256) return f.template go<8, 1, 256>();
    if (p <= 512) return f.template go<8, 2, 256>();
    if (p <= 1024) return f.template go<8, 4, 256>();
    return f.template go<8, 8, 256>();
  }
  if (d <= 16) return f.template go<1, 1, 16>();
  if (d <= 64) return f.template go<1, 1, 64>();
  if (d <= 256) return f.template go<1, 4, 64>();
  if (d <= 1024) return f.template go<1, 4, 256>();
  if (d <= 2048) return f.template go<1, 8, 256>();
  if (d <= 4096) return f.template go<1, 16, 256>();
  return f.template go<1, 64, 256>();
}

int after_launch(const char* who) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? GDN_OK : set_error(GDN_EHIP, "%s: launch: %s", who, hipGetErrorString(e));
}

// Workgroups for `rows` rows of teams of G threads: up to eight a CU, each with
// rows in turn.
template <int G>
unsigned blocks_for(unsigned rows) {
  const unsigned teams = kThreads / G;
  return std::min((rows - 1) / teams + 1, 2048u);
}

struct GateLaunch {
  const GateNormArgs& a;
  Types ty;
  hipStream_t stream;
  template <int V, int K, int G>
  int go() const {
    gate_norm_kernel<V, K, G><<<blocks_for<G>(unsigned(a.N) * unsigned(a.H)), kThreads, 0, stream>>>(a, ty);
    return after_launch("gate_norm");
  }
};

struct AddLaunch {
  const AddNormArgs& a;
  Types ty;
  hipStream_t stream;
  template <int V, int K, int G>
  int go() const {
    add_norm_kernel<V, K, G><<<blocks_for<G>(unsigned(a.N)), kThreads, 0, stream>>>(a, ty);
    return after_launch("add_norm");
  }
};

bool at16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }
bool rows16(long long ld, int dtype) { return ld * (dtype == GDN_BF16 ? 2 : 4) % 16 == 0; }

}  // namespace

int launch_gate_norm(const GateNormArgs& a, int x_dtype, int gate_dtype, int out_dtype, hipStream_t stream) {
  const bool packs = a.d % 8 == 0 && at16(a.x) && rows16(a.ldx, x_dtype) && at16(a.gate) &&
                     (!a.gate || rows16(a.ldg, gate_dtype)) && at16(a.weight) && at16(a.out);
  return for_rows(a.d, packs, GateLaunch{a, {x_dtype, gate_dtype, out_dtype}, stream});
}

int launch_add_norm(const AddNormArgs& a, int x_dtype, int res_dtype, int out_dtype, hipStream_t stream) {
  const bool packs = a.D % 8 == 0 && at16(a.x) && at16(a.residual) && at16(a.res_out) && at16(a.out) && at16(a.weight) &&
                     at16(a.post_weight) && at16(a.scale);
  return for_rows(a.D, packs, AddLaunch{a, {x_dtype, res_dtype, out_dtype}, stream});
}

}  // namespace gdn
