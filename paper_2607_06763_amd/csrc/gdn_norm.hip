// gdn_norm.hip -- norms around a block: every head's norm times a gate, and the
// residual stream with the norms before and after the block.
//
// A team of threads holds a row (a head) in registers, K packs of 8 values a
// thread, so that a row is read once however many sums it takes.  A pack is read
// and written whole at the alignment of its elements (the hardware takes 16
// bytes at any address; 999 rows of 2051 fp32 channels: 9 us where single
// values took 15); only a row's last pack, if not full, goes value by value.
// Element types are uniform branches, not template arguments: they cost a scalar
// compare a pack.
#include <algorithm>

#include "gdn_layer.h"

namespace gdn {
namespace {

constexpr int kThreads = 256;
constexpr int kV = 8;  // values of a pack

// 16 bytes at the alignment of an element
typedef u32x4 Bytes2 __attribute__((aligned(2)));
typedef f32x4 Bytes4 __attribute__((aligned(4)));

// The first n (up to 8) of the values from element i on; others are 0.
__device__ __forceinline__ void fetch(const void* p, size_t i, int dtype, int n, float (&x)[kV]) {
  if (n >= kV) {
    if (dtype == GDN_BF16) {
      const u32x4 u = *reinterpret_cast<const Bytes2*>(static_cast<const BF16*>(p) + i);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[2 * e] = __uint_as_float(u[e] << 16);
        x[2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u);
      }
    } else {
      const float* q = static_cast<const float*>(p) + i;
      const f32x4 y = *reinterpret_cast<const Bytes4*>(q), z = *reinterpret_cast<const Bytes4*>(q + 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = y[e], x[4 + e] = z[e];
    }
  } else {
#pragma unroll
    for (int e = 0; e < kV; ++e) {
      x[e] = 0.0f;
      if (e < n) x[e] = dtype == GDN_BF16 ? to_f32(static_cast<const BF16*>(p)[i + e]) : static_cast<const float*>(p)[i + e];
    }
  }
}

__device__ __forceinline__ void store(void* p, size_t i, int dtype, int n, const float (&x)[kV]) {
  if (n >= kV) {
    if (dtype == GDN_BF16) {
      bf16x8 y;
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = (__bf16)x[e];
      *reinterpret_cast<Bytes2*>(static_cast<BF16*>(p) + i) = __builtin_bit_cast(u32x4, y);
    } else {
      float* q = static_cast<float*>(p) + i;
      *reinterpret_cast<Bytes4*>(q) = f32x4{x[0], x[1], x[2], x[3]};
      *reinterpret_cast<Bytes4*>(q + 4) = f32x4{x[4], x[5], x[6], x[7]};
    }
  } else {
#pragma unroll
    for (int e = 0; e < kV; ++e)
      if (e < n) {
        if (dtype == GDN_BF16) put(static_cast<BF16*>(p) + i + e, x[e]);
        else static_cast<float*>(p)[i + e] = x[e];
      }
  }
}

// fp32 parameters of a row: from memory where they are used, or with few packs
// a thread held in registers for all rows of the workgroup.
template <int K, int G>
struct Param {
  static constexpr bool kKeep = K <= 2;
  const float* p;
  float w[kKeep ? K : 1][kV];
  __device__ __forceinline__ Param(const float* from, int d, int at) : p(from) {
    if constexpr (kKeep) {
#pragma unroll
      for (int k = 0; k < K; ++k) read(k, d, at, w[k]);
    }
  }
  __device__ __forceinline__ void read(int k, int d, int at, float (&x)[kV]) const {
    const int c = (k * G + at) * kV;
    if (p && c < d) {
      fetch(p, size_t(c), GDN_F32, d - c, x);
    } else {
#pragma unroll
      for (int e = 0; e < kV; ++e) x[e] = 1.0f;
    }
  }
  __device__ __forceinline__ void get(int k, int d, int at, float (&x)[kV]) const {
    if constexpr (kKeep) {
#pragma unroll
      for (int e = 0; e < kV; ++e) x[e] = w[k][e];
    } else {
      read(k, d, at, x);
    }
  }
};

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

// Bound by the bytes: 8192 rows of 48 heads of 128, fp32 in, bf16 gates and
// outputs, 403 MB in 75 to 77 us, 5.3 TB/s (a large copy reaches 5.1 to 5.3); one
// row 2.3 us.
template <int K, int G>
__global__ __launch_bounds__(kThreads) void gate_norm_kernel(GateNormArgs a, Types ty) {
  __shared__ float s_sum[2][4];
  const int at = threadIdx.x % G, teams = kThreads / G, d = a.d;
  const float inv = 1.0f / float(d);
  const unsigned rows = unsigned(a.N) * unsigned(a.H), step = gridDim.x * teams;
  const Param<K, G> weight(a.weight, d, at);
  int turn = 0;
  for (unsigned r = blockIdx.x * teams + threadIdx.x / G; r < rows; r += step, turn ^= 1) {
    const unsigned n = r / unsigned(a.H), h = r - n * unsigned(a.H);
    const size_t ix = size_t(n) * a.ldx + size_t(h) * d, ig = size_t(n) * a.ldg + size_t(h) * d, io = size_t(r) * d;
    float x[K][kV], g[K][kV], sum = 0.0f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = (k * G + at) * kV;
#pragma unroll
      for (int e = 0; e < kV; ++e) x[k][e] = 0.0f;
      if (c >= d) continue;
      fetch(a.x, ix + c, ty.x, d - c, x[k]);
      if (a.gate) fetch(a.gate, ig + c, ty.other, d - c, g[k]);
    }
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int e = 0; e < kV; ++e) sum += x[k][e] * x[k][e];
    const float f = rsqrt_hw(team_sum<G>(sum, s_sum[turn]) * inv + a.eps);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = (k * G + at) * kV;
      if (c >= d) continue;
      float w[kV];
      weight.get(k, d, at, w);
#pragma unroll
      for (int e = 0; e < kV; ++e) {
        float y = x[k][e] * f * w[e];
        if (a.gate) {
          const float s = __builtin_amdgcn_rcpf(1.0f + __expf(-g[k][e]));
          y *= a.act == GDN_SILU ? g[k][e] * s : s;
        }
        x[k][e] = y;
      }
      store(a.out, io + c, ty.out, d - c, x[k]);
    }
  }
}

// Bound by the bytes: 8192 rows of 4096 channels, bf16 branch, fp32 residual read
// and written, both norms, bf16 out, 403 MB in 86 us, 4.7 TB/s; the second sum waits
// for the first.  999 rows of 2051 fp32 channels 9.8 us, one row 3 to 4 us.
template <int K, int G>
__global__ __launch_bounds__(kThreads) void add_norm_kernel(AddNormArgs a, Types ty) {
  __shared__ float s_sum[4][4];
  const int at = threadIdx.x % G, teams = kThreads / G, D = a.D;
  const float inv = 1.0f / float(D);
  const unsigned rows = unsigned(a.N), step = gridDim.x * teams;
  const Param<K, G> weight(a.weight, D, at), post(a.post ? a.post_weight : nullptr, D, at), scale(a.scale, D, at);
  int turn = 0;
  for (unsigned r = blockIdx.x * teams + threadIdx.x / G; r < rows; r += step, turn ^= 2) {
    const size_t i = size_t(r) * D;
    float x[K][kV], y[K][kV];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = (k * G + at) * kV;
#pragma unroll
      for (int e = 0; e < kV; ++e) x[k][e] = y[k][e] = 0.0f;
      if (c >= D) continue;
      fetch(a.x, i + c, ty.x, D - c, x[k]);
      if (a.residual) fetch(a.residual, i + c, ty.other, D - c, y[k]);
    }
    float f = 1.0f;
    if (a.post) {
      float sum = 0.0f;
#pragma unroll
      for (int k = 0; k < K; ++k)
#pragma unroll
        for (int e = 0; e < kV; ++e) sum += x[k][e] * x[k][e];
      f = rsqrt_hw(team_sum<G>(sum, s_sum[turn]) * inv + a.eps);
    }
    float sum = 0.0f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = (k * G + at) * kV;
      if (c >= D) continue;
      float w[kV], s[kV];
      post.get(k, D, at, w);
      scale.get(k, D, at, s);
#pragma unroll
      for (int e = 0; e < kV; ++e) {
        y[k][e] += x[k][e] * f * w[e] * s[e];
        sum += c + e < D ? y[k][e] * y[k][e] : 0.0f;
      }
      if (a.res_out) store(a.res_out, i + c, ty.other, D - c, y[k]);
    }
    if (!a.out) continue;
    f = rsqrt_hw(team_sum<G>(sum, s_sum[turn + 1]) * inv + a.eps);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = (k * G + at) * kV;
      if (c >= D) continue;
      float w[kV];
      weight.get(k, D, at, w);
#pragma unroll
      for (int e = 0; e < kV; ++e) y[k][e] *= f * w[e];
      store(a.out, i + c, ty.out, D - c, y[k]);
    }
  }
}

// Runs launch.template go<K, G>() for rows of d values.
template <typename F>
int for_rows(int d, const F& f) {
  const int p = (d + kV - 1) / kV;
  if (p <= 1) return f.template go<1, 1>();
  if (p <= 2) return f.template go<1, 2>();
  if (p <= 4) return f.template go<1, 4>();
  if (p <= 8) return f.template go<1, 8>();
  if (p <= 16) return f.template go<1, 16>();
  if (p <= 32) return f.template go<1, 32>();
  if (p <= 64) return f.template go<1, 64>();
  if (p <= 256) return f.template go<1, 256>();
  if (p <= 512) return f.template go<2, 256>();
  if (p <= 1024) return f.template go<4, 256>();
  return f.template go<8, 256>();
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
  template <int K, int G>
  int go() const {
    gate_norm_kernel<K, G><<<blocks_for<G>(unsigned(a.N) * unsigned(a.H)), kThreads, 0, stream>>>(a, ty);
    return after_launch("gate_norm");
  }
};

struct AddLaunch {
  const AddNormArgs& a;
  Types ty;
  hipStream_t stream;
  template <int K, int G>
  int go() const {
    add_norm_kernel<K, G><<<blocks_for<G>(unsigned(a.N)), kThreads, 0, stream>>>(a, ty);
    return after_launch("add_norm");
  }
};

}  // namespace

int launch_gate_norm(const GateNormArgs& a, int x_dtype, int gate_dtype, int out_dtype, hipStream_t stream) {
  return for_rows(a.d, GateLaunch{a, {x_dtype, gate_dtype, out_dtype}, stream});
}

int launch_add_norm(const AddNormArgs& a, int x_dtype, int res_dtype, int out_dtype, hipStream_t stream) {
  return for_rows(a.D, AddLaunch{a, {x_dtype, res_dtype, out_dtype}, stream});
}

}  // namespace gdn
