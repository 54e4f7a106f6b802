// gdn_chain.hip -- the gated delta rule token by token, for sequences of few
// tokens (single-token decoding).
#include <algorithm>

#include "gdn_layer.h"

namespace gdn {
namespace {

constexpr int kThreads = 256;
constexpr int kOwn = 2;  // channels that a thread convolves

// One token of a row of the state in the stored orientation,
//   S <- alpha S + beta (v - alpha S.k) k^T,  o = scale S.q,
// with the rows in registers: kLanes lanes a row, RP rows a lane.  One
// workgroup per (slice of rows, value head, sequence); every workgroup
// convolves the key head's channels and its own value channels, and keeps the
// last three raw inputs of each in registers.
//
// Bound by the state, read and written once a call: one token of 32 sequences of
// 16 / 48 heads of 128, 210 MB, in 33 us called again and again (part of it stays
// in the caches), 45 us in turn with other work; a copy of as much takes 41.  A
// token of one sequence takes 5 us, the latency of a launch, of the loads, which go
// out together, and of the stores; each further one 0.9 us, for a barrier and the
// sums over a row's lanes.
template <typename TIn, typename TOut, int DK, int RP>
__global__ __launch_bounds__(kThreads) void chain_step_kernel(ChainArgs a) {
  constexpr int kLanes = DK >= 32 ? 8 : 4, kCols = DK / kLanes, kRows = kThreads / kLanes * RP;
  __shared__ __align__(16) float s_f[2][2 * DK + kRows];
  const int tid = threadIdx.x, slice = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
  const int per = a.Hv / a.Hk, hk = h / per, row0 = slice * kRows, rows = min(kRows, a.dv - row0);
  const int C = 2 * a.Hk * DK + a.Hv * a.dv;
  const Tokens tk = tokens_of(a, b);
  if (a.status && slice == 0 && h == 0 && tid == 0) a.status[b] = tk.status;

  // this thread's channels: queries, keys, values of the slice
  const TIn* src[kOwn];
  size_t stride[kOwn];
  float4 w[kOwn];
  float x0[kOwn], x1[kOwn], x2[kOwn], raw[kOwn];
  int chan[kOwn];
#pragma unroll
  for (int i = 0; i < kOwn; ++i) {
    const int c = tid + i * kThreads;
    chan[i] = -1;
    if (c < 2 * DK) {
      const bool key = c >= DK;
      chan[i] = (key ? a.Hk + hk : hk) * DK + (key ? c - DK : c);
      src[i] = reinterpret_cast<const TIn*>(key ? a.k : a.q) + hk * DK + (key ? c - DK : c);
      stride[i] = size_t(a.Hk) * DK;
    } else if (c < 2 * DK + rows) {
      const int r = h * a.dv + row0 + c - 2 * DK;
      chan[i] = 2 * a.Hk * DK + r;
      src[i] = reinterpret_cast<const TIn*>(a.v) + r;
      stride[i] = size_t(a.Hv) * a.dv;
    }
    x0[i] = x1[i] = x2[i] = raw[i] = 0.0f;
    if (chan[i] < 0) continue;
    const float* cs = a.conv_state + size_t(b) * 3 * C + chan[i];
    x0[i] = cs[0];
    x1[i] = cs[C];
    x2[i] = cs[2 * size_t(C)];
    w[i] = *reinterpret_cast<const float4*>(a.conv_w + size_t(chan[i]) * 4);
    src[i] += size_t(tk.first) * stride[i];
    if (tk.n > 0) raw[i] = to_f32(*src[i]);
  }

  const int lane = tid % kLanes, r0 = tid / kLanes * RP;  // of the slice
  float* S = a.S + ((size_t(b) * a.Hv + h) * a.dv + row0 + r0) * DK + 4 * lane;
  float st[RP][kCols];
  if (tk.n > 0) {
#pragma unroll
    for (int p = 0; p < RP; ++p)
#pragma unroll
      for (int e = 0; e < kCols; e += 4) {
        const float4 y = r0 + p < rows ? *reinterpret_cast<const float4*>(S + p * DK + e * kLanes) : make_float4(0, 0, 0, 0);
        st[p][e] = y.x, st[p][e + 1] = y.y, st[p][e + 2] = y.z, st[p][e + 3] = y.w;
      }
  }
  const TIn *al = reinterpret_cast<const TIn*>(a.alpha) + size_t(tk.first) * a.Hv + h,
            *be = reinterpret_cast<const TIn*>(a.beta) + size_t(tk.first) * a.Hv + h;
  float alpha = 0.0f, beta = 0.0f;
  if (tk.n > 0) alpha = to_f32(*al), beta = to_f32(*be);
  TOut* out = reinterpret_cast<TOut*>(a.out) + (size_t(tk.first) * a.Hv + h) * a.dv + row0 + r0;
  for (int t = 0; t < tk.n; ++t) {
    float* f = s_f[t & 1];
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      if (chan[i] < 0) continue;
      const float x = raw[i];
      f[tid + i * kThreads] = silu(w[i].x * x0[i] + w[i].y * x1[i] + w[i].z * x2[i] + w[i].w * x);
      x0[i] = x1[i], x1[i] = x2[i], x2[i] = x;
      if (t + 1 < tk.n) raw[i] = to_f32(*(src[i] += stride[i]));
    }
    const float al1 = alpha, be1 = beta;
    if (t + 1 < tk.n) alpha = to_f32(*(al += a.Hv)), beta = to_f32(*(be += a.Hv));
    __syncthreads();  // the other buffer's readers are a token ahead of its writers
    float q[kCols], k[kCols], qq = 0.0f, kk = 0.0f;
#pragma unroll
    for (int e = 0; e < kCols; e += 4) {
      const float4 y = *reinterpret_cast<const float4*>(f + 4 * lane + e * kLanes);
      const float4 z = *reinterpret_cast<const float4*>(f + DK + 4 * lane + e * kLanes);
      q[e] = y.x, q[e + 1] = y.y, q[e + 2] = y.z, q[e + 3] = y.w;
      k[e] = z.x, k[e + 1] = z.y, k[e + 2] = z.z, k[e + 3] = z.w;
    }
#pragma unroll
    for (int e = 0; e < kCols; ++e) qq += q[e] * q[e], kk += k[e] * k[e];
    const float iq = rsqrt_hw(group_sum<kLanes>(qq) + 1e-6f), ik = rsqrt_hw(group_sum<kLanes>(kk) + 1e-6f);
#pragma unroll
    for (int e = 0; e < kCols; ++e) k[e] *= ik;
#pragma unroll
    for (int p = 0; p < RP; ++p) {
      float u = 0.0f, o = 0.0f;
#pragma unroll
      for (int e = 0; e < kCols; ++e) u += st[p][e] * k[e];
      u = group_sum<kLanes>(u);
      const float v = r0 + p < rows ? f[2 * DK + r0 + p] : 0.0f, d = be1 * (v - al1 * u);
#pragma unroll
      for (int e = 0; e < kCols; ++e) {
        st[p][e] = al1 * st[p][e] + d * k[e];
        o += st[p][e] * q[e];
      }
      o = group_sum<kLanes>(o);
      if (lane == 0 && r0 + p < rows) put(out + p, a.scale * iq * o);
    }
    out += size_t(a.Hv) * a.dv;
  }

#pragma unroll
  for (int i = 0; i < kOwn; ++i) {
    // queries and keys: one workgroup of a key head
    if (chan[i] < 0 || (tid + i * kThreads < 2 * DK && (slice != 0 || h % per != 0))) continue;
    float* cs = a.conv_state_out + size_t(b) * 3 * C + chan[i];
    cs[0] = x0[i];
    cs[C] = x1[i];
    cs[2 * size_t(C)] = x2[i];
  }
  if (tk.n == 0) return;
#pragma unroll
  for (int p = 0; p < RP; ++p)
#pragma unroll
    for (int e = 0; e < kCols; e += 4)
      if (r0 + p < rows)
        *reinterpret_cast<float4*>(S + p * DK + e * kLanes) = make_float4(st[p][e], st[p][e + 1], st[p][e + 2], st[p][e + 3]);
}

template <typename TIn, typename TOut, int DK, int RP>
int launch_rows(const ChainArgs& a, hipStream_t stream) {
  constexpr int kRows = kThreads / (DK >= 32 ? 8 : 4) * RP;
  chain_step_kernel<TIn, TOut, DK, RP><<<dim3((a.dv + kRows - 1) / kRows, a.Hv, a.B), kThreads, 0, stream>>>(a);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? GDN_OK : set_error(GDN_EHIP, "chain: launch: %s", hipGetErrorString(e));
}

template <typename TIn, typename TOut, int DK>
int launch_dk(const ChainArgs& a, hipStream_t stream) {
  if ((long long)(a.B) * a.Hv >= 512 && a.dv > 64) return launch_rows<TIn, TOut, DK, 4>(a, stream);
  return launch_rows<TIn, TOut, DK, 1>(a, stream);
}

template <typename TIn, typename TOut>
int launch_types(const ChainArgs& a, hipStream_t stream) {
  switch (a.dk) {
    case 16: return launch_dk<TIn, TOut, 16>(a, stream);
    case 32: return launch_dk<TIn, TOut, 32>(a, stream);
    case 64: return launch_dk<TIn, TOut, 64>(a, stream);
    default: return launch_dk<TIn, TOut, 128>(a, stream);
  }
}

}  // namespace

int launch_chain_steps(const ChainArgs& a, hipStream_t stream) {
  const bool out32 = a.out_dtype == GDN_F32;
  if (a.in_dtype == GDN_BF16)
    return out32 ? launch_types<BF16, float>(a, stream) : launch_types<BF16, BF16>(a, stream);
  return out32 ? launch_types<float, float>(a, stream) : launch_types<float, BF16>(a, stream);
}

}  // namespace gdn
