// gdn_attend.hip -- softmax attention of a step's slots over the paged cache.
#include "gdn_attn.h"

namespace gdn {
namespace {

// One wave per (slot, query head, sequence): 64 keys at a time, a key per
// lane in the scores, channels over the lanes in the sums.
template <typename T>
__global__ __launch_bounds__(kWave) void attend_kernel(AttnArgs a) {
  constexpr int X = Pack<T>::kN;
  constexpr int kMaxD = 256;
  __shared__ float s_q[kMaxD], s_p[kWave];
  const int i = blockIdx.x, hq = blockIdx.y, b = blockIdx.z, lane = threadIdx.x;
  const int d = a.c.d, h = hq / (a.Hq / a.c.Hkv);
  const int ctx = a.ctx_len[b], span = span_of(a, b);
  const MetaPtrs m = meta_ptrs(a.meta, a.B, a.T);
  const size_t bt = size_t(b) * a.T;
  const bool real = !(a.meta && m.status[b] != 0) && len_status(a, ctx, span) == 0 &&
                    (a.meta ? m.depth[bt + i] >= 0 : i < span);
  T* out = reinterpret_cast<T*>(a.out) + ((bt + i) * a.Hq + hq) * d;
  float o[kMaxD / kWave] = {};
  float mx = -INFINITY, sum = 0.0f;
  if (real) {
    const T* q = reinterpret_cast<const T*>(a.q) + ((bt + i) * a.Hq + hq) * d;
    for (int e = lane; e < d; e += kWave) s_q[e] = to_f32(q[e]) * a.scale;
    __syncthreads();
    const int32_t* row = a.page_table + size_t(b) * a.c.max_pages;
    const int mask = (1 << a.c.page_shift) - 1;
    const T *kc = reinterpret_cast<const T*>(a.k_cache), *vc = reinterpret_cast<const T*>(a.v_cache);
    for (int p0 = 0; p0 < ctx + span; p0 += kWave) {
      const int p = p0 + lane, j = p - ctx;
      bool seen = p < ctx + span;
      if (seen && j >= 0)
        seen = j == i || (a.meta ? ((m.anc[(bt + i) * m.W + (j >> 6)] >> (j & 63)) & 1) != 0 : j < i);
      const int pg = seen ? page_of(a.c, row, p) : -1;
      float z = -INFINITY;
      if (pg >= 0) {
        const T* k = kc + block_of(a.c, pg, h) + size_t(p & mask) * X;
        z = 0.0f;
        for (int c = 0; c < d / X; ++c)
          for (int e = 0; e < X; ++e) z += s_q[c * X + e] * to_f32(k[(size_t(c) << a.c.page_shift) * X + e]);
      }
      float top = z;
      for (int s = 1; s < kWave; s <<= 1) top = fmaxf(top, __shfl_xor(top, s));
      const float next = fmaxf(mx, top);
      if (next == -INFINITY) continue;  // the same in every lane
      const float fix = __expf(mx - next), w = pg >= 0 ? __expf(z - next) : 0.0f;
      mx = next;
      sum = sum * fix + wave_sum(w);
      s_p[lane] = w;
      for (int r = 0; r < kMaxD / kWave; ++r) o[r] *= fix;
      __syncthreads();
      for (int t = 0; t < kWave; ++t) {
        const int pt = __shfl(pg, t);
        if (pt < 0) continue;
        const int off = (p0 + t) & mask;
        const T* v = vc + block_of(a.c, pt, h) + size_t(off / X) * d * X + off % X;
        for (int r = 0; r < kMaxD / kWave; ++r)
          if (r * kWave + lane < d) o[r] += s_p[t] * to_f32(v[(r * kWave + lane) * X]);
      }
      __syncthreads();
    }
  }
  for (int r = 0; r < kMaxD / kWave; ++r)
    if (r * kWave + lane < d) st(out + r * kWave + lane, sum > 0.0f || sum != sum ? o[r] / sum : 0.0f);
}

}  // namespace

int launch_attend(const AttnArgs& a, hipStream_t stream) {
  const dim3 grid(a.T, a.Hq, a.B);
  if (a.dtype == GDN_BF16)
    attend_kernel<BF16><<<grid, kWave, 0, stream>>>(a);
  else
    attend_kernel<float><<<grid, kWave, 0, stream>>>(a);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? GDN_OK : set_error(GDN_EHIP, "attend: launch: %s", hipGetErrorString(e));
}

}  // namespace gdn
