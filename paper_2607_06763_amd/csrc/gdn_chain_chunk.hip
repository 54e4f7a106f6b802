// gdn_chain_chunk.hip -- the gated delta rule in chunks of 64 tokens, for
// sequences of any length.
//
// Inside a chunk, with g_i the sum of log(alpha) up to token i and S0 the state
// before it,
//   (I + A) V' = diag(beta) (V - diag(e^g) K S0^T),  A_ij = beta_i k_i.k_j e^(g_i - g_j), j < i
//   O = scale (diag(e^g) Q S0^T + Y V'),             Y_ij = q_i.k_j e^(g_i - g_j), j <= i
//   S = e^g_last S0 + V'^T diag(e^(g_last - g)) K.
// Keys, queries, (I + A)^-1 and Y do not depend on the state and are computed
// for many chunks at once (chunk_kernel); the rest goes chunk by chunk
// (scan_kernel), with the state in registers: a wave holds 16 value channels,
// the columns of its matrix tiles, and needs nothing from the other waves.
//
// What passes between the two bounds both: 170 KB a chunk and key head with
// three value heads of 128.  With (I + A)^-1 diag(beta) applied to V and K
// beforehand, as first built, it was 295 KB, and chunk_kernel, which then
// convolves the values too, took three times as long.
//
// Products.  Each operand is a pair of fp16 values, hi + lo, 22 bits together, and
// a product is three on the matrix units (hi hi, hi lo, lo hi) with 32-bit sums:
// lo lo, 2^-22 of a product, is left out, and the outputs come out as near as
// those of fp32 products.  Scales are powers of two, exact: 2^15 for what is at
// most 1 (unit keys, queries), else they take the largest value of the matrix or of
// the operand's column to 2^14 .. 2^15.  A pair has its 22 bits down to 2^-16 of
// that value; what is smaller is off by up to 2^-39 of it (lo's last step is 2^-24).
// So a value that is forgotten inside its chunk, 10^6 times what follows it, costs
// that 1e-6 of its accuracy where fp32 loses nothing.
//
// Operand order.  A tile's accumulators hold rows 4 q + r (q = lane / 16) of
// column lane % 16, and an operand 8 values of one row or column.  Two tiles of
// 16 rows are taken as the 32 products of a step in the order
// 16 (j / 4) + 4 q + j % 4 (slot 8 q + j), so that accumulators become
// operands without leaving their lane; what multiplies them is stored in that
// order.  (I + A) is inverted in blocks of 16, each by substitution.
#include <algorithm>

#include "gdn_layer.h"
#include "gdn_workspace.h"

namespace gdn {
namespace {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

constexpr int kC = 64;          // tokens of a chunk
constexpr int kPrepThreads = 512;
constexpr int kPrepWaves = kPrepThreads / kWave;
constexpr int kHeads = 3;       // value heads that are inverted at once
constexpr int kLd = kC + 4;     // floats of a row of a chunk's matrix in LDS
constexpr float kUnit = 32768.0f;  // scale of what is at most 1
constexpr int kFrag = 1024;     // bytes of an operand tile: 64 lanes of 8 fp16 values

// ---------------------------------------------------------------------------
// Workspace of a slot (a chunk of a sequence).  Operand tiles of a pair: hi,
// then lo.
// ---------------------------------------------------------------------------
__host__ __device__ constexpr int padded_dk(int dk) { return dk < 32 ? 32 : dk; }

struct SlotLayout {
  int ks;        // steps of 32 key channels
  size_t key;    // bytes of a key head: K and Q [ks][4 token tiles], K^T [2 ks][2 token steps]
  size_t total;
  __host__ __device__ size_t q_bytes() const { return size_t(ks) * 8 * kFrag; }
};
constexpr size_t kYAt = 12 * kFrag, kScalarsAt = 24 * kFrag;  // of a value head: (I + A)^-1 [6], Y [6], scalars
constexpr size_t kValue = 25 * kFrag;

__host__ __device__ inline SlotLayout slot_layout(int Hk, int Hv, int dk) {
  SlotLayout l;
  l.ks = padded_dk(dk) / 32;
  l.key = 3 * l.q_bytes();
  l.total = Hk * l.key + Hv * kValue;
  return l;
}

// What a launch takes: chunks c0 .. c0 + M - 1 of sequences b0 .. b0 + G - 1.
struct Part {
  int b0, G, c0, M;
  char* ws;
};

__device__ __forceinline__ char* slot_at(const ChainArgs& a, const Part& p, int g, int m) {
  return p.ws + (size_t(g) * p.M + m) * slot_layout(a.Hk, a.Hv, a.dk).total;
}
__device__ __forceinline__ char* key_at(const ChainArgs& a, char* slot, int hk) {
  return slot + hk * slot_layout(a.Hk, a.Hv, a.dk).key;
}
__device__ __forceinline__ char* value_at(const ChainArgs& a, char* slot, int h) {
  return slot + a.Hk * slot_layout(a.Hk, a.Hv, a.dk).key + h * kValue;
}

// Step s of token tile t of a lower triangular operand (6 of them: a step holds
// the columns of two tiles).
__device__ __forceinline__ constexpr int lower_step(int t, int s) { return t < 2 ? t : 2 + (t - 2) * 2 + s; }
__device__ __forceinline__ constexpr int lower_tile(int u) { return u < 2 ? u : 2 + (u - 2) / 2; }
__device__ __forceinline__ constexpr int lower_col(int u) { return u < 2 ? 0 : (u - 2) % 2; }

// ---------------------------------------------------------------------------
// fp16 pairs
// ---------------------------------------------------------------------------
struct Pair {
  f16x8 hi, lo;
};

// hi of two values times a scale; lo
__device__ __forceinline__ unsigned split2(float x, float y, float scale, unsigned& lo) {
  f16x2 h = {(_Float16)(x * scale), (_Float16)(y * scale)};
  // a value of its own: were it computed again for the difference, with another
  // rounding of the product, hi + lo would miss x by a step of hi
  asm("" : "+v"(h));
  const f16x2 l = {(_Float16)__builtin_fmaf(x, scale, -(float)h[0]), (_Float16)__builtin_fmaf(y, scale, -(float)h[1])};
  lo = __builtin_bit_cast(unsigned, l);
  return __builtin_bit_cast(unsigned, h);
}
__device__ __forceinline__ Pair split(const float (&x)[8], float scale) {
  u32x4 hi, lo;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    unsigned l;
    hi[e] = split2(x[2 * e], x[2 * e + 1], scale, l);
    lo[e] = l;
  }
  return {__builtin_bit_cast(f16x8, hi), __builtin_bit_cast(f16x8, lo)};
}

__device__ __forceinline__ f32x4 mma(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

__device__ __forceinline__ f32x4 mma3(const Pair& a, const Pair& b, f32x4 c) {
  c = mma(a.lo, b.hi, c);
  c = mma(a.hi, b.lo, c);
  return mma(a.hi, b.hi, c);
}

// Power of two that takes m to 2^14 .. 2^15, and its inverse (both normal
// floats: m is clamped to 2^-112 .. 2^126).
__device__ __forceinline__ void f16_scale(float m, float& scale, float& inv) {
  int ex = int((__float_as_uint(m) >> 23) & 0xffu);
  ex = ex < 15 ? 15 : ex > 253 ? 253 : ex;
  scale = __uint_as_float(unsigned(268 - ex) << 23);
  inv = __uint_as_float(unsigned(ex - 14) << 23);
}

// Of values >= 0 (their bits compare as they do, which spares the instructions that
// quiet a NaN), over the four lanes of a column (lane % 16): rows of 16 lanes trade
// places.
__device__ __forceinline__ float column_max(float x) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  const unsigned y = max(r[0], r[1]);
  r = __builtin_amdgcn_permlane32_swap(y, y, false, false);
  return __uint_as_float(max(r[0], r[1]));
}
__device__ __forceinline__ Pair load_pair(const char* p, int tile, int lane) {
  const char* q = p + size_t(tile) * 2 * kFrag + lane * 16;
  return {*reinterpret_cast<const f16x8*>(q), *reinterpret_cast<const f16x8*>(q + kFrag)};
}
__device__ __forceinline__ void store_pair(char* p, int tile, int lane, const Pair& x) {
  char* q = p + size_t(tile) * 2 * kFrag + lane * 16;
  *reinterpret_cast<f16x8*>(q) = x.hi;
  *reinterpret_cast<f16x8*>(q + kFrag) = x.lo;
}

template <int DKP>
struct Prep {
  static constexpr int kPacks = DKP / 8, kKs = DKP / 32;
  static constexpr int kPlane = kPacks * (kC + 1) * 16;       // bytes of hi or lo of K or Q: [pack][token]
  static constexpr int kMat = kC * kLd * int(sizeof(float));  // a chunk's matrix
  static constexpr int kRows = 4 * kPlane > kHeads * kMat ? 4 * kPlane : kHeads * kMat;
  static constexpr int kLds = kRows + kHeads * (kC * 12 + 8);
};

// ---------------------------------------------------------------------------
// What does not depend on the state.  One workgroup per (key head, chunk) with
// all of its value heads: keys and queries are convolved once.  Loads have no
// branch around them (rows are clamped and values selected): a branch each made
// them wait for one another.
//
// Bound by its own chain of steps, convolution, products, inversion, stores, each
// behind a barrier: 14 us for a single chunk.  1365 workgroups, a third of 4
// sequences of 4096 tokens of 16 / 48 heads of 128, take 73 us and write 233 MB,
// 3.2 TB/s; a workgroup has 69 KB of LDS, two are on a CU, and half of the wave
// cycles are spent waiting.
// ---------------------------------------------------------------------------
template <typename TIn, int DKP>
__global__ __launch_bounds__(kPrepThreads, 4) void chunk_kernel(ChainArgs a, Part part) {
  typedef Prep<DKP> P;
  constexpr int kKs = P::kKs, kPacks = P::kPacks;
  extern __shared__ __align__(16) char s_raw[];
  char* s_kq = s_raw;                            // K hi, K lo, Q hi, Q lo; then the heads' matrices
  float* s_t = reinterpret_cast<float*>(s_raw);  // [head][64][kLd]
  double* s_log = reinterpret_cast<double*>(s_raw + P::kRows);  // [head][64]
  float* s_beta = reinterpret_cast<float*>(s_log + kHeads * kC);
  float *s_scale = s_beta + kHeads * kC, *s_yscale = s_scale + kHeads;  // of (I + A)^-1, of Y
  const int tid = threadIdx.x, lane = tid % kWave, w = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int n16 = lane & 15, q4 = lane >> 4;
  const int hk = blockIdx.x, m = blockIdx.y, b = part.b0 + blockIdx.z;
  const Tokens tk = tokens_of<false>(a, b);  // only its own slot is written
  const int n0 = (part.c0 + m) * kC, nt = min(kC, tk.n - n0);
  if (nt <= 0) return;
  const int dk = a.dk, dv = a.dv, per = a.Hv / a.Hk, C = 2 * a.Hk * dk + a.Hv * dv;
  const SlotLayout layout = slot_layout(a.Hk, a.Hv, dk);
  char* slot = slot_at(a, part, blockIdx.z, m);
  const float* cs = a.conv_state + size_t(b) * 3 * C;
  const size_t row0 = size_t(tk.first) + n0;  // of the chunk's first token

  // decays and strengths of a head, a token a lane
  float al = 1.0f, be = 0.0f;
  auto fetch_gates = [&](int r0, int nr) {
    const size_t at = (row0 + min(lane, nt - 1)) * a.Hv + hk * per + r0 + min(w, nr - 1);
    al = to_f32(reinterpret_cast<const TIn*>(a.alpha)[at]);
    be = to_f32(reinterpret_cast<const TIn*>(a.beta)[at]);
    if (lane >= nt) al = 1.0f, be = 0.0f;
  };
  fetch_gates(0, min(kHeads, per));

  // keys and queries: 4 channels a thread, kLpt threads a token
  {
    constexpr int kLpt = DKP / 4, kTok = kC * kLpt / kPrepThreads;
    static_assert(kTok >= 1, "every thread has a token");
    const int p = tid % kLpt, t0 = tid / kLpt * kTok, c4 = min(p * 4, dk - 4);
    const bool in = p * 4 < dk;
    float4 win[2][kTok + 3], cw[2][4];  // all loads before the first is waited for
#pragma unroll
    for (int isq = 0; isq < 2; ++isq) {
      const TIn* x = reinterpret_cast<const TIn*>(isq ? a.q : a.k) + hk * dk + c4;
#pragma unroll
      for (int i = 0; i < kTok + 3; ++i) {
        const int t = min(max(t0 - 3 + i, n0 ? -3 : 0), nt - 1);
        win[isq][i] = ld4(x + (long long)(row0 + t) * a.Hk * dk);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)
        cw[isq][e] = *reinterpret_cast<const float4*>(a.conv_w + size_t((isq ? hk : a.Hk + hk) * dk + c4 + e) * 4);
    }
    if (n0 == 0 && t0 < 3) {  // before the sequence's first token
#pragma unroll
      for (int isq = 0; isq < 2; ++isq)
#pragma unroll
        for (int i = 0; i < 3; ++i)
          if (t0 + i < 3) win[isq][i] = ld4(cs + size_t(t0 + i) * C + (isq ? hk : a.Hk + hk) * dk + c4);
    }
#pragma unroll
    for (int isq = 0; isq < 2; ++isq) {
#pragma unroll
      for (int i = 0; i < kTok; ++i) {
        const float4 *x = &win[isq][i], *f = cw[isq];
        float y[4] = {silu(f[0].x * x[0].x + f[0].y * x[1].x + f[0].z * x[2].x + f[0].w * x[3].x),
                      silu(f[1].x * x[0].y + f[1].y * x[1].y + f[1].z * x[2].y + f[1].w * x[3].y),
                      silu(f[2].x * x[0].z + f[2].y * x[1].z + f[2].z * x[2].z + f[2].w * x[3].z),
                      silu(f[3].x * x[0].w + f[3].y * x[1].w + f[3].z * x[2].w + f[3].w * x[3].w)};
        float sum = 0.0f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (!in || t0 + i >= nt) y[e] = 0.0f;
          sum += y[e] * y[e];
        }
        const float scale = rsqrt_hw(group_sum<kLpt>(sum) + 1e-6f) * kUnit;
        unsigned lo0, lo1;
        const unsigned hi0 = split2(y[0], y[1], scale, lo0), hi1 = split2(y[2], y[3], scale, lo1);
        char* d = s_kq + isq * 2 * P::kPlane + (p / 2 * (kC + 1) + t0 + i) * 16 + p % 2 * 8;
        *reinterpret_cast<uint2*>(d) = make_uint2(hi0, hi1);
        *reinterpret_cast<uint2*>(d + P::kPlane) = make_uint2(lo0, lo1);
      }
    }
  }
  __syncthreads();

  auto rows_of = [&](int isq, int t, int s) {  // operand rows: 16 tokens, 32 channels in order
    const char* d = s_kq + isq * 2 * P::kPlane + ((4 * s + q4) * (kC + 1) + 16 * t + n16) * 16;
    return Pair{*reinterpret_cast<const f16x8*>(d), *reinterpret_cast<const f16x8*>(d + P::kPlane)};
  };
  // k_j.k_i and k_j.q_i, rows j, columns i, in the units of a lower triangular
  // operand, one a wave (what is above the diagonal stays 0)
  const int unit = min(w, 5), tile = lower_tile(unit), step = lower_col(unit);
  f32x4 kk[2] = {}, kq[2] = {};
  if (w < 6) {
#pragma unroll
    for (int s = 0; s < kKs; ++s) {
      const Pair k = rows_of(0, tile, s), q = rows_of(1, tile, s);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        if (2 * step + e > tile) continue;
        const Pair x = rows_of(0, 2 * step + e, s);
        kk[e] = mma3(x, k, kk[e]);
        kq[e] = mma3(x, q, kq[e]);
      }
    }
  }
  // K and Q: rows are tokens, 32 channels; K^T: rows are channels, 32 tokens; in
  // the order of accumulators
  char* kws = key_at(a, slot, hk);
#pragma unroll
  for (int n = 0; n < kKs * 8 / kPrepWaves; ++n) {
    const int u = n * kPrepWaves + w, isq = u / (kKs * 4), s = u / 4 % kKs, t = u % 4;
    Pair x;
#pragma unroll
    for (int hl = 0; hl < 2; ++hl) {
      f16x4 y[2];
#pragma unroll
      for (int e = 0; e < 2; ++e)
        y[e] = *reinterpret_cast<const f16x4*>(s_kq + (2 * isq + hl) * P::kPlane +
                                               ((4 * s + 2 * e + q4 / 2) * (kC + 1) + 16 * t + n16) * 16 + q4 % 2 * 8);
      const f16x8 z = {y[0][0], y[0][1], y[0][2], y[0][3], y[1][0], y[1][1], y[1][2], y[1][3]};
      if (hl) x.lo = z;
      else x.hi = z;
    }
    store_pair(kws, u, lane, x);
  }
#pragma unroll
  for (int n = 0; n < (kKs * 4 + kPrepWaves - 1) / kPrepWaves; ++n) {
    const int u = n * kPrepWaves + w, c = u / 2 * 16 + n16, s = u % 2;
    if (u >= kKs * 4) continue;
    Pair x;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int t = 32 * s + 16 * (j / 4) + 4 * q4 + j % 4;
      const char* d = s_kq + (c / 8 * (kC + 1) + t) * 16 + c % 8 * 2;
      x.hi[j] = *reinterpret_cast<const _Float16*>(d);
      x.lo[j] = *reinterpret_cast<const _Float16*>(d + P::kPlane);
    }
    store_pair(kws + 2 * layout.q_bytes(), u, lane, x);
  }
  __syncthreads();  // K and Q are read

  for (int r0 = 0; r0 < per; r0 += kHeads) {
    const int nr = min(kHeads, per - r0);
    if (r0) fetch_gates(r0, nr);
    if (w < nr) {
      // 64-bit sums: far into a chunk of strong decays the difference of two of
      // them is small
      double g = double(logf(al < 0x1p-126f ? 0x1p-126f : al));
#pragma unroll
      for (int d = 1; d < kWave; d *= 2) {
        const double x = __shfl_up(g, d);
        if (lane >= d) g += x;
      }
      s_log[w * kC + lane] = g;
      s_beta[w * kC + lane] = be;
      // a token a lane; its decay from the chunk's start, to the chunk's end
      float* sc = reinterpret_cast<float*>(value_at(a, slot, hk * per + r0 + w) + kScalarsAt);
      const float f = __expf(float(g));
      sc[lane] = be;
      sc[kC + lane] = f;
      sc[2 * kC + lane] = __expf(float(__shfl(g, kC - 1) - g));
      float grown = 1.0f, ys, yi;  // the most that a "decay" above 1 makes of a value
      if (__any(al > 1.0f)) grown = __expf(group_sum<kWave>(al > 1.0f ? __logf(al) : 0.0f));
      f16_scale(grown, ys, yi);
      if (lane == kC - 1) {
        sc[3 * kC] = f;
        sc[3 * kC + 2] = yi;
        s_yscale[w] = ys * (1.0f / (kUnit * kUnit));
      }
    }
    __syncthreads();
    // A, to be inverted, and Y
    if (w < 6) {
      for (int r = 0; r < nr; ++r) {
        const int n16 = opaque(lane & 15), q4 = opaque(lane >> 4);  // addresses are computed here, not held
        const int i = 16 * tile + n16, j0 = 32 * step + 4 * q4;
        const double *lg = s_log + r * kC, li = lg[i];
        const float bi = s_beta[r * kC + i] * (1.0f / (kUnit * kUnit));
        float y[8];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          f32x4 x;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int j = j0 + 16 * e + k;
            const float f = j <= i ? __expf(float(li - lg[j])) : 0.0f;
            x[k] = j < i ? bi * kk[e][k] * f : 0.0f;
            y[4 * e + k] = kq[e][k] * f;
          }
          *reinterpret_cast<f32x4*>(s_t + (r * kC + i) * kLd + j0 + 16 * e) = x;
        }
        store_pair(value_at(a, slot, hk * per + r0 + r) + kYAt, unit, lane, split(y, s_yscale[r]));
      }
    }
    __syncthreads();
    // (I + A)^-1 of a head by one wave
    if (w < nr) {
      // blocks of the diagonal: a block per 16 lanes, a column a lane
      float* x = s_t + w * kC * kLd;
      const int n16 = opaque(lane & 15), q4 = opaque(lane >> 4);  // as above
      {
        float *d = x + 16 * q4 * kLd + 16 * q4, t[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          float y = i == n16 ? 1.0f : 0.0f;
#pragma unroll
          for (int j = 0; j < i; j += 4) {
            const float4 l = *reinterpret_cast<const float4*>(d + i * kLd + j);
            y -= l.x * t[j];
            if (j + 1 < i) y -= l.y * t[j + 1];
            if (j + 2 < i) y -= l.z * t[j + 2];
            if (j + 3 < i) y -= l.w * t[j + 3];
          }
          t[i] = y;
        }
        wave_lds_order();  // rows are read before they are replaced
#pragma unroll
        for (int i = 0; i < 16; ++i) d[i * kLd + n16] = t[i];
      }
      wave_lds_order();
      // blocks below: X_j = T_jj, X_i = -T_ii sum_k A_ik X_k down a column of blocks
      auto block = [&](int i, int k) { return *reinterpret_cast<const f32x4*>(x + (16 * i + n16) * kLd + 16 * k + 4 * q4); };
      auto diagonal = [&](int j) {
        f32x4 c;
#pragma unroll
        for (int r = 0; r < 4; ++r) c[r] = x[(16 * j + 4 * q4 + r) * kLd + 16 * j + n16];
        return c;
      };
      auto times = [&](f32x4 y, f32x4 z, f32x4 c) {
#pragma unroll
        for (int r = 0; r < 4; ++r) c = __builtin_amdgcn_mfma_f32_16x16x4f32(y[r], z[r], c, 0, 0, 0);
        return c;
      };
      const f32x4 zero = {}, a10 = block(1, 0), a20 = block(2, 0), a21 = block(2, 1), a30 = block(3, 0), a31 = block(3, 1),
                  a32 = block(3, 2), t1 = block(1, 1), t2 = block(2, 2), t3 = block(3, 3);
      const f32x4 x0 = diagonal(0), x1 = diagonal(1), x2 = diagonal(2);
      const f32x4 x10 = -times(t1, times(a10, x0, zero), zero), x21 = -times(t2, times(a21, x1, zero), zero),
                  x32 = -times(t3, times(a32, x2, zero), zero);
      const f32x4 x20 = -times(t2, times(a21, x10, times(a20, x0, zero)), zero),
                  x31 = -times(t3, times(a32, x21, times(a31, x1, zero)), zero);
      const f32x4 x30 = -times(t3, times(a32, x20, times(a31, x10, times(a30, x0, zero))), zero);
      wave_lds_order();
      auto put_block = [&](int i, int j, f32x4 c) {
#pragma unroll
        for (int r = 0; r < 4; ++r) x[(16 * i + 4 * q4 + r) * kLd + 16 * j + n16] = c[r];
      };
      put_block(1, 0, x10), put_block(2, 1, x21), put_block(3, 2, x32);
      put_block(2, 0, x20), put_block(3, 1, x31), put_block(3, 0, x30);
      float most = 1.0f, scale, inv;  // the diagonal
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        most = fmaxf(most, fmaxf(fmaxf(fabsf(x0[r]), fabsf(x1[r])), fmaxf(fabsf(x2[r]), fabsf(x[(48 + 4 * q4 + r) * kLd + 48 + n16]))));
        most = fmaxf(most, fmaxf(fmaxf(fabsf(x10[r]), fabsf(x21[r])), fabsf(x32[r])));
        most = fmaxf(most, fmaxf(fmaxf(fabsf(x20[r]), fabsf(x31[r])), fabsf(x30[r])));
      }
      most = column_max(group_max<16>(most));
      f16_scale(most, scale, inv);
      if (lane == 0) {
        s_scale[w] = scale;
        float* sc = reinterpret_cast<float*>(value_at(a, slot, hk * per + r0 + w) + kScalarsAt) + 3 * kC;
        sc[1] = inv;
      }
    }
    __syncthreads();

    if (w < 6) {
      for (int r = 0; r < nr; ++r) {
        const float* x = s_t + (r * kC + 16 * tile + n16) * kLd + 32 * step + 4 * q4;
        const float4 y = *reinterpret_cast<const float4*>(x), z = *reinterpret_cast<const float4*>(x + 16);
        const float f[8] = {y.x, y.y, y.z, y.w, z.x, z.y, z.z, z.w};
        store_pair(value_at(a, slot, hk * per + r0 + r), unit, lane, split(f, s_scale[r]));
      }
    }
    __syncthreads();  // the matrices are read
  }
}

// ---------------------------------------------------------------------------
// The chunks of a sequence in turn: parts of both forms of the scan.
// ---------------------------------------------------------------------------
// Two tiles of accumulators as an operand.
__device__ __forceinline__ Pair operand(const f32x4& x, const f32x4& y, float scale) {
  const float z[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
  return split(z, scale);
}

// Products of K or Q (rows: tokens, kKs steps of channels) with the state.
// Group n: token tiles 2 (n / kPer) and the next, kSteps steps from
// n % kPer kSteps on; two accumulators in turn.
template <int kKs>
struct Rows {
  static constexpr int kPer = kKs > 1 ? kKs / 2 : 1, kGroups = 2 * kPer, kSteps = kKs > 1 ? 2 : 1;
  typedef Pair Group[2 * kSteps];
  static __device__ __forceinline__ void read(Group& f, const char* from, int n, int lane) {
#pragma unroll
    for (int k = 0; k < 2 * kSteps; ++k) f[k] = load_pair(from, (n % kPer * kSteps + k / 2) * 4 + n / kPer * 2 + k % 2, lane);
  }
  static __device__ __forceinline__ void times(const Group& f, const Pair (&sp)[kKs], f32x4 (&c)[4], int n) {
    const int t = n / kPer * 2, s = n % kPer * kSteps;
#pragma unroll
    for (int k = 0; k < kSteps; ++k) {
      const Pair& y = sp[s + k];
      c[t] = mma(f[2 * k].lo, y.hi, c[t]);
      c[t + 1] = mma(f[2 * k + 1].lo, y.hi, c[t + 1]);
      c[t] = mma(f[2 * k].hi, y.lo, c[t]);
      c[t + 1] = mma(f[2 * k + 1].hi, y.lo, c[t + 1]);
      c[t] = mma(f[2 * k].hi, y.hi, c[t]);
      c[t + 1] = mma(f[2 * k + 1].hi, y.hi, c[t + 1]);
    }
  }
};

// Products of a lower triangular operand: n = 0: tiles 0, 1 and the first step
// of 2, 3; n = 1: their second.
__device__ __forceinline__ void read_lower(Pair (&f)[4], const char* from, int n, int lane) {
#pragma unroll
  for (int k = 0; k < 4 - 2 * n; ++k) f[k] = load_pair(from, n ? lower_step(2 + k, 1) : lower_step(k, 0), lane);
}
__device__ __forceinline__ void times_lower(const Pair (&f)[4], const Pair& y, f32x4 (&c)[4], int n) {
#pragma unroll
  for (int k = 0; k < 4 - 2 * n; ++k) c[2 * n + k] = mma(f[k].lo, y.hi, c[2 * n + k]);
#pragma unroll
  for (int k = 0; k < 4 - 2 * n; ++k) c[2 * n + k] = mma(f[k].hi, y.lo, c[2 * n + k]);
#pragma unroll
  for (int k = 0; k < 4 - 2 * n; ++k) c[2 * n + k] = mma(f[k].hi, y.hi, c[2 * n + k]);
}

// Products of K^T: group n: tiles 2 n and 2 n + 1 of 16 key channels.
__device__ __forceinline__ void read_kt(Pair (&f)[4], const char* from, int n, int lane) {
#pragma unroll
  for (int k = 0; k < 4; ++k) f[k] = load_pair(from, 4 * n + k, lane);
}
__device__ __forceinline__ void times_kt(const Pair (&f)[4], const Pair (&vd)[2], f32x4 (&c)[2]) {
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    c[0] = mma(f[s].lo, vd[s].hi, c[0]);
    c[1] = mma(f[2 + s].lo, vd[s].hi, c[1]);
    c[0] = mma(f[s].hi, vd[s].lo, c[0]);
    c[1] = mma(f[2 + s].hi, vd[s].lo, c[1]);
    c[0] = mma(f[s].hi, vd[s].hi, c[0]);
    c[1] = mma(f[2 + s].hi, vd[s].hi, c[1]);
  }
}

// What a chunk's scalars give: the decay over it, 1 / scale of (I + A)^-1 and of Y.
struct ChunkScalars {
  float last, inv, y;
};
__device__ __forceinline__ ChunkScalars scalars_of(const float* s_sc) {
  const float4 x = *reinterpret_cast<const float4*>(s_sc + 3 * kC);
  return {x.x, x.y, x.z};
}

// V' as operands, plain and decayed to the chunk's end, and the scale of the
// state behind the chunk.  V' and V' decayed have scales from their own largest
// values in the column: a bound from the largest value in the chunk would keep
// one that the decays have forgotten by its end, and what is left would lose its
// bits to it, without limit.  The state's comes from a bound, so that it does not
// wait for the state: at most `last` times what it was plus 64 times the largest
// decayed V'.  A unit key leaves at least 1 / sqrt(dk) of that V', so the bound is
// up to 2^10 too large: the state's pairs have 22 bits down to 2^-6 of its largest
// value, and what is smaller is off by up to 2^-29 of that.
struct Scales {
  float iv, id, s, is;  // 1 / scale of V', of V' decayed; scale of the state, 1 / it
};
// x: accumulators of (I + A)^-1 times its operand, in units of 1 / ix; mx: the
// state's largest value
__device__ __forceinline__ Scales value_operands(const f32x4 (&x)[4], const float* s_sc, int q4, float ix, float last, float mx,
                                                 Pair (&vp)[2], Pair (&vd)[2]) {
  f32x4 xd[4];
  float mv = 0.0f, md = 0.0f, sv, sd;
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    xd[t] = x[t] * *reinterpret_cast<const f32x4*>(s_sc + 2 * kC + 16 * t + 4 * q4);
#pragma unroll
    for (int r = 0; r < 4; ++r) mv = fmaxf(mv, fabsf(x[t][r])), md = fmaxf(md, fabsf(xd[t][r]));
  }
  Scales k;
  md = column_max(md);
  f16_scale(column_max(mv), sv, k.iv);
  f16_scale(md, sd, k.id);
  f16_scale(fabsf(last) * mx + kC * (md * ix), k.s, k.is);
  k.iv *= ix;
  k.id *= ix;
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    vd[s] = operand(xd[2 * s], xd[2 * s + 1], sd);
    vp[s] = operand(x[2 * s], x[2 * s + 1], sv);
  }
  return k;
}

// This wave's loads and stores are done and its LDS reads; then the workgroup's.
template <int NW>
__device__ __forceinline__ void arrive() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
  if constexpr (NW > 1) __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// 64 lanes of 16 bytes to consecutive places of LDS: from base + at
typedef __attribute__((address_space(3))) char* LdsPtr;
__device__ __forceinline__ void to_lds(const char* base, unsigned at, LdsPtr dst) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(base + at),
                                   (__attribute__((address_space(3))) void*)(dst), 16, 0, 0);
}

// Raw values of a chunk's tokens and the three before, of NG groups of 16
// channels: row i at i kPieces, its pieces of 16 bytes traded by the quarter of
// i, so that the four rows of a read lie on different banks.  Rows outside the
// sequence are read as its first or last.
template <typename TIn, int NG>
struct RawRows {
  static constexpr int kOwn = int(sizeof(TIn)), kPieces = NG * kOwn;  // of a group, of a row
  static constexpr int kFrags = ((kC + 3) * kPieces + kWave - 1) / kWave;
  static __device__ __forceinline__ int place(int row, int piece) { return piece ^ (((row >> 2) & 3) * kOwn & (kPieces - 1)); }
  // load u of chunk c; values: the sequence's first row
  static __device__ __forceinline__ void load(const char* values, size_t stride, int n, int c, int u, int lane, LdsPtr to) {
    const int slot = u * kWave + lane, row = slot / kPieces, piece = place(row, slot % kPieces);
    const int i = min(max(c * kC - 3 + row, 0), n - 1);
    to_lds(values + size_t(i) * stride + piece * 16, 0, to + u * kFrag);
  }
  static __device__ __forceinline__ float get(const char* s_v, int row, int group, int n16) {
    return to_f32(*reinterpret_cast<const TIn*>(s_v + (row * kPieces + place(row, (group * 16 + n16) * kOwn / 16)) * 16 +
                                                n16 * kOwn % 16));
  }
};

// Raw values that token tile t of channel n16 needs, rows 16 t + 4 q4 - 3 ..;
// old: those before the sequence, first: whether the chunk is its first.
template <typename TIn, int NG>
__device__ __forceinline__ void window(float (&x)[7], const char* s_v, int t, int group, int n16, int q4, const float (&old)[3], bool first) {
#pragma unroll
  for (int i = 0; i < 7; ++i) {
    x[i] = RawRows<TIn, NG>::get(s_v, 16 * t + 4 * q4 + i, group, n16);
    if (t == 0 && i < 3) x[i] = first && q4 == 0 ? old[i] : x[i];
  }
}
__device__ __forceinline__ f32x4 convolved(const float (&x)[7], float4 cw) {
  f32x4 v;
#pragma unroll
  for (int r = 0; r < 4; ++r) v[r] = silu(cw.x * x[r] + cw.y * x[r + 1] + cw.z * x[r + 2] + cw.w * x[r + 3]);
  return v;
}

// Outputs of a chunk whose first row is `to` and that has n tokens left.
template <typename TOut>
__device__ __forceinline__ void store_chunk(TOut* to, size_t stride, int n, int q4, const f32x4 (&o)[4]) {
  to += 4 * q4 * stride;
  if (n >= kC) {
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) put(to + (16 * t + r) * stride, o[t][r]);
  } else {
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (16 * t + 4 * q4 + r < n) put(to + (16 * t + r) * stride, o[t][r]);
  }
  asm volatile("" ::: "memory");
}

// Head and slice of a workgroup.  Workgroups go to the 8 XCDs in turn: those of
// a key head to one, whose L2 gives them K, Q and K^T.
__device__ __forceinline__ int2 head_of() {
  const int each = gridDim.x * gridDim.y, id = blockIdx.y * gridDim.x + blockIdx.x;
  const int place = each % 8 == 0 ? id % 8 * (each / 8) + id / 8 : id;
  return make_int2(place / gridDim.x, place % gridDim.x);
}

// What a workgroup of the scan writes beside outputs and state: the status (one of
// a sequence, with its first part), and behind the last token the conv state of
// its `many` value channels from v0 on (of a head) and, one of a key head, of
// that head's queries and keys.  By `threads` threads; true where there are no
// chunks to take.
template <typename TIn>
__device__ __forceinline__ bool tail(const ChainArgs& a, const Part& part, const Tokens& tk, int b, int h, int v0, int many, int tid,
                                     int threads) {
  const int chunks = (tk.n + kC - 1) / kC, per = a.Hv / a.Hk, hk = h / per, nq = a.Hk * a.dk, nv = a.Hv * a.dv;
  const bool one = v0 == 0 && h % per == 0;
  if (part.c0 == 0 && one && hk == 0 && tid == 0 && a.status) a.status[b] = tk.status;
  const bool last = part.c0 + part.M >= chunks && (part.c0 < chunks || part.c0 == 0);
  if (last) {
    const int all = many + (one ? 2 * a.dk : 0);
    for (int i = tid; i < 3 * all; i += threads) {
      const int s = i / all, c = i % all, t = tk.n - 3 + s;
      const int which = c < many ? 2 : c < many + a.dk ? 0 : 1;  // values, queries, keys
      const int at = which == 2 ? h * a.dv + v0 + c : hk * a.dk + (c - many) % a.dk, width = which == 2 ? nv : nq;
      const size_t row = size_t(b) * 3 * (2 * nq + nv) + which * size_t(nq) + at;
      float x;
      if (t < 0) x = a.conv_state[row + size_t(t + 3) * (2 * nq + nv)];
      else x = to_f32(static_cast<const TIn*>(which == 2 ? a.v : which == 0 ? a.q : a.k)[size_t(tk.first + t) * width + at]);
      a.conv_state_out[row + size_t(s) * (2 * nq + nv)] = x;
    }
  }
  return part.c0 >= chunks;
}

// ---------------------------------------------------------------------------
// Many heads.  A wave holds the state of 16 value channels and does all with it;
// the waves of a workgroup share the chunk's operands in LDS.
//
// Operands come into LDS past the registers, each into the place of the last
// chunk's as soon as that is read: K, Q and (I + A)^-1 behind the products with
// the state, Y and K^T behind those with V'; the raw values of the next chunk
// with these.  The compiler has no loads of its own in the loop: it would wait
// for all.
//
// With one wave a SIMD nothing hides an LDS read but the wave's own products:
// operand pairs are read a group of four ahead of them, two accumulators in turn
// (12 products of 16 clocks over about 130 of a read).
//
// Bound by the vector and matrix instructions of a wave, which do not overlap
// enough: 4 sequences of 4096 tokens of 48 value heads of 128, 192 workgroups of
// eight waves, 597 us, 15000 to 17000 clocks a chunk; the matrix units are busy for
// 33 % of them, the vector units for 48 % (operands made of values and of V', scales).
// ---------------------------------------------------------------------------
template <typename TIn, int DKP, int NW>
struct Scan {
  static constexpr int kKs = DKP / 32;
  static constexpr int kQ = kKs * 8 * kFrag;  // bytes of K, of Q, of K^T
  static constexpr int kAtQ = kQ, kAtKt = 2 * kQ, kAtT = 3 * kQ, kAtY = kAtT + 12 * kFrag, kAtScalars = kAtY + 12 * kFrag,
                       kAtV = kAtScalars + 2 * kFrag;
  static constexpr int kLds = kAtV + RawRows<TIn, NW>::kFrags * kFrag;
};

template <typename TIn, typename TOut, int DKP, int NW>
__global__ __launch_bounds__(NW * kWave) void scan_kernel(ChainArgs a, Part part) {
  typedef Scan<TIn, DKP, NW> S;
  typedef Rows<S::kKs> R;
  typedef RawRows<TIn, NW> Raw;
  constexpr int kKs = S::kKs, kGroups = R::kGroups, kQFrags = S::kQ / kFrag;
  extern __shared__ __align__(16) char s_raw[];
  const char *s_k = s_raw, *s_q = s_raw + S::kAtQ, *s_kt = s_raw + S::kAtKt, *s_t = s_raw + S::kAtT, *s_y = s_raw + S::kAtY,
             *s_v = s_raw + S::kAtV;
  const LdsPtr lds = (LdsPtr)s_raw;
  const int tid = threadIdx.x, lane = tid % kWave, w = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int n16 = lane & 15, q4 = lane >> 4;
  const int2 hs = head_of();
  const int group = hs.y * NW + w, h = hs.x, b = part.b0 + blockIdx.z, hk = h / (a.Hv / a.Hk);
  const Tokens tk = tokens_of(a, b);
  const int dk = a.dk, dv = a.dv, end = min(part.c0 + part.M, (tk.n + kC - 1) / kC);
  if (tail<TIn>(a, part, tk, b, h, hs.y * NW * 16, NW * 16, tid, NW * kWave)) return;
  const SlotLayout l = slot_layout(a.Hk, a.Hv, dk);
  const int ch = group * 16 + n16;  // value channel
  const char* vws = value_at(a, slot_at(a, part, blockIdx.z, 0), h);
  const char* kws = key_at(a, slot_at(a, part, blockIdx.z, 0), hk);
  const unsigned at = lane * 16;
  auto shared = [&](const char* src, int to, int frags) {  // by all waves
#pragma unroll
    for (int n = 0; n < (frags + NW - 1) / NW; ++n) {
      const int u = n * NW + w;
      if (frags % NW == 0 || u < frags) to_lds(src + u * kFrag, at, lds + to + u * kFrag);
    }
  };
  const size_t vstride = size_t(a.Hv) * dv;
  const char* values = reinterpret_cast<const char*>(reinterpret_cast<const TIn*>(a.v) + size_t(tk.first) * vstride + h * dv + hs.y * NW * 16);
  auto load_values = [&](int m) {
#pragma unroll
    for (int n = 0; n < (Raw::kFrags + NW - 1) / NW; ++n)
      if (n * NW + w < Raw::kFrags) Raw::load(values, vstride * sizeof(TIn), tk.n, part.c0 + m, n * NW + w, lane, lds + S::kAtV);
  };
  auto load_first = [&](int m) {  // K, Q, (I + A)^-1, scalars
    const char *k = kws + size_t(m) * l.total, *v = vws + size_t(m) * l.total;
    shared(k, 0, 2 * kQFrags);
    shared(v, S::kAtT, 12);
    shared(v + kScalarsAt, S::kAtScalars + (m & 1) * kFrag, 1);
    asm volatile("" ::: "memory");
  };
  auto load_second = [&](int m, int next) {  // Y, K^T, the next chunk's raw values
    shared(vws + size_t(m) * l.total + kYAt, S::kAtY, 12);
    shared(kws + size_t(m) * l.total + 2 * S::kQ, S::kAtKt, kQFrags);
    load_values(next);
    asm volatile("" ::: "memory");
  };
  load_values(0);
  load_first(0);

  float* state = a.S + ((size_t(b) * a.Hv + h) * dv + ch) * dk + 4 * q4;
  f32x4 st[DKP / 16];  // key channels 16 n + 4 q4 ..
#pragma unroll
  for (int n = 0; n < DKP / 16; ++n) st[n] = 16 * n < dk ? *reinterpret_cast<const f32x4*>(state + 16 * n) : f32x4{};
  const size_t C = 2 * size_t(a.Hk) * dk + vstride, channel = 2 * size_t(a.Hk) * dk + h * dv + ch;
  const float4 cw = *reinterpret_cast<const float4*>(a.conv_w + channel * 4);
  float old[3];  // before the sequence's first token
#pragma unroll
  for (int i = 0; i < 3; ++i) old[i] = a.conv_state[(size_t(b) * 3 + i) * C + channel];
  TOut* out = reinterpret_cast<TOut*>(a.out) + size_t(tk.first) * vstride + h * dv + ch;
  auto store = [&](int m, const f32x4 (&o)[4]) {
    const int n0 = (part.c0 + m) * kC;
    store_chunk(out + size_t(n0) * vstride, vstride, tk.n - n0, q4, o);
  };
  float mx = 0.0f;  // the largest of this lane's values
#pragma unroll
  for (int n = 0; n < DKP / 16; ++n)
#pragma unroll
    for (int r = 0; r < 4; ++r) mx = fmaxf(mx, fabsf(st[n][r]));
  f32x4 v[4];  // convolved values of a chunk
  auto values_of = [&](int m, int t) {
    float x[7];
    window<TIn, NW>(x, s_v, t, w, n16, q4, old, part.c0 + m == 0);
    v[t] = convolved(x, cw);
    asm volatile("" : "+v"(v[t]));  // here, not at its use a chunk later
  };
  arrive<NW>();
#pragma unroll
  for (int t = 0; t < 4; ++t) values_of(0, t);

  f32x4 o[4];  // outputs of a chunk
  float is;    // the state as operands
  Pair sp[kKs];
  {
    float ss;
    f16_scale(column_max(mx), ss, is);
#pragma unroll
    for (int s = 0; s < kKs; ++s) sp[s] = operand(st[2 * s], st[2 * s + 1], ss);
  }
  for (int m = 0; m < end - part.c0; ++m) {
    const int next = min(m + 1, end - part.c0 - 1);  // the last chunk's again: they are not used
    const float* s_sc = reinterpret_cast<const float*>(s_raw + S::kAtScalars + (m & 1) * kFrag);
    arrive<NW>();  // K, Q, (I + A)^-1, scalars; the last chunk's Y and K^T, the raw values are read
    if (m) store(m - 1, o);  // here: the next wait is a part away
    load_second(m, next);

    typename R::Group f[2];
    f32x4 x[4] = {};
#pragma unroll
    for (int t = 0; t < 4; ++t) o[t] = f32x4{};
    R::read(f[0], s_k, 0, lane);
#pragma unroll
    for (int n = 0; n < kGroups; ++n) {
      if (n + 1 < kGroups) R::read(f[(n + 1) & 1], s_k, n + 1, lane);
      else R::read(f[kGroups & 1], s_q, 0, lane);
      __builtin_amdgcn_sched_barrier(0);
      R::times(f[n & 1], sp, x, n);
      __builtin_amdgcn_sched_barrier(0);
    }
    // beta (V - e^g K S^T), beside half of the queries' products
    float mr = 0.0f, sr, ir;
    const float ik = is * (1.0f / kUnit);
#pragma unroll
    for (int n = 0; n < kGroups / 2; ++n) {
      R::read(f[(kGroups + n + 1) & 1], s_q, n + 1, lane);
      __builtin_amdgcn_sched_barrier(0);
      R::times(f[(kGroups + n) & 1], sp, o, n);
#pragma unroll
      for (int t = n * 8 / kGroups; t < (n + 1) * 8 / kGroups; ++t) {
        const f32x4 be = *reinterpret_cast<const f32x4*>(s_sc + 16 * t + 4 * q4);
        const f32x4 dec = *reinterpret_cast<const f32x4*>(s_sc + kC + 16 * t + 4 * q4);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          x[t][r] = be[r] * (v[t][r] - dec[r] * (x[t][r] * ik));
          mr = fmaxf(mr, fabsf(x[t][r]));
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    mr = column_max(mr);
    f16_scale(mr, sr, ir);
    const Pair r0 = operand(x[0], x[1], sr), r1 = operand(x[2], x[3], sr);
    Pair g[2][4];
    read_lower(g[0], s_t, 0, lane);
    read_lower(g[1], s_t, 1, lane);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int t = 0; t < 4; ++t) x[t] = f32x4{};
    times_lower(g[0], r0, x, 0);
    times_lower(g[1], r1, x, 1);
    __builtin_amdgcn_sched_barrier(0);
    const ChunkScalars cs = scalars_of(s_sc);
    Scales sc;
    Pair vp[2], vd[2];
#pragma unroll
    for (int n = kGroups / 2; n < kGroups; ++n) {
      if (n + 1 < kGroups) R::read(f[(kGroups + n + 1) & 1], s_q, n + 1, lane);
      __builtin_amdgcn_sched_barrier(0);
      R::times(f[(kGroups + n) & 1], sp, o, n);
      if (n == kGroups / 2) sc = value_operands(x, s_sc, q4, ir * cs.inv, cs.last, column_max(mx), vp, vd);  // beside the others
      __builtin_amdgcn_sched_barrier(0);
    }
    arrive<NW>();  // Y, K^T, raw values; K, Q and (I + A)^-1 are read
    load_first(next);

    // outputs: Y V' beside Q S^T; then the state behind the chunk, and the next
    // chunk's values
    f32x4 y[4] = {};
    read_lower(g[0], s_y, 0, lane);
    read_lower(g[1], s_y, 1, lane);
    __builtin_amdgcn_sched_barrier(0);
    times_lower(g[0], vp[0], y, 0);
    read_kt(g[0], s_kt, 0, lane);
    __builtin_amdgcn_sched_barrier(0);
    times_lower(g[1], vp[1], y, 1);
    const float iv = sc.iv * cs.y * a.scale, io = ik * a.scale, id = sc.id * (1.0f / kUnit);
    mx = 0.0f;
    f32x4 c[2][2];
    auto state_of = [&](int n) {
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          st[2 * n + e][r] = cs.last * st[2 * n + e][r] + c[n & 1][e][r] * id;
          mx = fmaxf(mx, fabsf(st[2 * n + e][r]));
        }
      sp[n] = operand(st[2 * n], st[2 * n + 1], sc.s);
    };
#pragma unroll
    for (int n = 0; n < kKs; ++n) {
      if (n + 1 < kKs) read_kt(g[(n + 1) & 1], s_kt, n + 1, lane);
      __builtin_amdgcn_sched_barrier(0);
      c[n & 1][0] = c[n & 1][1] = f32x4{};
      times_kt(g[n & 1], vd, c[n & 1]);
      if (n) state_of(n - 1);
      // a share of the outputs and of the next values beside these products
#pragma unroll
      for (int t = n * 4 / kKs; t < (n + 1) * 4 / kKs; ++t) {
        const f32x4 dec = *reinterpret_cast<const f32x4*>(s_sc + kC + 16 * t + 4 * q4);
#pragma unroll
        for (int r = 0; r < 4; ++r) o[t][r] = o[t][r] * dec[r] * io + y[t][r] * iv;
        values_of(next, t);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    state_of(kKs - 1);
    is = sc.is;
  }
  store(end - part.c0 - 1, o);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // nothing arrives in LDS after the end
#pragma unroll
  for (int n = 0; n < DKP / 16; ++n)
    if (16 * n < dk) *reinterpret_cast<f32x4*>(state + 16 * n) = st[n];
}

// ---------------------------------------------------------------------------
// Few heads: the recurrence is what takes time, a chunk behind the other, and
// half of the SIMDs have nothing.  The work of 16 value channels goes to two
// waves: one takes the state from chunk to chunk (K S^T, V', the new state), the
// other, a part behind, makes the outputs and convolves the next chunk's values.
// They pass the state, V' and the values as operands through LDS.  Two more waves
// do all loads (a wave has at most 64 on their way).
//
// Bound by the state's wave, whose steps wait for one another (8192 tokens of one
// sequence of 48 heads of 128: 412 us, 6500 to 7000 clocks a chunk, matrix units 22 %
// busy).  The loads, 126 KB a chunk and workgroup (K, Q, K^T 96, the inverse and Y 24,
// raw values 5), come to 19 bytes a clock and CU.  With one wave for both 1024 tokens of
// 32 such heads take 109 us, with two 73.
// ---------------------------------------------------------------------------
constexpr int kLoaders = 2;

template <typename TIn, int DKP, int NG>
struct ScanPair {
  typedef Scan<TIn, DKP, NG> Base;
  static constexpr int kKs = DKP / 32, kThreads = (2 * NG + kLoaders) * kWave;
  static constexpr int kAtS = Base::kLds;                       // of a group: the state's operands [ks]
  static constexpr int kAtX = kAtS + NG * kKs * 2 * kFrag;      // of a group: the values, then V' [2 steps]
  static constexpr int kAtScale = kAtX + NG * 4 * kFrag;        // of a group: 1 / scale of the state, of V' [2][16]
  static constexpr int kAtScrap = kAtScale + NG * 128;
  static constexpr int kLds = kAtScrap + 256;
};

template <typename TIn, typename TOut, int DKP, int NG>
__global__ __launch_bounds__((2 * NG + kLoaders) * kWave) void scan_pair_kernel(ChainArgs a, Part part) {
  typedef ScanPair<TIn, DKP, NG> S;
  typedef typename S::Base B;
  typedef Rows<S::kKs> R;
  typedef RawRows<TIn, NG> Raw;
  constexpr int kKs = S::kKs, kGroups = R::kGroups, kQFrags = B::kQ / kFrag, kWaves = 2 * NG + kLoaders;
  extern __shared__ __align__(16) char s_raw[];
  const char *s_k = s_raw, *s_q = s_raw + B::kAtQ, *s_kt = s_raw + B::kAtKt, *s_t = s_raw + B::kAtT, *s_y = s_raw + B::kAtY,
             *s_v = s_raw + B::kAtV;
  const int tid = threadIdx.x, lane = tid % kWave, w = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int n16 = lane & 15, q4 = lane >> 4;
  const int2 hs = head_of();
  const int mine = w % NG, h = hs.x, b = part.b0 + blockIdx.z, hk = h / (a.Hv / a.Hk);
  const Tokens tk = tokens_of(a, b);
  const int dk = a.dk, dv = a.dv, end = min(part.c0 + part.M, (tk.n + kC - 1) / kC), count = end - part.c0;
  if (count <= 0) {
    tail<TIn>(a, part, tk, b, h, hs.y * NG * 16, NG * 16, tid, kWaves * kWave);
    return;
  }
  const size_t vstride = size_t(a.Hv) * dv;

  if (w >= 2 * NG) {  // loads, every other one of a list by each of the two waves
    const LdsPtr lds = (LdsPtr)s_raw;
    const SlotLayout l = slot_layout(a.Hk, a.Hv, dk);
    const char* vws = value_at(a, slot_at(a, part, blockIdx.z, 0), h);
    const char* kws = key_at(a, slot_at(a, part, blockIdx.z, 0), hk);
    const char* values = reinterpret_cast<const char*>(reinterpret_cast<const TIn*>(a.v) + size_t(tk.first) * vstride + h * dv + hs.y * NG * 16);
    const unsigned at = lane * 16;
    auto copy = [&](const char* src, int to, int frags) {
#pragma unroll 4
      for (int u = w - 2 * NG; u < frags; u += kLoaders) to_lds(src + u * kFrag, at, lds + to + u * kFrag);
    };
    auto load_values = [&](int m) {
      for (int u = w - 2 * NG; u < Raw::kFrags; u += kLoaders)
        Raw::load(values, vstride * sizeof(TIn), tk.n, part.c0 + m, u, lane, lds + B::kAtV);
    };
    auto load_first = [&](int m) {  // K, (I + A)^-1, scalars
      const char* v = vws + size_t(m) * l.total;
      copy(kws + size_t(m) * l.total, 0, kQFrags);
      copy(v + kScalarsAt, B::kAtScalars + (m & 1) * kFrag, 1);
      copy(v, B::kAtT, 12);
    };
    // Lines of a chunk into L2, a chunk ahead of the loads, a lane a line: those of
    // a key head by its workgroups in turn
    const int per = a.Hv / a.Hk, turns = per * gridDim.x, turn = h % per * gridDim.x + hs.y;
    auto touch = [&](const char* p) {
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(p),
                                       (__attribute__((address_space(3))) void*)(lds + S::kAtScrap), 4, 0, 0);
    };
    auto ahead = [&](int m) {
      if (w != 2 * NG || m >= count) return;
      for (int u = turn; u < 3 * B::kQ / 8192; u += turns) touch(kws + size_t(m) * l.total + u * 8192 + lane * 128);
      for (int u = hs.y; u < 4; u += gridDim.x) touch(vws + size_t(m) * l.total + min(u * 8192 + lane * 128, int(kValue) - 128));
      const int i = min((part.c0 + m + 1) * kC + lane, tk.n - 1);
      touch(values + size_t(i) * vstride * sizeof(TIn));
    };
    load_values(0);
    arrive<kWaves>();
    load_first(0);
    arrive<kWaves>();
    load_values(min(1, count - 1));
    for (int m = 0; m < count; ++m) {
      arrive<kWaves>();
      ahead(m + 1);
      copy(kws + size_t(m) * l.total + B::kQ, B::kAtQ, 2 * kQFrags);  // and K^T
      copy(vws + size_t(m) * l.total + kYAt, B::kAtY, 12);
      arrive<kWaves>();
      if (m + 2 < count) load_values(m + 2);
      if (m + 1 < count) load_first(m + 1);
    }
    tail<TIn>(a, part, tk, b, h, hs.y * NG * 16, NG * 16, tid - 2 * NG * kWave, kLoaders * kWave);
    return;
  }

  const int ch = (hs.y * NG + mine) * 16 + n16;  // value channel
  char* s_s = s_raw + S::kAtS + mine * kKs * 2 * kFrag;
  char* s_x = s_raw + S::kAtX + mine * 4 * kFrag;
  float* s_scale = reinterpret_cast<float*>(s_raw + S::kAtScale + mine * 128) + n16;
  if (w < NG) {  // the state
    float* state = a.S + ((size_t(b) * a.Hv + h) * dv + ch) * dk + 4 * q4;
    f32x4 st[DKP / 16];
    float mx = 0.0f;
#pragma unroll
    for (int n = 0; n < DKP / 16; ++n) {
      st[n] = 16 * n < dk ? *reinterpret_cast<const f32x4*>(state + 16 * n) : f32x4{};
#pragma unroll
      for (int r = 0; r < 4; ++r) mx = fmaxf(mx, fabsf(st[n][r]));
    }
    float is;
    Pair sp[kKs];
    {
      float ss;
      f16_scale(column_max(mx), ss, is);
#pragma unroll
      for (int s = 0; s < kKs; ++s) {
        sp[s] = operand(st[2 * s], st[2 * s + 1], ss);
        store_pair(s_s, s, lane, sp[s]);
      }
    }
    arrive<kWaves>();
    arrive<kWaves>();
    for (int m = 0; m < count; ++m) {
      const float* s_sc = reinterpret_cast<const float*>(s_raw + B::kAtScalars + (m & 1) * kFrag);
      s_scale[0] = is;
      arrive<kWaves>();  // K, (I + A)^-1, scalars; values, the state
      typename R::Group f[2];
      f32x4 x[4] = {};
      R::read(f[0], s_k, 0, lane);
      Pair g[2][4];
#pragma unroll
      for (int n = 0; n < kGroups; ++n) {
        if (n + 1 < kGroups) R::read(f[(n + 1) & 1], s_k, n + 1, lane);
        __builtin_amdgcn_sched_barrier(0);
        R::times(f[n & 1], sp, x, n);
        __builtin_amdgcn_sched_barrier(0);
      }
      read_lower(g[0], s_t, 0, lane);
      read_lower(g[1], s_t, 1, lane);
      float mr = 0.0f, sr, ir;
      const float ik = is * (1.0f / kUnit);
#pragma unroll
      for (int t = 0; t < 4; ++t) {  // beta (V - e^g K S^T)
        const f32x4 be = *reinterpret_cast<const f32x4*>(s_sc + 16 * t + 4 * q4);
        const f32x4 dec = *reinterpret_cast<const f32x4*>(s_sc + kC + 16 * t + 4 * q4);
        const f32x4 v = *reinterpret_cast<const f32x4*>(s_x + t * kFrag + lane * 16);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          x[t][r] = be[r] * (v[r] - dec[r] * (x[t][r] * ik));
          mr = fmaxf(mr, fabsf(x[t][r]));
        }
      }
      mr = column_max(mr);
      f16_scale(mr, sr, ir);
      const Pair r0 = operand(x[0], x[1], sr), r1 = operand(x[2], x[3], sr);
#pragma unroll
      for (int t = 0; t < 4; ++t) x[t] = f32x4{};
      times_lower(g[0], r0, x, 0);
      times_lower(g[1], r1, x, 1);
      const ChunkScalars cs = scalars_of(s_sc);
      Pair vp[2], vd[2];
      const Scales sc = value_operands(x, s_sc, q4, ir * cs.inv, cs.last, column_max(mx), vp, vd);
      store_pair(s_x, 0, lane, vp[0]);  // in place of the values, which this wave has read
      store_pair(s_x, 1, lane, vp[1]);
      s_scale[16] = sc.iv;
      const float id = sc.id * (1.0f / kUnit);
      arrive<kWaves>();  // K^T; V'
      read_kt(g[0], s_kt, 0, lane);
      mx = 0.0f;
      f32x4 c[2][2];
      auto state_of = [&](int n) {
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            st[2 * n + e][r] = cs.last * st[2 * n + e][r] + c[n & 1][e][r] * id;
            mx = fmaxf(mx, fabsf(st[2 * n + e][r]));
          }
        sp[n] = operand(st[2 * n], st[2 * n + 1], sc.s);
        store_pair(s_s, n, lane, sp[n]);
      };
#pragma unroll
      for (int n = 0; n < kKs; ++n) {
        if (n + 1 < kKs) read_kt(g[(n + 1) & 1], s_kt, n + 1, lane);
        __builtin_amdgcn_sched_barrier(0);
        c[n & 1][0] = c[n & 1][1] = f32x4{};
        times_kt(g[n & 1], vd, c[n & 1]);
        if (n) state_of(n - 1);
        __builtin_amdgcn_sched_barrier(0);
      }
      state_of(kKs - 1);
      is = sc.is;
    }
#pragma unroll
    for (int n = 0; n < DKP / 16; ++n)
      if (16 * n < dk) *reinterpret_cast<f32x4*>(state + 16 * n) = st[n];
    return;
  }

  // the outputs
  const size_t C = 2 * size_t(a.Hk) * dk + vstride, channel = 2 * size_t(a.Hk) * dk + h * dv + ch;
  const float4 cw = *reinterpret_cast<const float4*>(a.conv_w + channel * 4);
  float old[3];  // before the sequence's first token
#pragma unroll
  for (int i = 0; i < 3; ++i) old[i] = a.conv_state[(size_t(b) * 3 + i) * C + channel];
  TOut* out = reinterpret_cast<TOut*>(a.out) + size_t(tk.first) * vstride + h * dv + ch;
  f32x4 v[4];
  auto values_of = [&](int m) {
    float x[4][7];
#pragma unroll
    for (int t = 0; t < 4; ++t) window<TIn, NG>(x[t], s_v, t, mine, n16, q4, old, part.c0 + m == 0);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      v[t] = convolved(x[t], cw);
      asm volatile("" : "+v"(v[t]));  // here, not at its use a part later
    }
  };
  auto pass_values = [&]() {
#pragma unroll
    for (int t = 0; t < 4; ++t) *reinterpret_cast<f32x4*>(s_x + t * kFrag + lane * 16) = v[t];
  };
  arrive<kWaves>();  // raw values
  values_of(0);
  pass_values();
  arrive<kWaves>();
  f32x4 o[4];
  for (int m = 0; m < count; ++m) {
    const float* s_sc = reinterpret_cast<const float*>(s_raw + B::kAtScalars + (m & 1) * kFrag);
    arrive<kWaves>();  // raw values of the next chunk; the state
    if (m) {
      const int n0 = (part.c0 + m - 1) * kC;
      store_chunk(out + size_t(n0) * vstride, vstride, tk.n - n0, q4, o);
    }
    Pair sp[kKs];
#pragma unroll
    for (int s = 0; s < kKs; ++s) sp[s] = load_pair(s_s, s, lane);
    const float io = s_scale[0] * (a.scale * (1.0f / kUnit));
    values_of(m + 1);  // behind the last chunk: not used
    arrive<kWaves>();  // Q, Y; V'
    const Pair v0 = load_pair(s_x, 0, lane), v1 = load_pair(s_x, 1, lane);
    const float iv = s_scale[16] * scalars_of(s_sc).y * a.scale;
    typename R::Group f[2];
    Pair g[2][4];
#pragma unroll
    for (int t = 0; t < 4; ++t) o[t] = f32x4{};
    R::read(f[0], s_q, 0, lane);
#pragma unroll
    for (int n = 0; n < kGroups; ++n) {
      if (n + 1 < kGroups) R::read(f[(n + 1) & 1], s_q, n + 1, lane);
      else read_lower(g[0], s_y, 0, lane);
      __builtin_amdgcn_sched_barrier(0);
      R::times(f[n & 1], sp, o, n);
      if (n == 0) pass_values();  // V' is read
      __builtin_amdgcn_sched_barrier(0);
    }
    read_lower(g[1], s_y, 1, lane);
    f32x4 y[4] = {};
    times_lower(g[0], v0, y, 0);
    times_lower(g[1], v1, y, 1);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const f32x4 dec = *reinterpret_cast<const f32x4*>(s_sc + kC + 16 * t + 4 * q4);
#pragma unroll
      for (int r = 0; r < 4; ++r) o[t][r] = o[t][r] * dec[r] * io + y[t][r] * iv;
    }
  }
  const int n0 = (end - 1) * kC;
  store_chunk(out + size_t(n0) * vstride, vstride, tk.n - n0, q4, o);
}

int after_launch() {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? GDN_OK : set_error(GDN_EHIP, "chain: launch: %s", hipGetErrorString(e));
}

template <typename TIn, int DKP>
int launch_prep(const ChainArgs& a, const Part& p, hipStream_t stream) {
  constexpr int lds = Prep<DKP>::kLds;
  const int rc = ensure_dynamic_lds(reinterpret_cast<const void*>(chunk_kernel<TIn, DKP>), lds, "chain");
  if (rc != GDN_OK) return rc;
  chunk_kernel<TIn, DKP><<<dim3(a.Hk, p.M, p.G), kPrepThreads, lds, stream>>>(a, p);
  return after_launch();
}

template <typename TIn, typename TOut, int DKP, int NW>
int launch_waves(const ChainArgs& a, const Part& p, hipStream_t stream) {
  constexpr int lds = Scan<TIn, DKP, NW>::kLds;
  const int rc = ensure_dynamic_lds(reinterpret_cast<const void*>(scan_kernel<TIn, TOut, DKP, NW>), lds, "chain");
  if (rc != GDN_OK) return rc;
  scan_kernel<TIn, TOut, DKP, NW><<<dim3(a.dv / 16 / NW, a.Hv, p.G), NW * kWave, lds, stream>>>(a, p);
  return after_launch();
}

template <typename TIn, typename TOut, int DKP, int NG>
int launch_pairs(const ChainArgs& a, const Part& p, hipStream_t stream) {
  typedef ScanPair<TIn, DKP, NG> S;
  const int rc = ensure_dynamic_lds(reinterpret_cast<const void*>(scan_pair_kernel<TIn, TOut, DKP, NG>), S::kLds, "chain");
  if (rc != GDN_OK) return rc;
  scan_pair_kernel<TIn, TOut, DKP, NG><<<dim3(a.dv / 16 / NG, a.Hv, p.G), S::kThreads, S::kLds, stream>>>(a, p);
  return after_launch();
}

// The fewest of a head's channels a workgroup that leave at most one for each of the
// 256 CUs, else all of them.  us for 1024 tokens and heads of 128, one key head a value
// head (pairs of waves: 1 and 2 of them; waves: 2, 4 and 8):
//   32 heads    73  77   111 109 134
//   48         120  84   118 117 143
//   64         127  93   125 123 148
//   80         176 144   214 135 160
//   128        284 207   262 187 210
//   144        362 291   390 305 248
//   256        589 431   549 381 330
template <typename TIn, typename TOut, int DKP>
int launch_scan(const ChainArgs& a, const Part& p, hipStream_t stream) {
  const int groups = a.dv / 16;  // of 16 value channels
  const long long all = (long long)(p.G) * a.Hv * groups;
  if (groups == 1 || all <= 256) return launch_pairs<TIn, TOut, DKP, 1>(a, p, stream);
  if (all <= 512) return launch_pairs<TIn, TOut, DKP, 2>(a, p, stream);
  if (groups == 2) return launch_waves<TIn, TOut, DKP, 2>(a, p, stream);
  if (groups == 4 || all <= 1024) return launch_waves<TIn, TOut, DKP, 4>(a, p, stream);
  return launch_waves<TIn, TOut, DKP, 8>(a, p, stream);
}

template <typename TIn, int DKP>
int launch_part(const ChainArgs& a, const Part& p, hipStream_t stream) {
  const int rc = launch_prep<TIn, DKP>(a, p, stream);
  if (rc != GDN_OK) return rc;
  return a.out_dtype == GDN_BF16 ? launch_scan<TIn, BF16, DKP>(a, p, stream) : launch_scan<TIn, float, DKP>(a, p, stream);
}

template <typename TIn>
int launch_type(const ChainArgs& a, const Part& p, hipStream_t stream) {
  if (padded_dk(a.dk) == 32) return launch_part<TIn, 32>(a, p, stream);
  return a.dk == 64 ? launch_part<TIn, 64>(a, p, stream) : launch_part<TIn, 128>(a, p, stream);
}

}  // namespace

int launch_chain_chunks(const ChainArgs& a, hipStream_t stream) {
  const StreamOrder order(stream);
  const size_t slot = slot_layout(a.Hk, a.Hv, a.dk).total;
  const int chunks = (a.T + kC - 1) / kC;
  const long long slots = std::max<long long>(1, (long long)(GDN_CHAIN_WORKSPACE / slot));
  Part p;
  p.G = int(std::min<long long>(a.B, slots));
  p.M = int(std::min<long long>(chunks, slots / p.G));
  if (p.M > 65535) p.M = 65535;
  int rc = GDN_OK;
  p.ws = static_cast<char*>(stream_workspace(slot * p.G * p.M, stream, &rc));
  if (!p.ws) return rc;
  const int G = p.G;
  for (p.b0 = 0; p.b0 < a.B; p.b0 += G) {
    p.G = std::min(G, a.B - p.b0);
    for (p.c0 = 0; p.c0 < chunks; p.c0 += p.M) {
      rc = a.in_dtype == GDN_BF16 ? launch_type<BF16>(a, p, stream) : launch_type<float>(a, p, stream);
      if (rc != GDN_OK) return rc;
    }
  }
  return GDN_OK;
}

}  // namespace gdn
