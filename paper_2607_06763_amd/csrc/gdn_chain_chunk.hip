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
// Products.  The outputs have 32-bit accuracy, so each operand is a pair of fp16
// values, hi + lo, 22 bits together, and a product is three on the matrix units
// (hi hi, hi lo, lo hi) with 32-bit sums: 2^-22 of an operand is lost.  Scales
// are powers of two, exact: 2^10 for what is at most 1 (unit keys, queries, Y),
// else by the largest value of the matrix or of the operand's column.
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
constexpr int kPrepThreads = 256;
constexpr int kPrepWaves = kPrepThreads / kWave;
constexpr int kHeads = 3;       // value heads that are inverted at once
constexpr int kLd = kC + 4;     // floats of a row of a chunk's matrix in LDS
constexpr float kUnit = 1024.0f;  // scale of what is at most 1
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

__device__ __forceinline__ Pair split(const float (&x)[8], float scale) {
  u32x4 hi, lo;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    f16x2 h = {(_Float16)(x[2 * e] * scale), (_Float16)(x[2 * e + 1] * scale)};
    // a value of its own: were it computed again for the difference, with another
    // rounding of the product, hi + lo would miss x by a step of hi
    asm("" : "+v"(h));
    const f16x2 l = {(_Float16)__builtin_fmaf(x[2 * e], scale, -(float)h[0]),
                     (_Float16)__builtin_fmaf(x[2 * e + 1], scale, -(float)h[1])};
    hi[e] = __builtin_bit_cast(unsigned, h);
    lo[e] = __builtin_bit_cast(unsigned, l);
  }
  return {__builtin_bit_cast(f16x8, hi), __builtin_bit_cast(f16x8, lo)};
}

__device__ __forceinline__ f32x4 mma(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

__device__ __forceinline__ f32x4 mma3(const Pair& a, const Pair& b, f32x4 c) {
  c = mma(a.lo, b.hi, c);
  c = mma(a.hi, b.lo, c);
  return mma(a.hi, b.hi, c);
}

// Power of two that takes m to 2^13 .. 2^14, and its inverse (both normal
// floats: m is clamped to 2^-113 .. 2^126).
__device__ __forceinline__ void f16_scale(float m, float& scale, float& inv) {
  int ex = int((__float_as_uint(m) >> 23) & 0xffu);
  ex = ex < 14 ? 14 : ex > 253 ? 253 : ex;
  scale = __uint_as_float(unsigned(267 - ex) << 23);
  inv = __uint_as_float(unsigned(ex - 13) << 23);
}

// Over the four lanes of a column (lane % 16): rows of 16 lanes trade places.
__device__ __forceinline__ float column_max(float x) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
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

// ---------------------------------------------------------------------------
// Raw inputs
// ---------------------------------------------------------------------------
// 8 channels of a row.
__device__ __forceinline__ void fetch8(const float* p, float (&x)[8]) {
  const float4 y = ld4(p), z = ld4(p + 4);
  x[0] = y.x, x[1] = y.y, x[2] = y.z, x[3] = y.w, x[4] = z.x, x[5] = z.y, x[6] = z.z, x[7] = z.w;
}
__device__ __forceinline__ void fetch8(const BF16* p, float (&x)[8]) {
  const u32x4 u = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[2 * e] = __uint_as_float(u[e] << 16);
    x[2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u);
  }
}

template <int DKP>
struct Prep {
  static constexpr int kPacks = DKP / 8, kKs = DKP / 32;
  static constexpr int kPlane = kPacks * (kC + 1) * 16;       // bytes of hi or lo of K or Q: [pack][token]
  static constexpr int kMat = kC * kLd * int(sizeof(float));  // a chunk's matrix
  static constexpr int kRows = 4 * kPlane > kHeads * kMat ? 4 * kPlane : kHeads * kMat;
  static constexpr int kLds = kRows + kHeads * (kC * 12 + 4);
};

// ---------------------------------------------------------------------------
// What does not depend on the state.  One workgroup per (key head, chunk) with
// all of its value heads: keys and queries are convolved once.  Loads have no
// branch around them (rows are clamped and values selected): a branch each made
// them wait for one another.
// ---------------------------------------------------------------------------
template <typename TIn, int DKP>
__global__ __launch_bounds__(kPrepThreads, 2) void chunk_kernel(ChainArgs a, Part part) {
  typedef Prep<DKP> P;
  constexpr int kKs = P::kKs, kPacks = P::kPacks;
  extern __shared__ __align__(16) char s_raw[];
  char* s_kq = s_raw;                            // K hi, K lo, Q hi, Q lo; then the heads' matrices
  float* s_t = reinterpret_cast<float*>(s_raw);  // [head][64][kLd]
  double* s_log = reinterpret_cast<double*>(s_raw + P::kRows);  // [head][64]
  float* s_beta = reinterpret_cast<float*>(s_log + kHeads * kC);
  float* s_scale = s_beta + kHeads * kC;  // of (I + A)^-1
  const int tid = threadIdx.x, lane = tid % kWave, w = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int n16 = lane & 15, q4 = lane >> 4;
  const int hk = blockIdx.x, m = blockIdx.y, b = part.b0 + blockIdx.z;
  const Tokens tk = tokens_of(a, b);
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

  // keys and queries: 8 channels a thread, kLpt threads a token
  {
    constexpr int kLpt = kPacks, kGroups = kPrepThreads / kLpt, kTok = kC / kGroups;
    static_assert(kTok * kGroups == kC, "every thread has tokens");
    const int p = tid % kLpt, t0 = tid / kLpt * kTok, c8 = min(p * 8, dk - 8);
    const bool in = p * 8 < dk;
    float win[2][kTok + 3][8];
#pragma unroll
    for (int isq = 0; isq < 2; ++isq) {
      const TIn* x = reinterpret_cast<const TIn*>(isq ? a.q : a.k) + hk * dk + c8;
#pragma unroll
      for (int i = 0; i < kTok + 3; ++i) {
        const int t = min(max(t0 - 3 + i, n0 ? -3 : 0), nt - 1);
        fetch8(x + (long long)(row0 + t) * a.Hk * dk, win[isq][i]);
      }
    }
    if (n0 == 0 && t0 < 3) {  // before the sequence's first token
#pragma unroll
      for (int isq = 0; isq < 2; ++isq)
#pragma unroll
        for (int i = 0; i < 3; ++i)
          if (t0 + i < 3) fetch8(cs + size_t(t0 + i) * C + (isq ? hk : a.Hk + hk) * dk + c8, win[isq][i]);
    }
#pragma unroll
    for (int isq = 0; isq < 2; ++isq) {
      float4 cw[8];
#pragma unroll
      for (int e = 0; e < 8; ++e)
        cw[e] = *reinterpret_cast<const float4*>(a.conv_w + size_t((isq ? hk : a.Hk + hk) * dk + c8 + e) * 4);
#pragma unroll
      for (int i = 0; i < kTok; ++i) {
        float y[8], sum = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const auto& x = win[isq];
          y[e] = silu(cw[e].x * x[i][e] + cw[e].y * x[i + 1][e] + cw[e].z * x[i + 2][e] + cw[e].w * x[i + 3][e]);
          if (!in || t0 + i >= nt) y[e] = 0.0f;
          sum += y[e] * y[e];
        }
        const Pair x8 = split(y, rsqrt_hw(group_sum<kLpt>(sum) + 1e-6f) * kUnit);
        char* d = s_kq + isq * 2 * P::kPlane + (p * (kC + 1) + t0 + i) * 16;
        *reinterpret_cast<f16x8*>(d) = x8.hi;
        *reinterpret_cast<f16x8*>(d + P::kPlane) = x8.lo;
      }
    }
  }
  __syncthreads();

  auto rows_of = [&](int isq, int t, int s) {  // operand rows: 16 tokens, 32 channels in order
    const char* d = s_kq + isq * 2 * P::kPlane + ((4 * s + q4) * (kC + 1) + 16 * t + n16) * 16;
    return Pair{*reinterpret_cast<const f16x8*>(d), *reinterpret_cast<const f16x8*>(d + P::kPlane)};
  };
  // k_j.k_i and k_j.q_i, rows j, columns i, in the units of a lower triangular
  // operand: w and w + 4 (what is above the diagonal stays 0)
  f32x4 kk[2][2] = {}, kq[2][2] = {};
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    const int u = w + 4 * n, t = lower_tile(u);
    if (u >= 6) continue;
#pragma unroll
    for (int s = 0; s < kKs; ++s) {
      const Pair k = rows_of(0, t, s), q = rows_of(1, t, s);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int j = 2 * lower_col(u) + e;
        if (j > t) continue;
        const Pair x = rows_of(0, j, s);
        kk[n][e] = mma3(x, k, kk[n][e]);
        kq[n][e] = mma3(x, q, kq[n][e]);
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
  for (int n = 0; n < kKs * 4 / kPrepWaves; ++n) {
    const int u = n * kPrepWaves + w, c = u / 2 * 16 + n16, s = u % 2;
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
      if (lane == kC - 1) sc[3 * kC] = f;
    }
    __syncthreads();
    // A, to be inverted, and Y
    for (int r = 0; r < nr; ++r) {
      const double* lg = s_log + r * kC;
      const int n16 = opaque(lane & 15), q4 = opaque(lane >> 4);
      char* y_out = value_at(a, slot, hk * per + r0 + r) + kYAt;
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const int u = w + 4 * n, i = 16 * lower_tile(u) + n16, j0 = 32 * lower_col(u) + 4 * q4;
        if (u >= 6) continue;
        const double li = lg[i];
        const float bi = s_beta[r * kC + i] * (1.0f / (kUnit * kUnit));
        float y[8];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          f32x4 x;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int j = j0 + 16 * e + k;
            const float f = j <= i ? __expf(float(li - lg[j])) : 0.0f;
            x[k] = j < i ? bi * kk[n][e][k] * f : 0.0f;
            y[4 * e + k] = kq[n][e][k] * f;
          }
          *reinterpret_cast<f32x4*>(s_t + (r * kC + i) * kLd + j0 + 16 * e) = x;
        }
        store_pair(y_out, u, lane, split(y, 1.0f / kUnit));
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
        __builtin_amdgcn_wave_barrier();  // rows are read before they are replaced
#pragma unroll
        for (int i = 0; i < 16; ++i) d[i * kLd + n16] = t[i];
      }
      __builtin_amdgcn_wave_barrier();
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
      __builtin_amdgcn_wave_barrier();
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
      f16_scale(column_max(group_max<16>(most)), scale, inv);
      if (lane == 0) {
        s_scale[w] = scale;
        reinterpret_cast<float*>(value_at(a, slot, hk * per + r0 + w) + kScalarsAt)[3 * kC + 1] = inv;
      }
    }
    __syncthreads();

    for (int r = 0; r < nr; ++r) {
      char* t_out = value_at(a, slot, hk * per + r0 + r);
      const int n16 = opaque(lane & 15), q4 = opaque(lane >> 4);
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const int u = w + 4 * n;
        if (u >= 6) continue;
        const float* x = s_t + (r * kC + 16 * lower_tile(u) + n16) * kLd + 32 * lower_col(u) + 4 * q4;
        const float4 y = *reinterpret_cast<const float4*>(x), z = *reinterpret_cast<const float4*>(x + 16);
        const float f[8] = {y.x, y.y, y.z, y.w, z.x, z.y, z.z, z.w};
        store_pair(t_out, u, lane, split(f, s_scale[r]));
      }
    }
    __syncthreads();  // the matrices are read
  }
}

// ---------------------------------------------------------------------------
// The chunks of a sequence in turn.  A wave holds the state of 16 value
// channels; the waves of a workgroup share the chunk's operands in LDS.
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
// ---------------------------------------------------------------------------
template <typename TIn, int DKP, int NW>
struct Scan {
  static constexpr int kKs = DKP / 32;
  static constexpr int kQ = kKs * 8 * kFrag;  // bytes of K, of Q, of K^T
  static constexpr int kPieces = NW * int(sizeof(TIn));  // 16 bytes each, of a row of raw values
  static constexpr int kRaw = ((kC + 3) * kPieces + kWave - 1) / kWave * kFrag;
  static constexpr int kLds = 3 * kQ + 24 * kFrag + 2 * kFrag + kRaw;
};

// This wave's loads and stores are done and its LDS reads; then the workgroup's.
template <int NW>
__device__ __forceinline__ void arrive() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
  if constexpr (NW > 1) __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// 64 lanes of 16 bytes to consecutive places of LDS
typedef __attribute__((address_space(3))) char* LdsPtr;
__device__ __forceinline__ void to_lds(const char* src, LdsPtr dst) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(src),
                                   (__attribute__((address_space(3))) void*)(dst), 16, 0, 0);
}

template <typename TIn, typename TOut, int DKP, int NW>
__global__ __launch_bounds__(NW * kWave) void scan_kernel(ChainArgs a, Part part) {
  typedef Scan<TIn, DKP, NW> S;
  constexpr int kKs = S::kKs;
  extern __shared__ __align__(16) char s_raw[];
  constexpr int kAtQ = S::kQ, kAtKt = 2 * S::kQ, kAtT = 3 * S::kQ, kAtY = kAtT + 12 * kFrag, kAtScalars = kAtY + 12 * kFrag,
                kAtV = kAtScalars + 2 * kFrag;
  const char *s_k = s_raw, *s_q = s_raw + kAtQ, *s_kt = s_raw + kAtKt, *s_t = s_raw + kAtT, *s_y = s_raw + kAtY, *s_v = s_raw + kAtV;
  const LdsPtr lds = (LdsPtr)s_raw;
  const int tid = threadIdx.x, lane = tid % kWave, w = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int n16 = lane & 15, q4 = lane >> 4;
  // workgroups go to the 8 XCDs in turn: those of a key head to one, whose L2
  // gives them K, Q and K^T
  const int each = gridDim.x * gridDim.y, id = blockIdx.y * gridDim.x + blockIdx.x;
  const int place = each % 8 == 0 ? id % 8 * (each / 8) + id / 8 : id;
  const int group = place % gridDim.x * NW + w, h = place / gridDim.x, b = part.b0 + blockIdx.z, hk = h / (a.Hv / a.Hk);
  const Tokens tk = tokens_of(a, b);
  const int dk = a.dk, dv = a.dv, end = min(part.c0 + part.M, (tk.n + kC - 1) / kC);
  if (part.c0 >= end) return;
  const SlotLayout l = slot_layout(a.Hk, a.Hv, dk);
  const int ch = group * 16 + n16;  // value channel
  const char* vws = value_at(a, slot_at(a, part, blockIdx.z, 0), h);
  const char* kws = key_at(a, slot_at(a, part, blockIdx.z, 0), hk);
  auto shared = [&](const char* src, int to, int frags) {  // by all waves
#pragma unroll
    for (int n = 0; n < (frags + NW - 1) / NW; ++n) {
      const int u = n * NW + w;
      if (frags % NW == 0 || u < frags) to_lds(src + u * kFrag + lane * 16, lds + to + u * kFrag);
    }
  };
  auto load_first = [&](int m) {  // K, Q, (I + A)^-1, scalars
    const char *k = kws + size_t(m) * l.total, *v = vws + size_t(m) * l.total;
    shared(k, 0, 2 * S::kQ / kFrag);
    shared(v, kAtT, 12);
    shared(v + kScalarsAt, kAtScalars + (m & 1) * kFrag, 1);
    asm volatile("" ::: "memory");
  };
  // Raw values of chunk m's tokens and the three before: row i at i kPieces,
  // its pieces traded by the quarter of i, so that the four rows of a read lie
  // on different banks.  Rows outside the sequence are read as its first or last.
  constexpr int kOwn = int(sizeof(TIn));  // pieces of 16 channels
  auto piece_of = [](int row, int piece) { return piece ^ (((row >> 2) & 3) * kOwn & (S::kPieces - 1)); };
  const char* values = reinterpret_cast<const char*>(reinterpret_cast<const TIn*>(a.v) + size_t(tk.first) * a.Hv * dv + h * dv +
                                                     (group - w) * 16);
  auto load_values = [&](int m) {
    const int n0 = (part.c0 + m) * kC - 3;
#pragma unroll
    for (int n = 0; n < (S::kRaw / kFrag + NW - 1) / NW; ++n) {
      const int u = n * NW + w, slot = u * kWave + lane, row = slot / S::kPieces, piece = piece_of(row, slot % S::kPieces);
      const int i = min(max(n0 + row, 0), tk.n - 1);
      if (u < S::kRaw / kFrag) to_lds(values + size_t(i) * a.Hv * dv * sizeof(TIn) + piece * 16, lds + kAtV + u * kFrag);
    }
  };
  auto load_second = [&](int m, int next) {  // Y, K^T, the next chunk's raw values
    shared(vws + size_t(m) * l.total + kYAt, kAtY, 12);
    shared(kws + size_t(m) * l.total + 2 * S::kQ, kAtKt, S::kQ / kFrag);
    load_values(next);
    asm volatile("" ::: "memory");
  };
  load_values(0);
  load_first(0);

  float* state = a.S + ((size_t(b) * a.Hv + h) * dv + ch) * dk + 4 * q4;
  f32x4 st[DKP / 16];  // key channels 16 n + 4 q4 ..
#pragma unroll
  for (int n = 0; n < DKP / 16; ++n) st[n] = 16 * n < dk ? *reinterpret_cast<const f32x4*>(state + 16 * n) : f32x4{};
  const size_t C = 2 * size_t(a.Hk) * dk + size_t(a.Hv) * dv, channel = 2 * size_t(a.Hk) * dk + h * dv + ch;
  const float4 cw = *reinterpret_cast<const float4*>(a.conv_w + channel * 4);
  float old[3];  // before the sequence's first token
#pragma unroll
  for (int i = 0; i < 3; ++i) old[i] = a.conv_state[(size_t(b) * 3 + i) * C + channel];
  TOut* out = reinterpret_cast<TOut*>(a.out) + (size_t(tk.first) * a.Hv + h) * dv + ch;
  float mx = 0.0f;  // the largest of this lane's values
#pragma unroll
  for (int n = 0; n < DKP / 16; ++n)
#pragma unroll
    for (int r = 0; r < 4; ++r) mx = fmaxf(mx, fabsf(st[n][r]));

  f32x4 v[4];  // convolved values of a chunk, rows 16 t + 4 q4 ..
  auto convolve = [&](int m, int t) {
    float x[7];
#pragma unroll
    for (int i = 0; i < 7; ++i) {
      const int row = 16 * t + 4 * q4 + i;
      x[i] = to_f32(*reinterpret_cast<const TIn*>(s_v + (row * S::kPieces + piece_of(row, (w * 16 + n16) * kOwn / 16)) * 16 +
                                                  n16 * kOwn % 16));
      if (t == 0 && i < 3 && part.c0 + m == 0 && q4 == 0) x[i] = old[i];
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) v[t][r] = silu(cw.x * x[r] + cw.y * x[r + 1] + cw.z * x[r + 2] + cw.w * x[r + 3]);
  };
  arrive<NW>();
#pragma unroll
  for (int t = 0; t < 4; ++t) convolve(0, t);

  f32x4 o[4];  // outputs of a chunk
  auto store = [&](int m) {
    const int n0 = (part.c0 + m) * kC;
    TOut* to = out + size_t(n0 + 4 * q4) * a.Hv * dv;
    if (n0 + kC <= tk.n) {
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) put(to + size_t(16 * t + r) * a.Hv * dv, o[t][r]);
    } else {
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (n0 + 16 * t + 4 * q4 + r < tk.n) put(to + size_t(16 * t + r) * a.Hv * dv, o[t][r]);
    }
    asm volatile("" ::: "memory");
  };

  for (int m = 0; m < end - part.c0; ++m) {
    const int next = min(m + 1, end - part.c0 - 1);  // the last chunk's again: they are not used
    const float* s_sc = reinterpret_cast<const float*>(s_raw + kAtScalars + (m & 1) * kFrag);
    float ss, is;  // the state as an operand
    f16_scale(column_max(mx), ss, is);
    Pair sp[kKs];
#pragma unroll
    for (int s = 0; s < kKs; ++s) {
      const float y[8] = {st[2 * s][0], st[2 * s][1], st[2 * s][2], st[2 * s][3],
                          st[2 * s + 1][0], st[2 * s + 1][1], st[2 * s + 1][2], st[2 * s + 1][3]};
      sp[s] = split(y, ss);
    }
    arrive<NW>();  // K, Q, (I + A)^-1, scalars; the last chunk's Y and K^T, the raw values are read
    if (m) store(m - 1);  // here: the next wait is a part away
    load_second(m, next);

    // K S^T and Q S^T.  Group n: token tiles 2 (n / kPer) and the next, kSteps
    // steps from n % kPer kSteps on.
    constexpr int kPer = kKs > 1 ? kKs / 2 : 1, kGroups = 2 * kPer, kSteps = kKs > 1 ? 2 : 1;
    Pair f[2][2 * kSteps];
    auto read = [&](Pair (&f)[2 * kSteps], const char* from, int n) {
#pragma unroll
      for (int k = 0; k < 2 * kSteps; ++k)
        f[k] = load_pair(from, (n % kPer * kSteps + k / 2) * 4 + n / kPer * 2 + k % 2, lane);
    };
    auto times = [&](const Pair (&f)[2 * kSteps], f32x4 (&c)[4], int n) {
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
    };
    // A lower triangular operand: tiles 0, 1 and the first step of 2, 3; then their second.
    Pair g[2][4];
    auto read_lower = [&](Pair (&f)[4], const char* from, int n) {
#pragma unroll
      for (int k = 0; k < 4 - 2 * n; ++k) f[k] = load_pair(from, n ? lower_step(2 + k, 1) : lower_step(k, 0), lane);
    };
    auto times_lower = [&](const Pair (&f)[4], const Pair& y, f32x4 (&c)[4], int n) {
#pragma unroll
      for (int k = 0; k < 4 - 2 * n; ++k) c[2 * n + k] = mma(f[k].lo, y.hi, c[2 * n + k]);
#pragma unroll
      for (int k = 0; k < 4 - 2 * n; ++k) c[2 * n + k] = mma(f[k].hi, y.lo, c[2 * n + k]);
#pragma unroll
      for (int k = 0; k < 4 - 2 * n; ++k) c[2 * n + k] = mma(f[k].hi, y.hi, c[2 * n + k]);
    };
    f32x4 x[4] = {};
#pragma unroll
    for (int t = 0; t < 4; ++t) o[t] = f32x4{};
    read(f[0], s_k, 0);
#pragma unroll
    for (int n = 0; n < kGroups; ++n) {
      if (n + 1 < kGroups) read(f[(n + 1) & 1], s_k, n + 1);
      else read(f[kGroups & 1], s_q, 0);
      __builtin_amdgcn_sched_barrier(0);
      times(f[n & 1], x, n);
      __builtin_amdgcn_sched_barrier(0);
    }
    // beta (V - e^g K S^T), beside half of the queries' products
    float mr = 0.0f, sr, ir;
    const float ik = is * (1.0f / kUnit);
#pragma unroll
    for (int n = 0; n < kGroups / 2; ++n) {
      read(f[(kGroups + n + 1) & 1], s_q, n + 1);
      __builtin_amdgcn_sched_barrier(0);
      times(f[(kGroups + n) & 1], o, n);
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
    f16_scale(column_max(mr), sr, ir);
    Pair rp[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const float y[8] = {x[2 * s][0], x[2 * s][1], x[2 * s][2], x[2 * s][3],
                          x[2 * s + 1][0], x[2 * s + 1][1], x[2 * s + 1][2], x[2 * s + 1][3]};
      rp[s] = split(y, sr);
    }
    read_lower(g[0], s_t, 0);
    read_lower(g[1], s_t, 1);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int t = 0; t < 4; ++t) x[t] = f32x4{};
    times_lower(g[0], rp[0], x, 0);
    times_lower(g[1], rp[1], x, 1);
    __builtin_amdgcn_sched_barrier(0);
    // V', and decayed to the chunk's end, beside the others
    float mv = 0.0f, md = 0.0f, sv, iv, sd, id;
    const float it = s_sc[3 * kC + 1] * ir, last = s_sc[3 * kC];
    f32x4 xd[4];
#pragma unroll
    for (int n = kGroups / 2; n < kGroups; ++n) {
      if (n + 1 < kGroups) read(f[(kGroups + n + 1) & 1], s_q, n + 1);
      __builtin_amdgcn_sched_barrier(0);
      times(f[(kGroups + n) & 1], o, n);
#pragma unroll
      for (int t = n * 8 / kGroups - 4; t < (n + 1) * 8 / kGroups - 4; ++t) {
        const f32x4 dec = *reinterpret_cast<const f32x4*>(s_sc + 2 * kC + 16 * t + 4 * q4);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          x[t][r] *= it;
          xd[t][r] = x[t][r] * dec[r];
          mv = fmaxf(mv, fabsf(x[t][r]));
          md = fmaxf(md, fabsf(xd[t][r]));
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    f16_scale(column_max(mv), sv, iv);
    f16_scale(column_max(md), sd, id);
    Pair vp[2], vd[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const float y[8] = {x[2 * s][0], x[2 * s][1], x[2 * s][2], x[2 * s][3],
                          x[2 * s + 1][0], x[2 * s + 1][1], x[2 * s + 1][2], x[2 * s + 1][3]};
      const float z[8] = {xd[2 * s][0], xd[2 * s][1], xd[2 * s][2], xd[2 * s][3],
                          xd[2 * s + 1][0], xd[2 * s + 1][1], xd[2 * s + 1][2], xd[2 * s + 1][3]};
      vp[s] = split(y, sv);
      vd[s] = split(z, sd);
    }
    arrive<NW>();  // Y, K^T, raw values; K, Q and (I + A)^-1 are read
    load_first(next);

    // outputs: Y V' beside Q S^T; then the state behind the chunk, and the next
    // chunk's values
    f32x4 y[4] = {};
    auto read_k = [&](Pair (&f)[4], int n) {
#pragma unroll
      for (int k = 0; k < 4; ++k) f[k] = load_pair(s_kt, 4 * n + k, lane);
    };
    read_lower(g[0], s_y, 0);
    read_lower(g[1], s_y, 1);
    __builtin_amdgcn_sched_barrier(0);
    times_lower(g[0], vp[0], y, 0);
    read_k(g[0], 0);
    __builtin_amdgcn_sched_barrier(0);
    times_lower(g[1], vp[1], y, 1);
    iv *= a.scale * (1.0f / kUnit);
    const float io = ik * a.scale;
    id *= 1.0f / kUnit;
    mx = 0.0f;
#pragma unroll
    for (int n = 0; n < DKP / 32; ++n) {
      if (n + 1 < DKP / 32) read_k(g[(n + 1) & 1], n + 1);
      __builtin_amdgcn_sched_barrier(0);
      f32x4 c[2] = {};
      const Pair(&f)[4] = g[n & 1];
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        c[0] = mma(f[s].lo, vd[s].hi, c[0]);
        c[1] = mma(f[2 + s].lo, vd[s].hi, c[1]);
        c[0] = mma(f[s].hi, vd[s].lo, c[0]);
        c[1] = mma(f[2 + s].hi, vd[s].lo, c[1]);
        c[0] = mma(f[s].hi, vd[s].hi, c[0]);
        c[1] = mma(f[2 + s].hi, vd[s].hi, c[1]);
      }
      // a share of the outputs and of the next values beside these products
#pragma unroll
      for (int t = n * 4 / (DKP / 32); t < (n + 1) * 4 / (DKP / 32); ++t) {
        const f32x4 dec = *reinterpret_cast<const f32x4*>(s_sc + kC + 16 * t + 4 * q4);
#pragma unroll
        for (int r = 0; r < 4; ++r) o[t][r] = o[t][r] * dec[r] * io + y[t][r] * iv;
        convolve(next, t);
      }
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          st[2 * n + e][r] = last * st[2 * n + e][r] + c[e][r] * id;
          mx = fmaxf(mx, fabsf(st[2 * n + e][r]));
        }
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  store(end - part.c0 - 1);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // nothing arrives in LDS after the end
#pragma unroll
  for (int n = 0; n < DKP / 16; ++n)
    if (16 * n < dk) *reinterpret_cast<f32x4*>(state + 16 * n) = st[n];
}

// The conv state behind the last token, and the statuses.
template <typename TIn>
__global__ __launch_bounds__(256) void tail_kernel(ChainArgs a) {
  const int b = blockIdx.y, nq = a.Hk * a.dk, nv = a.Hv * a.dv, C = 2 * nq + nv;
  const Tokens tk = tokens_of(a, b);
  if (a.status && blockIdx.x == 0 && threadIdx.x == 0) a.status[b] = tk.status;
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= C) return;
  const size_t at = size_t(b) * 3 * C + c;
#pragma unroll
  for (int s = 0; s < 3; ++s) {
    const int t = tk.n - 3 + s;
    float x;
    if (t < 0) x = a.conv_state[at + size_t(t + 3) * C];
    else if (c < nq) x = to_f32(reinterpret_cast<const TIn*>(a.q)[size_t(tk.first + t) * nq + c]);
    else if (c < 2 * nq) x = to_f32(reinterpret_cast<const TIn*>(a.k)[size_t(tk.first + t) * nq + c - nq]);
    else x = to_f32(reinterpret_cast<const TIn*>(a.v)[size_t(tk.first + t) * nv + c - 2 * nq]);
    a.conv_state_out[at + size_t(s) * C] = x;
  }
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

template <typename TIn, typename TOut, int DKP>
int launch_scan(const ChainArgs& a, const Part& p, hipStream_t stream) {
  // waves of a workgroup: as many as share a head, but a workgroup a CU
  const int groups = a.dv / 16;
  int nw = groups;
  while (nw > 1 && (long long)(p.G) * a.Hv * (groups / nw) < 192) nw /= 2;
  if (nw >= 8) return launch_waves<TIn, TOut, DKP, 8>(a, p, stream);
  if (nw == 4) return launch_waves<TIn, TOut, DKP, 4>(a, p, stream);
  if (nw == 2) return launch_waves<TIn, TOut, DKP, 2>(a, p, stream);
  return launch_waves<TIn, TOut, DKP, 1>(a, p, stream);
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
  const int C = 2 * a.Hk * a.dk + a.Hv * a.dv, G = p.G;
  if (a.in_dtype == GDN_BF16) tail_kernel<BF16><<<dim3((C + 255) / 256, a.B), 256, 0, stream>>>(a);
  else tail_kernel<float><<<dim3((C + 255) / 256, a.B), 256, 0, stream>>>(a);
  if ((rc = after_launch()) != GDN_OK) return rc;
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
