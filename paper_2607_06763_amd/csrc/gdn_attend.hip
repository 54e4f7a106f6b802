// gdn_attend.hip -- softmax attention of a step's slots over the paged cache.
//
// Rows.  The G = Hq / Hkv query heads of a key / value head read the same
// keys, so the queries of a (sequence, key head) are M = T G rows, row
// r = slot G + g.  Everything is computed transposed, with the rows as matrix
// columns: S^T = K Q^T, then O^T = V^T P^T on 32 x 32 tiles.  A lane then
// holds one row (lane mod 32) and half of a tile's keys or channels: softmax
// statistics are per lane, with one exchange between the halves, and P^T
// feeds the second product from the registers it was computed in.  For that,
// row m of a key tile holds key key_of(m), so that the accumulators of a lane
// are runs of kN consecutive keys, the packs in which the values are stored.
//
// Work.  The key tiles of all sequences, one after the other, are cut into S
// equal runs; a workgroup takes one run for one key head and one tile of
// rows.  A run may end one sequence and begin the next.  A sequence that one
// run covers is written at once; the parts of one that several runs share go
// to the workspace with their maximum and sum and are joined by a second
// kernel.  The lengths are on the device: every workgroup finds its run by a
// scan over them.
#include "gdn_attn.h"

namespace gdn {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef unsigned long long u64;

constexpr float kLog2e = 1.44269504088896340736f;
// The running maximum follows a larger score only past 8 octaves: weights
// stay below 2^8 and the sums in range, and most tiles rescale nothing.
constexpr float kSlack = 8.0f;

// ---------------------------------------------------------------------------
// Matrix tiles of either type
// ---------------------------------------------------------------------------
template <typename T>
struct Mat;

template <>
struct Mat<BF16> {
  typedef bf16x8 Frag;  // one pack
  static __device__ __forceinline__ f32x16 mma(Frag a, Frag b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
  // key of row m: bits 2 and 3 traded
  static __device__ __forceinline__ int key_of(int m) { return (m & 0x13) | ((m & 4) << 1) | ((m & 8) >> 1); }
  static __device__ __forceinline__ Frag pack(const float* p) {
    Frag f;
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = (__bf16)p[e];
    return f;
  }
  // bits of value e, and the pack without it
  static __device__ __forceinline__ unsigned bits(Frag f, int e) {
    return __builtin_bit_cast(u32x4, f)[e / 2] << (e & 1 ? 0 : 16) & 0xffff0000u;
  }
  static __device__ __forceinline__ Frag without(Frag f, int e) {
    u32x4 w = __builtin_bit_cast(u32x4, f);
    w[e / 2] &= e & 1 ? 0x0000ffffu : 0xffff0000u;
    return __builtin_bit_cast(Frag, w);
  }
};

template <>
struct Mat<float> {
  typedef f32x4 Frag;
  static __device__ __forceinline__ f32x16 mma(Frag a, Frag b, f32x16 c) {
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
    return c;
  }
  static __device__ __forceinline__ int key_of(int m) { return m; }
  static __device__ __forceinline__ Frag pack(const float* p) { return Frag{p[0], p[1], p[2], p[3]}; }
  static __device__ __forceinline__ unsigned bits(Frag f, int e) { return __float_as_uint(f[e]); }
  static __device__ __forceinline__ Frag without(Frag f, int e) {
    f[e] = 0.0f;
    return f;
  }
};

// The exponent of infinities and NaN, in the upper half of either type.
constexpr unsigned kExp = 0x7f800000u;

template <typename F>
__device__ __forceinline__ F load16(const void* p) {
  return *reinterpret_cast<const F*>(p);
}

// the other half's value: lane l gets max / sum of lanes l and l ^ 32
__device__ __forceinline__ float half_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// ---------------------------------------------------------------------------
// Schedule
// ---------------------------------------------------------------------------
// Positions of sequence b; -1 if it is skipped.
__device__ __forceinline__ int length_of(const AttnArgs& a, int b) {
  const int ctx = a.ctx_len[b], span = span_of(a, b);
  if (a.meta && meta_ptrs(a.meta, a.B, a.T).status[b] != 0) return -1;
  return len_status(a, ctx, span) ? -1 : ctx + span;
}

// A sequence without keys still has a tile: someone clears its outputs.
__device__ __forceinline__ int tiles_of(const AttnArgs& a, int b, int kt) {
  const int n = b < a.B ? length_of(a, b) : 0;
  return b < a.B ? (n > kt ? (n + kt - 1) / kt : 1) : 0;
}

// A value that every lane holds, in scalar registers.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ long long uniform(long long v) {
  return (long long)(unsigned(uniform(int(v)))) | (long long)(uniform(int(v >> 32))) << 32;
}

__device__ __forceinline__ long long wave_sum_ll(long long v) {
  for (int s = 1; s < kWave; s <<= 1) v += __shfl_xor(v, s);
  return uniform(v);
}

// Tiles of a run: all tiles over S, at least one.
__device__ __forceinline__ long long run_length(const AttnArgs& a, int S, int kt, long long* total) {
  long long n = 0;
  for (int b = threadIdx.x % kWave; b < (a.B + kWave - 1) / kWave * kWave; b += kWave) n += tiles_of(a, b, kt);
  n = wave_sum_ll(n);
  *total = n;
  return (n + S - 1) / S;
}

// Sequence that holds global tile g, and the tile at which it begins.
__device__ __forceinline__ void find_tile(const AttnArgs& a, long long g, int kt, int* b, long long* start) {
  const int lane = threadIdx.x % kWave;
  long long run = 0;
  for (int b0 = 0; b0 < a.B; b0 += kWave) {
    const int n = tiles_of(a, b0 + lane, kt);
    long long inc = n;
    for (int d = 1; d < kWave; d <<= 1) {
      const long long up = __shfl_up(inc, d);
      if (lane >= d) inc += up;
    }
    const u64 past = __ballot(run + inc > g);
    if (past) {
      const int at = __builtin_ctzll(past);
      *b = b0 + at;
      *start = uniform(run + __shfl(inc, at) - __shfl(n, at));
      return;
    }
    run = uniform(run + __shfl(inc, kWave - 1));
  }
  *b = a.B;
  *start = run;
}

// First global tile of sequence b.
__device__ __forceinline__ long long first_tile(const AttnArgs& a, int b, int kt) {
  long long n = 0;
  for (int i = threadIdx.x % kWave; i < b; i += kWave) n += tiles_of(a, i, kt);
  return wave_sum_ll(n);
}

// Workspace of the parts: slot 2 u + 1 of run u for a part that begins inside
// the run, 2 u for one that begins with it.
struct Parts {
  float* o;    // [2 S][Hkv][M][d]
  float2* ml;  // [2 S][Hkv][M]
};

// ---------------------------------------------------------------------------
// What a row sees
// ---------------------------------------------------------------------------
// Visibility of positions p0 .. p0 + 63 for slot i (bit 0 = p0).
__device__ __forceinline__ u64 seen_bits(const AttnArgs& a, const MetaPtrs& m, int b, int i, int ctx, int p0) {
  const int j0 = p0 - ctx;
  if (j0 <= -64) return ~u64(0);
  if (!a.meta) {
    const int n = ctx + i + 1 - p0;
    return n >= 64 ? ~u64(0) : n <= 0 ? 0 : (u64(1) << n) - 1;
  }
  const uint64_t* anc = m.anc + (size_t(b) * a.T + i) * m.W;
  auto word = [&](int k) {
    if (k < 0) return ~uint64_t(0);
    if (k >= m.W) return uint64_t(0);
    return anc[k] | (i >> 6 == k ? uint64_t(1) << (i & 63) : 0);
  };
  const int k = j0 >> 6, r = j0 & 63;
  const u64 lo = word(k);
  return r ? (lo >> r) | (word(k + 1) << (64 - r)) : lo;
}

// ---------------------------------------------------------------------------
// State of one wave's 32 rows
// ---------------------------------------------------------------------------
template <typename T, int D>
struct Rows {
  static constexpr int X = Pack<T>::kN;
  typedef Mat<T> M;
  typedef typename M::Frag Frag;
  Frag q[D / (2 * X)];
  f32x16 o[D / 32];
  float m, l;

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int k = 0; k < D / 32; ++k) o[k] = f32x16{};
    m = -INFINITY;
    l = 0.0f;
  }

  // queries of this lane's row (nullptr: zeros)
  __device__ __forceinline__ void load_q(const T* row, int h) {
#pragma unroll
    for (int k = 0; k < D / (2 * X); ++k) q[k] = row ? load16<Frag>(row + (2 * k + h) * X) : Frag{};
  }

  // Scores of N tiles of 32 keys to weights; c = scale log2(e).
  template <int N>
  __device__ __forceinline__ void softmax(float (&s)[N][16], float c) {
    float mx = s[0][0];
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[n][i]);
    mx = half_max(mx) * c;
    if (__any(mx > m + kSlack)) {
      const float to = fmaxf(m, mx);
      const float fix = to == m ? 1.0f : __builtin_amdgcn_exp2f(m - to);
#pragma unroll
      for (int k = 0; k < D / 32; ++k) o[k] *= fix;
      l *= fix;
      m = to;
    }
    const float ref = m == -INFINITY ? 0.0f : m;  // nothing seen yet
    float sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[n][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[n][i], c, -ref));
        sum[i & 1] += s[n][i];
      }
    l += sum[0] + sum[1];
  }

  // Values that are not finite take part by themselves, after a product that
  // ran without them: the matrix units count, for every row and channel, the
  // visible keys that hold +inf (or NaN) and -inf (or NaN).  value(q, k): the
  // pack as the cache holds it, seen: this lane's visible keys of 32.
  template <typename V>
  __device__ __forceinline__ void add_bad(unsigned seen, V value) {
    const int half = (threadIdx.x >> 5) & 1;
    const float one = 1.0f, none = 0.0f;
#pragma unroll
    for (int k = 0; k < D / 32; ++k) {
      f32x16 up = {}, down = {};
#pragma unroll
      for (int q = 0; q < 32 / (2 * X); ++q) {
        const Frag f = value(q, k);
        float on[X], hi[X], lo[X];
#pragma unroll
        for (int e = 0; e < X; ++e) {
          const unsigned x = M::bits(f, e);
          const bool inf = (x & kExp) == kExp, nan = inf && (x & 0x7fffffu);
          on[e] = (seen >> (q * 2 * X + half * X + e)) & 1 ? one : none;
          hi[e] = nan || (inf && !(x >> 31)) ? one : none;
          lo[e] = nan || (inf && (x >> 31)) ? one : none;
        }
        up = M::mma(M::pack(hi), M::pack(on), up);
        down = M::mma(M::pack(lo), M::pack(on), down);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        o[k][i] += up[i] > 0.0f ? INFINITY : 0.0f;
        o[k][i] += down[i] > 0.0f ? -INFINITY : 0.0f;
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }
};

// Position of a lane's row: slot, and whether the slot is real.
struct RowAt {
  int slot, head;  // head: query head
  bool real;
};

__device__ __forceinline__ RowAt row_at(const AttnArgs& a, const MetaPtrs& m, int b, int h, int r, int M, bool skip) {
  const int G = a.Hq / a.c.Hkv;
  RowAt w;
  w.slot = r < M ? r / G : 0;
  w.head = h * G + (r < M ? r % G : 0);
  w.real = r < M && !skip;
  if (w.real) w.real = a.meta ? m.depth[size_t(b) * a.T + w.slot] >= 0 : w.slot < span_of(a, b);
  return w;
}

template <typename T>
__device__ __forceinline__ size_t row_offset(const AttnArgs& a, int b, const RowAt& w) {
  return ((size_t(b) * a.T + w.slot) * a.Hq + w.head) * a.c.d;
}

// 4 outputs of a row
__device__ __forceinline__ void store4(float* p, float4 x) { *reinterpret_cast<float4*>(p) = x; }
__device__ __forceinline__ void store4(BF16* p, float4 x) {
  typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
  *reinterpret_cast<bf16x4*>(p) = bf16x4{(__bf16)x.x, (__bf16)x.y, (__bf16)x.z, (__bf16)x.w};
}

// ---------------------------------------------------------------------------
// Few rows: a workgroup's four waves share a tile of 32 rows and take 32 keys
// each of a tile of 128.  Keys and values go from memory to the operand
// registers (512 contiguous bytes per 32 lanes), a tile ahead of their use.
// ---------------------------------------------------------------------------
constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kStreamKeys = 32 * kWaves;

template <int D>
constexpr size_t stream_lds() {
  return sizeof(float) * kWaves * 32 * (D + 4) + sizeof(float2) * kWaves * 32;
}

// Registers of a wave: Q, K, V of 32 keys and O take D (2 X 4 / X^2 ..) each;
// a workgroup per SIMD wave pair up to here, one above.
template <typename T, int D>
constexpr int stream_groups() {
  return D * int(sizeof(T)) <= 256 ? 2 : 1;
}

template <typename T, int D>
__global__ __launch_bounds__(kThreads, (stream_groups<T, D>())) void attend_stream_kernel(AttnArgs a, int S, Parts ws) {
  constexpr int X = Pack<T>::kN, NK = D / (2 * X), NS = 32 / (2 * X);
  constexpr bool kAhead = D * int(sizeof(T)) <= 512;  // registers for a tile of keys and values ahead
  typedef Mat<T> Mt;
  typedef typename Mt::Frag Frag;
  extern __shared__ __align__(16) char s_raw[];
  float* s_o = reinterpret_cast<float*>(s_raw);                       // [wave][row][D + 4]
  float2* s_ml = reinterpret_cast<float2*>(s_o + kWaves * 32 * (D + 4));  // [wave][row]
  const int tid = threadIdx.x, lane = tid % kWave, w = uniform(tid / kWave), n32 = lane & 31, h2 = lane >> 5;
  const int u = blockIdx.x, h = blockIdx.y, rt = blockIdx.z;
  const int M = a.T * (a.Hq / a.c.Hkv);
  long long total;
  const long long run = run_length(a, S, kStreamKeys, &total);
  long long g = u * run;
  const long long end = g + run < total ? g + run : total;
  if (g >= end) return;
  int b;
  long long start;
  find_tile(a, g, kStreamKeys, &b, &start);

  const MetaPtrs m = meta_ptrs(a.meta, a.B, a.T);
  const T *kc = reinterpret_cast<const T*>(a.k_cache), *vc = reinterpret_cast<const T*>(a.v_cache);
  const int mask = (1 << a.c.page_shift) - 1, shift = a.c.page_shift;
  const float c = a.scale * kLog2e;
  for (; g < end; ++b) {
    const int tiles = uniform(tiles_of(a, b, kStreamKeys));
    const int t0 = int(g - start), n = int(min((long long)(tiles), end - start)) - t0;
    const bool whole = n == tiles;
    const int slot = 2 * u + (g > u * run ? 1 : 0);
    start += tiles;
    g = start;

    const int len = uniform(length_of(a, b)), ctx = uniform(a.ctx_len[b]);
    const int r = rt * 32 + n32;
    const RowAt at = row_at(a, m, b, h, r, M, len < 0);
    const int32_t* row = a.page_table + size_t(b) * a.c.max_pages;
    Rows<T, D> st;
    st.clear();
    st.load_q(at.real ? reinterpret_cast<const T*>(a.q) + row_offset<T>(a, b, at) : nullptr, h2);

    // 32 keys from p0: their two pages (16 keys never cross one)
    int p0 = (t0 * kWaves + w) * 32;
    const int key = Mt::key_of(n32);
    const T *vp0, *vp1;  // values of the first and the last 16 keys
    const T* kp;         // the lane's key
    unsigned valid;
    auto pages = [&](int p) {
      const int id0 = uniform(p < len ? page_of(a.c, row, p) : -1);
      const int id1 = uniform(p + 16 < len ? page_of(a.c, row, p + 16) : -1);
      const unsigned all = len - p >= 32 ? ~0u : (1u << (len - p)) - 1;  // p < len
      valid = (id0 >= 0 ? all & 0xffffu : 0) | (id1 >= 0 ? all & 0xffff0000u : 0);
      const size_t b0 = block_of(a.c, id0 < 0 ? 0 : id0, h), b1 = block_of(a.c, id1 < 0 ? 0 : id1, h);
      vp0 = vc + b0 + size_t(p & mask) * D;
      vp1 = vc + b1 + size_t((p + 16) & mask) * D;
      kp = kc + (key & 16 ? b1 : b0) + size_t((p + key) & mask) * X;
    };
    auto k_pack = [&](const T* p, int k) { return load16<Frag>(p + ((size_t(2 * k + h2) << shift) * X)); };
    auto v_pack = [&](int q, int k) {
      return load16<Frag>((q < NS / 2 ? vp0 : vp1) + ((2 * (q % (NS / 2)) + h2) * D + k * 32 + n32) * X);
    };
    // waves past the end have nothing to load
    const int last = min((t0 + n) * kStreamKeys, len < 0 ? 0 : len);
    if (p0 < last) pages(p0);
    if constexpr (kAhead) {
      // context: every row sees every key.  The next tile's keys load behind
      // the scores, its values behind the second product.
      if (p0 < last && p0 + 32 <= ctx && valid == ~0u) {
        Frag kf[NK], vf[NS][D / 32];
        auto load_k = [&]() {
#pragma unroll
          for (int k = 0; k < NK; ++k) kf[k] = k_pack(kp, k);
        };
        auto load_v = [&]() {
#pragma unroll
          for (int q = 0; q < NS; ++q)
#pragma unroll
            for (int k = 0; k < D / 32; ++k) vf[q][k] = v_pack(q, k);
        };
        load_k();
        load_v();
        for (bool more = true; more;) {
          f32x16 acc = {};
#pragma unroll
          for (int k = 0; k < NK; ++k) acc = Mt::mma(kf[k], st.q[k], acc);
          p0 += kStreamKeys;
          more = p0 < last;
          if (more) {
            pages(p0);
            more = p0 + 32 <= ctx && valid == ~0u;
          }
          if (more) load_k();
          float s[1][16];
#pragma unroll
          for (int i = 0; i < 16; ++i) s[0][i] = acc[i];
          st.template softmax<1>(s, c);
#pragma unroll
          for (int q = 0; q < NS; ++q) {
            const Frag p = Mt::pack(&s[0][q * X]);
#pragma unroll
            for (int k = 0; k < D / 32; ++k) st.o[k] = Mt::mma(vf[q][k], p, st.o[k]);
          }
          if (more) load_v();
        }
      }
    }
    // slots of the tree, the end of the cache and pages that are left out
    for (; p0 < last; p0 += kStreamKeys) {
      pages(p0);
      f32x16 acc = {};
#pragma unroll
      for (int k = 0; k < NK; ++k) acc = Mt::mma(k_pack(kp, k), st.q[k], acc);
      const bool masked = p0 + 32 > ctx || valid != ~0u;
      const unsigned seen = masked ? unsigned(seen_bits(a, m, b, at.slot, ctx, p0)) & valid : ~0u;
      float s[1][16];
#pragma unroll
      for (int i = 0; i < 16; ++i) s[0][i] = (seen >> (i / X * 2 * X + h2 * X + i % X)) & 1 ? acc[i] : -INFINITY;
      st.template softmax<1>(s, c);
      bool bad = false;
#pragma unroll
      for (int q = 0; q < NS; ++q) {
        const Frag p = Mt::pack(&s[0][q * X]);
        const unsigned ok = valid >> (q * 2 * X + h2 * X);
#pragma unroll
        for (int k = 0; k < D / 32; ++k) {
          Frag f = v_pack(q, k);
          if (masked) {  // a masked weight is 0, and must stay so whatever it meets
#pragma unroll
            for (int e = 0; e < X; ++e)
              if (!((ok >> e) & 1) || (Mt::bits(f, e) & kExp) == kExp) {
                bad = bad || ((ok >> e) & 1);
                f = Mt::without(f, e);
              }
          }
          st.o[k] = Mt::mma(f, p, st.o[k]);
        }
        __builtin_amdgcn_sched_barrier(0);  // one row of value packs in registers at a time
      }
      if (__any(bad))
        st.add_bad(seen, [&](int q, int k) {
          Frag f = v_pack(q, k);
#pragma unroll
          for (int e = 0; e < X; ++e)
            if (!((valid >> (q * 2 * X + h2 * X + e)) & 1)) f = Mt::without(f, e);
          return f;
        });
    }

    // join the waves
    const float l = half_sum(st.l);
    if (h2 == 0) s_ml[w * 32 + n32] = make_float2(st.m, l);
    if (r < M) {
#pragma unroll
      for (int k = 0; k < D / 32; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *reinterpret_cast<float4*>(s_o + (w * 32 + n32) * (D + 4) + k * 32 + 8 * i + 4 * h2) =
              make_float4(st.o[k][4 * i], st.o[k][4 * i + 1], st.o[k][4 * i + 2], st.o[k][4 * i + 3]);
    }
    __syncthreads();
    const int rows = min(32, M - rt * 32);
    for (int x = tid; x < rows * (D / 4); x += kThreads) {
      const int rr = x / (D / 4), d = x % (D / 4) * 4;
      float mx = -INFINITY;
#pragma unroll
      for (int k = 0; k < kWaves; ++k) mx = fmaxf(mx, s_ml[k * 32 + rr].x);
      float sum = 0.0f;
      float4 o = make_float4(0, 0, 0, 0);
#pragma unroll
      for (int k = 0; k < kWaves; ++k) {
        const float2 ml = s_ml[k * 32 + rr];
        const float f = ml.x == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(ml.x - mx);
        const float4 y = *reinterpret_cast<const float4*>(s_o + (k * 32 + rr) * (D + 4) + d);
        if (ml.x == -INFINITY && ml.y == 0.0f) continue;
        sum += f * ml.y;
        o.x += f * y.x, o.y += f * y.y, o.z += f * y.z, o.w += f * y.w;
      }
      if (whole) {
        const RowAt to = row_at(a, m, b, h, rt * 32 + rr, M, len < 0);
        const float inv = to.real && sum != 0.0f ? 1.0f / sum : 0.0f;
        const bool on = to.real && sum != 0.0f;
        store4(reinterpret_cast<T*>(a.out) + row_offset<T>(a, b, to) + d,
               on ? make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv) : make_float4(0, 0, 0, 0));
      } else {
        const size_t i = (size_t(slot) * a.c.Hkv + h) * M + rt * 32 + rr;
        *reinterpret_cast<float4*>(ws.o + i * D + d) = o;
        if (d == 0) ws.ml[i] = make_float2(mx, sum);
      }
    }
    __syncthreads();  // before the next sequence's part overwrites the waves' rows
  }
}

// ---------------------------------------------------------------------------
// Joins the parts of the sequences that several runs share.
// ---------------------------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(kThreads) void attend_join_kernel(AttnArgs a, int S, int kt, Parts ws) {
  const int b = blockIdx.z, h = blockIdx.y, D = a.c.d, M = a.T * (a.Hq / a.c.Hkv);
  long long total;
  const long long run = run_length(a, S, kt, &total);
  const long long t0 = first_tile(a, b, kt), t1 = t0 + tiles_of(a, b, kt) - 1;
  const int u0 = int(t0 / run), u1 = int(t1 / run);
  if (u0 == u1) return;
  const int per = kThreads / (D / 4), r = blockIdx.x * per + threadIdx.x / (D / 4), d = threadIdx.x % (D / 4) * 4;
  if (r >= M) return;
  const MetaPtrs m = meta_ptrs(a.meta, a.B, a.T);
  const RowAt at = row_at(a, m, b, h, r, M, false);
  auto part = [&](int u) { return (size_t(2 * u + (u == u0 && t0 > u0 * run ? 1 : 0)) * a.c.Hkv + h) * M + r; };
  float mx = -INFINITY;
  for (int u = u0; u <= u1; ++u) mx = fmaxf(mx, ws.ml[part(u)].x);
  float sum = 0.0f;
  float4 o = make_float4(0, 0, 0, 0);
  for (int u = u0; u <= u1; ++u) {
    const size_t i = part(u);
    const float2 ml = ws.ml[i];
    if (ml.x == -INFINITY && ml.y == 0.0f) continue;
    const float f = ml.x == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(ml.x - mx);
    const float4 y = *reinterpret_cast<const float4*>(ws.o + i * D + d);
    sum += f * ml.y;
    o.x += f * y.x, o.y += f * y.y, o.z += f * y.z, o.w += f * y.w;
  }
  const bool on = at.real && sum != 0.0f;
  const float inv = on ? 1.0f / sum : 0.0f;
  store4(reinterpret_cast<T*>(a.out) + row_offset<T>(a, b, at) + d,
         on ? make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv) : make_float4(0, 0, 0, 0));
}

int after_launch() {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? GDN_OK : set_error(GDN_EHIP, "attend: launch: %s", hipGetErrorString(e));
}

// Runs for `blocks` workgroups per run on `slots` workgroup places: as many as
// fill the places, in up to four rounds where fewer would leave more than a
// tenth of them empty.
int runs_for(long long blocks, long long slots) {
  long long best = 1;
  double fill = 0.0;
  for (int rounds = 1; rounds <= 4; ++rounds) {
    const long long S = rounds * slots / blocks;
    if (S < 1) continue;
    const double f = double(S * blocks) / double(rounds * slots);
    if (f > fill) fill = f, best = S;
    if (fill >= 0.9) break;
  }
  return int(best);
}

template <typename T, int D>
int launch_stream(const AttnArgs& a, hipStream_t stream) {
  const int M = a.T * (a.Hq / a.c.Hkv), rt = (M + 31) / 32;
  const int S = runs_for((long long)(a.c.Hkv) * rt, 256 * stream_groups<T, D>());
  const size_t rows = size_t(2) * S * a.c.Hkv * M;
  int rc = GDN_OK;
  char* p = static_cast<char*>(stream_workspace(rows * (D * sizeof(float) + sizeof(float2)), stream, &rc));
  if (!p) return rc;
  const Parts ws = {reinterpret_cast<float*>(p), reinterpret_cast<float2*>(p + rows * D * sizeof(float))};
  constexpr size_t lds = stream_lds<D>();
  rc = ensure_dynamic_lds(reinterpret_cast<const void*>(attend_stream_kernel<T, D>), int(lds), "attend");
  if (rc != GDN_OK) return rc;
  attend_stream_kernel<T, D><<<dim3(S, a.c.Hkv, rt), kThreads, lds, stream>>>(a, S, ws);
  if ((rc = after_launch()) != GDN_OK || S == 1) return rc;
  const int per = kThreads / (D / 4);
  attend_join_kernel<T><<<dim3((M + per - 1) / per, a.c.Hkv, a.B), kThreads, 0, stream>>>(a, S, kStreamKeys, ws);
  return after_launch();
}

template <typename T>
int launch_type(const AttnArgs& a, hipStream_t stream) {
  switch (a.c.d) {
    case 32: return launch_stream<T, 32>(a, stream);
    case 64: return launch_stream<T, 64>(a, stream);
    case 128: return launch_stream<T, 128>(a, stream);
    default: return launch_stream<T, 256>(a, stream);
  }
}

}  // namespace

int launch_attend(const AttnArgs& a, hipStream_t stream) {
  return a.dtype == GDN_BF16 ? launch_type<BF16>(a, stream) : launch_type<float>(a, stream);
}

}  // namespace gdn
