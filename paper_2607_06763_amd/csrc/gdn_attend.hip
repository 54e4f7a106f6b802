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
#include <limits.h>

#include <algorithm>

#include "gdn_attn.h"
#include "gdn_workspace.h"

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
  // weights as the second product's operand: bf16, as the instruction takes them
  // (at most 2^-8 of each; sums and maxima stay in 32 bits).  Outputs are off by
  // 0.0023 of their norm, 0.0017 of it from their own rounding.
  static __device__ __forceinline__ Frag pack(const float* p) {
    Frag f;
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = (__bf16)p[e];
    return f;
  }
  // whether any value is infinite or NaN: a full exponent reaches the sign's place
  static __device__ __forceinline__ bool odd(Frag f) {
    const u32x4 t = (__builtin_bit_cast(u32x4, f) & 0x7f807f80u) + 0x00800080u;
    return (t[0] | t[1] | t[2] | t[3]) & 0x80008000u;
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
// A sequence: its cached positions, those with the step's (-1 if it is
// skipped), and its tiles.  One without keys still has a tile: someone clears
// its outputs.
struct Seq {
  int ctx, len, tiles;
};

__device__ __forceinline__ Seq seq_of(const AttnArgs& a, int b, int kt) {
  if (b >= a.B) return {0, 0, 0};
  const int ctx = a.ctx_len[b], span = span_of(a, b);
  const bool bad = a.meta && meta_ptrs(a.meta, a.B, a.T).status[b] != 0;
  const int len = bad || len_status(a, ctx, span) ? -1 : ctx + span;
  return {ctx, len, len > kt ? (len + kt - 1) / kt : 1};
}

// A value that every lane holds, in scalar registers.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ long long uniform(long long v) {
  return (long long)(unsigned(uniform(int(v)))) | (long long)(uniform(int(v >> 32))) << 32;
}

// Inclusive prefix over the lanes, in DPP steps (the shuffles of a wider type
// through LDS took a microsecond of the smallest calls).
__device__ __forceinline__ unsigned wave_scan(unsigned v) {
#define GDN_STEP(ctrl, rows) v += unsigned(__builtin_amdgcn_update_dpp(0, int(v), ctrl, rows, 0xF, false))
  GDN_STEP(0x111, 0xF);  // row_shr by 1, 2, 4, 8
  GDN_STEP(0x112, 0xF);
  GDN_STEP(0x114, 0xF);
  GDN_STEP(0x118, 0xF);
  GDN_STEP(0x142, 0xA);  // row 0's last lane to row 1, row 2's to row 3
  GDN_STEP(0x143, 0xC);  // lane 31 to rows 2 and 3
#undef GDN_STEP
  return v;
}

// The tiles of all sequences in a row, cut into S equal runs.  Lane l keeps
// sequence l of the first 64, so that these are loaded once.  Tiles of 64
// sequences stay below 2^32 (a page table's row spans at most 2^30 positions, a
// tile at least 32).
struct Schedule {
  Seq own;
  unsigned upto;        // tiles of sequences 0 .. lane
  long long total, run;  // tiles of all sequences, of a run
};

__device__ __forceinline__ Schedule schedule(const AttnArgs& a, int S, int kt) {
  const int lane = threadIdx.x % kWave;
  Schedule r;
  r.own = seq_of(a, lane, kt);
  r.upto = wave_scan(r.own.tiles);
  r.total = unsigned(__builtin_amdgcn_readlane(int(r.upto), kWave - 1));
  for (int b0 = kWave; b0 < a.B; b0 += kWave)
    r.total += unsigned(__builtin_amdgcn_readlane(int(wave_scan(seq_of(a, b0 + lane, kt).tiles)), kWave - 1));
  r.total = uniform(r.total);
  const long long most = r.total + S - 1;
  r.run = uniform(most >> 32 ? most / S : (long long)(unsigned(most) / unsigned(S)));
  return r;
}

__device__ __forceinline__ Seq seq_at(const AttnArgs& a, const Schedule& w, int b, int kt) {
  if (b < kWave)
    return {__builtin_amdgcn_readlane(w.own.ctx, b), __builtin_amdgcn_readlane(w.own.len, b),
            __builtin_amdgcn_readlane(w.own.tiles, b)};
  const Seq x = seq_of(a, b, kt);
  return {uniform(x.ctx), uniform(x.len), uniform(x.tiles)};
}

// Sequence that holds global tile g, and the tile at which it begins.
__device__ __forceinline__ void find_tile(const AttnArgs& a, const Schedule& w, long long g, int kt, int* b, long long* start) {
  const int lane = threadIdx.x % kWave;
  long long before = 0;
  int n = w.own.tiles;
  unsigned inc = w.upto;
  for (int b0 = 0;;) {
    const u64 past = __ballot(before + inc > g);
    if (past) {
      const int at = __builtin_ctzll(past);
      *b = b0 + at;
      *start = uniform(before + unsigned(__builtin_amdgcn_readlane(int(inc), at)) - __builtin_amdgcn_readlane(n, at));
      return;
    }
    before = uniform(before + unsigned(__builtin_amdgcn_readlane(int(inc), kWave - 1)));
    b0 += kWave;
    if (b0 >= a.B) break;
    n = seq_of(a, b0 + lane, kt).tiles;
    inc = wave_scan(n);
  }
  *b = a.B;
  *start = before;
}

// First global tile of sequence b.
__device__ __forceinline__ long long first_tile(const AttnArgs& a, const Schedule& w, int b, int kt) {
  const int lane = threadIdx.x % kWave;
  long long n = 0;
  if (b < kWave) return b ? unsigned(__builtin_amdgcn_readlane(int(w.upto), b - 1)) : 0;
  for (int b0 = 0; b0 < b; b0 += kWave) {
    const int i = b0 + lane;
    n += unsigned(__builtin_amdgcn_readlane(int(wave_scan(i < b ? seq_of(a, i, kt).tiles : 0)), kWave - 1));
  }
  return uniform(n);
}

// Workspace of the parts: slot 2 u + 1 of run u for a part that begins inside
// the run, 2 u for one that begins with it.  A row that sees nothing there,
// and one of a padding slot, has maximum -inf and sum 0.
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

// First position that no row up to `r` sees: in a chain that of the next slot
// (prompts from their start, heads of 128: 2 x 400 tokens in fp32 63 us, 87 with
// all tiles, 2 x 512 in bf16 36 and 40); the slots of a tree are in any order.
__device__ __forceinline__ int end_of_rows(const AttnArgs& a, int ctx, int len, int r) {
  if (len < 0) return 0;  // a skipped sequence
  return a.meta ? len : min(len, ctx + r / (a.Hq / a.c.Hkv) + 1);
}

// x where bit n of seen is set, else -inf.
__device__ __forceinline__ float where_seen(float x, unsigned seen, int n) {
  const int on = __builtin_amdgcn_sbfe(int(seen), n, 1);  // 0 or -1
  return __int_as_float((__float_as_int(x) & on) | (0xff800000 & ~on));
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

  // The running maximum for N tiles of 32 scores (c = scale log2(e)); returns
  // what a weight's exponent is counted from.
  template <int N>
  __device__ __forceinline__ float follow(const float (&s)[N][16], float c) {
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
    return m == -INFINITY ? 0.0f : m;  // nothing seen yet
  }

  // Scores to weights.
  template <int N>
  __device__ __forceinline__ void softmax(float (&s)[N][16], float c) {
    const float ref = follow<N>(s, c);
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
};

// Position of a lane's row: slot, and whether the slot is real.
struct RowAt {
  int slot, head;  // head: query head
  bool real;
};

__device__ __forceinline__ RowAt row_of(const AttnArgs& a, int h, int r) {
  const int G = a.Hq / a.c.Hkv;
  return {r / G, h * G + r % G, true};
}

__device__ __forceinline__ RowAt row_at(const AttnArgs& a, const MetaPtrs& m, int b, int h, int r, int M, bool skip) {
  RowAt w = row_of(a, h, r < M ? r : 0);
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

__device__ __forceinline__ float4 fetch4(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ float4 fetch4(const BF16* p) { return ld4(p); }

// Where some slots are masked, the product runs without the values that are
// not finite (0 times infinity is not 0).  This adds them to 4 channels of
// what a row has written: those of the keys from position `from` up to `to`
// that the row sees.
template <typename T, typename O>
__device__ void add_not_finite(const AttnArgs& a, const MetaPtrs& m, int b, int h, int slot, int ctx, int from, int to,
                               int d, O* out) {
  constexpr int X = Pack<T>::kN;
  const int32_t* row = a.page_table + size_t(b) * a.c.max_pages;
  const int mask = (1 << a.c.page_shift) - 1;
  float x[4] = {};
  for (int p0 = from; p0 < to; p0 += 64) {
    u64 seen = seen_bits(a, m, b, slot, ctx, p0);
    if (to - p0 < 64) seen &= (u64(1) << (to - p0)) - 1;
    for (; seen; seen &= seen - 1) {
      const int p = p0 + __builtin_ctzll(seen), id = page_of(a.c, row, p);
      if (id < 0) continue;
      const T* v = reinterpret_cast<const T*>(a.v_cache) + block_of(a.c, id, h) +
                   (size_t((p & mask) / X) * a.c.d + d) * X + p % X;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float y = to_f32(v[e * X]);
        if ((__float_as_uint(y) & kExp) == kExp) x[e] += y;
      }
    }
  }
  const float4 o = fetch4(out);
  store4(out, make_float4(o.x + x[0], o.y + x[1], o.z + x[2], o.w + x[3]));
}

// ---------------------------------------------------------------------------
// Few rows: a workgroup's four waves share a tile of 32 rows and take 32 keys
// each of a tile of 128.  Keys and values go from memory to the operand
// registers (512 contiguous bytes per 32 lanes), ahead of their use.
//
// Bound by the bytes of the cache (32 x 1 token, 32 + 8 heads of 128 in bf16,
// up to 8 k tokens: 656 MB in 117 to 120 us, 5.5 TB/s; a large copy reaches 5.1), with
// a short cache by the chain lengths - pages - keys - values - parts (10 us),
// in fp32 by the products, which take 16 times those of bf16: 6 x 14 nodes,
// 48 + 8 heads of 128, 9 k tokens 159 us, of which about 136 are products (a
// quarter on rows that fill up the tiles); 8 x 99 nodes, 16 + 4 heads of 64,
// 1 k tokens 45 us, of which the products (2.6 GFLOP with the rows that fill up
// the tiles) take 17 at the matrix units' rate and the join 6: a run is 5 or 6
// key tiles behind the chain.  32 x 1 token in fp32: 1312 MB in 245 us.
//
// Scalar registers spill into lanes of vector registers (up to 121 of them);
// to memory only fp32 heads of 256 do, two registers.
// ---------------------------------------------------------------------------
constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kStreamKeys = 32 * kWaves;

template <int D>
constexpr size_t stream_lds() {
  return sizeof(float) * kWaves * 32 * (D + 4) + sizeof(float2) * kWaves * 32 + 16;
}

// Workgroups a CU: two where the registers allow (Q, O and 32 keys and values
// ahead).  fp32 heads of 64 dims, 8 x 99 nodes: 45 us, 55 with one; bf16 of 128,
// 16 x 1 token over 8 k: 40.8 and 42.0, over 600 (4 x 1): 13.1 and 12.2.
template <typename T, int D>
constexpr int stream_groups() {
  return D * int(sizeof(T)) <= 256 ? 2 : 1;
}

template <typename T, int D>
__global__ __launch_bounds__(kThreads, (stream_groups<T, D>())) void attend_stream_kernel(AttnArgs a, int S, Parts ws) {
  constexpr int X = Pack<T>::kN, NK = D / (2 * X), NS = 32 / (2 * X);
  // A whole tile of keys and values ahead, where registers hold it: fp32 heads
  // of 128 dims 159 us (167 without; 6 x 14 nodes, 9 k tokens).  bf16 heads of
  // 256, which it fits only with spills: 49 us, 42 without (16 x 1, 8 k).
  constexpr bool kAhead = D <= 128;
  typedef Mat<T> Mt;
  typedef typename Mt::Frag Frag;
  extern __shared__ __align__(16) char s_raw[];
  float* s_o = reinterpret_cast<float*>(s_raw);                       // [wave][row][D + 4]
  float2* s_ml = reinterpret_cast<float2*>(s_o + kWaves * 32 * (D + 4));  // [wave][row]
  int* s_from = reinterpret_cast<int*>(s_ml + kWaves * 32);  // first tile with values left out, two segments in turn
  int turn = 0;
  const int tid = threadIdx.x, lane = tid % kWave, w = uniform(tid / kWave), n32 = lane & 31, h2 = lane >> 5;
  const int u = blockIdx.x, h = blockIdx.y, rt = blockIdx.z;
  const int M = a.T * (a.Hq / a.c.Hkv);
  const Schedule plan = schedule(a, S, kStreamKeys);
  const long long run = plan.run, total = plan.total;
  long long g = u * run;
  const long long end = g + run < total ? g + run : total;
  if (g >= end) return;
  int b;
  long long start;
  find_tile(a, plan, g, kStreamKeys, &b, &start);

  const MetaPtrs m = meta_ptrs(a.meta, a.B, a.T);
  const T *kc = reinterpret_cast<const T*>(a.k_cache), *vc = reinterpret_cast<const T*>(a.v_cache);
  const int mask = (1 << a.c.page_shift) - 1, shift = a.c.page_shift;
  const float c = a.scale * kLog2e;
  for (; g < end; ++b, s_from += turn ? -1 : 1, turn ^= 1) {
    const Seq seq = seq_at(a, plan, b, kStreamKeys);
    const int tiles = seq.tiles, len = seq.len, ctx = seq.ctx;
    const int t0 = int(g - start), n = int(min((long long)(tiles), end - start)) - t0;
    const bool whole = n == tiles;
    const int slot = 2 * u + (g > u * run ? 1 : 0);
    start += tiles;
    g = start;

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
    const T* kp;         // the lane's first pack of its key
    unsigned valid;
    auto entry = [&](int p) { return row[p < len ? p >> shift : 0]; };
    auto set_pages = [&](int p, int e0, int e1) {  // of their page-table entries
      const bool on0 = p < len && unsigned(e0) < unsigned(a.c.n_pages);
      const bool on1 = p + 16 < len && unsigned(e1) < unsigned(a.c.n_pages);
      const unsigned all = len - p >= 32 ? ~0u : (1u << (len - p)) - 1;  // p < len
      valid = (on0 ? all & 0xffffu : 0) | (on1 ? all & 0xffff0000u : 0);
      const size_t b0 = block_of(a.c, on0 ? e0 : 0, h), b1 = block_of(a.c, on1 ? e1 : 0, h);
      vp0 = vc + b0 + size_t(p & mask) * D;
      vp1 = vc + b1 + size_t((p + 16) & mask) * D;
      kp = kc + (key & 16 ? b1 : b0) + (size_t((p + key) & mask) + (size_t(h2) << shift)) * X;
    };
    auto pages = [&](int p) {
      const int e0 = entry(p), e1 = entry(p + 16);
      set_pages(p, uniform(e0), uniform(e1));
    };
    auto k_pack = [&](const T* p, int k) { return load16<Frag>(p + (2 * k * X << shift)); };
    auto v_pack = [&](int q, int k) {
      return load16<Frag>((q < NS / 2 ? vp0 : vp1) + ((2 * (q % (NS / 2)) + h2) * D + k * 32 + n32) * X);
    };
    // waves past what the rows see have nothing to load
    const int last = min((t0 + n) * kStreamKeys, end_of_rows(a, ctx, len, rt * 32 + 31));
    int from = INT_MAX;
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
    // slots of the tree, the end of the cache and pages that are left out, and
    // all keys where the registers do not hold a tile ahead: packs load a group
    // ahead of their products, the next tile's first keys behind the last values
    constexpr int kG = NK < 4 ? NK : 4;
    Frag kf[2][kG], vf[2][D / 32];
    auto k_group = [&](Frag (&f)[kG], int n) {
#pragma unroll
      for (int k = 0; k < kG; ++k) f[k] = k_pack(kp, n * kG + k);
    };
    auto v_row = [&](Frag (&f)[D / 32], int q) {
#pragma unroll
      for (int k = 0; k < D / 32; ++k) f[k] = v_pack(q, k);
    };
    if (p0 < last) k_group(kf[0], 0);
    while (p0 < last) {
      const int e0 = entry(p0 + kStreamKeys), e1 = entry(p0 + kStreamKeys + 16);
      f32x16 acc = {};
#pragma unroll
      for (int n = 0; n < NK / kG; ++n) {
        if (n + 1 < NK / kG) k_group(kf[(n + 1) & 1], n + 1);
        else v_row(vf[0], 0);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int k = 0; k < kG; ++k) acc = Mt::mma(kf[n & 1][k], st.q[n * kG + k], acc);
        __builtin_amdgcn_sched_barrier(0);
      }
      const bool masked = p0 + 32 > ctx || valid != ~0u;
      const unsigned seen = masked ? unsigned(seen_bits(a, m, b, at.slot, ctx, p0)) & valid : ~0u;
      const unsigned there = valid;
      float s[1][16];
#pragma unroll
      for (int i = 0; i < 16; ++i) s[0][i] = where_seen(acc[i], seen >> (h2 * X), i / X * 2 * X + i % X);
      st.template softmax<1>(s, c);
      bool left = false;
      const int now = p0;
#pragma unroll
      for (int q = 0; q < NS; ++q) {
        if (q + 1 < NS) {
          v_row(vf[(q + 1) & 1], q + 1);
        } else {
          p0 += kStreamKeys;
          if (p0 < last) {
            set_pages(p0, uniform(e0), uniform(e1));
            k_group(kf[0], 0);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
        const Frag p = Mt::pack(&s[0][q * X]);
        const unsigned ok = there >> (q * 2 * X + h2 * X);
#pragma unroll
        for (int k = 0; k < D / 32; ++k) {
          Frag f = vf[q & 1][k];
          if (masked) {  // a masked weight is 0, and must stay so whatever it meets
#pragma unroll
            for (int e = 0; e < X; ++e)
              if (!((ok >> e) & 1) || (Mt::bits(f, e) & kExp) == kExp) {
                left = left || ((ok >> e) & 1);
                f = Mt::without(f, e);
              }
          }
          st.o[k] = Mt::mma(f, p, st.o[k]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      if (from == INT_MAX && __any(left)) from = now;
    }

    // join the waves
    if (tid == 0) *s_from = INT_MAX;
    const float l = half_sum(st.l);
    if (h2 == 0) s_ml[w * 32 + n32] = at.real ? make_float2(st.m, l) : make_float2(-INFINITY, 0.0f);
    if (r < M) {
#pragma unroll
      for (int k = 0; k < D / 32; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *reinterpret_cast<float4*>(s_o + (w * 32 + n32) * (D + 4) + k * 32 + 8 * i + 4 * h2) =
              make_float4(st.o[k][4 * i], st.o[k][4 * i + 1], st.o[k][4 * i + 2], st.o[k][4 * i + 3]);
    }
    __syncthreads();
    if (from != INT_MAX && lane == 0) atomicMin(s_from, from);
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
        const bool on = sum != 0.0f;
        const float inv = on ? 1.0f / sum : 0.0f;
        store4(reinterpret_cast<T*>(a.out) + row_offset<T>(a, b, row_of(a, h, rt * 32 + rr)) + d,
               on ? make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv) : make_float4(0, 0, 0, 0));
      } else {
        const size_t i = (size_t(slot) * a.c.Hkv + h) * M + rt * 32 + rr;
        *reinterpret_cast<float4*>(ws.o + i * D + d) = o;
        if (d == 0) ws.ml[i] = make_float2(mx, sum);
      }
    }
    __syncthreads();  // before the next sequence's part overwrites the waves' rows
    if (*s_from != INT_MAX) {
      from = *s_from;
      for (int x = tid; x < rows * (D / 4); x += kThreads) {
        const int rr = x / (D / 4), d = x % (D / 4) * 4;
        const RowAt to = row_at(a, m, b, h, rt * 32 + rr, M, false);
        if (!to.real) continue;
        const int upto = min((t0 + n) * kStreamKeys, len);
        if (whole)
          add_not_finite<T>(a, m, b, h, to.slot, ctx, from, upto, d, reinterpret_cast<T*>(a.out) + row_offset<T>(a, b, to) + d);
        else
          add_not_finite<T>(a, m, b, h, to.slot, ctx, from, upto, d,
                            ws.o + ((size_t(slot) * a.c.Hkv + h) * M + rt * 32 + rr) * D + d);
      }
      __syncthreads();
    }
  }
}

// ---------------------------------------------------------------------------
// Many rows (bf16): four waves of 32 rows each share key and value tiles in
// LDS, double-buffered and loaded past the registers.  The cache's packs are
// the operand layout, so a tile is copied as it stands and read without bank
// conflicts (32 lanes read 512 contiguous bytes).
//
// A wave issues in order, so the scores of the next tile are computed between
// the exponentials of this one, a product and the work of 256 / d scores in
// turn: the matrix units run while the others do.  Operands come from LDS a
// group ahead of their products (left to itself the compiler waits for each).
// Up to d = 128 two workgroups a CU (16 x 128 nodes over 8 k tokens 240 us, 299
// with one; 16 x 16 nodes 62.8 and 58.9); at 256 one, with the registers of both.
//
// 32 + 8 heads of 128, 16 x 128 nodes, up to 8 k tokens: 177 GFLOP in 239 to
// 255 us with the join (20), 690 to 740 TFLOP/s; a large bf16 product reaches
// 1270.  The matrix units are busy 39 % of the time and the vector units 44 %
// (counters), so neither bounds it alone: a tile takes the two waves of a SIMD
// 5300 clocks, 2048 of them products.  Each product has an operand read of its
// own from LDS, 1 KB (5.6 M of each), because a wave holds 32 rows: products
// without a pause on all four SIMDs would take the 128 bytes a clock that LDS
// gives, before the tiles' own way into it.  The first tile and the outputs of a
// run are not overlapped, which is what the short calls wait for (27 x 90 nodes
// over 850 tokens 26 us).  Heads of 256, two chunks of 512 over 12 k tokens: 156
// GFLOP in 228 to 235 us, one wave a SIMD, matrix units 27 % busy.
// ---------------------------------------------------------------------------
template <int D>
struct Tile {
  static constexpr int kKeys = 64, kPerCu = D <= 128 ? 2 : 1;  // workgroups a CU
  static constexpr int kPacks = kKeys * D / 8;          // of keys, and of values
  static constexpr int kPer = kPacks / kThreads;        // loads of a thread
  static constexpr size_t kLds = 2 * 2 * kPacks * 16 + 16;
};
constexpr int kTileRows = 32 * kWaves;

__device__ __forceinline__ void load_to_lds(const void* src, void* dst) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(src),
                                   (__attribute__((address_space(3))) void*)(dst), 16, 0, 0);
}

template <int D>
__global__ __launch_bounds__(kThreads, Tile<D>::kPerCu) void attend_tile_kernel(AttnArgs a, int S, int rts, Parts ws) {
  typedef Tile<D> Tl;
  typedef Mat<BF16> Mt;
  typedef Mt::Frag Frag;
  constexpr int KT = Tl::kKeys, NB = KT / 32;
  extern __shared__ __align__(16) char s_raw[];
  uint4* s_kv = reinterpret_cast<uint4*>(s_raw);  // two of K [D / 8][KT], two of V [KT / 8][D]
  int* s_from = reinterpret_cast<int*>(s_kv + 4 * Tl::kPacks);  // first tile with values left out
  const int tid = threadIdx.x, lane = tid % kWave, w = uniform(tid / kWave), n32 = lane & 31, h2 = lane >> 5;
  const int M = a.T * (a.Hq / a.c.Hkv);
  // the row tiles of a run and key head on one XCD, whose L2 they share
  const int x = blockIdx.x % 8, y = blockIdx.x / 8, rt = y % rts, uh = y / rts * 8 + x;
  const int u = uh / a.c.Hkv, h = uh % a.c.Hkv;
  if (u >= S) return;
  const Schedule plan = schedule(a, S, KT);
  const long long run = plan.run, total = plan.total;
  long long g = u * run;
  const long long end = g + run < total ? g + run : total;
  if (g >= end) return;
  int b;
  long long start;
  find_tile(a, plan, g, KT, &b, &start);

  const MetaPtrs m = meta_ptrs(a.meta, a.B, a.T);
  const BF16 *kc = reinterpret_cast<const BF16*>(a.k_cache), *vc = reinterpret_cast<const BF16*>(a.v_cache);
  const int shift = a.c.page_shift, mask = (1 << shift) - 1;
  const size_t page_size = block_of(a.c, 1, 0);
  const BF16 *kh = kc + block_of(a.c, 0, h), *vh = vc + block_of(a.c, 0, h);
  const float c = a.scale * kLog2e;
  for (; g < end; ++b) {
    const Seq seq = seq_at(a, plan, b, KT);
    const int tiles = seq.tiles, len = seq.len, ctx = seq.ctx;
    const int t0 = int(g - start), t1 = int(min((long long)(tiles), end - start));
    const bool whole = t1 - t0 == tiles;
    const int slot = 2 * u + (g > u * run ? 1 : 0);
    start += tiles;
    g = start;

    const int r = rt * kTileRows + w * 32 + n32;
    const RowAt at = row_at(a, m, b, h, r, M, len < 0);
    const int32_t* row = a.page_table + size_t(b) * a.c.max_pages;
    Rows<BF16, D> st;
    st.clear();
    st.load_q(at.real ? reinterpret_cast<const BF16*>(a.q) + row_offset<BF16>(a, b, at) : nullptr, h2);

    // page-table entry of the lane's key of a tile.  Nothing looks at it before
    // the next tile: a wait for it would be one for the tile's loads too.
    const int last_entry = (len - 1) >> shift;
    auto entry_at = [&](int t) { return row[min((t * KT + lane) >> shift, last_entry)]; };
    auto page_in = [&](int t, int entry) { return t * KT + lane < len && unsigned(entry) < unsigned(a.c.n_pages) ? entry : -1; };
    auto stage_k = [&](int t, int id, int buf) {
      const BF16* kl = kh + size_t(id < 0 ? 0 : id) * page_size + size_t((t * KT + lane) & mask) * 8;
#pragma unroll
      for (int n = 0; n < Tl::kPer; ++n) {
        const int at0 = (n * kWaves + w) * kWave;  // packs at0 + lane: one key a lane
        load_to_lds(kl + (size_t(at0 / KT) << shift) * 8, s_kv + buf * Tl::kPacks + at0);
      }
    };
    auto stage_v = [&](int t, int id, int buf) {
#pragma unroll
      for (int n = 0; n < Tl::kPer; ++n) {
        const int at0 = (n * kWaves + w) * kWave, grp = at0 / D;  // packs at0 + lane: of one page
        const int vid = __builtin_amdgcn_readlane(id, grp * 8);
        const BF16* vl = vh + size_t(vid < 0 ? 0 : vid) * page_size + size_t((t * KT + grp * 8) & mask) * D + at0 % D * 8;
        load_to_lds(vl + lane * 8, s_kv + (2 + buf) * Tl::kPacks + at0);
      }
    };
    // operands in groups: 64 packs each, the keys of a tile, then its values
    constexpr int kGroup = 4, kOps = Tl::kPacks / 64, kGroups = kOps / kGroup;
    const uint4 *sk, *sv;
    auto k_group = [&](Frag (&f)[kGroup], int n) {
#pragma unroll
      for (int k = 0; k < kGroup; ++k) {
        const int j = n * kGroup + k, nb = j / (D / 16), c = j % (D / 16);
        f[k] = load16<Frag>(sk + (2 * c + h2) * KT + nb * 32 + Mt::key_of(n32));
      }
    };
    auto v_group = [&](Frag (&f)[kGroup], int n) {
#pragma unroll
      for (int k = 0; k < kGroup; ++k) {
        const int j = n * kGroup + k, q = j / (D / 32), c = j % (D / 32);
        f[k] = load16<Frag>(sv + (2 * q + h2) * D + c * 32 + n32);
      }
    };
    auto score = [&](f32x16 (&acc)[NB], Frag f, int j) { acc[j / (D / 16)] = Mt::mma(f, st.q[j % (D / 16)], acc[j / (D / 16)]); };

    // tiles past what the rows see have nothing to load
    const int stop = min(t1, (end_of_rows(a, ctx, len, (rt + 1) * kTileRows - 1) + KT - 1) / KT);
    int id = -1, id1 = -1, next = 0;     // pages of this tile and the next, entry of the one after
    Frag f[2][kGroup];
    float s[NB][16];
    __syncthreads();  // the buffers are free
    if (tid == 0) *s_from = INT_MAX;
    if (t0 < stop) {
      id = page_in(t0, entry_at(t0));
      id1 = page_in(t0 + 1, entry_at(t0 + 1));
      next = entry_at(t0 + 2);
      stage_k(t0, id, 0);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      stage_v(t0, id, 0);
      if (t0 + 1 < stop) stage_k(t0 + 1, id1, 1);
      sk = s_kv;
      f32x16 acc[NB] = {};
#pragma unroll
      for (int n = 0; n < kGroups; ++n) {
        k_group(f[0], n);
#pragma unroll
        for (int k = 0; k < kGroup; ++k) score(acc, f[0][k], n * kGroup + k);
      }
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[nb][i] = acc[nb][i];
    }
    for (int t = t0; t < stop; ++t) {
      const int p0 = t * KT, r = (t - t0) & 1;
      // the keys of the next tile and the values of this one are there, the
      // buffers of their predecessors are free
      const u64 valid = __ballot(id >= 0);
      u64 seen = ~u64(0);
      if (p0 + KT > ctx) seen = seen_bits(a, m, b, at.slot, ctx, p0);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      id = id1;
      id1 = page_in(t + 2, next);
      next = entry_at(t + 3);
      if (t + 2 < stop) stage_k(t + 2, id1, r);
      if (t + 1 < stop) stage_v(t + 1, id, r ^ 1);
      sk = s_kv + (r ^ 1) * Tl::kPacks;
      sv = s_kv + (2 + r) * Tl::kPacks;
      if (p0 + KT > ctx || valid != ~u64(0)) {
        // slots of the tree, the end of the cache, pages that are left out:
        // values of absent keys, and those that are not finite, leave the
        // product (a masked weight is 0, and must stay so whatever it meets)
        bool mine = false;
        for (int q = tid; q < Tl::kPacks; q += kThreads) {
          const unsigned ok = unsigned(valid >> (q / D * 8)) & 0xffu;
          Frag y = load16<Frag>(sv + q);
          if (ok == 0xffu && !Mt::odd(y)) continue;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const bool on = (ok >> e) & 1;
            if (!on || (Mt::bits(y, e) & kExp) == kExp) {
              mine = mine || on;
              y = Mt::without(y, e);
            }
          }
          *reinterpret_cast<Frag*>(const_cast<uint4*>(sv + q)) = y;
        }
        if (mine) atomicMin(s_from, p0);
        __syncthreads();
        seen &= valid;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int i = 0; i < 16; ++i) s[nb][i] = where_seen(s[nb][i], unsigned(seen >> (nb * 32)) >> (h2 * 8), i / 8 * 16 + i % 8);
      }
      __builtin_amdgcn_s_setprio(1);  // before the waves in their products alone
      k_group(f[0], 0);
      const float ref = st.template follow<NB>(s, c);
      f32x16 acc[NB] = {};  // scores of the next tile (of nothing, after the last)
      Frag p[NB * 2];
      float sum[2] = {0.0f, 0.0f};
#pragma unroll
      for (int j = 0; j < kOps; ++j) {
        if (j % kGroup == 0) {
          if (j / kGroup + 1 < kGroups) k_group(f[(j / kGroup + 1) & 1], j / kGroup + 1);
          else v_group(f[kGroups & 1], 0);
        }
        score(acc, f[j / kGroup & 1][j % kGroup], j);
        constexpr int kEach = NB * 16 / kOps;
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
          const int x = j * kEach + e;
          float& y = s[x / 16][x % 16];
          y = __builtin_amdgcn_exp2f(__builtin_fmaf(y, c, -ref));
          sum[x & 1] += y;
          if (x % 8 == 7) p[x / 8] = Mt::pack(&s[x / 16][x % 16 - 7]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      __builtin_amdgcn_s_setprio(0);
      st.l += sum[0] + sum[1];
#pragma unroll
      for (int n = 0; n < kGroups; ++n) {
        if (n + 1 < kGroups) v_group(f[(kGroups + n + 1) & 1], n + 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int k = 0; k < kGroup; ++k) {
          const int j = n * kGroup + k;
          st.o[j % (D / 32)] = Mt::mma(f[(kGroups + n) & 1][k], p[j / (D / 32)], st.o[j % (D / 32)]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[nb][i] = acc[nb][i];
    }

    __syncthreads();
    const int from = *s_from;
    const float l = half_sum(st.l);
    if (r < M) {
      const bool on = at.real && l != 0.0f;
      const float inv = on ? 1.0f / l : 0.0f;
      const size_t i = (size_t(slot) * a.c.Hkv + h) * M + r;
      BF16* out = reinterpret_cast<BF16*>(a.out) + row_offset<BF16>(a, b, at);
      if (!whole && h2 == 0) ws.ml[i] = at.real ? make_float2(st.m, l) : make_float2(-INFINITY, 0.0f);
#pragma unroll
      for (int k = 0; k < D / 32; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int d = k * 32 + 8 * e + 4 * h2;
          float4 o = make_float4(st.o[k][4 * e], st.o[k][4 * e + 1], st.o[k][4 * e + 2], st.o[k][4 * e + 3]);
          if (whole)
            store4(out + d, on ? make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv) : make_float4(0, 0, 0, 0));
          else
            *reinterpret_cast<float4*>(ws.o + i * D + d) = o;
        }
      if (from != INT_MAX && at.real) {  // on what this lane has written
        const int upto = min(t1 * KT, len);
#pragma unroll 1
        for (int x = 0; x < D / 8; ++x) {
          const int d = 8 * x + 4 * h2;
          if (whole) add_not_finite<BF16>(a, m, b, h, at.slot, ctx, from, upto, d, out + d);
          else add_not_finite<BF16>(a, m, b, h, at.slot, ctx, from, upto, d, ws.o + i * D + d);
        }
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Joins the parts of the sequences that several runs share.  Four channels of
// a row a thread; with few rows and many parts `lanes` threads share these
// (taken by one thread in turn they cost 0.15 us each: 20 us where two
// sequences share 512 runs, 5 us this way).  What it costs otherwise is a trip
// for the lengths, one for the parts and one for the outputs.
// ---------------------------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(kThreads) void attend_join_kernel(AttnArgs a, int S, int kt, int lanes, Parts ws) {
  __shared__ float4 s_o[kThreads];
  __shared__ float2 s_ml[kThreads];
  const int b = blockIdx.z, h = blockIdx.y, D = a.c.d, M = a.T * (a.Hq / a.c.Hkv);
  const Schedule plan = schedule(a, S, kt);
  const long long run = plan.run, t0 = first_tile(a, plan, b, kt), t1 = t0 + seq_at(a, plan, b, kt).tiles - 1;
  const int u0 = plan.total >> 31 ? int(t0 / run) : int(t0) / int(run);
  const int u1 = plan.total >> 31 ? int(t1 / run) : int(t1) / int(run);
  if (u0 == u1) return;
  const int q = D / 4, per = kThreads / q / lanes;
  const int d = threadIdx.x % q * 4, at = threadIdx.x / q % lanes, rr = threadIdx.x / q / lanes;
  const int first = 2 * u0 + (t0 > u0 * run ? 1 : 0);
  for (int r0 = blockIdx.x * per; r0 < M; r0 += gridDim.x * per) {
    const int r = min(r0 + rr, M - 1);
    float mx = -INFINITY, sum = 0.0f;
    float4 o = make_float4(0, 0, 0, 0);
    constexpr int kAhead = 8;  // parts in flight
    for (int v = u0; v <= u1; v += kAhead * lanes) {
      float2 ml[kAhead];
      float4 y[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        if (v + k * lanes > u1) continue;
        const int u = min(v + k * lanes + at, u1);
        const size_t i = (size_t(u == u0 ? first : 2 * u) * a.c.Hkv + h) * M + r;
        ml[k] = ws.ml[i];
        y[k] = *reinterpret_cast<const float4*>(ws.o + i * D + d);
      }
      float top = mx;
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
        if (v + k * lanes <= u1) top = fmaxf(top, ml[k].x);
      const float fix = mx == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mx - top);
      if (mx > -INFINITY) sum *= fix, o.x *= fix, o.y *= fix, o.z *= fix, o.w *= fix;
      mx = top;
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        // a part without a visible key has nothing (one whose scores are not
        // numbers has a sum that is none)
        if (v + k * lanes + at > u1 || (ml[k].x == -INFINITY && ml[k].y == 0.0f)) continue;
        const float f = ml[k].x == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(ml[k].x - mx);
        sum += f * ml[k].y;
        o.x += f * y[k].x, o.y += f * y[k].y, o.z += f * y[k].z, o.w += f * y[k].w;
      }
    }
    if (lanes > 1) {
      __syncthreads();  // the row before is read
      s_o[threadIdx.x] = o;
      s_ml[threadIdx.x] = make_float2(mx, sum);
      __syncthreads();
      if (at) continue;
      for (int k = 1; k < lanes; ++k) mx = fmaxf(mx, s_ml[threadIdx.x + k * q].x);
      sum = 0.0f;
      o = make_float4(0, 0, 0, 0);
      for (int k = 0; k < lanes; ++k) {
        const float2 ml = s_ml[threadIdx.x + k * q];
        const float4 y = s_o[threadIdx.x + k * q];
        if (ml.x == -INFINITY && ml.y == 0.0f) continue;
        const float f = ml.x == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(ml.x - mx);
        sum += f * ml.y;
        o.x += f * y.x, o.y += f * y.y, o.z += f * y.z, o.w += f * y.w;
      }
    }
    if (r0 + rr >= M) continue;
    const bool on = sum != 0.0f;
    const float inv = on ? 1.0f / sum : 0.0f;
    store4(reinterpret_cast<T*>(a.out) + row_offset<T>(a, b, row_of(a, h, r)) + d,
           on ? make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv) : make_float4(0, 0, 0, 0));
  }
}

int after_launch() {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? GDN_OK : set_error(GDN_EHIP, "attend: launch: %s", hipGetErrorString(e));
}

// Runs for `blocks` workgroups per run on `slots` workgroup places: as many as
// fill the places, in up to four rounds where fewer would leave more than a
// tenth of them empty (a key head and row tile count that does not divide the
// places; calls whose count does are the same with one round).
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

// Workspace of S runs.
int parts_for(const AttnArgs& a, int S, hipStream_t stream, Parts* ws) {
  *ws = {nullptr, nullptr};
  if (S == 1) return GDN_OK;  // every sequence is whole
  const size_t rows = size_t(2) * S * a.c.Hkv * a.T * (a.Hq / a.c.Hkv);
  int rc = GDN_OK;
  char* p = static_cast<char*>(stream_workspace(rows * (a.c.d * sizeof(float) + sizeof(float2)), stream, &rc));
  if (!p) return rc;
  *ws = {reinterpret_cast<float*>(p), reinterpret_cast<float2*>(p + rows * a.c.d * sizeof(float))};
  return GDN_OK;
}

template <typename T>
int launch_join(const AttnArgs& a, int S, int kt, const Parts& ws, hipStream_t stream) {
  if (S == 1) return GDN_OK;  // no sequence is shared
  const int M = a.T * (a.Hq / a.c.Hkv), q = a.c.d / 4;
  // threads for the parts of a sequence (S / B on average): more than one while
  // each has over four and the rows alone give under two workgroups a CU
  int lanes = 1;
  while (lanes < kThreads / q && 4LL * lanes * a.B < S && (long long)(M) * q * lanes * a.c.Hkv * a.B < 512 * kThreads)
    lanes *= 2;
  const int per = kThreads / q / lanes, blocks = (M + per - 1) / per;
  // a round of workgroups, if there are rows for more
  const int most = std::max(1, 2048 / (a.c.Hkv * a.B));
  attend_join_kernel<T><<<dim3(std::min(blocks, most), a.c.Hkv, a.B), kThreads, 0, stream>>>(a, S, kt, lanes, ws);
  return after_launch();
}

template <typename T, int D>
int launch_stream(const AttnArgs& a, hipStream_t stream) {
  const int M = a.T * (a.Hq / a.c.Hkv), rt = (M + 31) / 32;
  const int S = runs_for((long long)(a.c.Hkv) * rt, 256 * stream_groups<T, D>());
  Parts ws;
  int rc = parts_for(a, S, stream, &ws);
  if (rc != GDN_OK) return rc;
  constexpr size_t lds = stream_lds<D>();
  rc = ensure_dynamic_lds(reinterpret_cast<const void*>(attend_stream_kernel<T, D>), int(lds), "attend");
  if (rc != GDN_OK) return rc;
  attend_stream_kernel<T, D><<<dim3(S, a.c.Hkv, rt), kThreads, lds, stream>>>(a, S, ws);
  rc = after_launch();
  return rc != GDN_OK ? rc : launch_join<T>(a, S, kStreamKeys, ws, stream);
}

template <int D>
int launch_tile(const AttnArgs& a, hipStream_t stream) {
  const int M = a.T * (a.Hq / a.c.Hkv), rt = (M + kTileRows - 1) / kTileRows;
  const int S = runs_for((long long)(a.c.Hkv) * rt, 256 * Tile<D>::kPerCu);
  Parts ws;
  int rc = parts_for(a, S, stream, &ws);
  if (rc != GDN_OK) return rc;
  constexpr size_t lds = Tile<D>::kLds;
  rc = ensure_dynamic_lds(reinterpret_cast<const void*>(attend_tile_kernel<D>), int(lds), "attend");
  if (rc != GDN_OK) return rc;
  const int groups = (S * a.c.Hkv + 7) / 8 * 8;
  attend_tile_kernel<D><<<groups * rt, kThreads, lds, stream>>>(a, S, rt, ws);
  rc = after_launch();
  return rc != GDN_OK ? rc : launch_join<BF16>(a, S, Tile<D>::kKeys, ws, stream);
}

template <int D>
int launch_dim(const AttnArgs& a, hipStream_t stream) {
  // One tile of rows: every wave would load and multiply three empty ones.  4 key
  // heads of 128, 16 sequences of 8 k tokens: 8 rows 40.8 us, 45.2 with shared
  // tiles; 32 rows 47.4, 48.7; 64 rows 53.7 and 54.4; 128 rows 73.4 and 62.8.
  if (a.dtype != GDN_BF16) return launch_stream<float, D>(a, stream);
  if (a.T * (a.Hq / a.c.Hkv) > 32) return launch_tile<D>(a, stream);
  return launch_stream<BF16, D>(a, stream);
}

}  // namespace

int launch_attend(const AttnArgs& a, hipStream_t stream) {
  const StreamOrder order(stream);  // the parts, then their join
  switch (a.c.d) {
    case 32: return launch_dim<32>(a, stream);
    case 64: return launch_dim<64>(a, stream);
    case 128: return launch_dim<128>(a, stream);
    default: return launch_dim<256>(a, stream);
  }
}

}  // namespace gdn
