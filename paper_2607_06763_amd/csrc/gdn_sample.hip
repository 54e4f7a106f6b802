// gdn_sample.hip -- tokens from logits with given random numbers, and the
// acceptance of a draft tree along them.
#include "gdn_attn.h"

namespace gdn {
namespace {

// ---------------------------------------------------------------------------
// Sampling: one workgroup per slot.
//
// A token's mass is a whole number, w = round(2^31 2^((z - top) c)) with
// c = log2(e) / temperature, so sums are exact and do not depend on their
// order.  What top_k and top_p leave is everything up to one last logit in
// the order (z falling, index rising): its value and index are the cut.
//
// The first pass over the row takes every thread's maximum.  Where a floor
// under all that can stay is known from them, only the threads with a larger
// maximum read their part again, and what is above the floor is listed in LDS,
// where the cut and the draw are made:
//   top_k   at least k logits are as large as the k-th largest of the threads'
//           maxima
//   min_p   the floor itself
// top_p alone (or a k above the number of threads) takes the masses of bins of
// (top - z) c, the logits of the bin that holds the cut, and the masses that
// stay in vocabulary order; no cut at all takes the last of these only.
// Rows for which LDS is too small (thousands of equal logits) take the cuts by
// halving the value.
//
// Bound by the passes of a row in turn, not by bytes: under top_p a logit is
// read three times at 10 to 20 instructions, with barriers and the bins'
// bookkeeping between.  512 rows of 131072 in bf16, every kind of cut: 113 to
// 117 us, 1.2 TB/s of logits (1.7 times these fetched, vector units 22 % busy: one
// round of workgroups, in which greedy and min_p rows leave their places empty);
// 1056 rows of 50001 in fp32 with top_p: 112 to 121 us, 1.6 TB/s (padding slots,
// up to a third of a tree, left out).  One row of 131072: 21 to 25 us, the
// passes of one workgroup.
//
// The kernel is held to 128 registers, for 16 waves a CU: in fp32 8 to 12 of
// them spill to memory, in bf16 5 with 1024 threads and none with fewer.
// ---------------------------------------------------------------------------
constexpr int kBins = 1024;
constexpr float kBinsPerOctave = kBins / 32.0f;  // w is 0 beyond 32 octaves
constexpr int kFew = 128;  // logits up to here are ranked as they are

typedef unsigned long long u64;

struct Cut {
  float z;  // what stays: logits above z, and those equal to z up to index i
  int i;
};

// A listed logit: its place in the order as one number (larger is ahead: the
// value's ordered bits, then the inverted index) and its mass.
struct alignas(16) Item {
  u64 key;
  unsigned w, none;
};

// ordered image of a float: larger value, larger image
__device__ __forceinline__ unsigned ordered(float z) {
  const unsigned b = __float_as_uint(z + 0.0f);  // -0 as 0
  return b >> 31 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float unordered(unsigned k) { return __uint_as_float(k >> 31 ? k & 0x7fffffffu : ~k); }
__device__ __forceinline__ u64 key_of(float z, int i) { return u64(ordered(z)) << 32 | unsigned(~i); }
__device__ __forceinline__ float value_of(u64 key) { return unordered(unsigned(key >> 32)); }
__device__ __forceinline__ int index_of(u64 key) { return int(~unsigned(key)); }

// What a cut asks of a logit, given the count and the mass of those ahead.
struct Before {
  bool by_count;
  int k;
  double want;
  __device__ __forceinline__ bool operator()(u64 cnt, u64 mass) const {
    return by_count ? cnt < u64(k) : mass == 0 || double(mass) < want;
  }
};

template <int NT>
struct Shared {
  static constexpr int kWaves = NT / kWave, kList = 4 * NT;
  u64 mass[kBins];
  unsigned cnt[kBins];
  Item list[kList];  // listed logits, their indices and masses
  alignas(16) unsigned short sub[kList];  // places in the list
  u64 red[kWaves];
  unsigned redc[kWaves];
  float redf[kWaves];
  int n, m;
  int bin;
  u64 mass_before, sum;
  unsigned cnt_before;
  Cut cut;
  int token;
};

__device__ __forceinline__ unsigned weight_near(float z, float top, float c) {
  // NaN converts to 0
  return unsigned(__builtin_fmaf(__builtin_amdgcn_exp2f((z - top) * c), 2147483648.0f, 0.5f));
}
// The same where top or c may be infinite.
__device__ __forceinline__ unsigned weight(float z, float top, float c) {
  return z == top ? 0x80000000u : weight_near(z, top, c);
}

__device__ __forceinline__ int bin_of(float z, float top, float c) {
  return z == top ? 0 : int(fminf((top - z) * c * kBinsPerOctave, float(kBins - 1)));
}

__device__ __forceinline__ u64 wave_sum64(u64 v) {
  for (int s = 1; s < kWave; s <<= 1) v += __shfl_xor(v, s);
  return v;
}

__device__ __forceinline__ u64 wave_scan64(u64 v) {
  const int lane = threadIdx.x % kWave;
  for (int d = 1; d < kWave; d <<= 1) {
    const u64 up = __shfl_up(v, d);
    if (lane >= d) v += up;
  }
  return v;
}

// Sum over the workgroup, in every thread.
template <int NT>
__device__ __forceinline__ u64 block_sum(u64 v, Shared<NT>& s) {
  v = wave_sum64(v);
  __syncthreads();
  if (threadIdx.x % kWave == 0) s.red[threadIdx.x / kWave] = v;
  __syncthreads();
  u64 t = 0;
#pragma unroll
  for (int w = 0; w < NT / kWave; ++w) t += s.red[w];
  return t;
}

// loaded for a row without a whole vector
__device__ u32x4 g_low = {0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u};

// A row of logits in 16-byte vectors.  A row may start anywhere: vector j
// holds elements j X - lead .. + X - 1, those outside the row are -inf.  Wave
// w holds the vectors from w per kWave on, in order.  A last vector that is
// not whole is never loaded as one (it may pass the end of the buffer).
template <typename T, int NT>
struct Row {
  static constexpr int X = Pack<T>::kN;
  static constexpr unsigned kLow = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;  // -inf
  const u32x4* vec;
  int V, lead, n, per;  // n vectors, per of them a thread
  int whole;            // vectors that end inside the row
  u32x4 head, tail;     // bits of the first vector that are the row's; a last vector that is not whole
  __device__ __forceinline__ Row(const T* p, int v) : V(v) {
    lead = int((reinterpret_cast<uintptr_t>(p) & 15) / sizeof(T));
    n = (lead + V + X - 1) / X;
    per = (n + NT - 1) / NT;
    whole = (lead + V) / X;
    vec = whole ? reinterpret_cast<const u32x4*>(p - lead) : &g_low;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      constexpr int kPer = X / 4;
      unsigned h = 0, t = 0;
#pragma unroll
      for (int k = 0; k < kPer; ++k) {
        const int at = e * kPer + k, i = whole * X - lead + at;
        const unsigned all = sizeof(T) == 2 ? 0xffffu : 0xffffffffu;
        if (at >= lead) h |= all << (16 * k);
        unsigned bits = kLow & all;
        if (i >= 0 && i < V) {
          if constexpr (sizeof(T) == 2) bits = p[i].bits;
          else bits = __float_as_uint(p[i]);
        }
        t |= bits << (16 * k);
      }
      head[e] = h;
      tail[e] = t;
    }
  }
  // first vector of wave w's j-th load; the lane's
  __device__ __forceinline__ int base(int w, int j) const { return (w * per + j) * kWave; }
  __device__ __forceinline__ int at(int w, int j) const { return base(w, j) + int(threadIdx.x) % kWave; }
  __device__ __forceinline__ int first(int v) const { return v * X - lead; }
  __device__ __forceinline__ int wave_of(int i) const { return (i + lead) / X / kWave / per; }
  // what is in memory of vector v, or of another one
  __device__ __forceinline__ u32x4 load(int v) const { return vec[max(0, min(v, whole - 1))]; }
  // whether the load needs mending: the row's ends, and past them
  __device__ __forceinline__ bool edge(int w, int j) const { return (base(w, j) == 0 && lead > 0) || base(w, j) + kWave > whole; }
  __device__ __forceinline__ u32x4 mend(u32x4 x, int v) const {
    const u32x4 low = {kLow, kLow, kLow, kLow};
    if (v >= whole) x = v == whole && whole < n ? tail : low;
    if (v == 0) x = (x & head) | (low & ~head);
    return x;
  }
  __device__ __forceinline__ u32x4 get(int w, int j) const {
    const u32x4 x = load(at(w, j));
    return edge(w, j) ? mend(x, at(w, j)) : x;
  }
  static __device__ __forceinline__ float value(u32x4 x, int e) {
    if constexpr (sizeof(T) == 2) return __uint_as_float(e & 1 ? x[e / 2] & 0xffff0000u : x[e / 2] << 16);
    else return __uint_as_float(x[e]);
  }
};

// f(z, i) for every logit of the loads j0 .. j1 - 1 of wave w's part, a few at
// a time.  A NaN fails every comparison of f.
template <int kAhead, typename T, int NT, typename F>
__device__ __forceinline__ void each_of(const Row<T, NT>& row, int w, int j0, int j1, F f) {
  constexpr int X = Row<T, NT>::X;
  for (int j = j0; j < j1; j += kAhead) {
    u32x4 x[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) x[k] = row.load(row.at(w, j + k));
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (j + k >= j1) break;
      if (row.edge(w, j + k)) x[k] = row.mend(x[k], row.at(w, j + k));
      const int i0 = row.first(row.at(w, j + k));
#pragma unroll
      for (int e = 0; e < X; ++e) f(Row<T, NT>::value(x[k], e), i0 + e);
    }
  }
}

// test(z) for every logit; f(z, i) for all of a vector in which it was true for
// one: few instructions a logit where few vectors are hit.
template <typename T, int NT, typename P, typename F>
__device__ __forceinline__ void each_if(const Row<T, NT>& row, P test, F f) {
  constexpr int X = Row<T, NT>::X, kAhead = 8;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  for (int j = 0; j < row.per; j += kAhead) {
    u32x4 x[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) x[k] = row.load(row.at(w, j + k));
    __builtin_amdgcn_sched_barrier(0);
    unsigned hits = 0;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (j + k >= row.per) break;
      if (row.edge(w, j + k)) x[k] = row.mend(x[k], row.at(w, j + k));
      bool hit = false;
#pragma unroll
      for (int e = 0; e < X; ++e) hit = hit | test(Row<T, NT>::value(x[k], e));
      hits |= (hit ? 1u : 0u) << k;
    }
    for (; hits; hits &= hits - 1) {
      const int v = row.at(w, j + __builtin_ctz(hits));
      const u32x4 y = row.mend(row.load(v), v);
#pragma unroll
      for (int e = 0; e < X; ++e) f(Row<T, NT>::value(y, e), row.first(v) + e);
    }
  }
}

template <int kAhead, typename T, int NT, typename F>
__device__ __forceinline__ void each(const Row<T, NT>& row, F f) {
  each_of<kAhead>(row, __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), 0, row.per, f);
}

// without branches: they run in loops over LDS
__device__ __forceinline__ bool stays(float z, int i, const Cut& c) { return (z > c.z) | ((z == c.z) & (i <= c.i)); }

// The last logit in the order (z falling, index rising) for which
// before(count of those ahead, mass of those ahead) holds; it holds for the
// first one and, once it fails, for none after.  Only logits that stay under
// `cut` count.  By halving the value, then the index: for bins of more
// logits than the list holds (many equal ones).
template <typename T, int NT>
__device__ __forceinline__ Cut bisect(const Row<T, NT>& row, float top, float c, Cut cut, Before before, Shared<NT>& s) {
  unsigned lo = ordered(-INFINITY), hi = ordered(top);  // hi holds at index 0
  int a = 0, b = row.V - 1;                      // then the last index that holds
  while (lo < hi || a < b) {
    const bool values = lo < hi;
    const unsigned k = values ? lo + (hi - lo) / 2 : hi;
    const int i = values ? 0 : a + (b - a + 1) / 2;
    u64 mass = 0, cnt = 0;
    each<4>(row, [&](float z, int j) {
      if (!stays(z, j, cut)) return;
      const unsigned kz = ordered(z);
      if (kz > k || (kz == k && j < i)) {
        const unsigned w = weight(z, top, c);
        mass += w;
        cnt += w > 0;
      }
    });
    cnt = block_sum(cnt, s);
    mass = block_sum(mass, s);
    const bool holds = before(cnt, mass);
    if (values) (holds ? hi : lo) = holds ? k : k + 1;
    else if (holds) a = i;
    else b = i - 1;
  }
  return {unordered(hi), a};
}

template <int NT>
__device__ __forceinline__ void clear_bins(Shared<NT>& s) {
  for (int q = threadIdx.x; q < kBins; q += NT) s.mass[q] = 0, s.cnt[q] = 0;
  __syncthreads();
}

// Prefix over the bins: s.bin = the last bin that holds a mass and for whose
// first logit `before` holds, s.cnt_before and s.mass_before what lies ahead
// of it in the bins; mb and cb lie ahead of all bins.
template <int NT>
__device__ __forceinline__ void find_bin(Before before, u64 mb, unsigned cb, Shared<NT>& s) {
  constexpr int kPer = kBins / NT;
  const int tid = threadIdx.x, lane = tid % kWave, w = __builtin_amdgcn_readfirstlane(tid / kWave);
  u64 mass = 0;
  unsigned cnt = 0;
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    mass += s.mass[tid * kPer + e];
    cnt += s.cnt[tid * kPer + e];
  }
  const u64 im = wave_scan64(mass);
  unsigned ic = cnt;
  for (int d = 1; d < kWave; d <<= 1) {
    const unsigned up = __shfl_up(ic, d);
    if (lane >= d) ic += up;
  }
  __syncthreads();
  if (lane == kWave - 1) s.red[w] = im, s.redc[w] = ic;
  if (tid == 0) s.bin = 0;
  __syncthreads();
  u64 m = im - mass;
  unsigned n = ic - cnt;
#pragma unroll 1
  for (int k = 0; k < w; ++k) m += s.red[k], n += s.redc[k];
  // each thread's last bin that holds; the largest of them is the answer
  int best = -1;
  u64 bm = 0;
  unsigned bn = 0;
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    const u64 q = s.mass[tid * kPer + e];
    if (q && before(u64(n) + cb, m + mb)) best = tid * kPer + e, bm = m, bn = n;
    m += q;
    n += s.cnt[tid * kPer + e];
  }
  if (best >= 0) atomicMax(&s.bin, best);
  __syncthreads();
  if (best == s.bin) s.cnt_before = bn, s.mass_before = bm;
  __syncthreads();
}

// f(item) for the m list places in s.sub (or, of `shares` shares of them, one),
// eight in flight: one LDS latency a place would be most of the time.  A place
// past the end has the smallest key and no mass.
template <int NT, typename F>
__device__ __forceinline__ void each_of_sub(int m, int share, int shares, const Shared<NT>& s, F f) {
  for (int q = 8 * share; q < m; q += 8 * shares) {
    const u32x4 at = *reinterpret_cast<const u32x4*>(&s.sub[q]);
    Item y[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) y[k] = s.list[q + k < m ? (k & 1 ? at[k / 2] >> 16 : at[k / 2] & 0xffffu) : 0u];
    __builtin_amdgcn_sched_barrier(0);  // or each load is waited for by itself
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (q + k >= m) y[k].key = 0, y[k].w = 0;
      f(y[k]);
    }
  }
}

// The cut for `before` among the n listed logits that stay under `old`; mb and
// cb lie ahead of all, and all lie between (top - z) scale = 0 and kBins.
// *kept = the mass up to and with it.
template <int NT>
__device__ __forceinline__ Cut cut_of_list(int n, float top, float scale, u64 mb, unsigned cb, Cut old, Before before, u64* kept,
                                           Shared<NT>& s) {
  const int tid = threadIdx.x;
  const u64 least = key_of(old.z, old.i);  // what stays has this key or a larger one
  auto bin = [&](u64 key) {
    const float z = value_of(key);
    return z == top ? 0 : int(fmaxf(0.0f, fminf((top - z) * scale, float(kBins - 1))));
  };
  const bool few = n <= kFew;
  clear_bins(s);
  if (!few) {
    for (int a = tid; a < n; a += NT) {
      const Item x = s.list[a];
      if (x.key >= least) {
        const int q = bin(x.key);
        atomicAdd(&s.mass[q], u64(x.w));
        atomicAdd(&s.cnt[q], 1u);
      }
    }
    __syncthreads();
    find_bin(before, mb, cb, s);
    mb += s.mass_before;
    cb += s.cnt_before;
    __syncthreads();
    clear_bins(s);
  }
  if (tid == 0) s.m = 0, s.sum = 0;
  __syncthreads();
  for (int a = tid; a < n; a += NT) {
    const Item x = s.list[a];
    if (x.key >= least && (few || bin(x.key) == s.bin)) s.sub[atomicAdd(&s.m, 1)] = a;
  }
  __syncthreads();
  // every member against every other one; several threads a member where there
  // are fewer of them, their shares added up in the bins
  const int m = s.m;
  int width = kWave;
  while (width < m && width < NT) width *= 2;
  const int share = width <= NT ? NT / width : 1;
  u64 mine = 0, best_key = 0;
  for (int a = tid % width; a < m; a += width) {
    const Item x = s.list[s.sub[a]];
    u64 mass = 0;
    unsigned cnt = 0;
    each_of_sub(m, tid / width, share, s, [&](const Item& y) {
      mass += y.key > x.key ? y.w : 0u;
      cnt += y.key > x.key;
    });
    if (share > 1) {  // m <= width < NT: one member a thread
      atomicAdd(&s.mass[a], mass);
      atomicAdd(&s.cnt[a], cnt);
    } else if (before(cnt + cb, mass + mb) && mass + mb + x.w > mine) {
      // masses rise along the order (no listed mass is 0): the largest that
      // holds is the last one
      mine = mass + mb + x.w, best_key = x.key;
    }
  }
  __syncthreads();
  if (share > 1 && tid < m) {
    const Item x = s.list[s.sub[tid]];
    const u64 mass = s.mass[tid] + mb;
    if (before(u64(s.cnt[tid]) + cb, mass)) mine = mass + x.w, best_key = x.key;
  }
  if (mine) atomicMax(&s.sum, mine);
  __syncthreads();
  const u64 best = s.sum;
  if (mine == best) s.cut = {value_of(best_key), index_of(best_key)};
  __syncthreads();
  *kept = best;
  const Cut cut = s.cut;
  __syncthreads();
  return cut;
}

// First place at which a running mass exceeds u times the whole.
__device__ __forceinline__ u64 goal_of(float u, u64 total) {
  const double want = double(u) * double(total);
  const u64 goal = want > 0.0 ? u64(want) : 0;
  return goal < total ? goal : total - 1;
}

// The draw among the n listed logits, in the order of their indices.
template <int NT>
__device__ __forceinline__ void draw_from_list(int n, float u, Cut cut, u64 least, int V, int32_t* token, Shared<NT>& s) {
  const int tid = threadIdx.x, lane = tid % kWave, w = tid / kWave;
  const bool few = n <= kFew;
  const int shift = max(0, 32 - __builtin_clz(unsigned(V)) - (31 - __builtin_clz(unsigned(NT))));  // V >> shift < NT
  const u64 last = key_of(cut.z, cut.i);
  if (!few) clear_bins(s);
  for (int a = tid; a < n; a += NT) {
    const Item x = s.list[a];
    const bool on = x.key >= last && x.w >= least;
    if (!on) s.list[a].w = 0;
    else if (!few) atomicAdd(&s.mass[index_of(x.key) >> shift], u64(x.w));
  }
  if (tid == 0) s.m = 0;
  __syncthreads();
  if (few) {
    if (tid >= n) return;
    const Item x = s.list[tid];
    const int i = index_of(x.key);
    u64 run = 0, total = 0;
    for (int q = 0; q < n; q += 8) {
      Item y[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) y[k] = s.list[min(q + k, n - 1)];
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const unsigned w = q + k < n ? y[k].w : 0u;
        total += w;
        run += index_of(y[k].key) < i ? w : 0u;
      }
    }
    const u64 goal = goal_of(u, total);
    if (goal >= run && goal < run + x.w) *token = i;
    return;
  }
  const u64 mine = s.mass[tid], inc = wave_scan64(mine);
  if (lane == kWave - 1) s.red[w] = inc;
  __syncthreads();
  u64 before = inc - mine, total = 0;
#pragma unroll
  for (int k = 0; k < NT / kWave; ++k) {
    const u64 v = s.red[k];
    before += k < w ? v : 0;
    total += v;
  }
  const u64 goal = goal_of(u, total);
  if (goal >= before && goal < before + mine) s.bin = tid, s.mass_before = before;
  __syncthreads();
  const int bucket = s.bin;
  for (int a = tid; a < n; a += NT) {
    const Item x = s.list[a];
    if (x.w && index_of(x.key) >> shift == bucket) s.sub[atomicAdd(&s.m, 1)] = a;
  }
  __syncthreads();
  const int m = s.m;
  for (int a = tid; a < m; a += NT) {
    const Item x = s.list[s.sub[a]];
    const int i = index_of(x.key);
    u64 run = s.mass_before;
    each_of_sub(m, 0, 1, s, [&](const Item& y) { run += index_of(y.key) < i ? y.w : 0u; });
    if (goal >= run && goal < run + x.w) *token = i;
  }
}

// The draw over the row in vocabulary order: the wave's part whose masses hold
// the goal, a share of that part, a vector, a logit.  mine: the mass of this
// wave's part.
template <typename T, int NT, typename F>
__device__ __forceinline__ void draw_from_row(const Row<T, NT>& row, float u, u64 mine, F mass_of, int32_t* token, Shared<NT>& s) {
  constexpr int X = Row<T, NT>::X, kWaves = NT / kWave;
  const int lane = threadIdx.x % kWave, w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  __syncthreads();
  if (lane == 0) s.red[w] = mine;
  __syncthreads();
  u64 total = 0, before = 0;
  int part = 0;
  for (int k = 0; k < kWaves; ++k) total += s.red[k];
  const u64 goal = goal_of(u, total);
  for (int k = 0; k < kWaves - 1 && goal >= before + s.red[k]; ++k) before += s.red[k], part = k + 1;
  part = __builtin_amdgcn_readfirstlane(part);
  __syncthreads();
  const int step = (row.per + kWaves - 1) / kWaves;
  const int j0 = min(w * step, row.per), j1 = min(j0 + step, row.per);
  u64 sub = 0;
  each_of<4>(row, part, j0, j1, [&](float z, int i) { sub += mass_of(z, i); });
  sub = wave_sum64(sub);
  if (lane == 0) s.red[w] = sub;
  __syncthreads();
  for (int k = 0; k < w; ++k) before += s.red[k];
  if (goal < before || goal >= before + sub) return;
  for (int j = j0; j < j1; ++j) {
    const int v = row.at(part, j);
    const u32x4 x = row.get(part, j);
    u64 m = 0;
#pragma unroll
    for (int e = 0; e < X; ++e) m += mass_of(Row<T, NT>::value(x, e), row.first(v) + e);
    const u64 inc = wave_scan64(m), all = __shfl(inc, kWave - 1);
    if (goal < before + all) {
      u64 run = before + inc - m;
      if (goal >= run && goal < run + m) {
        int at = -1;
#pragma unroll
        for (int e = 0; e < X; ++e) {
          run += mass_of(Row<T, NT>::value(x, e), row.first(v) + e);
          if (at < 0 && run > goal) at = row.first(v) + e;
        }
        *token = at;
      }
      return;
    }
    before += all;
  }
}

// Settings of a row's sequence.
struct Settings {
  float t, p, least;
  int k;
  bool greedy, use_k, use_p, use_m;
  float c;
  u64 thr;  // min_p as a mass
  __device__ __forceinline__ Settings(const SampleArgs& a, int b) {
    t = a.temperature ? a.temperature[b] : 1.0f;
    k = a.top_k ? a.top_k[b] : 0;
    p = a.top_p ? a.top_p[b] : 1.0f;
    least = a.min_p ? a.min_p[b] : 0.0f;
    greedy = !(t > 0.0f);
    c = greedy ? 1.0f : (1.0f / t) * 1.44269504088896340736f;
    use_k = !greedy && k > 0 && k < a.V;
    use_p = !greedy && !(p >= 1.0f);
    use_m = !greedy && least > 0.0f;
    thr = use_m ? u64(ceil(double(fminf(least, 1.0f)) * 2147483648.0)) : 0;
  }
};

// A row that LDS is too small for (seldom any): the cuts by halving, the draw
// over the row.
template <typename T, int NT>
__device__ __forceinline__ void sample_rest(const Row<T, NT>& row, const Settings& o, float top, float u, int32_t* token,
                                            Shared<NT>& s) {
  const float c = o.c;
  if (o.greedy) {
    int best = row.V;
    each<4>(row, [&](float z, int i) {
      if (z == top) best = min(best, i);
    });
    if (best < row.V) atomicMin(&s.token, best);
    __syncthreads();
    if (threadIdx.x == 0) *token = s.token;
    return;
  }
  Cut cut = {-INFINITY, row.V};
#pragma unroll 1
  for (int stage = 0; stage < 2; ++stage) {
    if (stage == 0 ? !o.use_k : !o.use_p) continue;
    u64 m = 0;
    each<4>(row, [&](float z, int i) { m += stays(z, i, cut) ? weight(z, top, c) : 0u; });
    m = block_sum(m, s);
    cut = bisect(row, top, c, cut, Before{stage == 0, o.k, double(o.p) * double(m)}, s);
  }
  auto mass_of = [&](float z, int i) {
    if (!stays(z, i, cut)) return u64(0);
    const u64 w = weight(z, top, c);
    return w >= o.thr ? w : u64(0);
  };
  u64 part = 0;
  each<4>(row, [&](float z, int i) { part += mass_of(z, i); });
  draw_from_row(row, u, wave_sum64(part), mass_of, token, s);
}

template <typename T, int NT>
__global__ __launch_bounds__(NT, 4) void sample_kernel(SampleArgs a) {
  constexpr int kList = Shared<NT>::kList;
  __shared__ Shared<NT> s;
  const int r = blockIdx.x, b = r / a.T, tid = threadIdx.x, lane = tid % kWave;
  const int wave = tid / kWave;
  if (a.meta) {
    const MetaPtrs m = meta_ptrs(a.meta, a.B, a.T);
    if (m.status[b] != 0 || m.depth[r] < 0) {
      if (tid == 0) a.token[r] = -1;
      return;
    }
  }
  const Row<T, NT> row(reinterpret_cast<const T*>(a.logits) + (long long)(r) * a.ld, a.V);
  const Settings o(a, b);
  const float u = a.u[r], c = o.c;
  float mine = -INFINITY;  // this thread's maximum
  each<8>(row, [&](float z, int) { mine = fmaxf(mine, z); });
  float top = mine;
  for (int d = 1; d < kWave; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
  if (lane == 0) s.redf[wave] = top;
  if (tid == 0) s.token = a.V, s.n = 0;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NT / kWave; ++w) top = fmaxf(top, s.redf[w]);
  if (top == -INFINITY) {
    if (tid == 0) a.token[r] = -1;
    return;
  }

  // the floor, where there is one
  const bool flat = o.greedy || top == INFINITY || c == INFINITY;  // only the logits equal to top have a mass
  float floor = -INFINITY;
  if (flat) {
    floor = top;
  } else if (o.use_k && o.k <= NT) {
    clear_bins(s);
    if (mine > -INFINITY) {
      const int q = bin_of(mine, top, c);
      atomicAdd(&s.cnt[q], 1u);
      atomicAdd(&s.mass[q], u64(1));
    }
    __syncthreads();
    find_bin(Before{true, o.k, 0.0}, 0, 0, s);  // the bin of the k-th maximum
    const int bin = s.bin;
    const u64 n = u64(s.cnt_before) + s.cnt[bin];
    float low = mine > -INFINITY && bin_of(mine, top, c) <= bin ? mine : INFINITY;
    for (int d = 1; d < kWave; d <<= 1) low = fminf(low, __shfl_xor(low, d));
    __syncthreads();
    if (lane == 0) s.redf[wave] = low;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NT / kWave; ++w) low = fminf(low, s.redf[w]);
    if (n >= u64(o.k)) floor = low;  // else fewer than k threads have any logit
  } else if (!o.use_k && !o.use_p && o.use_m) {
    // a mass that rounds to thr may be up to a half below it
    const float down = (log2f(float(o.thr) - 0.5f) - 31.0f - 0.01f) / c;
    floor = fmaxf(-3.4028235e38f, top + down - 1e-6f * (fabsf(top) + fabsf(down)));
  }
  bool listed = floor > -INFINITY;

  Cut cut = {-INFINITY, a.V};
  // lists a logit (of that bin) that stays under the cut
  auto list = [&](float z, int i, int bin) {
    if ((bin >= 0 && bin_of(z, top, c) != bin) || !stays(z, i, cut)) return;
    const unsigned w = weight(z, top, c);
    if (w == 0) return;
    const int at = atomicAdd(&s.n, 1);
    if (at < kList) s.list[at] = {key_of(z, i), w, 0};
  };
  const unsigned thr = unsigned(o.thr);
  u64 part = 0;  // mass of this thread's logits that stay
  bool counted = false;
  int n = 0;
  u64 total = 0;
  if (listed) {
    if (mine >= floor)  // few threads have anything
      each_if(row, [&](float z) { return z >= floor; }, [&](float z, int i) {
        if (z >= floor) list(z, i, -1);
      });
    __syncthreads();
    n = s.n;
    if (n > kList) {
      if (flat) {
        sample_rest(row, o, top, u, a.token + r, s);
        return;
      }
      listed = false;
    }
  }
  if (listed) {
    if (o.greedy) {
      int best = a.V;
      for (int q = tid; q < n; q += NT) best = min(best, index_of(s.list[q].key));
      if (best < a.V) atomicMin(&s.token, best);
      __syncthreads();
      if (tid == 0) a.token[r] = s.token;
      return;
    }
    u64 m = 0;
    for (int q = tid; q < n; q += NT) m += s.list[q].w;
    total = block_sum(m, s);
  }
#pragma unroll 1
  for (int stage = 0; stage < 2; ++stage) {  // top_k, then top_p
    if (stage == 0 ? !o.use_k || (listed && n <= o.k) : !o.use_p) continue;
    float from = top, scale = c * kBinsPerOctave;
    u64 mb = 0;
    unsigned cb = 0;
    if (!listed) {
      clear_bins(s);
      const bool count = stage == 0;
      each<4>(row, [&](float z, int) {  // without a branch: a mass of 0 changes nothing, NaN has the last bin
        const float y = (z - top) * c;
        const unsigned w = unsigned(__builtin_fmaf(__builtin_amdgcn_exp2f(y), 2147483648.0f, 0.5f));
        const int q = int(fminf(y * -kBinsPerOctave, float(kBins - 1)));
        atomicAdd(&s.mass[q], u64(w));
        if (count) atomicAdd(&s.cnt[q], w ? 1u : 0u);
      });
      __syncthreads();
      if (tid == 0) s.n = 0;
      if (!o.use_k) {
        u64 m = 0;
        for (int q = tid; q < kBins; q += NT) m += s.mass[q];
        total = block_sum(m, s);
      }
    }
    // bins past the top_k cut hold logits that are gone; none of them can
    // hold the top_p cut, because the mass ahead of them is at least total
    const Before before = {stage == 0, o.k, double(o.p) * double(total)};
    if (!listed) {
      find_bin(before, 0, 0, s);
      const int bin = s.bin;
      mb = s.mass_before;
      cb = s.cnt_before;
      // a little more than the bin (bounds that are not numbers, of a c near 0, leave nothing out)
      const float step = 1.0f / scale, slack = 0.01f * step + 1e-6f * (fabsf(top) + float(bin + 1) * step);
      const float low = bin < kBins - 1 ? top - float(bin + 1) * step - slack : -3.4028235e38f;
      const float high = top - float(bin) * step + slack;
      if (stage == 0 && o.use_p) {
        each_if(row, [&](float z) { return !(z < low) & !(z > high); }, [&](float z, int i) { list(z, i, bin); });
      } else {  // nothing more is cut: the masses of the bins ahead, in the same pass
        counted = true;
        each_if(row,
                [&](float z) {
                  const float y = (z - top) * c;
                  const unsigned w = unsigned(__builtin_fmaf(__builtin_amdgcn_exp2f(y), 2147483648.0f, 0.5f));
                  const int q = int(fminf(y * -kBinsPerOctave, float(kBins - 1)));
                  part += (q < bin) & (w >= thr) ? w : 0u;
                  return q == bin;
                },
                [&](float z, int i) { list(z, i, bin); });
      }
      __syncthreads();
      n = s.n;
      if (n > kList) {
        sample_rest(row, o, top, u, a.token + r, s);
        return;
      }
      from = fminf(high, top);  // bins of the bin
      scale = from > low ? float(kBins) / (from - low) : 0.0f;
    }
    cut = cut_of_list(n, from, scale, mb, cb, cut, before, &total, s);
  }
  if (listed) {
    draw_from_list(n, u, cut, o.thr, a.V, a.token + r, s);
    return;
  }
  auto mass_of = [&](float z, int i) {
    const unsigned w = weight_near(z, top, c);
    return u64(stays(z, i, cut) & (w >= thr) ? w : 0u);
  };
  if (!counted) {
    each<4>(row, [&](float z, int i) { part += mass_of(z, i); });
    part = wave_sum64(part);
  } else {  // and what stays of the listed bin
    part = wave_sum64(part);
    clear_bins(s);
    const u64 last = key_of(cut.z, cut.i);
    for (int q = tid; q < n; q += NT) {
      const Item x = s.list[q];
      if (x.key >= last && x.w >= thr) atomicAdd(&s.mass[row.wave_of(index_of(x.key))], u64(x.w));
    }
    __syncthreads();
    part += s.mass[wave];
  }
  draw_from_row(row, u, part, mass_of, a.token + r, s);
}

// ---------------------------------------------------------------------------
// Acceptance: one workgroup per tree.  A slot is taken if its draft token was
// sampled at its parent and no lower slot of that parent has it too; the
// accepted node is the deepest whose ancestors are all taken.  A chain of three
// loads (parents, their tokens, ancestors): 4 to 5 us, 8 x 64 and 32 x 33 slots.
// ---------------------------------------------------------------------------
__global__ __launch_bounds__(GDN_MAX_T) void accept_kernel(int B, int T, const void* meta, const int32_t* draft,
                                                          const int32_t* token, int32_t* accepted,
                                                          int32_t* n_emitted, int32_t* emitted) {
  __shared__ int s_child[GDN_MAX_T];  // lowest matching child of a slot
  __shared__ u64 s_ok[GDN_MAX_T / 64];
  __shared__ int s_best;
  const int b = blockIdx.x, i = threadIdx.x, lane = i % kWave;
  const MetaPtrs m = meta_ptrs(meta, B, T);
  const size_t bt = size_t(b) * T;
  const bool valid = !meta || m.status[b] == 0;
  int par = kPad, dep = -1;
  if (i < T && valid) {
    par = meta ? m.parent[bt + i] : i - 1;
    dep = meta ? m.depth[bt + i] : i;
  }
  if (i < T) s_child[i] = T;
  if (i == 0) s_best = -1;
  __syncthreads();
  const int tok = i < T ? draft[bt + i] : -1;
  bool ok = dep >= 0 && par >= 0 && par < T && tok >= 0 && tok == token[bt + par];
  if (ok) atomicMin(&s_child[par], i);
  __syncthreads();
  ok = dep == 0 || (ok && s_child[par] == i);
  const u64 bits = __ballot(ok);
  if (lane == 0) s_ok[i / kWave] = bits;
  __syncthreads();
  bool on = ok;
  if (meta) {
    for (int w = 0; on && w < m.W; ++w) on = (m.anc[(bt + i) * m.W + w] & ~s_ok[w]) == 0;
  } else {
    for (int w = 0; on && w <= i / kWave; ++w) {
      const u64 need = w < i / kWave ? ~u64(0) : (u64(1) << lane) - 1;
      on = (need & ~s_ok[w]) == 0;
    }
  }
  // depths of the slots that are on are 0, 1, .., one slot each
  if (on) atomicMax(&s_best, dep);
  if (i < T) emitted[bt + i] = -1;
  __syncthreads();
  const int last = s_best;
  if (on && dep > 0) emitted[bt + dep - 1] = tok;
  if (on && dep == last) {
    emitted[bt + last] = token[bt + i];
    accepted[b] = i;
  }
  if (i == 0) {
    n_emitted[b] = last + 1;
    if (last < 0) accepted[b] = -1;
  }
}

int after_launch(const char* who) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? GDN_OK : set_error(GDN_EHIP, "%s: launch: %s", who, hipGetErrorString(e));
}

}  // namespace

// Threads for a row.  Between the passes over a row every wave takes part in
// the same bookkeeping, so with many rows fewer waves a row are faster.  In us
// with 256 / 512 / 1024 threads, without the acceptance:
//   one row of 131072 in fp32, top_p            104 /  62 /  55
//   256 rows of 131072 in bf16, top_p           124 /  78 /  72
//   528 rows of 131072 in bf16, top_p           209 / 172 / 170
//   1056 rows of 50001 in fp32, top_p           145 / 131 / 173
//   2048 rows of 17000 in bf16, top_p            77 / 108 / 211
//   2048 rows of 17000 in fp32, top_k            60 /  79 / 144
//   4096 rows of 33000 in bf16, top_p           204 / 275 / 513
//   4096 rows of 8000 in fp32, top_k             72 / 127 / 269
// From 2048 rows on only rows of 65000 in fp32 do better with 512 (287 and 268).
// A short row leaves many threads nothing to load: one of 8000 takes 15 / 14 / 17.
template <typename T>
static int launch_type(const SampleArgs& a, hipStream_t stream) {
  const long long rows = (long long)(a.B) * a.T, vectors = a.V / Pack<T>::kN;
  if (rows >= 2048 || vectors <= 2048) sample_kernel<T, 256><<<rows, 256, 0, stream>>>(a);
  else if (rows > 256 || vectors <= 4096) sample_kernel<T, 512><<<rows, 512, 0, stream>>>(a);
  else sample_kernel<T, 1024><<<rows, 1024, 0, stream>>>(a);
  return after_launch("sample");
}

int launch_sample(const SampleArgs& a, hipStream_t stream) {
  return a.dtype == GDN_BF16 ? launch_type<BF16>(a, stream) : launch_type<float>(a, stream);
}

int launch_accept(int B, int T, const void* meta, const int32_t* draft, const int32_t* token, int32_t* accepted,
                  int32_t* n_emitted, int32_t* emitted, hipStream_t stream) {
  accept_kernel<<<B, (T + kWave - 1) / kWave * kWave, 0, stream>>>(B, T, meta, draft, token, accepted, n_emitted,
                                                                   emitted);
  return after_launch("accept");
}

}  // namespace gdn
