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
// Rows for which LDS is too small (thousands of equal logits, a low min_p) are
// left to a second kernel.
// ---------------------------------------------------------------------------
constexpr int kBins = 1024;
constexpr float kBinsPerOctave = kBins / 32.0f;  // w is 0 beyond 32 octaves
constexpr int kFew = 128;  // logits up to here are ranked as they are

typedef unsigned long long u64;

struct Cut {
  float z;  // what stays: logits above z, and those equal to z up to index i
  int i;
};

struct alignas(16) Item {
  float z;
  int i;
  unsigned w, none;
};

template <int NT>
struct Shared {
  static constexpr int kWaves = NT / kWave, kList = 4 * NT;
  u64 mass[kBins];
  unsigned cnt[kBins];
  Item list[kList];  // listed logits, their indices and masses
  unsigned short sub[kList];  // places in the list
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
__device__ const u32x4 g_low = {0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u};

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
template <typename T, int NT, typename F>
__device__ __forceinline__ void each_of(const Row<T, NT>& row, int w, int j0, int j1, F f) {
  constexpr int X = Row<T, NT>::X, kAhead = 8;
  for (int j = j0; j < j1; j += kAhead) {
    u32x4 x[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) x[k] = row.load(row.at(w, j + k));
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

// The same for the vectors that hold a logit for which test(z) is true: a
// comparison or two a logit where few vectors do.
template <typename T, int NT, typename P, typename F>
__device__ __forceinline__ void each_if(const Row<T, NT>& row, P test, F f) {
  constexpr int X = Row<T, NT>::X, kAhead = 8;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  for (int j = 0; j < row.per; j += kAhead) {
    u32x4 x[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) x[k] = row.load(row.at(w, j + k));
    unsigned hits = 0;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (row.edge(w, j + k)) x[k] = row.mend(x[k], row.at(w, j + k));
      bool hit = false;
#pragma unroll
      for (int e = 0; e < X; ++e) hit = hit | test(Row<T, NT>::value(x[k], e));
      hits |= (hit && j + k < row.per ? 1u : 0u) << k;
    }
    for (; hits; hits &= hits - 1) {
      const int v = row.at(w, j + __builtin_ctz(hits));
      const u32x4 y = row.mend(row.load(v), v);
#pragma unroll
      for (int e = 0; e < X; ++e) {
        const float z = Row<T, NT>::value(y, e);
        if (test(z)) f(z, row.first(v) + e);
      }
    }
  }
}

template <typename T, int NT, typename F>
__device__ __forceinline__ void each(const Row<T, NT>& row, F f) {
  each_of(row, __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), 0, row.per, f);
}

__device__ __forceinline__ bool stays(float z, int i, const Cut& c) { return z > c.z || (z == c.z && i <= c.i); }
__device__ __forceinline__ bool ahead_of(float y, int j, float z, int i) { return y > z || (y == z && j < i); }

// The last logit in the order (z falling, index rising) for which
// before(count of those ahead, mass of those ahead) holds; it holds for the
// first one and, once it fails, for none after.  Only logits that stay under
// `cut` count.  By halving the value, then the index: for bins of more
// logits than the list holds (many equal ones).
template <typename T, int NT, typename F>
__device__ __forceinline__ Cut bisect(const Row<T, NT>& row, float top, float c, Cut cut, F before, Shared<NT>& s) {
  // ordered image of a float: larger value, larger key
  auto key = [](float z) {
    const unsigned b = __float_as_uint(z + 0.0f);  // -0 as 0
    return b >> 31 ? ~b : b | 0x80000000u;
  };
  unsigned lo = key(-INFINITY), hi = key(top);  // hi holds at index 0
  int a = 0, b = row.V - 1;                      // then the last index that holds
  while (lo < hi || a < b) {
    const bool values = lo < hi;
    const unsigned k = values ? lo + (hi - lo) / 2 : hi;
    const int i = values ? 0 : a + (b - a + 1) / 2;
    u64 mass = 0, cnt = 0;
    each(row, [&](float z, int j) {
      if (!stays(z, j, cut)) return;
      const unsigned kz = key(z);
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
  const unsigned bits = hi >> 31 ? hi & 0x7fffffffu : ~hi;
  return {__uint_as_float(bits), a};
}

template <int NT>
__device__ __forceinline__ void clear_bins(Shared<NT>& s) {
  for (int q = threadIdx.x; q < kBins; q += NT) s.mass[q] = 0, s.cnt[q] = 0;
  __syncthreads();
}

// Prefix over the bins: s.bin = the last bin that holds a mass and for whose
// first logit `before` holds, s.cnt_before and s.mass_before what lies ahead
// of it.
template <int NT, typename F>
__device__ __forceinline__ void find_bin(F before, Shared<NT>& s) {
  constexpr int kPer = kBins / NT;
  const int tid = threadIdx.x, lane = tid % kWave, w = tid / kWave;
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
#pragma unroll
  for (int k = 0; k < NT / kWave; ++k) {
    const u64 rm = s.red[k];
    const unsigned rn = s.redc[k];
    m += k < w ? rm : 0;
    n += k < w ? rn : 0;
  }
  // each thread's last bin that holds; the largest of them is the answer
  int best = -1;
  u64 bm = 0;
  unsigned bn = 0;
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    const u64 q = s.mass[tid * kPer + e];
    if (q && before(n, m)) best = tid * kPer + e, bm = m, bn = n;
    m += q;
    n += s.cnt[tid * kPer + e];
  }
  if (best >= 0) atomicMax(&s.bin, best);
  __syncthreads();
  if (best == s.bin) s.cnt_before = bn, s.mass_before = bm;
  __syncthreads();
}

// The last of the m list places in s.sub (or, identity: of the first m) for
// which `before` holds, counting those that stay under `old`; cb and mb lie
// ahead of all.  *kept = the mass up to and with it.
template <bool kIdentity, int NT, typename F>
__device__ __forceinline__ Cut rank_cut(int m, u64 mb, unsigned cb, Cut old, F before, u64* kept, Shared<NT>& s) {
  if (threadIdx.x == 0) s.sum = 0;
  __syncthreads();
  u64 mine = 0;
  Cut cut = {0.0f, 0};
  for (int a = threadIdx.x; a < m; a += NT) {
    const Item x = s.list[kIdentity ? a : s.sub[a]];
    if (!stays(x.z, x.i, old)) continue;
    u64 mass = mb;
    unsigned cnt = cb;
#pragma unroll 4
    for (int q = 0; q < m; ++q) {
      const Item y = s.list[kIdentity ? q : s.sub[q]];
      const bool first = ahead_of(y.z, y.i, x.z, x.i);
      mass += first ? y.w : 0u;
      cnt += first ? 1u : 0u;
    }
    // masses rise along the order (no listed mass is 0): the largest that
    // holds is the last one
    if (before(cnt, mass) && mass + x.w > mine) mine = mass + x.w, cut = {x.z, x.i};
  }
  if (mine) atomicMax(&s.sum, mine);
  __syncthreads();
  const u64 best = s.sum;
  if (mine == best) s.cut = cut;
  __syncthreads();
  *kept = best;
  cut = s.cut;
  __syncthreads();
  return cut;
}

// The cut for `before` among the n listed logits that stay under `old`; mb and
// cb lie ahead of all, and all lie between (top - z) scale = 0 and kBins.
template <int NT, typename F>
__device__ __forceinline__ Cut cut_of_list(int n, float top, float scale, u64 mb, unsigned cb, Cut old, F before, u64* kept,
                                           Shared<NT>& s) {
  const int tid = threadIdx.x;
  if (n <= kFew) return rank_cut<true>(n, mb, cb, old, before, kept, s);
  auto bin = [&](float z) { return z == top ? 0 : int(fmaxf(0.0f, fminf((top - z) * scale, float(kBins - 1)))); };
  clear_bins(s);
  for (int a = tid; a < n; a += NT) {
    const Item x = s.list[a];
    if (stays(x.z, x.i, old)) {
      const int q = bin(x.z);
      atomicAdd(&s.mass[q], u64(x.w));
      atomicAdd(&s.cnt[q], 1u);
    }
  }
  if (tid == 0) s.m = 0;
  __syncthreads();
  find_bin([&](u64 cnt, u64 mass) { return before(cnt + cb, mass + mb); }, s);
  for (int a = tid; a < n; a += NT) {
    const Item x = s.list[a];
    if (stays(x.z, x.i, old) && bin(x.z) == s.bin) s.sub[atomicAdd(&s.m, 1)] = a;
  }
  __syncthreads();
  return rank_cut<false>(s.m, mb + s.mass_before, cb + s.cnt_before, old, before, kept, s);
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
  if (!few) clear_bins(s);
  for (int a = tid; a < n; a += NT) {
    const Item x = s.list[a];
    const bool on = stays(x.z, x.i, cut) && x.w >= least;
    if (!on) s.list[a].w = 0;
    else if (!few) atomicAdd(&s.mass[x.i >> shift], u64(x.w));
  }
  if (tid == 0) s.m = 0;
  __syncthreads();
  if (few) {
    if (tid >= n) return;
    const Item x = s.list[tid];
    u64 run = 0, total = 0;
#pragma unroll 4
    for (int q = 0; q < n; ++q) {
      const Item y = s.list[q];
      total += y.w;
      run += y.i < x.i ? y.w : 0u;
    }
    const u64 goal = goal_of(u, total);
    if (goal >= run && goal < run + x.w) *token = x.i;
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
    if (x.w && x.i >> shift == bucket) s.sub[atomicAdd(&s.m, 1)] = a;
  }
  __syncthreads();
  const int m = s.m;
  for (int a = tid; a < m; a += NT) {
    const Item x = s.list[s.sub[a]];
    u64 run = s.mass_before;
#pragma unroll 4
    for (int q = 0; q < m; ++q) {
      const Item y = s.list[s.sub[q]];
      run += y.i < x.i ? y.w : 0u;
    }
    if (goal >= run && goal < run + x.w) *token = x.i;
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
  each_of(row, part, j0, j1, [&](float z, int i) { sub += mass_of(z, i); });
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

struct ByCount {
  int k;
  __device__ __forceinline__ bool operator()(u64 cnt, u64) const { return cnt < u64(k); }
};
struct ByMass {
  double want;
  __device__ __forceinline__ bool operator()(u64 cnt, u64 mass) const { return mass == 0 || double(mass) < want; }
};

constexpr int kPending = -2;  // token of a row that is left for the second kernel

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
  each(row, [&](float z, int) { mine = fmaxf(mine, z); });
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
  // only the logits equal to top have a mass
  const bool flat = o.greedy || top == INFINITY || c == INFINITY;

  if (!flat && !o.use_k && !o.use_p && !o.use_m) {  // no cut
    u64 part = 0;
    each(row, [&](float z, int) { part += weight_near(z, top, c); });
    draw_from_row(row, u, wave_sum64(part), [&](float z, int) { return u64(weight_near(z, top, c)); }, a.token + r, s);
    return;
  }
  // the floor, where there is one
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
    find_bin(ByCount{o.k}, s);  // the bin of the k-th maximum
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
  } else if (!o.use_k && !o.use_p) {
    const float down = (log2f(fminf(o.least, 1.0f)) - 0.01f) / c;
    floor = fmaxf(-3.4028235e38f, top + down - 1e-6f * (fabsf(top) + fabsf(down)));
  }
  if (floor == -INFINITY) {
    // masses by bins, the bin of the cut, what stays in vocabulary order
    const bool count = o.use_k;
    u64 total = 0;
    auto masses = [&]() {
      each(row, [&](float z, int) {  // without a branch: a mass of 0 changes nothing, NaN has the last bin
        const float y = (z - top) * c;
        const unsigned w = unsigned(__builtin_fmaf(__builtin_amdgcn_exp2f(y), 2147483648.0f, 0.5f));
        const int q = int(fminf(y * -kBinsPerOctave, float(kBins - 1)));
        atomicAdd(&s.mass[q], u64(w));
        if (count) atomicAdd(&s.cnt[q], w ? 1u : 0u);
      });
      __syncthreads();
    };
    clear_bins(s);
    masses();
    Cut cut = {-INFINITY, a.V};
    bool full = false;
    auto cut_row = [&](auto before, u64* kept) {
      find_bin(before, s);
      const int bin = s.bin;
      // a little more than the bin (bounds that are not numbers, of a c near 0, leave nothing out)
      const float step = 1.0f / (kBinsPerOctave * c), slack = 0.01f * step + 1e-6f * (fabsf(top) + float(bin + 1) * step);
      const float low = bin < kBins - 1 ? top - float(bin + 1) * step - slack : -3.4028235e38f;
      const float high = top - float(bin) * step + slack;
      const u64 mb = s.mass_before;
      const unsigned cb = s.cnt_before;
      each_if(row, [&](float z) { return !(z < low) & !(z > high); }, [&](float z, int i) {
        if (bin_of(z, top, c) != bin || !stays(z, i, cut)) return;
        const unsigned w = weight_near(z, top, c);
        if (w == 0) return;
        const int at = atomicAdd(&s.n, 1);
        if (at < kList) s.list[at] = {z, i, w, 0};
      });
      __syncthreads();
      const int m = s.n;
      __syncthreads();
      if (tid == 0) s.n = 0;
      if (m > kList) {
        full = true;
        return;
      }
      // bins of the bin
      const float from = fminf(high, top), scale = from > low ? float(kBins) / (from - low) : 0.0f;
      cut = cut_of_list(m, from, scale, mb, cb, cut, before, kept, s);
    };
    if (o.use_k) {
      cut_row(ByCount{o.k}, &total);
    } else {
      u64 m = 0;
      for (int q = tid; q < kBins; q += NT) m += s.mass[q];
      total = block_sum(m, s);
    }
    // bins past the top_k cut hold logits that are gone; none of them can
    // hold the next cut, because the mass ahead of them is at least total
    u64 kept;
    if (o.use_p && !full) {
      if (o.use_k) {  // the bins of the list took their place
        clear_bins(s);
        masses();
      }
      cut_row(ByMass{double(o.p) * double(total)}, &kept);
    }
    if (full) {
      if (tid == 0) a.token[r] = kPending;
      return;
    }
    const unsigned thr = unsigned(o.thr);
    auto mass_of = [&](float z, int i) {
      const unsigned w = weight_near(z, top, c);
      return u64((z > cut.z) | ((z == cut.z) & (i <= cut.i)) && w >= thr ? w : 0u);
    };
    u64 part = 0;
    each(row, [&](float z, int i) { part += mass_of(z, i); });
    draw_from_row(row, u, wave_sum64(part), mass_of, a.token + r, s);
    return;
  }

  // list what is above it: few threads have anything
  if (mine >= floor)
    each_if(row, [&](float z) { return z >= floor; }, [&](float z, int i) {
      const unsigned w = weight(z, top, c);
      if (w == 0) return;
      const int at = atomicAdd(&s.n, 1);
      if (at < kList) s.list[at] = {z, i, w, 0};
    });
  __syncthreads();
  const int n = s.n;
  if (n > kList) {
    if (tid == 0) a.token[r] = kPending;
    return;
  }
  if (o.greedy) {
    int best = a.V;
    for (int q = tid; q < n; q += NT) best = min(best, s.list[q].i);
    if (best < a.V) atomicMin(&s.token, best);
    __syncthreads();
    if (tid == 0) a.token[r] = s.token;
    return;
  }
  u64 total = 0, kept;
  const float scale = c * kBinsPerOctave;
  Cut cut = {-INFINITY, a.V};
  if (o.use_k && n > o.k) {
    cut = cut_of_list(n, top, scale, 0, 0, cut, ByCount{o.k}, &total, s);
  } else {
    u64 m = 0;
    for (int q = tid; q < n; q += NT) m += s.list[q].w;
    total = block_sum(m, s);
  }
  if (o.use_p) cut = cut_of_list(n, top, scale, 0, 0, cut, ByMass{double(o.p) * double(total)}, &kept, s);
  draw_from_list(n, u, cut, o.thr, a.V, a.token + r, s);
}

// The rows that LDS is too small for: the cuts by halving, the draw over the
// row.  Seldom any.
template <typename T, int NT>
__global__ __launch_bounds__(NT, 4) void sample_rest_kernel(SampleArgs a) {
  __shared__ Shared<NT> s;
  const int r = blockIdx.x, b = r / a.T, tid = threadIdx.x;
  if (a.token[r] != kPending) return;
  __syncthreads();  // every thread has read the token
  const Row<T, NT> row(reinterpret_cast<const T*>(a.logits) + (long long)(r) * a.ld, a.V);
  const Settings o(a, b);
  const float c = o.c;
  float top = -INFINITY;
  each(row, [&](float z, int) { top = fmaxf(top, z); });
  for (int d = 1; d < kWave; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
  if (tid % kWave == 0) s.redf[tid / kWave] = top;
  if (tid == 0) s.token = a.V;
  __syncthreads();
  for (int w = 0; w < NT / kWave; ++w) top = fmaxf(top, s.redf[w]);
  if (o.greedy) {
    int best = a.V;
    each(row, [&](float z, int i) {
      if (z == top) best = min(best, i);
    });
    if (best < a.V) atomicMin(&s.token, best);
    __syncthreads();
    if (tid == 0) a.token[r] = s.token;
    return;
  }
  Cut cut = {-INFINITY, a.V};
  auto mass_of = [&](float z, int i) {
    if (!stays(z, i, cut)) return u64(0);
    const u64 w = weight(z, top, c);
    return w >= o.thr ? w : u64(0);
  };
  auto mass = [&]() {
    u64 m = 0;
    each(row, [&](float z, int i) { m += stays(z, i, cut) ? weight(z, top, c) : 0u; });
    return block_sum(m, s);
  };
  if (o.use_k) cut = bisect(row, top, c, cut, ByCount{o.k}, s);
  if (o.use_p) cut = bisect(row, top, c, cut, ByMass{double(o.p) * double(mass())}, s);
  u64 part = 0;
  each(row, [&](float z, int i) { part += mass_of(z, i); });
  draw_from_row(row, a.u[r], wave_sum64(part), mass_of, a.token + r, s);
}

// ---------------------------------------------------------------------------
// Acceptance: one workgroup per tree.  A slot is taken if its draft token was
// sampled at its parent and no lower slot of that parent has it too; the
// accepted node is the deepest whose ancestors are all taken.
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

template <typename T, int NT>
static int launch_rows(const SampleArgs& a, hipStream_t stream) {
  sample_kernel<T, NT><<<a.B * a.T, NT, 0, stream>>>(a);
  const int rc = after_launch("sample");
  if (rc != GDN_OK || a.V <= Shared<NT>::kList) return rc;  // no row needs more than the list
  sample_rest_kernel<T, 1024><<<a.B * a.T, 1024, 0, stream>>>(a);
  return after_launch("sample");
}

// Threads for a row: up to 8 vectors each.
template <typename T>
static int launch_type(const SampleArgs& a, hipStream_t stream) {
  const int vectors = a.V / Pack<T>::kN;
  if (vectors <= 8 * 256) return launch_rows<T, 256>(a, stream);
  if (vectors <= 8 * 512) return launch_rows<T, 512>(a, stream);
  return launch_rows<T, 1024>(a, stream);
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
