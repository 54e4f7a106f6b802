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
//   1  largest logit
//   2  counts and masses of bins of (top - z) c, 64 per octave of the mass
//   3  the bin of the cut, its logits gathered and ranked exactly
//   4  masses that stay, in vocabulary order, and the place of u in them
// ---------------------------------------------------------------------------
constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / kWave;
constexpr int kBins = 2048;
constexpr float kBinsPerOctave = 64.0f;  // kBins / 32: w is 0 beyond 32 octaves
constexpr int kList = 2048;              // logits of one bin that are ranked in LDS

typedef unsigned long long u64;

struct Cut {
  float z;  // what stays: logits above z, and those equal to z up to index i
  int i;
};

struct Shared {
  u64 mass[kBins];
  unsigned cnt[kBins];
  float lz[kList];
  int li[kList];
  unsigned lw[kList];
  u64 red[kWaves];
  unsigned redc[kWaves];
  int n;
  int bin;
  u64 mass_before, sum;
  unsigned cnt_before;
  Cut cut;
  int token;
};

__device__ __forceinline__ unsigned weight(float z, float top, float c) {
  if (z == top) return 0x80000000u;
  // NaN (a masked logit under an infinite temperature) converts to 0
  return unsigned(__builtin_amdgcn_exp2f((z - top) * c) * 2147483648.0f + 0.5f);
}

__device__ __forceinline__ int bin_of(float z, float top, float c) {
  return z == top ? 0 : min(kBins - 1, int((top - z) * c * kBinsPerOctave));
}

__device__ __forceinline__ u64 wave_sum64(u64 v) {
  for (int s = 1; s < kWave; s <<= 1) v += __shfl_xor(v, s);
  return v;
}

// Sum over the workgroup, in every thread.
__device__ u64 block_sum(u64 v, Shared& s) {
  v = wave_sum64(v);
  __syncthreads();
  if (threadIdx.x % kWave == 0) s.red[threadIdx.x / kWave] = v;
  __syncthreads();
  u64 t = 0;
  for (int w = 0; w < kWaves; ++w) t += s.red[w];
  return t;
}

// A row of logits read in 16-byte vectors.  A row may start anywhere: vector
// j holds elements j X - lead .. + X - 1, those outside the row are -inf.
template <typename T>
struct Row {
  static constexpr int X = Pack<T>::kN;
  const T* p;
  int V, lead, n;  // vectors
  __device__ Row(const T* q, int v) : p(q), V(v) {
    lead = int((reinterpret_cast<uintptr_t>(q) & 15) / sizeof(T));
    n = (lead + V + X - 1) / X;
  }
  __device__ __forceinline__ int first(int j) const { return j * X - lead; }
  __device__ __forceinline__ void load(int j, float (&z)[X]) const {
    const int i0 = first(j);
    if (i0 >= 0 && i0 + X <= V) {
      __align__(16) T x[X];
      copy16(x, p + i0);
#pragma unroll
      for (int e = 0; e < X; ++e) z[e] = to_f32(x[e]);
    } else {
#pragma unroll
      for (int e = 0; e < X; ++e) z[e] = i0 + e >= 0 && i0 + e < V ? to_f32(p[i0 + e]) : -INFINITY;
    }
#pragma unroll
    for (int e = 0; e < X; ++e) z[e] = z[e] != z[e] ? -INFINITY : z[e];
  }
};

// f(z, i) for every logit of the row.  Wave w takes the w-th part of the row,
// in order.
template <typename T, typename F>
__device__ __forceinline__ void each(const Row<T>& row, F f) {
  constexpr int X = Row<T>::X;
  const int per = (row.n + kWaves * kWave - 1) / (kWaves * kWave);
  const int w = threadIdx.x / kWave, lane = threadIdx.x % kWave;
  for (int j = 0; j < per; ++j) {
    const int v = (w * per + j) * kWave + lane;
    if (v >= row.n) break;
    float z[X];
    row.load(v, z);
#pragma unroll
    for (int e = 0; e < X; ++e) f(z[e], row.first(v) + e);
  }
}

__device__ __forceinline__ bool stays(float z, int i, const Cut& c) { return z > c.z || (z == c.z && i <= c.i); }

// The last of the logits in the order (z falling, index rising) for which
// before(count of those ahead, mass of those ahead) holds; it holds for the
// first one and, once it fails, for none after.  Only logits that stay under
// `cut` count.  By halving the value, then the index: for bins of more
// logits than the list holds (many equal ones).
template <typename T, typename F>
__device__ Cut bisect(const Row<T>& row, float top, float c, Cut cut, F before, Shared& s) {
  // ordered image of a float: larger value, larger key
  auto key = [](float z) {
    const unsigned b = __float_as_uint(z + 0.0f);  // -0 as 0
    return b >> 31 ? ~b : b | 0x80000000u;
  };
  auto ahead = [&](unsigned k, int i) {  // holds for an element at (k, i)?
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
    return before(cnt, mass);
  };
  unsigned lo = key(-INFINITY), hi = key(top);  // hi holds at index 0
  while (lo < hi) {
    const unsigned mid = lo + (hi - lo) / 2;
    if (ahead(mid, 0)) hi = mid;
    else lo = mid + 1;
  }
  int a = 0, b = row.V - 1;  // the last index that holds
  while (a < b) {
    const int mid = a + (b - a + 1) / 2;
    if (ahead(hi, mid)) a = mid;
    else b = mid - 1;
  }
  const unsigned bits = hi >> 31 ? hi & 0x7fffffffu : ~hi;
  return {__uint_as_float(bits), a};
}

// Prefix over the bins: s.bin = the last bin for whose first logit `before`
// holds, s.cnt_before and s.mass_before what lies ahead of it, s.sum all mass.
template <typename F>
__device__ void find_bin(F before, Shared& s) {
  constexpr int kPer = kBins / kThreads;
  const int tid = threadIdx.x, lane = tid % kWave, w = tid / kWave;
  u64 mass = 0;
  unsigned cnt = 0;
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    mass += s.mass[tid * kPer + e];
    cnt += s.cnt[tid * kPer + e];
  }
  u64 im = mass;
  unsigned ic = cnt;
  for (int d = 1; d < kWave; d <<= 1) {
    const u64 um = __shfl_up(im, d);
    const unsigned uc = __shfl_up(ic, d);
    if (lane >= d) im += um, ic += uc;
  }
  __syncthreads();
  if (lane == kWave - 1) s.red[w] = im, s.redc[w] = ic;
  __syncthreads();
  u64 m = im - mass, all = 0;
  unsigned n = ic - cnt;
  for (int k = 0; k < kWaves; ++k) {
    if (k < w) m += s.red[k], n += s.redc[k];
    all += s.red[k];
  }
  // each thread's last bin that holds; the largest of them is the answer
  int best = -1;
  u64 bm = 0;
  unsigned bn = 0;
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    const unsigned c = s.cnt[tid * kPer + e];
    if (c && before(n, m)) best = tid * kPer + e, bm = m, bn = n;
    m += s.mass[tid * kPer + e];
    n += c;
  }
  if (tid == 0) s.bin = 0, s.sum = all;
  __syncthreads();
  if (best >= 0) atomicMax(&s.bin, best);
  __syncthreads();
  if (best == s.bin) s.cnt_before = bn, s.mass_before = bm;
  __syncthreads();
}

// The cut for `before`, inside bin s.bin; *kept = mass up to and with the cut.
template <typename T, typename F>
__device__ Cut find_cut(const Row<T>& row, float top, float c, Cut old, F before, u64* kept, Shared& s) {
  const int tid = threadIdx.x;
  if (tid == 0) s.n = 0;
  __syncthreads();
  const int bin = s.bin;
  const u64 mb = s.mass_before;
  const unsigned cb = s.cnt_before;
  each(row, [&](float z, int i) {
    if (!(z > -INFINITY && bin_of(z, top, c) == bin && stays(z, i, old))) return;
    const unsigned w = weight(z, top, c);
    if (w == 0) return;
    const int at = atomicAdd(&s.n, 1);
    if (at < kList) s.lz[at] = z, s.li[at] = i, s.lw[at] = w;
  });
  __syncthreads();
  const int n = s.n;
  if (n > kList) {
    const Cut cut = bisect(row, top, c, old, before, s);
    u64 mass = 0;
    each(row, [&](float z, int i) {
      if (stays(z, i, cut) && stays(z, i, old)) mass += weight(z, top, c);
    });
    *kept = block_sum(mass, s);
    return cut;
  }
  if (tid == 0) s.sum = 0;
  __syncthreads();
  u64 mine = 0;
  for (int a = tid; a < n; a += kThreads) {
    const float z = s.lz[a];
    const int i = s.li[a];
    u64 mass = mb;
    unsigned cnt = cb;
    for (int q = 0; q < n; ++q) {
      const float y = s.lz[q];
      if (y > z || (y == z && s.li[q] < i)) mass += s.lw[q], ++cnt;
    }
    if (before(cnt, mass)) {
      // the last one: nothing of the list after it holds
      const u64 next = mass + s.lw[a];
      mine = next > mine ? next : mine;
      atomicMax(&s.sum, next);
    }
  }
  __syncthreads();
  const u64 best = s.sum;
  // masses rise strictly along the order (w > 0), so one logit ends at best
  for (int a = tid; a < n && mine == best; a += kThreads) {
    const float z = s.lz[a];
    const int i = s.li[a];
    u64 mass = mb + s.lw[a];
    for (int q = 0; q < n; ++q) {
      const float y = s.lz[q];
      if (y > z || (y == z && s.li[q] < i)) mass += s.lw[q];
    }
    if (mass == best) s.cut = {z, i};
  }
  __syncthreads();
  *kept = best;
  return s.cut;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void sample_kernel(SampleArgs a) {
  __shared__ Shared s;
  const int r = blockIdx.x, b = r / a.T, tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  if (a.meta) {
    const MetaPtrs m = meta_ptrs(a.meta, a.B, a.T);
    if (m.status[b] != 0 || m.depth[r] < 0) {
      if (tid == 0) a.token[r] = -1;
      return;
    }
  }
  const Row<T> row(reinterpret_cast<const T*>(a.logits) + (long long)(r) * a.ld, a.V);
  const float t = a.temperature ? a.temperature[b] : 1.0f;
  const int k = a.top_k ? a.top_k[b] : 0;
  const float p = a.top_p ? a.top_p[b] : 1.0f;
  const float least = a.min_p ? a.min_p[b] : 0.0f;

  float top = -INFINITY;
  each(row, [&](float z, int) { top = fmaxf(top, z); });
  for (int d = 1; d < kWave; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
  float* redf = reinterpret_cast<float*>(s.red);
  if (lane == 0) redf[wave] = top;
  if (tid == 0) s.token = a.V;
  __syncthreads();
  for (int w = 0; w < kWaves; ++w) top = fmaxf(top, redf[w]);
  if (top == -INFINITY) {
    if (tid == 0) a.token[r] = -1;
    return;
  }
  if (!(t > 0.0f)) {
    int best = a.V;
    each(row, [&](float z, int i) {
      if (z == top) best = min(best, i);
    });
    if (best < a.V) atomicMin(&s.token, best);
    __syncthreads();
    if (tid == 0) a.token[r] = s.token;
    return;
  }
  const float c = (1.0f / t) * 1.44269504088896340736f;
  Cut cut = {-INFINITY, a.V};
  const bool use_k = k > 0 && k < a.V, use_p = !(p >= 1.0f);
  if (use_k || use_p) {
    for (int q = tid; q < kBins; q += kThreads) s.mass[q] = 0, s.cnt[q] = 0;
    __syncthreads();
    each(row, [&](float z, int) {
      const unsigned w = weight(z, top, c);
      if (w) {
        const int q = bin_of(z, top, c);
        atomicAdd(&s.mass[q], u64(w));
        atomicAdd(&s.cnt[q], 1u);
      }
    });
    __syncthreads();
    u64 total = 0;
    if (use_k) {
      auto before = [k](u64 cnt, u64) { return cnt < u64(k); };
      find_bin(before, s);
      cut = find_cut(row, top, c, cut, before, &total, s);
    }
    if (use_p) {
      if (!use_k) {
        find_bin([](u64, u64) { return true; }, s);
        total = s.sum;
      }
      const double want = double(p) * double(total);
      auto before = [want](u64 cnt, u64 mass) { return cnt == 0 || double(mass) < want; };
      // bins past the top_k cut hold only logits that are gone; none of them
      // can hold the p cut, because the mass before them is at least total
      __syncthreads();
      find_bin(before, s);
      u64 kept;
      cut = find_cut(row, top, c, cut, before, &kept, s);
    }
  }
  const u64 thr = least > 0.0f ? u64(ceil(double(fminf(least, 1.0f)) * 2147483648.0)) : 0;
  // masses in vocabulary order: of a wave's part, of its 64-vector rows, of
  // the lanes, of a vector
  auto mass_of = [&](float z, int i) {
    if (!stays(z, i, cut)) return u64(0);
    const u64 w = weight(z, top, c);
    return w >= thr ? w : u64(0);
  };
  u64 mine = 0;
  each(row, [&](float z, int i) { mine += mass_of(z, i); });
  mine = wave_sum64(mine);
  __syncthreads();
  if (lane == 0) s.red[wave] = mine;
  __syncthreads();
  u64 total = 0, before = 0;
  for (int w = 0; w < kWaves; ++w) total += s.red[w];
  const double want = double(a.u[r]) * double(total);
  u64 goal = want > 0.0 ? u64(want) : 0;  // the first running mass above it
  goal = goal < total ? goal : total - 1;
  for (int w = 0; w < wave; ++w) before += s.red[w];
  if (goal < before || goal >= before + mine) return;
  const int per = (row.n + kThreads - 1) / kThreads;
  for (int j = 0; j < per; ++j) {
    const int v = (wave * per + j) * kWave + lane;
    float z[Row<T>::X];
    u64 m = 0;
    if (v < row.n) {
      row.load(v, z);
#pragma unroll
      for (int e = 0; e < Row<T>::X; ++e) m += mass_of(z[e], row.first(v) + e);
    }
    u64 inc = m;
    for (int d = 1; d < kWave; d <<= 1) {
      const u64 up = __shfl_up(inc, d);
      if (lane >= d) inc += up;
    }
    const u64 all = __shfl(inc, kWave - 1);
    if (goal < before + all) {
      u64 run = before + inc - m;
      if (goal >= run && goal < run + m) {
        int at = -1;
#pragma unroll
        for (int e = 0; e < Row<T>::X; ++e) {
          run += mass_of(z[e], row.first(v) + e);
          if (at < 0 && run > goal) at = row.first(v) + e;
        }
        a.token[r] = at;
      }
      return;
    }
    before += all;
  }
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

int launch_sample(const SampleArgs& a, hipStream_t stream) {
  if (a.dtype == GDN_BF16)
    sample_kernel<BF16><<<a.B * a.T, kThreads, 0, stream>>>(a);
  else
    sample_kernel<float><<<a.B * a.T, kThreads, 0, stream>>>(a);
  return after_launch("sample");
}

int launch_accept(int B, int T, const void* meta, const int32_t* draft, const int32_t* token, int32_t* accepted,
                  int32_t* n_emitted, int32_t* emitted, hipStream_t stream) {
  accept_kernel<<<B, (T + kWave - 1) / kWave * kWave, 0, stream>>>(B, T, meta, draft, token, accepted, n_emitted,
                                                                   emitted);
  return after_launch("accept");
}

}  // namespace gdn
