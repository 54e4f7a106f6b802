// gdn_kv.hip -- the paged key / value cache of the softmax-attention layers:
// appending a step's rows with the position rotation, and moving the
// accepted path's rows to the front.
#include "gdn_attn.h"

namespace gdn {
namespace {

constexpr int kThreads = 256;
constexpr int kTok = 8;    // tokens per workgroup: one bf16 value pack
constexpr int kUnits = 4;  // units of a thread in flight

// (x, y) of a pack of pairs to (x cos - y sin, y cos + x sin)
template <typename T>
__device__ __forceinline__ void turn(u32x4& x, u32x4& y, const float2* cs) {
  constexpr int X = Pack<T>::kN;
  u32x4 xo = {}, yo = {};
#pragma unroll
  for (int e = 0; e < X; ++e) {
    const float2 r = cs[e];
    if constexpr (X == 8) {
      const float p = __uint_as_float(e & 1 ? x[e / 2] & 0xffff0000u : x[e / 2] << 16);
      const float n = __uint_as_float(e & 1 ? y[e / 2] & 0xffff0000u : y[e / 2] << 16);
      const unsigned a = __builtin_bit_cast(uint16_t, (__bf16)(p * r.x - n * r.y));
      const unsigned b = __builtin_bit_cast(uint16_t, (__bf16)(n * r.x + p * r.y));
      xo[e / 2] |= a << (e & 1 ? 16 : 0);
      yo[e / 2] |= b << (e & 1 ? 16 : 0);
    } else {
      const float p = __uint_as_float(x[e]), n = __uint_as_float(y[e]);
      xo[e] = __float_as_uint(p * r.x - n * r.y);
      yo[e] = __float_as_uint(n * r.x + p * r.y);
    }
  }
  x = xo;
  y = yo;
}

// ---------------------------------------------------------------------------
// Append.
//
// Workgroups of queries hold a share of 8 slots' (head, pack) units; those of
// keys and values hold a group of 8 positions (one value pack in bf16, two in
// fp32), so that a value pack whose 8 tokens are all new is written whole.
// Bound by the chain in front of the bytes (length and depths, then pages and
// angles), which every workgroup goes through; the queries, most of the bytes,
// are on their way before it.  32 x 128 slots, 24 + 4 heads of 256, cold caches:
// 44 to 50 us for 120 MB, 58 for the 238 MB of fp32
// (64 with every load behind the checks, 50 with ordinary loads where this
// took 44; non-temporal stores took 42, but the rows are read again by the
// attention).  One token: 5 us, the chain.
// ---------------------------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(kThreads) void append_kernel(AttnArgs a, int qparts, int kparts) {
  constexpr int X = Pack<T>::kN;
  __shared__ float2 s_cs[kTok][128];  // cos and sin of the group's tokens
  __shared__ int s_page[kTok];        // page of the token, -1: absent
  __shared__ int s_bad;
  const int b = blockIdx.z, tid = threadIdx.x, h2 = a.rot / 2, d = a.c.d;
  const bool isq = int(blockIdx.y) < qparts;
  const int part = isq ? blockIdx.y : blockIdx.y - qparts, parts = isq ? qparts : kparts;
  const int H = isq ? a.Hq : a.c.Hkv;
  const size_t tok0 = size_t(b) * a.T;
  const T* src = reinterpret_cast<const T*>(isq ? a.q : a.k);
  // units of a head where the half of the rotated part is whole packs: pairs of
  // packs (c, c + half), which one thread owns (q may be q_out), then the packs
  // that are not rotated
  const int half = h2 / X, np = d / X - half;
  const bool packs = h2 % X == 0;
  const int units = kTok * H * np;
  u32x4 x0[kUnits], x1[kUnits];
  // unit u as token, head and pack: queries along the packs, keys along the
  // tokens (8 lanes write 128 bytes)
  auto unit = [&](int u, int& t, int& h, int& c) {
    if (isq) {
      const int r = u / np;
      c = u - r * np;
      t = r / H;
      h = r - t * H;
    } else {
      t = u % kTok;
      h = u / kTok / np;
      c = u / kTok - h * np;
    }
    c = c < half ? c : c + half;
  };
  auto fetch = [&](int first, int u0) {
#pragma unroll
    for (int n = 0; n < kUnits; ++n) {
      const int u = u0 + n * kThreads;
      int t, h, c;
      unit(u, t, h, c);
      const int i = first + t;
      if (u >= units || i < 0 || i >= a.T) continue;
      const T* p = src + ((tok0 + i) * H + h) * d + c * X;
      x0[n] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));  // read once
      if (c < half) x1[n] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p + h2));
    }
  };
  int u0 = part * kUnits * kThreads + tid;
  if (packs && isq) fetch(blockIdx.x * kTok, u0);

  const MetaPtrs m = meta_ptrs(a.meta, a.B, a.T);
  const int32_t* dep = m.depth + size_t(b) * a.T;
  int own[GDN_MAX_T / kThreads];  // depths of slots tid, tid + kThreads
#pragma unroll
  for (int n = 0; n < GDN_MAX_T / kThreads; ++n) {
    const int i = tid + n * kThreads;
    own[n] = i < a.T ? (a.meta ? dep[i] : i) : -1;
  }
  const int ctx = a.ctx_len[b], span = span_of(a, b);
  int status = a.meta ? m.status[b] : 0;
  if (!status) status = len_status(a, ctx, span);
  const int32_t* row = a.page_table + size_t(b) * a.c.max_pages;
  // the group's first slot; positions from a multiple of 8 on for the caches
  // (may be < 0)
  const int i0 = isq || status ? int(blockIdx.x) * kTok : ((ctx >> 3) + int(blockIdx.x)) * kTok - ctx;
  if (i0 >= a.T || (!isq && status)) return;
  if (tid < kTok) s_page[tid] = -1;
  if (tid == 0) s_bad = 0;
  __syncthreads();
  // every workgroup checks the whole sequence and takes the same decision
  int bad = 0;
#pragma unroll
  for (int n = 0; n < GDN_MAX_T / kThreads; ++n) {
    const int i = tid + n * kThreads;
    if (!status && own[n] >= 0 && (a.meta || i < span)) {
      const int pg = page_of(a.c, row, ctx + i);
      if (a.rot && (long long)(ctx) + own[n] >= a.n_pos) bad |= 1;
      if (pg < 0) bad |= 2;
      if (i >= i0 && i < i0 + kTok) s_page[i - i0] = pg;
    }
  }
  for (int u = tid; u < (status ? 0 : kTok * h2); u += kThreads) {
    const int t = u / h2, e = u % h2, i = i0 + t;
    if (i < 0 || i >= a.T) continue;
    const int at = a.meta ? dep[i] : (i < span ? i : -1);
    if (at >= 0 && (long long)(ctx) + at < a.n_pos) s_cs[t][e] = reinterpret_cast<const float2*>(a.rope)[size_t(ctx + at) * h2 + e];
  }
  if (bad) atomicOr(&s_bad, bad);
  __syncthreads();
  bad = s_bad;
  if (!status && bad) status = bad & 1 ? GDN_KV_BAD_POS : GDN_KV_BAD_PAGE;
  if (isq && a.status && blockIdx.x == 0 && part == 0 && tid == 0) a.status[b] = status;
  if (bad) {  // nothing is real
    if (!isq) return;
    __syncthreads();
    if (tid < kTok) s_page[tid] = -1;
    __syncthreads();
  }

  const int mask = (1 << a.c.page_shift) - 1;
  T *qo = reinterpret_cast<T*>(a.out), *kc = reinterpret_cast<T*>(a.k_cache), *vc = reinterpret_cast<T*>(a.v_cache);
  const int p8 = (ctx + i0) & mask;  // keys, values: place of the group's first position in its page, which all 8 share
  if (packs) {
    for (; u0 - tid < units; u0 += parts * kUnits * kThreads) {
      if (!isq || u0 >= parts * kUnits * kThreads) fetch(i0, u0);
#pragma unroll
      for (int n = 0; n < kUnits; ++n) {
        const int u = u0 + n * kThreads;
        int t, h, c;
        unit(u, t, h, c);
        const int i = i0 + t;
        if (u >= units || i < 0 || i >= a.T) continue;
        const int pg = s_page[t];
        const bool pair = c < half;
        T* dst;
        size_t step = h2;  // from a pack to its partner
        if (isq) {
          dst = qo + ((tok0 + i) * H + h) * d + c * X;
          if (pg < 0) x0[n] = x1[n] = u32x4{0, 0, 0, 0};
        } else {
          if (pg < 0) continue;
          dst = kc + block_of(a.c, pg, h) + ((size_t(c) << a.c.page_shift) + p8 + t) * X;
          step <<= a.c.page_shift;
        }
        if (pair) {
          if (pg >= 0) turn<T>(x0[n], x1[n], &s_cs[t][c * X]);
          *reinterpret_cast<u32x4*>(dst + step) = x1[n];
        }
        *reinterpret_cast<u32x4*>(dst) = x0[n];
      }
    }
  } else {
    // a half that ends inside a pack: one thread per head, pair by pair
    for (int u = part * kThreads + tid; u < kTok * H; u += parts * kThreads) {
      const int h = u % H, t = u / H, i = i0 + t;
      if (i < 0 || i >= a.T) continue;
      const int pg = s_page[t];
      if (!isq && pg < 0) continue;
      const T* p = src + ((tok0 + i) * H + h) * d;
      for (int e = 0; e < d; ++e) {
        if (e >= h2 && e < 2 * h2) continue;
        const bool pair = e < h2;
        const float x = to_f32(p[e]), y = pair ? to_f32(p[e + h2]) : 0.0f;
        const float2 cs = pair && pg >= 0 ? s_cs[t][e] : make_float2(1.0f, 0.0f);
        const float z[2] = {x * cs.x - y * cs.y, y * cs.x + x * cs.y};
        for (int n = 0; n < (pair ? 2 : 1); ++n) {
          const int at = e + n * h2;
          T* dst = isq ? qo + ((tok0 + i) * H + h) * d + at
                       : kc + block_of(a.c, pg, h) + ((size_t(at / X) << a.c.page_shift) + p8 + t) * X + at % X;
          st(dst, pg < 0 ? 0.0f : z[n]);
        }
      }
    }
  }
  // Values: a unit is a pack of channels of X tokens, turned into a pack of
  // tokens of X channels.
  if (isq) return;
  const T* v = reinterpret_cast<const T*>(a.v);
  const int chunks = a.c.Hkv * (d / X);
  for (int u = part * kThreads + tid; u < (kTok / X) * chunks; u += parts * kThreads) {
    const int t0 = u / chunks * X, r = u % chunks, h = r / (d / X), e = r % (d / X) * X;
    u32x4 x[X];
    bool whole = true;
#pragma unroll
    for (int n = 0; n < X; ++n) {
      whole = whole && s_page[t0 + n] >= 0;
      if (s_page[t0 + n] >= 0)
        x[n] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(v + ((tok0 + i0 + t0 + n) * a.c.Hkv + h) * d + e));
    }
    const size_t at = (size_t((p8 + t0) / X) * d + e) * X;  // in the page's block
    if (whole) {
      T* dst = vc + block_of(a.c, s_page[t0], h) + at;
#pragma unroll
      for (int m = 0; m < X; ++m) {
        u32x4 y;
        if constexpr (X == 8) {
#pragma unroll
          for (int n = 0; n < 4; ++n) {  // tokens 2 n and 2 n + 1 of channel m
            const unsigned lo = x[2 * n][m / 2], hi = x[2 * n + 1][m / 2];
            y[n] = m & 1 ? (lo >> 16) | (hi & 0xffff0000u) : (lo & 0xffffu) | (hi << 16);
          }
        } else {
#pragma unroll
          for (int n = 0; n < 4; ++n) y[n] = x[n % X][m % 4];
        }
        *reinterpret_cast<u32x4*>(dst + m * X) = y;
      }
    } else {
#pragma unroll
      for (int n = 0; n < X; ++n) {
        if (s_page[t0 + n] < 0) continue;
        T* dst = vc + block_of(a.c, s_page[t0 + n], h) + at + n;
#pragma unroll
        for (int m = 0; m < X; ++m) {
          if constexpr (X == 8) dst[m * X].bits = uint16_t(x[n][m / 2] >> (m & 1 ? 16 : 0));
          else dst[m * X] = __uint_as_float(x[n][m % 4]);
        }
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Commit.
//
// Slots are numbered in any order, so a row's new place may be another path
// row's old one: all rows of a pack (keys) or of a channel (values) are
// loaded before any of them is stored, a barrier between.  One workgroup per
// (slice of channels, key head, sequence); slice 0 is the keys.
//
// Bound by its chain (status and lengths, ancestors, pages, rows) and, with many
// sequences, by the bytes around the rows: a value's row is 2 or 4 bytes of a
// 16-byte pack, one pack a channel, so a row of 128 fp32 values touches 128
// packs.  8 x 64 nodes 10 us, 32 x 128 nodes, fp32, 8 heads of 128: 16 us.
// ---------------------------------------------------------------------------
constexpr int kHold = 2;       // rows a thread holds between the load and the store
constexpr int kSliceV = 64;    // value channels of a workgroup

template <typename U>
__device__ __forceinline__ void move_rows(U* base, const size_t* s_src, const size_t* s_dst, int L, size_t stride, int n) {
  // n columns (stride elements apart) of L rows; whole columns per round
  const int cols = max(1, kHold * kThreads / L);
  for (int c0 = 0; c0 < n; c0 += cols) {
    U x[kHold];
    const int units = min(cols, n - c0) * L;
#pragma unroll
    for (int r = 0; r < kHold; ++r) {
      const int u = r * kThreads + int(threadIdx.x);
      if (u < units) x[r] = base[s_src[u % L] + size_t(c0 + u / L) * stride];
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kHold; ++r) {
      const int u = r * kThreads + int(threadIdx.x);
      if (u < units) base[s_dst[u % L] + size_t(c0 + u / L) * stride] = x[r];
    }
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void kv_commit_kernel(AttnArgs a) {
  constexpr int X = Pack<T>::kN;
  __shared__ int s_path[GDN_MAX_T];
  __shared__ size_t s_src[GDN_MAX_T], s_dst[GDN_MAX_T];
  __shared__ int s_flag[2];
  const int slice = blockIdx.x, h = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
  const int ctx = a.ctx_len[b], acc = a.accepted[b];
  const MetaPtrs m = meta_ptrs(a.meta, a.B, a.T);
  const size_t bt = size_t(b) * a.T;
  int status = a.meta ? m.status[b] : 0;
  int L = 0;
  if (!status) {
    if (acc < -1 || acc >= a.T) status = GDN_TREE_BAD_ACCEPTED;
    else if (acc >= 0) {
      L = (a.meta ? m.depth[bt + acc] : acc) + 1;
      if (L <= 0) status = GDN_TREE_BAD_ACCEPTED;
    }
  }
  if (!status) status = len_status(a, ctx, a.meta ? a.T : L);
  if (status) L = 0;
  if (tid < 2) s_flag[tid] = 0;
  __syncthreads();
  const int32_t* row = a.page_table + size_t(b) * a.c.max_pages;
  for (int j = tid; j < a.T; j += kThreads) {
    if (L == 0) break;
    const bool on = a.meta ? (j == acc || ((m.anc[(bt + acc) * m.W + (j >> 6)] >> (j & 63)) & 1)) : j <= acc;
    if (on) {
      const int at = a.meta ? m.depth[bt + j] : j;
      if (unsigned(at) < unsigned(GDN_MAX_T)) s_path[at] = j;
      if (at != j) s_flag[0] = 1;
      if (page_of(a.c, row, ctx + j) < 0 || page_of(a.c, row, ctx + at) < 0) s_flag[1] = 1;
    }
  }
  __syncthreads();
  if (L > 0 && s_flag[1]) {
    status = GDN_KV_BAD_PAGE;
    L = 0;
  }
  if (slice == 0 && h == 0 && tid == 0) {
    a.new_len[b] = ctx + L;
    if (a.status) a.status[b] = status;
  }
  if (L == 0 || !s_flag[0]) return;  // nothing to move
  const int mask = (1 << a.c.page_shift) - 1;
  for (int r = tid; r < L; r += kThreads) {
    const int ps = ctx + s_path[r], pd = ctx + r;
    const size_t bs = block_of(a.c, page_of(a.c, row, ps), h), bd = block_of(a.c, page_of(a.c, row, pd), h);
    if (slice == 0) {  // packs of 16 bytes
      s_src[r] = bs / X + (ps & mask);
      s_dst[r] = bd / X + (pd & mask);
    } else {
      s_src[r] = bs + size_t((ps & mask) / X) * a.c.d * X + ps % X;
      s_dst[r] = bd + size_t((pd & mask) / X) * a.c.d * X + pd % X;
    }
  }
  __syncthreads();
  if (slice == 0) {
    move_rows(reinterpret_cast<uint4*>(a.k_cache), s_src, s_dst, L, size_t(1) << a.c.page_shift, a.c.d / X);
  } else {
    const int e0 = (slice - 1) * kSliceV;
    move_rows(reinterpret_cast<T*>(a.v_cache) + size_t(e0) * X, s_src, s_dst, L, size_t(X), min(kSliceV, a.c.d - e0));
  }
}

int after_launch(const char* who) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? GDN_OK : set_error(GDN_EHIP, "%s: launch: %s", who, hipGetErrorString(e));
}

}  // namespace

int launch_kv_append(const AttnArgs& a, hipStream_t stream) {
  const int groups = (a.T + kTok - 1) / kTok + 1;  // a group more where ctx is not a multiple of 8
  const int x = a.dtype == GDN_BF16 ? 8 : 4, np = a.c.d / x - a.rot / 2 / x;
  const int qparts = (kTok * a.Hq * np + kUnits * kThreads - 1) / (kUnits * kThreads);
  const int kparts = (kTok * a.c.Hkv * np + kUnits * kThreads - 1) / (kUnits * kThreads);
  const dim3 grid(groups, qparts + kparts, a.B);
  if (a.dtype == GDN_BF16)
    append_kernel<BF16><<<grid, kThreads, 0, stream>>>(a, qparts, kparts);
  else
    append_kernel<float><<<grid, kThreads, 0, stream>>>(a, qparts, kparts);
  return after_launch("kv_append");
}

int launch_kv_commit(const AttnArgs& a, hipStream_t stream) {
  const dim3 grid(a.meta ? 1 + (a.c.d + kSliceV - 1) / kSliceV : 1, a.meta ? a.c.Hkv : 1, a.B);
  if (a.dtype == GDN_BF16)
    kv_commit_kernel<BF16><<<grid, kThreads, 0, stream>>>(a);
  else
    kv_commit_kernel<float><<<grid, kThreads, 0, stream>>>(a);
  return after_launch("kv_commit");
}

}  // namespace gdn
