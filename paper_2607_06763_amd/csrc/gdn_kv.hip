// gdn_kv.hip -- the paged key / value cache of the softmax-attention layers:
// appending a step's rows with the position rotation, and moving the
// accepted path's rows to the front.
#include "gdn_attn.h"

namespace gdn {
namespace {

constexpr int kThreads = 256;
constexpr int kTok = 8;  // tokens per workgroup: one bf16 value pack

// ---------------------------------------------------------------------------
// Append.
//
// A workgroup holds the slots of one group of 8 positions (one value pack in
// bf16, two in fp32) of a sequence, so that a value pack whose 8 tokens are
// all new is written whole, and one of `parts` shares of their (head, pack)
// units.  Bound by bytes.
// ---------------------------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(kThreads) void append_kernel(AttnArgs a, int parts) {
  constexpr int X = Pack<T>::kN;
  __shared__ float2 s_cs[kTok][128];  // cos and sin of the group's tokens
  __shared__ int s_page[kTok];        // page of the token, -1: absent
  __shared__ int s_red[3];
  const int b = blockIdx.z, tid = threadIdx.x, part = blockIdx.y;
  const int ctx = a.ctx_len[b], span = span_of(a, b);
  const MetaPtrs m = meta_ptrs(a.meta, a.B, a.T);
  int status = a.meta ? m.status[b] : 0;
  if (!status) status = len_status(a, ctx, span);
  const int32_t* row = a.page_table + size_t(b) * a.c.max_pages;

  // deepest real slot and bad pages of the whole sequence: every workgroup
  // takes the same decision
  if (tid < 3) s_red[tid] = tid == 0 ? -1 : 0;
  __syncthreads();
  for (int i = tid; i < (status ? 0 : a.T); i += kThreads) {
    const int dep = a.meta ? m.depth[size_t(b) * a.T + i] : (i < span ? i : -1);
    if (dep >= 0) {
      atomicMax(&s_red[0], dep);
      if (page_of(a.c, row, ctx + i) < 0) s_red[1] = 1;
    }
  }
  __syncthreads();
  if (!status && s_red[0] >= 0) {
    if (a.rot && (long long)(ctx) + s_red[0] >= a.n_pos) status = GDN_KV_BAD_POS;
    else if (s_red[1]) status = GDN_KV_BAD_PAGE;
  }
  if (a.status && blockIdx.x == 0 && part == 0 && tid == 0) a.status[b] = status;

  // slots of this group: positions g * 8 .. g * 8 + 7; a skipped sequence's
  // groups start at slot 0 (its queries are cleared all the same)
  const int base = status ? 0 : ctx;
  const int i0 = ((base >> 3) + int(blockIdx.x)) * kTok - base;  // slot of the group's first position, may be < 0
  if (i0 >= a.T) return;
  if (tid < kTok) {
    const int i = i0 + tid;
    int pg = -1;
    if (!status && i >= 0 && i < a.T) {
      const bool real = a.meta ? m.depth[size_t(b) * a.T + i] >= 0 : i < span;
      if (real) pg = page_of(a.c, row, ctx + i);
    }
    s_page[tid] = pg;
  }
  const int h2 = a.rot / 2;
  for (int u = tid; u < (status ? 0 : kTok * h2); u += kThreads) {
    const int t = u / h2, e = u % h2, i = i0 + t;
    if (i < 0 || i >= a.T) continue;
    const int dep = a.meta ? m.depth[size_t(b) * a.T + i] : (i < span ? i : -1);
    if (dep >= 0) s_cs[t][e] = reinterpret_cast<const float2*>(a.rope)[size_t(ctx + dep) * h2 + e];
  }
  __syncthreads();

  const int d = a.c.d, H = a.Hq + a.c.Hkv;
  const size_t tok0 = size_t(b) * a.T;
  // queries and keys.  Pairs of packs (c, c + h2 / X) where the half of the
  // rotated part is whole packs; a thread owns both, so q may be q_out.
  if (h2 % X == 0) {
    const int hp = h2 / X, np = d / X - hp;  // paired packs, units of a head
    for (int u = part * kThreads + tid; u < kTok * H * np; u += parts * kThreads) {
      const int c = u % np, r = u / np, h = r % H, t = r / H, i = i0 + t;
      if (i < 0 || i >= a.T) continue;
      const int pg = s_page[t];
      const bool isq = h < a.Hq;
      if (!isq && pg < 0) continue;
      const int kh = h - a.Hq;
      const T* src = isq ? reinterpret_cast<const T*>(a.q) + ((tok0 + i) * a.Hq + h) * d
                         : reinterpret_cast<const T*>(a.k) + ((tok0 + i) * a.c.Hkv + kh) * d;
      T *dst, *kc = reinterpret_cast<T*>(a.k_cache);
      size_t step;  // elements from one pack to the next
      if (isq) {
        dst = reinterpret_cast<T*>(a.out) + ((tok0 + i) * a.Hq + h) * d;
        step = X;
      } else {
        const int pos = ctx + i;
        dst = kc + block_of(a.c, pg, kh) + size_t(pos & ((1 << a.c.page_shift) - 1)) * X;
        step = size_t(X) << a.c.page_shift;
      }
      const bool pair = c < hp;
      const int c0 = pair ? c : c + hp;
      __align__(16) T x0[X], x1[X];
      if (pg < 0) {
        const uint4 zero = make_uint4(0, 0, 0, 0);
        *reinterpret_cast<uint4*>(dst + c0 * step) = zero;
        if (pair) *reinterpret_cast<uint4*>(dst + (c0 + hp) * step) = zero;
        continue;
      }
      copy16(x0, src + c0 * X);
      if (pair) {
        copy16(x1, src + (c0 + hp) * X);
#pragma unroll
        for (int e = 0; e < X; ++e) {
          const float2 cs = s_cs[t][c0 * X + e];
          const float p = to_f32(x0[e]), n = to_f32(x1[e]);
          st(&x0[e], p * cs.x - n * cs.y);
          st(&x1[e], n * cs.x + p * cs.y);
        }
        copy16(dst + (c0 + hp) * step, x1);
      }
      copy16(dst + c0 * step, x0);
    }
  } else {
    // a half that ends inside a pack: one thread per head, pair by pair
    for (int u = part * kThreads + tid; u < kTok * H; u += parts * kThreads) {
      const int h = u % H, t = u / H, i = i0 + t;
      if (i < 0 || i >= a.T) continue;
      const int pg = s_page[t];
      const bool isq = h < a.Hq;
      if (!isq && pg < 0) continue;
      const int kh = h - a.Hq;
      const T* src = isq ? reinterpret_cast<const T*>(a.q) + ((tok0 + i) * a.Hq + h) * d
                         : reinterpret_cast<const T*>(a.k) + ((tok0 + i) * a.c.Hkv + kh) * d;
      T* q = reinterpret_cast<T*>(a.out) + ((tok0 + i) * a.Hq + h) * d;
      T* kc = reinterpret_cast<T*>(a.k_cache);
      const int off = (ctx + i) & ((1 << a.c.page_shift) - 1);
      for (int e = 0; e < d; ++e) {
        if (e >= h2 && e < 2 * h2) continue;
        const bool pair = e < h2;
        const float p = to_f32(src[e]), n = pair ? to_f32(src[e + h2]) : 0.0f;
        const float2 cs = pair && pg >= 0 ? s_cs[t][e] : make_float2(1.0f, 0.0f);
        const float y0 = p * cs.x - n * cs.y, y1 = n * cs.x + p * cs.y;
        for (int k = 0; k < (pair ? 2 : 1); ++k) {
          const int at = e + k * h2;
          T* dst = isq ? q + at : kc + block_of(a.c, pg, kh) + ((size_t(at / X) << a.c.page_shift) + off) * X + at % X;
          st(dst, pg < 0 ? 0.0f : (k ? y1 : y0));
        }
      }
    }
  }
  // values: a thread holds one channel's tokens of a value pack
  if (status) return;
  const int per = kTok / X;
  T* vc = reinterpret_cast<T*>(a.v_cache);
  const T* v = reinterpret_cast<const T*>(a.v);
  for (int u = part * kThreads + tid; u < per * a.c.Hkv * d; u += parts * kThreads) {
    const int e = u % d, r = u / d, h = r % a.c.Hkv, t0 = r / a.c.Hkv * X;
    __align__(16) T x[X];
    bool whole = true;
#pragma unroll
    for (int k = 0; k < X; ++k) {
      const int i = i0 + t0 + k;
      whole = whole && s_page[t0 + k] >= 0;
      if (s_page[t0 + k] >= 0) x[k] = v[((tok0 + i) * a.c.Hkv + h) * d + e];
    }
    const int off = (ctx + i0 + t0) & ((1 << a.c.page_shift) - 1);
    if (whole) {  // 8 positions of one group share their page
      copy16(vc + block_of(a.c, s_page[t0], h) + (size_t(off / X) * d + e) * X, x);
    } else {
#pragma unroll
      for (int k = 0; k < X; ++k)
        if (s_page[t0 + k] >= 0) vc[block_of(a.c, s_page[t0 + k], h) + (size_t(off / X) * d + e) * X + k] = x[k];
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
  // enough workgroups for the chip, each with a unit per thread at least
  const int x = a.dtype == GDN_BF16 ? 8 : 4;
  const long long units = (long long)(kTok) * (a.Hq + a.c.Hkv) * (a.c.d / x) / 2 + 1;
  long long parts = (2048 + (long long)(groups) * a.B - 1) / ((long long)(groups) * a.B);
  parts = parts < units / kThreads + 1 ? parts : units / kThreads + 1;
  if (a.T == 1) parts = 1 + ((a.Hq + a.c.Hkv) * (a.c.d / x) / 2) / (4 * kThreads);
  const dim3 grid(groups, unsigned(parts), a.B);
  if (a.dtype == GDN_BF16)
    append_kernel<BF16><<<grid, kThreads, 0, stream>>>(a, int(parts));
  else
    append_kernel<float><<<grid, kThreads, 0, stream>>>(a, int(parts));
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
