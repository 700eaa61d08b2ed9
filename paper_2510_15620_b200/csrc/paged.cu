// The paged key/value cache: pages for new tokens, pages of leaving sequences, and the pass that normalises and rotates
// the new queries and keys and puts keys and values into their slots.
//
// Keys and values that outlive a call lie in pages of page_size tokens; a sequence owns the pages its block-table row
// names, in order, and token t of it lies in slot table[t / page_size] * page_size + t % page_size.
#include <math.h>

#include "paged.cuh"

namespace prism {
namespace {

constexpr int kThreads = 1024;
constexpr int kWarps = kThreads / 32;
constexpr int kRowsHere = 16384;

__device__ __forceinline__ unsigned cluster_rank() {
  unsigned r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ unsigned cluster_size() {
  unsigned r;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}
// All threads of all blocks of the cluster have passed; what they read before is read.
__device__ __forceinline__ void cluster_meet() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Exclusive scan over the block of one pair of sums per thread; tot receives the block's totals.
struct Pair {
  long long a, b;
};
__device__ __forceinline__ Pair block_scan(Pair v, Pair* warp_tot, Pair& tot) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  Pair inc = v;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const long long a = __shfl_up_sync(0xffffffffu, inc.a, d), b = __shfl_up_sync(0xffffffffu, inc.b, d);
    if (lane >= d) inc.a += a, inc.b += b;
  }
  if (lane == 31) warp_tot[warp] = inc;
  __syncthreads();
  if (warp == 0) {
    Pair w = warp_tot[lane];
    Pair wi = w;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const long long a = __shfl_up_sync(0xffffffffu, wi.a, d), b = __shfl_up_sync(0xffffffffu, wi.b, d);
      if (lane >= d) wi.a += a, wi.b += b;
    }
    warp_tot[lane] = Pair{wi.a - w.a, wi.b - w.b};
    if (lane == 31) warp_tot[32] = wi;
  }
  __syncthreads();
  tot = warp_tot[32];
  return Pair{warp_tot[warp].a + inc.a - v.a, warp_tot[warp].b + inc.b - v.b};
}

// Largest s in [0, n) with start[s] <= x (start is non-decreasing, start[0] == 0 <= x).
__device__ __forceinline__ int find_row(const int* start, int n, int x) {
  int lo = 0, hi = n;  // start[lo] <= x, and start[hi] > x or hi == n
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (start[mid] <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Pages and slots for the new tokens of every sequence.  One cluster: every block scans the lengths for itself (at most
// 4096 of them), the blocks meet once, so that lengths and pool size may be updated in place, and then share the writes.
// Bound by latency (two dependent loads, two scans of 1024 threads, the meeting); a cluster instead of a grid keeps it at one
// launch without any counter that outlives it.  Many rows would be bound by the searches and stores of eight SMs: above
// kRowsHere rows they are left to k_page_rows.
__global__ void __launch_bounds__(kThreads) k_page_append(const int* len_new, const int* kv_in, int* kv_out, int n, int shift,
                                                          int num_pages, int max_pages, long long table_stride,
                                                          int* table, const int* __restrict__ free_pages,
                                                          const int* n_free_in, int* n_free_out, int total, int* cu, int* pos,
                                                          int* slot, int* err, int vec, int rows_here) {
  pdl_sync();
  extern __shared__ int sm[];
  int* s_cu = sm;               // [n + 1] first row of each sequence
  int* s_first = s_cu + n + 1;  // [n + 1] first new page of each sequence, counted over the call
  int* s_kv = s_first + n + 1;  // [n] cached tokens
  __shared__ Pair warp_tot[33];
  const int tid = threadIdx.x;
  const int page = 1 << shift;
  const long long cap = (long long)max_pages << shift;
  const int per = (n + kThreads - 1) / kThreads, i0 = min(n, tid * per), i1 = min(n, i0 + per);
  Pair mine{0, 0};
  bool bad = false;
  for (int i = i0; i < i1; ++i) {
    const int kv = kv_in[i], add = len_new[i];
    if (kv < 0 || add < 0 || (long long)kv + add > cap) bad = true;
    else mine.a += add, mine.b += ((kv + (long long)add + page - 1) >> shift) - ((kv + (long long)page - 1) >> shift);
    s_kv[i] = kv;
  }
  Pair tot;
  Pair at = block_scan(mine, warp_tot, tot);
  for (int i = i0; i < i1; ++i) {
    s_cu[i] = (int)at.a;
    s_first[i] = (int)at.b;
    const int kv = s_kv[i];
    const long long add = len_new[i];
    at.a += add;
    at.b += ((kv + add + page - 1) >> shift) - ((kv + (long long)page - 1) >> shift);
  }
  const int n_free = *n_free_in;
  int code = __syncthreads_or(bad || tot.a > total) ? kErrBadOffsets : 0;
  if (!code && (n_free < 0 || n_free > num_pages || tot.b > n_free)) code = kErrPoolEmpty;
  const int rows = code ? 0 : (int)tot.a, pages = code ? 0 : (int)tot.b;
  if (tid == 0) s_cu[n] = rows, s_first[n] = pages;
  cluster_meet();  // every block has read the lengths and the pool's size: both may now be overwritten
  const int gid = (int)cluster_rank() * kThreads + tid, step = (int)cluster_size() * kThreads;
  if (gid == 0) {
    *n_free_out = n_free - pages;
    cu[n] = rows;
    if (code) atomicOr(err, code);
  }
  for (int i = gid; i < n; i += step) {
    cu[i] = code ? 0 : s_cu[i];
    kv_out[i] = s_kv[i] + (code ? 0 : s_cu[i + 1] - s_cu[i]);
  }
  bool bad_page = false;
  // page k of the call's new pages comes off the top of the stack of free ones
  for (int k = gid; k < pages; k += step) {
    const int s = find_row(s_first, n, k);
    const int j = ((s_kv[s] + page - 1) >> shift) + k - s_first[s];
    int id = free_pages[n_free - 1 - k];
    if ((unsigned)id >= (unsigned)num_pages) id = -1, bad_page = true;
    table[s * table_stride + j] = id;
  }
  // rows, four at a time: one search serves them, and they leave as 16-byte stores
  const int quads = rows_here ? (int)(((long long)total + 3) >> 2) : 0;
  for (int u = gid; u < quads; u += step) {
    const int t0 = u * 4, t1 = min(total, t0 + 4);
    int s = t0 < rows ? find_row(s_cu, n, t0) : n - 1;
    int ps[4], sl[4], last = -1, id = -1;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int t = t0 + e;
      ps[e] = 0, sl[e] = -1;
      if (t < rows) {
        while (t >= s_cu[s + 1]) ++s, last = -1;
        const int p = s_kv[s] + t - s_cu[s], j = p >> shift;
        if (j != last) {
          const int have = (s_kv[s] + page - 1) >> shift;
          id = j < have ? table[s * table_stride + j] : free_pages[n_free - 1 - (s_first[s] + j - have)];
          if ((unsigned)id >= (unsigned)num_pages) id = -1, bad_page = true;
          last = j;
        }
        ps[e] = p;
        sl[e] = id < 0 ? -1 : (id << shift) + (p & (page - 1));
      }
    }
    if (vec && t0 + 4 <= total) {
      *reinterpret_cast<int4*>(pos + t0) = make_int4(ps[0], ps[1], ps[2], ps[3]);
      *reinterpret_cast<int4*>(slot + t0) = make_int4(sl[0], sl[1], sl[2], sl[3]);
    } else {
      for (int e = 0; e < t1 - t0; ++e) pos[t0 + e] = ps[e], slot[t0 + e] = sl[e];
    }
  }
  if (bad_page) atomicOr(err, kErrBadPage);
}

// The rows of a large append, over the whole GPU: everything they need is in the first kernel's outputs (cu, kv_out and the
// table with its new entries; a refused call left cu = 0, which makes every row padding).
__global__ void __launch_bounds__(256) k_page_rows(const int* __restrict__ cu, const int* __restrict__ kv_out, int n, int shift,
                                                   int num_pages, long long table_stride, const int* __restrict__ table,
                                                   int total, int* __restrict__ pos, int* __restrict__ slot, int* err, int vec) {
  pdl_sync();
  const int page = 1 << shift, rows = cu[n];
  const int t0 = (int)min((long long)total, 4ll * ((long long)blockIdx.x * 256 + threadIdx.x)), t1 = min(total, t0 + 4);
  if (t0 >= total) return;
  int s = t0 < rows ? find_row(cu, n, t0) : n - 1;
  int ps[4], sl[4], beg = 0, end = 0, kv = 0, last = -1, id = -1;
  bool bad_page = false;
  if (t0 < rows) beg = cu[s], end = cu[s + 1], kv = kv_out[s] - (end - beg);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int t = t0 + e;
    ps[e] = 0, sl[e] = -1;
    if (t < rows) {
      while (t >= end) {
        ++s, last = -1;
        beg = end, end = cu[s + 1], kv = kv_out[s] - (end - beg);
      }
      const int p = kv + t - beg, j = p >> shift;
      if (j != last) id = table[s * table_stride + j], last = j;
      ps[e] = p;
      const bool out = (unsigned)id >= (unsigned)num_pages;
      bad_page |= out;
      sl[e] = out ? -1 : (id << shift) + (p & (page - 1));
    }
  }
  if (vec && t0 + 4 <= total) {
    *reinterpret_cast<int4*>(pos + t0) = make_int4(ps[0], ps[1], ps[2], ps[3]);
    *reinterpret_cast<int4*>(slot + t0) = make_int4(sl[0], sl[1], sl[2], sl[3]);
  } else {
    for (int e = 0; e < t1 - t0; ++e) pos[t0 + e] = ps[e], slot[t0 + e] = sl[e];
  }
  if (bad_page) atomicOr(err, kErrBadPage);
}

// Sequences that are not kept give their pages back; the kept ones' rows of the block table move to the front.
__global__ void __launch_bounds__(kThreads) k_page_release(const int* __restrict__ keep, int n_new, const int* kv_in, int* kv_out,
                                                           int n, int shift, int num_pages, int shared, int max_pages,
                                                           long long stride_in, const int* __restrict__ table_in,
                                                           long long stride_out, int* __restrict__ table_out, int* free_pages,
                                                           const int* n_free_in, int* n_free_out, int* err) {
  extern __shared__ int sm[];
  int* s_kv = sm;           // [n]
  int* s_new = s_kv + n;    // [n] new index, or -1
  int* s_base = s_new + n;  // [n] first place on the stack of a leaving sequence's pages
  __shared__ Pair warp_tot[33];
  const int tid = threadIdx.x, lane = tid & 31;
  const int page = 1 << shift;
  const long long cap = (long long)max_pages << shift;
  bool bad = false;
  for (int i = tid; i < n; i += kThreads) s_kv[i] = kv_in[i], s_new[i] = -1;
  const int n_free = *n_free_in;
  __syncthreads();
  for (int i = tid; i < n_new; i += kThreads) {
    const int s = keep[i];
    if ((unsigned)s >= (unsigned)n || atomicCAS(s_new + s, -1, i) != -1) bad = true;  // outside, or named twice
  }
  __syncthreads();
  const int per = (n + kThreads - 1) / kThreads, i0 = min(n, tid * per), i1 = min(n, i0 + per);
  auto leaving = [&](int i) {
    if (s_new[i] >= 0) return 0;
    const int have = (int)((s_kv[i] + (long long)page - 1) >> shift);
    return have > shared ? have - shared : 0;
  };
  Pair mine{0, 0};
  for (int i = i0; i < i1; ++i) {
    if (s_kv[i] < 0 || s_kv[i] > cap) bad = true;
    else mine.a += leaving(i);
  }
  Pair tot;
  Pair at = block_scan(mine, warp_tot, tot);
  int code = __syncthreads_or(bad) ? kErrBadOffsets : 0;
  if (!code && (n_free < 0 || tot.a + n_free > num_pages)) code = kErrPoolEmpty;
  if (!code)
    for (int i = i0; i < i1; ++i) {
      s_base[i] = (int)at.a;
      at.a += leaving(i);
    }
  cluster_meet();
  const int gid = (int)cluster_rank() * kThreads + tid, step = (int)cluster_size() * kThreads;
  if (gid == 0) {
    *n_free_out = n_free + (code ? 0 : (int)tot.a);
    if (code) atomicOr(err, code);
  }
  if (code) {  // refused as a whole: everything stays as it was
    for (int i = gid; i < n; i += step) kv_out[i] = s_kv[i];
    for (int i = gid >> 5; i < n; i += step >> 5)
      for (int j = lane; j < max_pages; j += 32) table_out[i * stride_out + j] = table_in[i * stride_in + j];
    return;
  }
  // one warp per old sequence: its pages to the stack, or its row to its new place
  bool bad_page = false;
  for (int i = gid >> 5; i < n; i += step >> 5) {
    const int to = s_new[i], have = (s_kv[i] + page - 1) >> shift;
    const int* row = table_in + i * stride_in;
    if (to < 0) {
      for (int j = shared + lane; j < have; j += 32) {
        const int id = row[j];
        if ((unsigned)id >= (unsigned)num_pages) bad_page = true;
        free_pages[n_free + s_base[i] + j - shared] = id;
      }
    } else {
      int* dst = table_out + to * stride_out;
      for (int j = lane; j < max_pages; j += 32) dst[j] = j < have ? row[j] : -1;
      if (lane == 0) kv_out[to] = s_kv[i];
    }
  }
  // rows behind the last survivor
  for (int i = n_new + (gid >> 5); i < n; i += step >> 5) {
    for (int j = lane; j < max_pages; j += 32) table_out[i * stride_out + j] = -1;
    if (lane == 0) kv_out[i] = 0;
  }
  if (bad_page) atomicOr(err, kErrBadPage);
}

// ------------------------------------------------------------------------------------------------
// Per-head RMSNorm of q and k, rotation, and the rows' keys and values into the cache, one pass over the row: read once,
// written once.  x' = x / sqrt(mean x^2 + eps) * gain, then (a, b) -> (a c - b s, b c + a s) for the pairs
// (j, j + dh/2) with angle pos * theta^(-2j/dh).
//
// Bound by HBM: (hq + 2 hkv) * dh elements in and out per row.  One block of four warps per row: a lane owns VEC
// consecutive elements of the first half of a head and the same of the second, so both members of every pair sit in one
// thread and a head's sum of squares is a short shuffle.  The angles are the row's, not the head's: the block forms them
// once, in shared memory, while the first loads are in flight.  q_out may be the q columns of qkv itself: every element is
// read by the thread that writes it, before it does.  The angle is taken in turns and in double
// (pos * theta^(-2j/dh) / 2 pi, reduced to an eighth of a turn before it becomes a float), so far positions lose nothing
// and no table bounds them.
struct RopeFreq {
  double turns[128];  // theta^(-2j/dh) / (2 pi)
};

template <typename T>
struct Vec16 {
  static constexpr int N = 16 / sizeof(T);
};
template <typename T>
__device__ __forceinline__ void unpack16(const uint4& u, float* f);
template <>
__device__ __forceinline__ void unpack16<float>(const uint4& u, float* f) {
  f[0] = __uint_as_float(u.x), f[1] = __uint_as_float(u.y), f[2] = __uint_as_float(u.z), f[3] = __uint_as_float(u.w);
}
template <>
__device__ __forceinline__ void unpack16<__nv_bfloat16>(const uint4& u, float* f) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) f[2 * i] = __uint_as_float(w[i] << 16), f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
}
template <typename T>
__device__ __forceinline__ uint4 pack16(const float* f);
template <>
__device__ __forceinline__ uint4 pack16<float>(const float* f) {
  return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}
template <>
__device__ __forceinline__ uint4 pack16<__nv_bfloat16>(const float* f) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    __nv_bfloat162 v = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
    w[i] = *reinterpret_cast<uint32_t*>(&v);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

template <typename T>
__global__ void __launch_bounds__(128) k_qknorm_rope_paged(const T* qkv, long long qkv_stride,
                                                           const int* __restrict__ pos, const int* __restrict__ slot_map, int hq,
                                                           int qk_norm, const T* __restrict__ g_q, const T* __restrict__ g_k,
                                                           float eps, const __grid_constant__ RopeFreq freq, T* q_out,
                                                           long long q_stride, PagedCache c, int shift, int lanes, int* err) {
  constexpr int V = Vec16<T>::N;
  __shared__ __align__(16) float s_cos[128], s_sin[128];
  const int row = blockIdx.x, dh = c.dh, half = dh >> 1, heads = hq + 2 * c.hkv;
  const int slot = slot_map[row], p = pos[row];
  const int per_block = 128 / lanes;  // heads a pass of the block covers
  const int sub = threadIdx.x & (lanes - 1), h_first = threadIdx.x / lanes;
  const bool live = sub * V < half;  // lanes of a head are rounded up to a power of two
  const T* src = qkv + row * qkv_stride;
  // two passes ahead: at 16 + 8 + 8 heads of 128 the whole row is in flight before anything waits
  uint4 ua[2], ub[2];
  auto fetch = [&](int h, int i) {
    ua[i] = ub[i] = make_uint4(0, 0, 0, 0);
    if (h < heads && live) {
      ua[i] = *reinterpret_cast<const uint4*>(src + (long long)h * dh + sub * V);
      ub[i] = *reinterpret_cast<const uint4*>(src + (long long)h * dh + half + sub * V);
    }
  };
  fetch(h_first, 0);
  fetch(h_first + per_block, 1);
  if (slot < 0) return;  // a padding row: nothing is written for it
  const int page = slot >> shift, off = slot & ((1 << shift) - 1);
  if (page >= c.num_pages) {
    if (threadIdx.x == 0) atomicOr(err, kErrBadPage);
    return;
  }
  for (int j = threadIdx.x; j < half; j += 128) {
    double t = p * freq.turns[j];
    t -= rint(t);                              // [-1/2, 1/2] turns
    const double quarter = rint(4.0 * t);      // -2 .. 2
    float sn, cs;
    sincospif((float)(2.0 * t - 0.5 * quarter), &sn, &cs);  // at most an eighth of a turn
    const int qd = (int)quarter & 3;
    const float c0 = (qd & 1) ? sn : cs, s0 = (qd & 1) ? cs : sn;
    s_cos[j] = (qd == 1 || qd == 2) ? -c0 : c0;
    s_sin[j] = qd >= 2 ? -s0 : s0;
  }
  __syncthreads();
  T* const kc = static_cast<T*>(c.k) + page * c.page_stride + (long long)off * dh;
  T* const vc = static_cast<T*>(c.v) + page * c.page_stride + (long long)off * dh;
  const long long head_step = (long long)dh << shift;
  // every lane of a warp takes the same number of passes, so the shuffles below always have all of them
  for (int h0 = 0; h0 < heads; h0 += per_block) {
    const int h = h0 + h_first;
    uint4 xa = ua[0], xb = ub[0];
    ua[0] = ua[1], ub[0] = ub[1];
    fetch(h + 2 * per_block, 1);
    float a[V], b[V];
    unpack16<T>(xa, a);
    unpack16<T>(xb, b);
    const bool rotate = h < hq + c.hkv;
    if (qk_norm) {
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < V; ++i) ss += a[i] * a[i] + b[i] * b[i];
      if (!live) ss = 0.f;
      for (int d = lanes >> 1; d > 0; d >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, d);
      if (rotate && live) {
        const float r = 1.0f / sqrtf(ss / (float)dh + eps);
        const T* g = h < hq ? g_q : g_k;
        float ga[V], gb[V];
        unpack16<T>(*reinterpret_cast<const uint4*>(g + sub * V), ga);
        unpack16<T>(*reinterpret_cast<const uint4*>(g + half + sub * V), gb);
#pragma unroll
        for (int i = 0; i < V; ++i) a[i] = a[i] * r * ga[i], b[i] = b[i] * r * gb[i];
      }
    }
    if (h >= heads || !live) continue;
    T* dst;
    if (rotate) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float cs = s_cos[sub * V + i], sn = s_sin[sub * V + i];
        const float x0 = a[i] * cs - b[i] * sn, x1 = b[i] * cs + a[i] * sn;
        a[i] = x0, b[i] = x1;
      }
      xa = pack16<T>(a);
      xb = pack16<T>(b);
      dst = h < hq ? q_out + row * q_stride + (long long)h * dh : kc + (h - hq) * head_step;
    } else {
      dst = vc + (h - hq - c.hkv) * head_step;
    }
    *reinterpret_cast<uint4*>(dst + sub * V) = xa;
    *reinterpret_cast<uint4*>(dst + half + sub * V) = xb;
  }
}

int log2_of(int x) {
  int s = 0;
  while ((1 << s) < x) ++s;
  return s;
}

template <typename... KArgs, typename... Args>
cudaError_t launch_cluster(void (*kernel)(KArgs...), int blocks, size_t smem, cudaStream_t st, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(blocks);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = blocks;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
}
// Blocks of the one cluster: 1, 2, 4 or 8 (the portable size), one per `per` units of work.
int cluster_blocks(long long work, long long per) {
  int b = 1;
  while (b < 8 && work > per * b) b *= 2;
  return b;
}

}  // namespace

cudaError_t launch_page_append(const int* len_new, const int* kv_in, int* kv_out, int n, int page_size, int num_pages,
                               int max_pages, long long table_stride, int* table, const int* free_pages, const int* n_free_in,
                               int* n_free_out, int total, int* cu, int* pos, int* slot, int* err, cudaStream_t st) {
  const size_t smem = (3 * (size_t)n + 2) * sizeof(int);
  static std::atomic<unsigned long long> set;
  if (cudaError_t e = ensure_dynamic_smem(k_page_append, (3 * kMaxCandidates + 2) * (int)sizeof(int), set)) return e;
  const int vec = !((reinterpret_cast<uintptr_t>(pos) | reinterpret_cast<uintptr_t>(slot)) & 15);
  const int shift = log2_of(page_size);
  const int rows_here = total <= kRowsHere;
  cudaError_t e = launch_cluster(k_page_append, cluster_blocks(rows_here ? total : total / 8, 4 * kThreads), smem, st, len_new,
                                 kv_in, kv_out, n, shift, num_pages, max_pages, table_stride, table, free_pages, n_free_in,
                                 n_free_out, total, cu, pos, slot, err, vec, rows_here);
  if (e != cudaSuccess || rows_here) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(((long long)total + 1023) / 1024));
  cfg.blockDim = dim3(256);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = pdl_enabled() ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, k_page_rows, (const int*)cu, (const int*)kv_out, n, shift, num_pages, table_stride,
                            (const int*)table, total, pos, slot, err, vec);
}

cudaError_t launch_page_release(const int* keep, int n_new, const int* kv_in, int* kv_out, int n, int page_size, int num_pages,
                                int shared_pages, int max_pages, long long stride_in, const int* table_in,
                                long long stride_out, int* table_out, int* free_pages, const int* n_free_in, int* n_free_out,
                                int* err, cudaStream_t st) {
  const size_t smem = 3 * (size_t)n * sizeof(int);
  static std::atomic<unsigned long long> set;
  if (cudaError_t e = ensure_dynamic_smem(k_page_release, 3 * kMaxCandidates * (int)sizeof(int), set)) return e;
  return launch_cluster(k_page_release, cluster_blocks(n, kWarps), smem, st, keep, n_new, kv_in, kv_out, n,
                        log2_of(page_size), num_pages, shared_pages, max_pages, stride_in, table_in, stride_out, table_out,
                        free_pages, n_free_in, n_free_out, err);
}

cudaError_t launch_qknorm_rope_paged(const void* qkv, long long qkv_stride, const int* pos, const int* slot, int rows, int hq,
                                     int qk_norm, const void* g_q, const void* g_k, float eps, double theta, void* q_out,
                                     long long q_stride, const PagedCache& c, int* err, cudaStream_t st) {
  if (rows <= 0) return cudaSuccess;
  RopeFreq f;
  const int half = c.dh / 2;
  for (int j = 0; j < 128; ++j)
    f.turns[j] = j < half ? pow(theta, -2.0 * j / c.dh) / 6.283185307179586476925286766559 : 0.0;
  const int shift = log2_of(c.page_size);
  if (c.dtype == 1) {
    const int lanes = 1 << log2_of((half + 7) / 8);
    k_qknorm_rope_paged<__nv_bfloat16><<<rows, 128, 0, st>>>((const __nv_bfloat16*)qkv, qkv_stride, pos, slot, hq, qk_norm,
                                                             (const __nv_bfloat16*)g_q, (const __nv_bfloat16*)g_k, eps, f,
                                                             (__nv_bfloat16*)q_out, q_stride, c, shift, lanes, err);
  } else {
    const int lanes = 1 << log2_of((half + 3) / 4);
    k_qknorm_rope_paged<float><<<rows, 128, 0, st>>>((const float*)qkv, qkv_stride, pos, slot, hq, qk_norm, (const float*)g_q,
                                                     (const float*)g_k, eps, f, (float*)q_out, q_stride, c, shift, lanes, err);
  }
  return cudaGetLastError();
}

}  // namespace prism
