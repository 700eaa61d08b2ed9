// Attention over a paged cache for few new tokens: at most 32 query rows (token, head of the group) per sequence and
// key/value head, 16 of them in an item, bf16, head_dim 64 or 128.
//
// Bound by reading the cache: every key and value is used for at most 16 rows, 2 * 16 flops a byte at best.  So the
// kernel is built around the loads.  A work unit is (item of the work list, key/value head); a producer warp keeps a ring
// of kStages stages of 64 keys and their values in flight, one TMA box per page (page numbers are read 32 boxes at a
// time, a batch ahead), and four warps each take 16 of a stage's keys with warp-level MMAs, a running maximum
// and a running sum of their own.  No warp waits for another until the end, where the four results meet in shared memory.
// The warp-level MMA is chosen on purpose: sixteen rows would leave seven eighths of a 128-row tcgen05 tile empty and put
// its tensor-memory round trips on the path of a kernel that only has to keep up with memory.
// Measured: 100 sequences of 500-32 k tokens, 32 / 8 heads of 128 (3.44 GB), 498 us, 6.9 TB/s; 20 of 500 tokens, 16 / 8 heads
// (36 MB), 11.2 us.  Rounding: probabilities become bf16 for the second product (relative 2^-8, as in the packed attention kernels); the sum
// they are divided by is taken in fp32 before that.
#include <math.h>

#include "paged.cuh"
#include "tc_common.cuh"

namespace prism {
namespace {

using namespace tc;

constexpr int kKeys = 64;          // keys of one stage
constexpr int kThreads = 160;      // producer warp, four MMA warps
__host__ __device__ constexpr int stage_bytes(int dh) { return 2 * kKeys * dh * 2; }  // keys and values
__host__ __device__ constexpr int n_stages(int dh) { return dh == 128 ? 3 : 6; }      // 96 KB: two blocks per SM
__host__ __device__ constexpr int tokens_smem(int dh) { return n_stages(dh) * stage_bytes(dh) + 1024 /*alignment*/ + 256; }
static_assert(4 * (16 * (128 + 4) + 32) * 4 <= 3 * 2 * 64 * 128 * 2, "the final meeting reuses the ring");

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t* r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t addr, uint32_t* r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma16816(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void tma_load_5d(uint32_t dst, const CUtensorMap* map, int c1, int c3, int c4, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];"
      ::"r"(dst), "l"(map), "r"(0), "r"(c1), "r"(0), "r"(c3), "r"(c4), "r"(bar)
      : "memory");
}

template <int DH>
__global__ void __launch_bounds__(kThreads, 2)
k_paged_tokens(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
               const __grid_constant__ PagedAttnArgs a, int shift, float scale_log2) {
  if (threadIdx.x == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_k) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_v) : "memory");
  }
  pdl_sync();
  constexpr int kStages = n_stages(DH), kStage = stage_bytes(DH), kHalf = kStage / 2;
  constexpr int NK = DH / 16, NO = DH / 8;  // MMA steps over head_dim; 8-column tiles of the output
  extern __shared__ unsigned char smem_raw[];
  const PagedPlanHeader* hd = static_cast<const PagedPlanHeader*>(a.plan);
  const int hkv = a.c.hkv, group = a.hq / hkv;
  const int4 h0 = reinterpret_cast<const int4*>(hd)[0], h1 = reinterpret_cast<const int4*>(hd)[1],
             h2 = reinterpret_cast<const int4*>(hd)[2];
  // the grid is not larger than the list's room, so the block's first item can be fetched beside the header that says whether
  // it exists
  PagedItem it = paged_item_raw(hd, blockIdx.x / hkv);
  if (h0.x != kPagedTokens || h1.x != a.hq || h1.y != hkv || h1.z != DH || h1.w != a.total_q || h2.x != a.n_seq ||
      h2.y != a.max_q) {
    if (threadIdx.x == 0 && blockIdx.x == 0) atomicOr(a.err, kErrBadOffsets);
    return;
  }
  const int total = h0.y * hkv;
  if ((int)blockIdx.x >= total) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  unsigned char* gen = smem_raw + (base - raw);
  uint64_t* bars = reinterpret_cast<uint64_t*>(gen + kStages * kStage);
  const uint32_t b_full = smem_u32(bars), b_empty = smem_u32(bars + kStages);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(bars + 2 * kStages);
  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(b_full + 8 * i, 1);
      mbar_init(b_empty + 8 * i, 4);
    }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();

  // The grid covers every uncut item; the pieces of cut ones beyond that are second helpings (a grid of all the pieces there
  // could be would be mostly blocks that only find out that they are not needed: 4 us at 20 sequences).
  uint32_t done = 0;  // blocks of 64 keys this CTA has been through
  for (int work = blockIdx.x;;) {
    const int h = work % hkv;
    paged_item_check(it, a.max_pages, shift, a.ws, a.err);
    const int n_blocks = it.k1 > it.k0 ? (it.k1 - it.k0 + kKeys - 1) / kKeys : 0;
    // rows of a TMA box: a page, or 64 rows of a larger one
    const int box_shift = shift < 6 ? shift : 6, box_rows = 1 << box_shift, boxes = kKeys >> box_shift;
    if (warp == 0) {
      const int* row = a.table + it.seq * a.table_stride;
      const uint32_t box_bytes = (uint32_t)box_rows * DH * 2;
      // Page numbers come 32 boxes at a time, one a lane, a batch ahead; lane i of the first `boxes` fetches box i of a stage.
      auto pages_of = [&](int batch) {
        const long long key = it.k0 + ((long long)(batch * 32 + lane) << box_shift);
        if (key >= it.k1) return 0;
        const int id = row[key >> shift];  // key < k1 <= max_pages << shift
        if ((unsigned)id >= (unsigned)a.c.num_pages) {
          atomicOr(a.err, kErrBadPage);
          return a.c.num_pages;  // beyond the tensor: the box arrives as zeros
        }
        return id;
      };
      int ids = 0, ids_next = pages_of(0), issued = 0;
      for (int j = 0; j < n_blocks; ++j) {
        const int first = j * boxes;  // of the stage's boxes
        if ((first & 31) == 0) {
          ids = ids_next;
          ids_next = pages_of((first >> 5) + 1);
        }
        const int id = __shfl_sync(0xffffffffu, ids, (first + lane) & 31);
        const uint32_t g = done + j, st = g % kStages;
        if (!warp_wait(b_empty + 8 * st, ((g / kStages) & 1) ^ 1, a.err, abort_flag)) break;
        const int keys = min(kKeys, it.k1 - it.k0 - j * kKeys), live = (keys + box_rows - 1) >> box_shift;
        if (lane == 0) mbar_expect_tx(b_full + 8 * st, 2 * live * box_bytes);
        __syncwarp();
        if (lane < live) {
          const int key = it.k0 + j * kKeys + (lane << box_shift);
          const uint32_t dst = base + st * kStage + lane * box_bytes;
          const int r = key & ((1 << shift) - 1);
          tma_load_5d(dst, &map_k, r, h, id, b_full + 8 * st);
          tma_load_5d(dst + kHalf, &map_v, r, h, id, b_full + 8 * st);
        }
        issued = j + 1;
      }
      __syncwarp();
      // every load has landed before the shared memory is reused below
      for (int j = max(0, issued - kStages); j < issued; ++j)
        mbar_drain(b_full + 8 * ((done + j) % kStages), ((done + j) / kStages) & 1);
    }

    const int w = warp - 1, r0 = lane >> 2, r1 = r0 + 8;  // this thread's two rows
    float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;
    float o[NO][4];
#pragma unroll
    for (int n = 0; n < NO; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;
    if (warp > 0) {
      uint32_t qf[NK][4];
      const int t0 = r0 / group, t1 = r1 / group;
      {
        const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(a.q);
        const __nv_bfloat16* p0 = q + (it.row0 + t0) * a.q_stride + (long long)(h * group + r0 % group) * DH + 2 * (lane & 3);
        const __nv_bfloat16* p1 = q + (it.row0 + t1) * a.q_stride + (long long)(h * group + r1 % group) * DH + 2 * (lane & 3);
        const bool v0 = t0 < it.n_tok, v1 = t1 < it.n_tok;
#pragma unroll
        for (int k = 0; k < NK; ++k) {
          qf[k][0] = v0 ? *reinterpret_cast<const uint32_t*>(p0 + 16 * k) : 0u;
          qf[k][1] = v1 ? *reinterpret_cast<const uint32_t*>(p1 + 16 * k) : 0u;
          qf[k][2] = v0 ? *reinterpret_cast<const uint32_t*>(p0 + 16 * k + 8) : 0u;
          qf[k][3] = v1 ? *reinterpret_cast<const uint32_t*>(p1 + 16 * k + 8) : 0u;
        }
      }
      const int causal = h0.w;
      const int lim0 = t0 < it.n_tok ? (causal ? min(it.k1, it.pos0 + t0 + 1) : it.k1) : it.k1;
      const int lim1 = t1 < it.n_tok ? (causal ? min(it.k1, it.pos0 + t1 + 1) : it.k1) : it.k1;
      const int lim_min = causal ? min(it.k1, it.pos0 + 1) : it.k1;  // the first token's: no row sees fewer
      // this warp's 16 keys inside a stage: all of one box
      const int kk = 16 * w, box = kk >> box_shift, in_box = kk & (box_rows - 1);
      const uint32_t off_box = (uint32_t)box * box_rows * DH * 2;
      // ldmatrix rows: K wants (keys 0-7, d 0-7), (keys 0-7, d 8-15), (keys 8-15, d 0-7), (keys 8-15, d 8-15);
      // V, transposed, (keys 0-7, d 0-7), (keys 8-15, d 0-7), (keys 0-7, d 8-15), (keys 8-15, d 8-15)
      const int mi = lane >> 3, mr = lane & 7;
      const int k_row = in_box + (mi >> 1) * 8 + mr, k_col = mi & 1;
      const int v_row = in_box + (mi & 1) * 8 + mr, v_col = mi >> 1;
      const uint32_t k_base = off_box + k_row * 128, v_base = kHalf + off_box + v_row * 128;
      auto swz = [&](uint32_t at, int row, int chunk) {  // 16-byte chunk `chunk` of the row (eight to a 64-column half)
        return at + (uint32_t)(chunk >> 3) * (box_rows * 128) + (uint32_t)(((chunk & 7) ^ (row & 7)) << 4);
      };
      for (int j = 0; j < n_blocks; ++j) {
        const uint32_t g = done + j, st = g % kStages;
        if (!warp_wait(b_full + 8 * st, (g / kStages) & 1, a.err, abort_flag)) break;
        const int key0 = it.k0 + j * kKeys + kk;  // first key of this warp
        if (key0 < it.k1) {
          const uint32_t sb = base + st * kStage;
          if (key0 + 16 > it.k1) {
            // keys beyond the end: whatever the page (or an earlier stage) holds there must not meet a zero probability
            const int first = it.k1 - key0;
            for (int u = lane; u < (16 - first) * (DH / 8); u += 32) {
              const int rr = in_box + first + u / (DH / 8);
              const uint32_t dst = swz(sb + kHalf + off_box + rr * 128, rr, u % (DH / 8));
              asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(dst), "r"(0) : "memory");
            }
            __syncwarp();
          }
          // two sums each, over even and odd steps: half the chain of dependent MMAs
          float s[2][4], s_odd[2][4];
#pragma unroll
          for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[n][e] = s_odd[n][e] = 0.f;
#pragma unroll
          for (int k = 0; k < NK; ++k) {
            uint32_t b[4];
            ldsm4(swz(sb + k_base, k_row, 2 * k + k_col), b);
            mma16816((k & 1) ? s_odd[0] : s[0], qf[k], b[0], b[1]);
            mma16816((k & 1) ? s_odd[1] : s[1], qf[k], b[2], b[3]);
          }
#pragma unroll
          for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[n][e] = (s[n][e] + s_odd[n][e]) * scale_log2;
          if (key0 + 16 > lim_min) {
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const int key = key0 + 8 * n + 2 * (lane & 3) + e;
                if (key >= lim0) s[n][e] = -INFINITY;
                if (key >= lim1) s[n][2 + e] = -INFINITY;
              }
          }
          float x0 = fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[1][0], s[1][1]));
          float x1 = fmaxf(fmaxf(s[0][2], s[0][3]), fmaxf(s[1][2], s[1][3]));
          x0 = fmaxf(x0, __shfl_xor_sync(0xffffffffu, x0, 1));
          x1 = fmaxf(x1, __shfl_xor_sync(0xffffffffu, x1, 1));
          x0 = fmaxf(x0, __shfl_xor_sync(0xffffffffu, x0, 2));
          x1 = fmaxf(x1, __shfl_xor_sync(0xffffffffu, x1, 2));
          if (__any_sync(0xffffffffu, x0 > m0 || x1 > m1)) {
            const float n0 = fmaxf(m0, x0), n1 = fmaxf(m1, x1);
            const float f0 = m0 == n0 ? 1.f : ex2(m0 - n0), f1 = m1 == n1 ? 1.f : ex2(m1 - n1);
            m0 = n0, m1 = n1;
            l0 *= f0, l1 *= f1;
#pragma unroll
            for (int n = 0; n < NO; ++n) o[n][0] *= f0, o[n][1] *= f0, o[n][2] *= f1, o[n][3] *= f1;
          }
          const float ref0 = m0 == -INFINITY ? 0.f : m0, ref1 = m1 == -INFINITY ? 0.f : m1;
#pragma unroll
          for (int n = 0; n < 2; ++n) {
            s[n][0] = ex2(s[n][0] - ref0), s[n][1] = ex2(s[n][1] - ref0);
            s[n][2] = ex2(s[n][2] - ref1), s[n][3] = ex2(s[n][3] - ref1);
            l0 += s[n][0] + s[n][1];
            l1 += s[n][2] + s[n][3];
          }
          const uint32_t p[4] = {pack_bf16(s[0][0], s[0][1]), pack_bf16(s[0][2], s[0][3]), pack_bf16(s[1][0], s[1][1]),
                                 pack_bf16(s[1][2], s[1][3])};
#pragma unroll
          for (int n = 0; n < NO; n += 2) {
            uint32_t b[4];
            ldsm4_t(swz(sb + v_base, v_row, n + v_col), b);
            mma16816(o[n], p, b[0], b[1]);
            mma16816(o[n + 1], p, b[2], b[3]);
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(b_empty + 8 * st);
      }
      l0 += __shfl_xor_sync(0xffffffffu, l0, 1);
      l1 += __shfl_xor_sync(0xffffffffu, l1, 1);
      l0 += __shfl_xor_sync(0xffffffffu, l0, 2);
      l1 += __shfl_xor_sync(0xffffffffu, l1, 2);
    }
    // The four warps' results meet in the ring's memory: [4][16][DH + 4] outputs, [4][16][2] references and sums.
    __syncthreads();
    float* so = reinterpret_cast<float*>(gen);
    float* sml = so + 4 * 16 * (DH + 4);
    if (warp > 0) {
      float* mine = so + w * 16 * (DH + 4);
#pragma unroll
      for (int n = 0; n < NO; ++n) {
        const int c = 8 * n + 2 * (lane & 3);
        *reinterpret_cast<float2*>(mine + r0 * (DH + 4) + c) = make_float2(o[n][0], o[n][1]);
        *reinterpret_cast<float2*>(mine + r1 * (DH + 4) + c) = make_float2(o[n][2], o[n][3]);
      }
      if ((lane & 3) == 0) {
        sml[(w * 16 + r0) * 2] = m0, sml[(w * 16 + r0) * 2 + 1] = l0;
        sml[(w * 16 + r1) * 2] = m1, sml[(w * 16 + r1) * 2 + 1] = l1;
      }
    }
    __syncthreads();
    const int live_rows = it.n_tok * group;
    __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.out);
    float* part = it.part < 0 ? nullptr : a.ws + ((long long)it.part * hkv + h) * paged_part_floats(16, DH);
    for (int u = threadIdx.x; u < live_rows * (DH / 4); u += kThreads) {
      const int r = u / (DH / 4), c = (u % (DH / 4)) * 4, tok = r / group;
      float mm[4], M = -INFINITY;
#pragma unroll
      for (int i = 0; i < 4; ++i) mm[i] = sml[(i * 16 + r) * 2], M = fmaxf(M, mm[i]);
      const float ref = M == -INFINITY ? 0.f : M;
      float l = 0.f, x0 = 0.f, x1 = 0.f, x2 = 0.f, x3 = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float f = ex2(mm[i] - ref);
        const float4 v = *reinterpret_cast<const float4*>(so + (i * 16 + r) * (DH + 4) + c);
        l += f * sml[(i * 16 + r) * 2 + 1];
        x0 += f * v.x, x1 += f * v.y, x2 += f * v.z, x3 += f * v.w;
      }
      if (part) {
        *reinterpret_cast<float4*>(part + ((c >> 2) * 16 + r) * 4) = make_float4(x0, x1, x2, x3);
        if (c == 0) *reinterpret_cast<float2*>(part + 16 * DH + 2 * r) = make_float2(M, l);
      } else {
        const bool any = (h0.w ? min(it.k1, it.pos0 + tok + 1) : it.k1) > it.k0;
        const float inv = 1.f / l;
        uint2 v = make_uint2(pack_bf16(x0 * inv, x1 * inv), pack_bf16(x2 * inv, x3 * inv));
        if (!any) v = make_uint2(0u, 0u);
        *reinterpret_cast<uint2*>(out + (it.row0 + tok) * a.out_stride + (long long)(h * group + r % group) * DH + c) = v;
      }
    }
    work += gridDim.x;
    if (work >= total || *abort_flag) return;
    done += n_blocks;
    it = paged_item_raw(hd, work / hkv);
    fence_async_smem();  // the meeting's and the cleared rows' plain accesses come before the next loads into the ring
    __syncthreads();
  }
}

template <int DH>
cudaError_t tokens_launch(const CUtensorMap& mk, const CUtensorMap& mv, const PagedAttnArgs& a, int grid, int shift,
                          cudaStream_t st) {
  static std::atomic<unsigned long long> set;
  if (cudaError_t e = ensure_dynamic_smem(k_paged_tokens<DH>, tokens_smem(DH), set)) return e;
  k_paged_tokens<DH><<<grid, kThreads, tokens_smem(DH), st>>>(mk, mv, a, shift, 1.4426950408889634f / sqrtf((float)DH));
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_paged_tokens(const PagedAttnArgs& a, const PagedPlanShape& s, int grid, cudaStream_t st) {
  (void)s;
  int shift = 0;
  while ((1 << shift) < a.c.page_size) ++shift;
  const uint64_t dh = a.c.dh, ps = a.c.page_size;
  const uint64_t dims[5] = {64, ps, dh / 64, (uint64_t)a.c.hkv, (uint64_t)a.c.num_pages};
  const uint64_t strides[4] = {dh * 2, 128, ps * dh * 2, (uint64_t)a.c.page_stride * 2};
  const uint32_t box[5] = {64, (uint32_t)(ps < 64 ? ps : 64), (uint32_t)(dh / 64), 1, 1};
  TmaDesc mk, mv;
  if (cudaError_t e = make_tma_nd_bf16(&mk, a.c.k, 5, dims, strides, box)) return e;
  if (cudaError_t e = make_tma_nd_bf16(&mv, a.c.v, 5, dims, strides, box)) return e;
  const CUtensorMap& k = reinterpret_cast<const CUtensorMap&>(mk);
  const CUtensorMap& v = reinterpret_cast<const CUtensorMap&>(mv);
  return a.c.dh == 128 ? tokens_launch<128>(k, v, a, grid, shift, st) : tokens_launch<64>(k, v, a, grid, shift, st);
}

}  // namespace prism
