// Attention over a paged cache on the 5th-generation tensor cores: chunks of new tokens, bf16, head_dim 64 or 128.
//
// A unit of work is (item of the work list, key/value head).  The query rows of a head group are (token, head of the
// group) pairs: 128 / group tokens times the group's heads fill one 128-row tile, so every key and value tile that is
// fetched serves all heads of the group.  An item has up to two such tiles, "A" and "B" (consecutive tokens), which share
// the key/value tiles of 128 keys: while one tile's softmax runs the other tile's MMAs do.  An item of few tokens has A
// only.  Long key ranges come cut into pieces (the work list decides); a piece leaves its unnormalised output, reference
// and sum as partial results.
//
// One persistent CTA per SM.  Units are handed out by the hardware's work distributor: the grid has one CTA per possible
// unit, and a running CTA takes over the next one that has not started (clusterlaunchcontrol.try_cancel), so there is no
// counter in memory that launches could share.  The request is made when a unit starts and answered long before it ends.
// Warp-specialised, 576 threads:
//   warp 0      producer: units, Q tiles, and key/value tiles page by page: every lane owns one (page, 64-column half) box of a
//               tile, so a tile of eight 16-token pages costs one instruction per lane; page numbers are read a tile ahead
//   warp 1      the only MMA issuer: S_x = Q_x K_j^T and O_x += P_x V_j (P from tensor memory, V as MN-major operand), in
//               the order PV_A(g) S_A(g+1) PV_B(g) S_B(g+1)
//   warps 2..9  softmax of A, warps 10..17 of B: two threads per row, exponentials against a per-row reference that starts
//               as the row's score on the piece's first key (a row that sees any key of a piece sees that one) and moves, by
//               whole powers of two, only when a row sum threatens fp32 range
// Tensor memory: S_A, S_B, O_A, O_B.  P_x(g) overlies S_x(g).  Rows that no token owns are not computed; a warp without any
// live row only keeps the barriers' phases.
// Values behind the last key of a piece (stale rows of the last page) are cleared in shared memory before the second
// product, so that nothing a page happens to hold meets a zero probability.
// Rounding: probabilities become bf16 for the second product; sums, references and outputs stay fp32 until the one
// rounding at the end.
// Every wait is bounded; on expiry the kernel records kErrTimeout and all roles drain to the common exit, which waits for
// the copies and MMAs in flight and frees the tensor memory.
#include "paged.cuh"
#include "tc_common.cuh"

namespace prism {
namespace {

using namespace tc;

constexpr int BM = 128, BN = 128;
constexpr int NK = 2, NV = 2;
constexpr int kStageBytes = 32 * 64;  // per softmax warp: 32 rows x 32 bf16 of output on their way to global memory
constexpr int kBarBytes = 640;
__host__ __device__ constexpr int tile_bytes(int dh) { return 128 * dh * 2; }
__host__ __device__ constexpr int smem_bytes(int dh) {
  return (2 + NK + NV) * tile_bytes(dh) + 16 * kStageBytes + 1024 /*alignment slack*/ + kBarBytes;
}
static_assert(smem_bytes(128) <= 232448, "exceeds the shared memory one CTA may have");
constexpr float kBigSum = 1.2089258e24f;  // 2^80: row sums of one block beyond this move the reference
constexpr int kThreads = 576;
constexpr int kTmemCols = 512;
constexpr int NI = 4;  // depth of the ring of published units

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void tmem_ld1(uint32_t taddr, uint32_t& v) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];" : "=r"(v) : "r"(taddr));
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
      ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, int c3, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
      ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(bar)
      : "memory");
}
// Ask the work distributor for a CTA of this grid that has not started; the 16-byte answer lands at `dst`.
__device__ __forceinline__ void request_unit(uint32_t dst, uint32_t bar) {
  asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(dst), "r"(bar)
               : "memory");
}
// The answer: that CTA's index, or -1 if there is none left.
__device__ __forceinline__ int answered_unit(uint32_t src) {
  uint32_t got, x;
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b128 r;\n\t"
      "ld.shared.b128 r, [%2];\n\t"
      "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, r;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t"
      "mov.u32 %1, 0;\n\t"
      "@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %1, r;\n\t}"
      : "=r"(got), "=r"(x)
      : "r"(src)
      : "memory");
  return got ? (int)x : -1;
}

struct Unit {
  int n_blocks;  // 0: no more units
  int row0, n_tok, pos0, k0, k1, part, h;
};
struct UnitReader {
  volatile Unit* ring;
  uint32_t b_full, b_empty, n;
  int n_blocks, n_tok;
  __device__ __forceinline__ void init(Unit* ring_, uint32_t b_full_, uint32_t b_empty_) {
    ring = ring_, b_full = b_full_, b_empty = b_empty_, n = 0, n_blocks = 0, n_tok = 0;
  }
  // Moves to the next unit; false at the end of the work or when the wait gave up.
  template <bool kWarp>
  __device__ __forceinline__ bool next(int* err, volatile int* abort_flag) {
    const uint32_t bar = b_full + 8 * (n % NI), parity = (n / NI) & 1;
    if (!(kWarp ? warp_wait(bar, parity, err, abort_flag) : mbar_wait(bar, parity, err, abort_flag))) return false;
    n_blocks = ring[n % NI].n_blocks;
    n_tok = ring[n % NI].n_tok;
    return n_blocks > 0;
  }
  __device__ __forceinline__ volatile Unit& rec() { return ring[n % NI]; }
  __device__ __forceinline__ void release() { mbar_arrive(b_empty + 8 * (n % NI)); }
  __device__ __forceinline__ void advance() { ++n; }
};

template <int DH>
__global__ void __launch_bounds__(kThreads, 1)
k_paged_tiles(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
              const __grid_constant__ CUtensorMap map_v, const __grid_constant__ PagedAttnArgs a, int shift, int tpt,
              float scale_log2) {
  pdl_sync();
  extern __shared__ unsigned char smem_raw[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int hkv = a.c.hkv, group = a.hq / hkv;
  const PagedPlanHeader* hd = static_cast<const PagedPlanHeader*>(a.plan);
  const int4 h0 = reinterpret_cast<const int4*>(hd)[0], h1 = reinterpret_cast<const int4*>(hd)[1],
             h2 = reinterpret_cast<const int4*>(hd)[2];
  if (h0.x != kPagedTiles || h1.x != a.hq || h1.y != hkv || h1.z != DH || h1.w != a.total_q || h2.x != a.n_seq ||
      h2.y != a.max_q) {
    if (threadIdx.x == 0 && blockIdx.x == 0) atomicOr(a.err, kErrBadOffsets);
    return;
  }
  const int total = min(h0.y * hkv, (int)gridDim.x), causal = h0.w;
  // more items than the launch was sized for: lengths beyond the block table's width
  if (threadIdx.x == 0 && blockIdx.x == 0 && h0.y * hkv > (int)gridDim.x) atomicOr(a.err, kErrBadPage);
  if ((int)blockIdx.x >= total) return;
  int* const err = a.err;
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  unsigned char* gen = smem_raw + (base - raw);
  constexpr int kTile = tile_bytes(DH), kSub = DH / 64;
  constexpr int kSubBytes = 128 * 128;
  const uint32_t s_q = base, s_k = base + 2 * kTile, s_v = s_k + NK * kTile, s_o = s_v + NV * kTile;
  uint64_t* bars = reinterpret_cast<uint64_t*>(gen + (2 + NK + NV) * kTile + 16 * kStageBytes);
  // q_full[2], q_empty[2], k_full[2], k_empty[2], v_full[2], v_empty[2], s_full[2], p_full[2], o_full[2]
  const uint32_t b_q_full = smem_u32(bars), b_q_empty = smem_u32(bars + 2);
  const uint32_t b_k_full = smem_u32(bars + 4), b_k_empty = smem_u32(bars + 6);
  const uint32_t b_v_full = smem_u32(bars + 8), b_v_empty = smem_u32(bars + 10);
  const uint32_t b_s_full = smem_u32(bars + 12), b_p_full = smem_u32(bars + 14), b_o_full = smem_u32(bars + 16);
  const uint32_t b_pair = smem_u32(bars + 18);                             // [8]: the two warps of a (tile, lane quarter)
  const uint32_t b_unit_full = smem_u32(bars + 26), b_unit_empty = b_unit_full + 8 * NI;
  const uint32_t b_clc = b_unit_empty + 8 * NI, b_done = b_clc + 8;
  const uint32_t clc_resp = smem_u32(bars + 36);                           // 16 bytes, 16-byte aligned
  Unit* ring = reinterpret_cast<Unit*>(bars + 38);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(ring + NI);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  uint32_t* votes = tmem_slot + 2;                                         // [8][3]
  static_assert(38 * 8 + NI * sizeof(Unit) + 8 + 24 * 4 <= kBarBytes, "barrier area too small");
  static_assert(26 + 2 * NI + 2 == 36, "barrier layout");

  if (threadIdx.x == 0) {
    for (int i = 0; i < 14; ++i) mbar_init(b_q_full + 8 * i, 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(b_p_full + 8 * i, 8);
      mbar_init(b_o_full + 8 * i, 1);
    }
    for (int i = 0; i < 8; ++i) mbar_init(b_pair + 8 * i, 2);
    for (int i = 0; i < 24; ++i) votes[i] = 0;
    for (int i = 0; i < NI; ++i) {
      mbar_init(b_unit_full + 8 * i, 1);
      mbar_init(b_unit_empty + 8 * i, 17);  // the MMA thread and sixteen softmax warps
    }
    mbar_init(b_clc, 1);
    mbar_init(b_done, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(kTmemCols));
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;

  if (warp == 0) {
    // ------------------------------------------------------------------ producer (the whole warp)
    const int box_shift = shift < 7 ? shift : 7, box_rows = 1 << box_shift, boxes = BN >> box_shift;
    const int my_box = lane & (boxes - 1), my_sub = lane >> (7 - box_shift);  // lane = sub * boxes + box
    const uint32_t box_bytes = (uint32_t)box_rows * 128;
    const uint32_t q_bytes = (uint32_t)(kSub * group * tpt) * 128;
    uint32_t kc = 0, vc = 0, ic = 0, qc[2] = {0, 0};
    int w = (int)blockIdx.x;
    bool ok = true;
    uint32_t asked = 0;
    for (;; ++asked) {
      if (lane == 0) {
        fence_async_smem();  // the previous answer has been read
        mbar_expect_tx(b_clc, 16);
        request_unit(clc_resp, b_clc);
      }
      if (w < total) {
        const PagedItem it = paged_item(hd, w / hkv, a.max_pages, shift, a.ws, err);
        const int h = w % hkv, nb = it.k1 > it.k0 ? (it.k1 - it.k0 + BN - 1) / BN : 0;
        if (nb == 0) {
          // no key is visible to these rows.  A piece without keys (a list made for a longer table) leaves an empty
          // partial result.
          __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.out);
          if (it.part < 0) {
            for (int u = lane; u < it.n_tok * group * (DH / 8); u += 32) {
              const int t = u / (group * (DH / 8)), rem = u % (group * (DH / 8));
              *reinterpret_cast<uint4*>(out + (it.row0 + t) * a.out_stride + (long long)h * group * DH + rem * 8) = make_uint4(0, 0, 0, 0);
            }
          } else {
            float* p = a.ws + ((long long)it.part * hkv + h) * paged_part_floats(256, DH);
            for (int u = lane; u < 256 * (DH / 4); u += 32) reinterpret_cast<float4*>(p)[u] = make_float4(0.f, 0.f, 0.f, 0.f);
            for (int u = lane; u < 256; u += 32) *reinterpret_cast<float2*>(p + 256 * DH + 2 * u) = make_float2(-INFINITY, 0.f);
          }
        } else {
          const uint32_t slot = ic % NI;
          ok = warp_wait(b_unit_empty + 8 * slot, ((ic / NI) & 1) ^ 1, err, abort_flag);
          if (!ok) break;
          if (lane == 0) {
            volatile Unit& u = ring[slot];
            u.n_blocks = nb, u.row0 = it.row0, u.n_tok = it.n_tok, u.pos0 = it.pos0;
            u.k0 = it.k0, u.k1 = it.k1, u.part = it.part, u.h = h;
            mbar_arrive(b_unit_full + 8 * slot);
          }
          ++ic;
          const int* row = a.table + it.seq * a.table_stride;
          auto page_of = [&](int t) {
            const int key = it.k0 + t * BN + (my_box << box_shift);
            if (my_sub >= kSub || key >= it.k1) return 0;
            const int id = row[key >> shift];  // key < k1 <= max_pages << shift
            if ((unsigned)id >= (unsigned)a.c.num_pages) {
              atomicOr(err, kErrBadPage);
              return a.c.num_pages;  // beyond the tensor: the box arrives as zeros
            }
            return id;
          };
          auto load_q = [&](int x) {
            if (!warp_wait(b_q_empty + 8 * x, (qc[x] & 1) ^ 1, err, abort_flag)) return false;
            if (lane == 0) {
              mbar_expect_tx(b_q_full + 8 * x, q_bytes);
#pragma unroll
              for (int sb = 0; sb < kSub; ++sb)
                tma_load_3d(s_q + x * kTile + sb * kSubBytes, &map_q, 64 * sb, h * group, it.row0 + x * tpt, b_q_full + 8 * x);
            }
            ++qc[x];
            return true;
          };
          auto load_kv = [&](const CUtensorMap* map, int t, int id, uint32_t ringbuf, uint32_t b_full, uint32_t b_empty,
                             uint32_t& cnt, int depth) {
            const uint32_t st = cnt % depth;
            if (!warp_wait(b_empty + 8 * st, ((cnt / depth) & 1) ^ 1, err, abort_flag)) return false;
            const int key0 = it.k0 + t * BN, live = (min(BN, it.k1 - key0) + box_rows - 1) >> box_shift;
            if (lane == 0) mbar_expect_tx(b_full + 8 * st, (uint32_t)(live * kSub) * box_bytes);
            __syncwarp();
            if (my_sub < kSub && my_box < live)
              tma_load_4d(ringbuf + st * kTile + my_sub * kSubBytes + my_box * box_bytes, map, 64 * my_sub,
                          (key0 + (my_box << box_shift)) & ((1 << shift) - 1), h, id, b_full + 8 * st);
            ++cnt;
            return true;
          };
          int id = page_of(0), id_prev = 0;
          ok = load_q(0) && load_kv(&map_k, 0, id, s_k, b_k_full, b_k_empty, kc, NK) && (it.n_tok <= tpt || load_q(1));
          for (int t = 1; ok && t <= nb; ++t) {
            id_prev = id;
            if (t < nb) {
              id = page_of(t);
              ok = load_kv(&map_k, t, id, s_k, b_k_full, b_k_empty, kc, NK);
            }
            if (ok) ok = load_kv(&map_v, t - 1, id_prev, s_v, b_v_full, b_v_empty, vc, NV);
          }
          if (!ok) break;
        }
      }
      __syncwarp();
      ok = warp_wait(b_clc, asked & 1, err, abort_flag);
      if (!ok) break;
      w = answered_unit(clc_resp);
      __syncwarp();  // every lane has read the answer before lane 0 asks again
      if (w < 0) break;
    }
    if (ok && lane == 0) {
      const uint32_t slot = ic % NI;
      if (mbar_wait(b_unit_empty + 8 * slot, ((ic / NI) & 1) ^ 1, err, abort_flag)) {
        ring[slot].n_blocks = 0;
        ring[slot].n_tok = 0;
        mbar_arrive(b_unit_full + 8 * slot);
      }
    }
    if (!ok) {
      // gave up: whatever is still in flight into this CTA's shared memory has to land first
      for (uint32_t i = kc > NK ? kc - NK : 0; i < kc; ++i) mbar_drain(b_k_full + 8 * (i % NK), (i / NK) & 1);
      for (uint32_t i = vc > NV ? vc - NV : 0; i < vc; ++i) mbar_drain(b_v_full + 8 * (i % NV), (i / NV) & 1);
      for (int x = 0; x < 2; ++x)
        if (qc[x]) mbar_drain(b_q_full + 8 * x, (qc[x] - 1) & 1);
      mbar_drain(b_clc, asked & 1);
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ MMA issuer
    if (lane == 0) {
      constexpr uint32_t kIdescS = idesc_bf16(BM, BN, 0), kIdescO = idesc_bf16(BM, DH, 1);
      constexpr int kDepthSteps = DH / 16;
      UnitReader its, itp;  // the block whose scores are issued next; the block whose P V is issued next
      its.init(ring, b_unit_full, b_unit_empty);
      itp.init(ring, b_unit_full, b_unit_empty);
      bool s_has = its.next<false>(err, abort_flag), p_has = itp.next<false>(err, abort_flag);
      int sj = 0, pj = 0;                               // block index inside its / itp
      uint32_t sq[2] = {0, 0}, pc[2] = {0, 0};          // Q tiles used up; blocks whose P V has been issued, per tile
      uint32_t kc = 0, vc = 0;
      bool ok = true;
      // S_x of block (its, sj).  The block's last tile also releases the keys and moves the score cursor on.
      auto issue_s = [&](int x, int last) {
        const uint32_t st = kc % NK;
        if (sj == 0 && !mbar_wait(b_q_full + 8 * x, sq[x] & 1, err, abort_flag)) return false;
        if (x == 0 && !mbar_wait(b_k_full + 8 * st, (kc / NK) & 1, err, abort_flag)) return false;
        tc_fence_after();
        const uint32_t aq = s_q + x * kTile, ak = s_k + st * kTile;
#pragma unroll
        for (int kk = 0; kk < kDepthSteps; ++kk) {
          const uint64_t da = smem_desc(aq + (kk >> 2) * kSubBytes + (kk & 3) * 32, 16, 1024);
          const uint64_t db = smem_desc(ak + (kk >> 2) * kSubBytes + (kk & 3) * 32, 16, 1024);
          umma_bf16(tmem + x * BN, da, db, kIdescS, kk != 0);
        }
        umma_commit(b_s_full + 8 * x);
        if (sj == its.n_blocks - 1) {
          umma_commit(b_q_empty + 8 * x);  // the unit's last use of Q_x
          ++sq[x];
        }
        if (x == last) {
          umma_commit(b_k_empty + 8 * st);
          ++kc;
          if (++sj == its.n_blocks) {
            sj = 0;
            its.advance();
            s_has = its.next<false>(err, abort_flag);
          }
        }
        return true;
      };
      auto issue_pv = [&](int x, int last) {
        const uint32_t st = vc % NV;
        if (!mbar_wait(b_p_full + 8 * x, pc[x] & 1, err, abort_flag)) return false;
        if (x == 0 && !mbar_wait(b_v_full + 8 * st, (vc / NV) & 1, err, abort_flag)) return false;
        tc_fence_after();
        const uint32_t av = s_v + st * kTile;
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) {
          const uint64_t db = smem_desc(av + kk * 2048, kSubBytes, 1024);
          umma_bf16_ts(tmem + 2 * BN + x * DH, tmem + x * BN + kk * 8, db, kIdescO, (pj | kk) != 0);
        }
        umma_commit(b_o_full + 8 * x);
        if (x == last) umma_commit(b_v_empty + 8 * st);
        ++pc[x];
        return true;
      };
      if (s_has) {
        const int last = its.n_tok > tpt;
        ok = issue_s(0, last);
        if (ok && last) ok = issue_s(1, last);
      }
      while (ok && p_has) {
        const int p_last = itp.n_tok > tpt;
        const bool s_now = s_has;
        const int s_last = s_now && its.n_tok > tpt;
        ok = issue_pv(0, p_last);
        if (ok && s_now) ok = issue_s(0, s_last);
        if (ok && p_last) ok = issue_pv(1, p_last);
        if (ok && s_last) ok = issue_s(1, s_last);
        ++vc;
        if (++pj == itp.n_blocks) {
          pj = 0;
          itp.release();  // the score cursor is past this unit too
          itp.advance();
          p_has = itp.next<false>(err, abort_flag);
        }
      }
      umma_commit(b_done);  // every MMA issued above has completed before the tensor memory is given back
      mbar_drain(b_done, 0);
    }
  } else {
    // ------------------------------------------------------------------ softmax + output, two threads per query row
    const int x = (warp - 2) >> 3;         // tile A or B
    const int hf = ((warp - 2) >> 2) & 1;  // which chunks of a block / which half of the output columns
    const int quarter = warp & 3;          // the TMEM lane quarter this warp may access
    const int r = quarter * 32 + lane;     // row inside the tile = TMEM lane
    const uint32_t lane_base = (uint32_t)(quarter * 32) << 16;
    const uint32_t t_s = tmem + lane_base + x * BN, t_o = tmem + lane_base + 2 * BN + x * DH + hf * (DH / 2);
    const uint32_t bar_s = b_s_full + 8 * x, bar_p = b_p_full + 8 * x, bar_o = b_o_full + 8 * x;
    const int tt = r / group, head = r % group;  // token inside the tile, head of the group
    // Meeting point of the two warps that share these 32 rows, carrying a vote: slot (u + 1) % 3 is cleared before the
    // arrival at meeting u; both warps read it after meeting u - 2 and before arriving at u - 1.
    const uint32_t pair_mb = b_pair + 8 * (x * 4 + quarter);
    volatile uint32_t* my_votes = votes + 3 * (x * 4 + quarter);
    uint32_t meet = 0;
    auto pair_meet = [&](bool flag) -> int {
      __syncwarp();
      const bool any = __any_sync(0xffffffffu, flag);
      if (lane == 0) {
        if (hf == 0) my_votes[(meet + 1) % 3] = 0;
        if (any) my_votes[meet % 3] = 1;
        mbar_arrive(pair_mb);
      }
      if (!warp_wait(pair_mb, meet & 1, err, abort_flag)) return -1;
      const int v = (int)my_votes[meet % 3];
      ++meet;
      return v;
    };
    const uint32_t stg = s_o + (uint32_t)(warp - 2) * kStageBytes;
    const uint32_t stg_other = s_o + (uint32_t)((warp - 2) ^ 4) * kStageBytes;
    const int c0 = hf, c1 = hf + 2;
    UnitReader it;
    it.init(ring, b_unit_full, b_unit_empty);
    uint32_t gc = 0;  // blocks of this tile handled so far
    bool ok = true;
    while (ok && it.next<true>(err, abort_flag)) {
      const int n_tok = x == 0 ? min(it.n_tok, tpt) : it.n_tok - tpt;  // tokens of this tile
      if (n_tok <= 0) {  // B of a unit that has A only
        __syncwarp();
        if (lane == 0) it.release();
        it.advance();
        continue;
      }
      const int row0 = it.rec().row0, pos0 = it.rec().pos0, k0 = it.rec().k0, k1 = it.rec().k1, part = it.rec().part;
      const int h = it.rec().h;
      const bool live = tt < n_tok;
      // keys below lim are visible to this row; rows without a token follow the tile's last one, so that they ask for no
      // masking of their own
      const int lim = causal ? min(k1, pos0 + x * tpt + min(tt, n_tok - 1) + 1) : k1;
      const int lim_min = __reduce_min_sync(0xffffffffu, lim), lim_max = __reduce_max_sync(0xffffffffu, lim);
      const bool warp_live = __any_sync(0xffffffffu, live);
      const bool sees = lim > k0;
      float ms = 0.f, l = 0.f;  // reference exponent; this thread's part of the row sum
      for (int j = 0; j < it.n_blocks; ++j, ++gc) {
        if (!warp_wait(bar_s, gc & 1, err, abort_flag)) { ok = false; break; }
        tc_fence_after();
        const int kb = k0 + j * BN;
        if (x == 0 && kb + BN > k1) {
          // the value tile's rows behind the last key: A's eight warps clear them.  A handles every block, so block gc is
          // value tile gc; its scores were issued after P V(gc - 1), whose wait saw every earlier phase of v_full.
          const uint32_t st = gc % NV;
          if (!warp_wait(b_v_full + 8 * st, (gc / NV) & 1, err, abort_flag)) { ok = false; break; }
          const int first = k1 - kb, n16 = (BN - first) * (DH / 8);
          for (int u = (warp - 2) * 32 + lane; u < n16; u += 256) {
            const int rr = first + u / (DH / 8), ch = u % (DH / 8);
            const uint32_t dst = s_v + st * kTile + (ch >> 3) * kSubBytes + rr * 128 + (((ch & 7) ^ (rr & 7)) << 4);
            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(dst), "r"(0) : "memory");
          }
          fence_async_smem();
        }
        if (warp_live) {
          uint32_t sa[32], pk[32];
          tmem_ld32(t_s + c0 * 32, sa);
          if (j == 0) {
            uint32_t s00;
            tmem_ld1(t_s, s00);
            tmem_ld_wait();
            ms = sees ? __uint_as_float(s00) * scale_log2 : 0.f;
          } else {
            tmem_ld_wait();
          }
          const uint64_t sc2 = f2_pack(scale_log2, scale_log2);
          uint64_t rs2;
          auto chunk = [&](int ch, uint32_t* cur, uint32_t* out16) {
            const int key = kb + ch * 32;
            if (key >= lim_max) {  // beyond every row of this warp
#pragma unroll
              for (int c = 0; c < 16; ++c) out16[c] = 0u;
              return;
            }
            if (key + 32 > lim_min) {
#pragma unroll
              for (int c = 0; c < 32; ++c)
                if (key + c >= lim) cur[c] = 0xff800000u;  // -inf
            }
            const uint64_t nm2 = f2_pack(-ms, -ms);
#pragma unroll
            for (int c = 0; c < 16; ++c) {
              float x0, x1;
              f2_unpack(f2_fma(f2_pack(__uint_as_float(cur[2 * c]), __uint_as_float(cur[2 * c + 1])), sc2, nm2), x0, x1);
              const float p0 = ex2(x0), p1 = ex2(x1);
              rs2 = f2_add(rs2, f2_pack(p0, p1));
              out16[c] = pack_bf16(p0, p1);
            }
          };
          rs2 = f2_pack(0.f, 0.f);
          chunk(c0, sa, pk);
          tmem_ld32(t_s + c1 * 32, sa);
          tmem_ld_wait();
          chunk(c1, sa, pk + 16);
          float rlo, rhi;
          f2_unpack(rs2, rlo, rhi);
          float rs = rlo + rhi;
          // The vote "some row sum is out of range" also orders the P stores below after both threads' score loads.
          const int vote = pair_meet(live && !(rs <= kBigSum));
          if (vote < 0) { ok = false; break; }
          if (vote) {
            // Rare: rows whose largest exponent is beyond 2^64 move their reference up by d = ceil(that exponent); what
            // was accumulated is scaled by 2^-d (exact).  Nothing of this block has been stored yet.
            float xmax = -INFINITY;
#pragma unroll 1
            for (int v = 0; v < 2; ++v) {
              const int ch = v ? c1 : c0;
              tmem_ld32(t_s + ch * 32, sa);
              tmem_ld_wait();
#pragma unroll
              for (int c = 0; c < 32; ++c)
                if (kb + ch * 32 + c < lim) xmax = fmaxf(xmax, fmaf(__uint_as_float(sa[c]), scale_log2, -ms));
            }
            asm volatile("st.shared.f32 [%0], %1;" ::"r"(stg + lane * 4), "f"(xmax) : "memory");
            if (pair_meet(false) < 0) { ok = false; break; }
            float xo;
            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(xo) : "r"(stg_other + lane * 4) : "memory");
            xmax = fmaxf(xmax, xo);
            const float d = xmax > 64.f ? ceilf(xmax) : 0.f;
            const float f = exp2f(-d);
            if (j > 0) {
              if (!warp_wait(bar_o, (gc - 1) & 1, err, abort_flag)) { ok = false; break; }  // complete already
              tc_fence_after();
#pragma unroll 1
              for (int c = 0; c < DH / 64; ++c) {
                uint32_t o[32];
                tmem_ld32(t_o + c * 32, o);
                tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                tmem_st32(t_o + c * 32, o);
              }
            }
            l *= f;
            ms += d;
            rs2 = f2_pack(0.f, 0.f);
            tmem_ld32(t_s + c0 * 32, sa);
            tmem_ld_wait();
            chunk(c0, sa, pk);
            tmem_ld32(t_s + c1 * 32, sa);
            tmem_ld_wait();
            chunk(c1, sa, pk + 16);
            f2_unpack(rs2, rlo, rhi);
            rs = rlo + rhi;
            if (pair_meet(false) < 0) { ok = false; break; }  // the partner has re-read its scores too
          }
          l += rs;
          tmem_st16(t_s + c0 * 16, pk);
          tmem_st16(t_s + c1 * 16, pk + 16);
          tmem_st_wait();
        }
        tc_fence_before();
        // The scores of block gc were issued after the wait for p_full(gc - 1), so that phase is over before any warp
        // gets here.
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_p);
      }
      if (!ok) break;
      if (!warp_wait(bar_o, (gc - 1) & 1, err, abort_flag)) { ok = false; break; }
      tc_fence_after();
      if (warp_live) {
        asm volatile("st.shared.f32 [%0], %1;" ::"r"(stg + lane * 4), "f"(l) : "memory");
        if (pair_meet(false) < 0) { ok = false; break; }
        float lo;
        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(lo) : "r"(stg_other + lane * 4) : "memory");
        if (pair_meet(false) < 0) { ok = false; break; }  // read before either warp stages output there
        if (part < 0) {
          // This thread's columns of O_x / l as bf16, 32 at a time through the warp's staging rows (64 bytes each,
          // 16-byte pieces XOR-swizzled), so that global stores are 64 contiguous bytes per row.
          const float inv = 1.f / (l + lo);
          const long long at = live ? (long long)(row0 + x * tpt + tt) * a.out_stride + (long long)(h * group + head) * DH : -1;
          __nv_bfloat16* ocol = static_cast<__nv_bfloat16*>(a.out) + hf * (DH / 2);
#pragma unroll 1
          for (int pt = 0; pt < DH / 64; ++pt) {
            uint32_t o[32];
            tmem_ld32(t_o + pt * 32, o);
            tmem_ld_wait();
#pragma unroll
            for (int v = 0; v < 4; ++v) {
              const uint32_t dst = stg + lane * 64 + ((v ^ ((lane >> 1) & 3)) << 4);
              uint32_t w4[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                w4[e] = pack_bf16(__uint_as_float(o[v * 8 + 2 * e]) * inv, __uint_as_float(o[v * 8 + 2 * e + 1]) * inv);
                if (!sees) w4[e] = 0u;  // no visible key: zero
              }
              asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst), "r"(w4[0]), "r"(w4[1]), "r"(w4[2]), "r"(w4[3])
                           : "memory");
            }
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int rr = i * 8 + (lane >> 2), chn = lane & 3;
              uint4 val;
              asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                           : "=r"(val.x), "=r"(val.y), "=r"(val.z), "=r"(val.w)
                           : "r"(stg + rr * 64 + ((chn ^ ((rr >> 1) & 3)) << 4)));
              const long long to = __shfl_sync(0xffffffffu, at, rr);
              if (to >= 0) *reinterpret_cast<uint4*>(ocol + to + pt * 32 + chn * 8) = val;
            }
            __syncwarp();
          }
        } else {
          // partial result, row fastest: the lanes of a warp write side by side
          float* p = a.ws + ((long long)part * hkv + h) * paged_part_floats(256, DH);
          const int rc = x * tpt * group + r;  // (token, head) index inside the unit
#pragma unroll 1
          for (int pt = 0; pt < DH / 64; ++pt) {
            uint32_t o[32];
            tmem_ld32(t_o + pt * 32, o);
            tmem_ld_wait();
            if (live) {
#pragma unroll
              for (int v = 0; v < 8; ++v)
                *reinterpret_cast<uint4*>(p + ((long long)(hf * (DH / 8) + pt * 8 + v) * 256 + rc) * 4) =
                    make_uint4(o[4 * v], o[4 * v + 1], o[4 * v + 2], o[4 * v + 3]);
            }
          }
          if (live && hf == 0) *reinterpret_cast<float2*>(p + 256 * DH + 2 * rc) = make_float2(ms, l + lo);
        }
      }
      // The next unit's first P V (which overwrites O_x) is issued only after this thread's arrival for that block.
      tc_fence_before();
      __syncwarp();
      if (lane == 0) it.release();
      it.advance();
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols));
  }
}

template <int DH>
cudaError_t tiles_launch(const TmaDesc& q, const TmaDesc& k, const TmaDesc& v, const PagedAttnArgs& a, int tpt, int grid, int shift,
                         cudaStream_t st) {
  static std::atomic<unsigned long long> set;
  if (cudaError_t e = ensure_dynamic_smem(k_paged_tiles<DH>, smem_bytes(DH), set)) return e;
  k_paged_tiles<DH><<<grid, kThreads, smem_bytes(DH), st>>>(
      reinterpret_cast<const CUtensorMap&>(q), reinterpret_cast<const CUtensorMap&>(k), reinterpret_cast<const CUtensorMap&>(v), a,
      shift, tpt, 1.4426950408889634f / sqrtf((float)DH));
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_paged_tiles(const PagedAttnArgs& a, const PagedPlanShape& s, int grid, cudaStream_t st) {
  int shift = 0;
  while ((1 << shift) < a.c.page_size) ++shift;
  const uint64_t dh = a.c.dh, ps = a.c.page_size;
  const int tpt = s.tokens / 2;
  TmaDesc mq, mk, mv;
  {
    const uint64_t dims[3] = {dh, (uint64_t)a.hq, (uint64_t)a.total_q};
    const uint64_t strides[2] = {dh * 2, (uint64_t)a.q_stride * 2};
    const uint32_t box[3] = {64, (uint32_t)s.group, (uint32_t)tpt};
    if (cudaError_t e = make_tma_nd_bf16(&mq, a.q, 3, dims, strides, box)) return e;
  }
  const uint64_t dims[4] = {dh, ps, (uint64_t)a.c.hkv, (uint64_t)a.c.num_pages};
  const uint64_t strides[3] = {dh * 2, ps * dh * 2, (uint64_t)a.c.page_stride * 2};
  const uint32_t box[4] = {64, (uint32_t)(ps < 128 ? ps : 128), 1, 1};
  if (cudaError_t e = make_tma_nd_bf16(&mk, a.c.k, 4, dims, strides, box)) return e;
  if (cudaError_t e = make_tma_nd_bf16(&mv, a.c.v, 4, dims, strides, box)) return e;
  return a.c.dh == 128 ? tiles_launch<128>(mq, mk, mv, a, tpt, grid, shift, st) : tiles_launch<64>(mq, mk, mv, a, tpt, grid, shift, st);
}

}  // namespace prism
