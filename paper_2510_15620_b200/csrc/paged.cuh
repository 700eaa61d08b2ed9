// Shared declarations of the paged key/value cache operators (internal; the public surface is include/prism_ops.h).
#pragma once

#include "common.cuh"

namespace prism {

constexpr int kErrBadPage = 16;   // a page id or slot outside the cache
constexpr int kErrPoolEmpty = 32; // not enough free pages (append), or no room to put them back (release)

// Where a cache lies: page p, key/value head h, row r of the page starts at p * page_stride + (h * page_size + r) * dh
// elements.  All of a head's rows of one page lie together, so that a page is fetched in one piece per head.
struct PagedCache {
  void* k;
  void* v;
  long long page_stride;  // elements
  int num_pages, page_size, hkv, dh, dtype;
};

// Attention over pages: which kernel serves a call.  The choice depends on host-known sizes only and is made by
// the same function for the work list and for the launch.
enum PagedKind : int {
  kPagedTokens = 0,  // up to 32 query rows per sequence and key/value head: warp-level MMA, bound by reading the cache
  kPagedTiles = 1,   // tcgen05, two 128-row tiles per item
  kPagedSimt = 2,    // CUDA cores: fp32, and head sizes without a tensor-core kernel
  kPagedFew = 3,     // the same for up to 8 query rows per sequence and key/value head: a warp per item and head
};

struct PagedPlanShape {
  int kind;
  int group;       // query heads per key/value head
  int rows;        // query rows (token, head of the group) an item has room for
  int tokens;      // tokens an item covers
  int min_piece;   // keys: tiles are never cut into pieces shorter than this
  int min_cut;     // keys: shorter tiles are not cut at all
  int piece_unit;  // keys: pieces are multiples of this
  int target;      // pieces are at least total keys * hkv / target long
  int slots;       // blocks that run at a time
  // What a launch is expected to take, in nanoseconds (measured): per key of a block's own, at least, and per key and running
  // block (they share the memory's rate); per item; per piece of a cut tile; once if any tile is cut.
  float ns_key, ns_key_block, ns_item, ns_part, ns_join;
};

// Work list of one step: header, items, joins.  A tile of query rows whose keys are cut into pieces has one item per
// piece (part >= 0: the piece's place among the partial results) and one join.
struct PagedPlanHeader {
  int kind, n_items, n_joins, causal;
  int hq, hkv, dh, total_q;
  int n_seq, max_q, rows, pad;
  int reserved[4];
};
struct PagedItem {
  int seq, row0, n_tok, pos0;  // sequence; first packed row; tokens; position of the first token
  int k0, k1, part, pad;       // keys [k0, k1) of the sequence; partial result or -1
};
#ifdef __CUDACC__
// Cuts an item's keys to what the block table can name (a list made from lengths beyond it must not keep a kernel busy).
// Without a workspace (a table too narrow for any tile to be cut) a cut tile can only come from such lengths too: its rows
// become zero.  Called by whole blocks or by one warp of a block whose first thread belongs to it.
__device__ __forceinline__ void paged_item_check(PagedItem& it, int max_pages, int shift, const float* ws, int* err) {
  const long long cap = (long long)max_pages << shift;
  if (it.k1 > cap) {
    if (threadIdx.x == 0) atomicOr(err, kErrBadPage);
    it.k1 = (int)cap, it.k0 = min(it.k0, it.k1);  // (what counts keys from k0 on stays below 2^31)
  }
  if (it.part >= 0 && !ws) it.k1 = it.k0 = 0, it.part = -1;
}
__device__ __forceinline__ PagedItem paged_item_raw(const PagedPlanHeader* hd, int i) {
  const int4* p = reinterpret_cast<const int4*>(reinterpret_cast<const PagedItem*>(hd + 1) + i);
  const int4 a = p[0], b = p[1];
  return PagedItem{a.x, a.y, a.z, a.w, b.x, b.y, b.z, 0};
}
__device__ __forceinline__ PagedItem paged_item(const PagedPlanHeader* hd, int i, int max_pages, int shift, const float* ws,
                                                int* err) {
  PagedItem it = paged_item_raw(hd, i);
  paged_item_check(it, max_pages, shift, ws, err);
  return it;
}
#endif
struct PagedJoin {
  int row0, n_tok, pos0, part0;
  int n_parts, piece, causal, pad;  // piece i covers keys from i * piece
};
static_assert(sizeof(PagedPlanHeader) == 64 && sizeof(PagedItem) == 32 && sizeof(PagedJoin) == 32, "plan layout");

// Returns false where no kernel serves the shape.
bool paged_plan_shape(int n_seq, int total_q, int max_q, int hq, int hkv, int dh, int dtype, int impl, PagedPlanShape* s);

// Upper bounds the buffers are sized by (the lengths live on the device).  An item covers s.tokens tokens of one
// sequence, so there are at most total_q / tokens + n_seq tiles; pieces are at least total keys * hkv / target long, so
// cutting adds at most target / hkv items, at most that many tiles are cut, and every cut tile adds at most one more.
struct PagedPlanBounds {
  long long items, joins, parts;
};
inline PagedPlanBounds paged_plan_bounds(const PagedPlanShape& s, int hkv, int n_seq, int total_q) {
  PagedPlanBounds b;
  const long long tiles = (long long)total_q / s.tokens + n_seq;
  const long long cuts = s.target / hkv + 1;
  b.items = tiles + cuts;
  b.joins = tiles < cuts ? tiles : cuts;
  b.parts = cuts + b.joins;
  return b;
}
inline long long paged_plan_bytes(const PagedPlanBounds& b) {
  return (long long)sizeof(PagedPlanHeader) + b.items * (long long)sizeof(PagedItem) + b.joins * (long long)sizeof(PagedJoin);
}
// Partial results: per part and key/value head, [dh / 4][rows] float4 of the unnormalised output (row fastest, so that
// threads that own rows write side by side), then [rows] (reference exponent, sum) pairs.
__host__ __device__ inline long long paged_part_floats(int rows, int dh) { return (long long)rows * (dh + 2); }
inline long long paged_ws_bytes(const PagedPlanShape& s, const PagedPlanBounds& b, int hkv, int dh) {
  return b.parts * hkv * paged_part_floats(s.rows, dh) * 4;
}

struct PagedAttnArgs {
  const void* q;
  long long q_stride;  // elements between tokens
  PagedCache c;
  const int* table;
  int max_pages;
  long long table_stride;
  const void* plan;
  int n_seq, total_q, max_q, hq;
  void* out;
  long long out_stride;
  float* ws;
  int* err;
};

cudaError_t launch_page_append(const int* len_new, const int* kv_in, int* kv_out, int n, int page_size, int num_pages,
                               int max_pages, long long table_stride, int* table, const int* free_pages, const int* n_free_in,
                               int* n_free_out, int total, int* cu, int* pos, int* slot, int* err, cudaStream_t st);
cudaError_t launch_page_release(const int* keep, int n_new, const int* kv_in, int* kv_out, int n, int page_size, int num_pages,
                                int shared_pages, int max_pages, long long stride_in, const int* table_in,
                                long long stride_out, int* table_out, int* free_pages, const int* n_free_in, int* n_free_out,
                                int* err, cudaStream_t st);
cudaError_t launch_qknorm_rope_paged(const void* qkv, long long qkv_stride, const int* pos, const int* slot, int rows, int hq,
                                     int qk_norm, const void* g_q, const void* g_k, float eps, double theta, void* q_out,
                                     long long q_stride, const PagedCache& c, int* err, cudaStream_t st);
cudaError_t launch_paged_plan(const int* cu, const int* kv_len, int n_seq, int total_q, int max_q, int hq, int hkv, int dh,
                              int causal, const PagedPlanShape& s, void* plan, int* err, cudaStream_t st);
cudaError_t launch_paged_tokens(const PagedAttnArgs& a, const PagedPlanShape& s, int grid_items, cudaStream_t st);
cudaError_t launch_paged_tiles(const PagedAttnArgs& a, const PagedPlanShape& s, int grid_items, cudaStream_t st);
cudaError_t launch_paged_simt(const PagedAttnArgs& a, const PagedPlanShape& s, int grid_items, cudaStream_t st);
cudaError_t launch_paged_few(const PagedAttnArgs& a, const PagedPlanShape& s, int grid_items, cudaStream_t st);
cudaError_t launch_paged_join(const PagedAttnArgs& a, const PagedPlanShape& s, int max_joins, cudaStream_t st);
// Uncached tensor map of a bf16 tensor with the 128-byte swizzle; strides in bytes for dimensions 1..rank-1.
cudaError_t make_tma_nd_bf16(TmaDesc* out, const void* base, int rank, const uint64_t* dims, const uint64_t* strides,
                             const uint32_t* box);

}  // namespace prism
