// Internal declarations of the decode-side operators (page tables, head norms with rotation, attention of new tokens
// over a paged cache, cache compaction).  Nothing here is part of the C ABI.
#pragma once

#include <utility>

#include "common.cuh"

namespace sp {

constexpr int kMaxRequests = 4096;   // requests per call: their prefix sums live in one CTA's shared memory
constexpr int kMaxMaskWords = 8;     // 32-bit words of a drafted token's visibility row: up to 256 drafted tokens

// Ids of device-side range failures (SP_ERR_RANGE in the status word).
enum { kWhereTreePage = 70, kWhereRopeSlot = 75, kWhereKeepPage = 80 };

// Whether an earlier failure of the context keeps a kernel from working.  A range failure does not: it is one request's
// (a page or slot that is not the cache's), and the others of the batch have to come out the same whichever CTA met it first.
__device__ __forceinline__ bool decode_poisoned(const int* status) {
  const int code = *reinterpret_cast<const volatile int*>(status);
  return code != 0 && code != (int)SP_ERR_RANGE;
}
__device__ __forceinline__ void report_range(int* status, int where) {
  if (atomicCAS(status, 0, (int)SP_ERR_RANGE) == 0) status[1] = where;
}

// The decode-side kernels take a few microseconds, of which a launch that waits for the kernel before it to drain is one
// or more.  They are launched as programmatic dependents: a kernel may be brought onto the device while the one before it
// still runs, does what needs no memory, and waits (wait_for_previous, in every CTA) until that one has ended and its
// writes are visible.
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
template <typename... Params, typename... Args>
cudaError_t launch_dependent(void (*kernel)(Params...), dim3 grid, dim3 block, size_t smem, cudaStream_t s, Args&&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, std::forward<Args>(args)...);
}

struct PageTablesArgs {
  const int32_t* past;        // [n_req]
  const int32_t* fresh;       // [n_req] new tokens
  const int32_t* free_pages;  // [n_free]
  const int32_t* parents;     // [rows] or null
  int32_t* table;             // [n_req, max_pages]
  int32_t* seq_lens;          // [n_req]
  int32_t* row_start;         // [n_req + 1]
  int32_t* positions;         // [rows]
  int32_t* slots;             // [rows]
  uint32_t* bits;             // [rows, words] or null
  int32_t* info;              // [4]
  int n_req, n_free, max_pages, page_log2, rows, words;
  const int* status;
};

struct PagedCache {            // one cache tensor [pages, heads, page, d]; strides in elements
  __nv_bfloat16* data;
  int64_t s_page, s_head, s_tok;
};

// Heads and pages as one dimension of a tensor map, in steps of `unit` elements (their strides' greatest common divisor):
// head h of page p is its element p * page + h * head.  False: more than 2^31 - 1 of them.
struct CacheSteps {
  int page, head, extent;
  int64_t unit;
};
inline bool cache_steps(const PagedCache& c, int heads, int pages, CacheSteps* s) {
  const int64_t sp = pages > 1 ? c.s_page : 0, sh = heads > 1 ? c.s_head : 0;       // never stepped: any stride
  int64_t a = sp, b = sh;
  while (b != 0) { const int64_t r = a % b; a = b; b = r; }
  s->unit = a != 0 ? a : 64;
  const int64_t page = sp / s->unit, head = sh / s->unit;
  if (page > INT32_MAX / (pages > 1 ? pages - 1 : 1) || head > INT32_MAX / (heads > 1 ? heads - 1 : 1)) return false;
  const int64_t extent = page * (pages - 1) + head * (heads - 1) + 1;
  if (extent > INT32_MAX) return false;
  s->page = (int)page; s->head = (int)head; s->extent = (int)extent;
  return true;
}

struct RopeArgs {
  const __nv_bfloat16* q;
  const __nv_bfloat16* k;
  const __nv_bfloat16* v;
  __nv_bfloat16* q_out;
  __nv_bfloat16* k_out;        // may be null
  __nv_bfloat16* v_out;        // may be null
  int64_t q_sh, q_sn, k_sh, k_sn, v_sh, v_sn, qo_sh, qo_sn, ko_sh, ko_sn, vo_sh, vo_sn;
  PagedCache kc, vc;           // data null: no cache
  const __nv_bfloat16* q_weight;
  const __nv_bfloat16* k_weight;
  const int32_t* positions;
  const int32_t* slots;
  int hq, hkv, tokens, d, rot, interleaved, page_log2;
  int n_slots;                 // pages * page
  int splits;                  // warps per token (launcher)
  float eps;
  int* status;
  uint64_t phase[64];          // turns per position of each rotated pair, in units of 2^-64
};

struct KeepArgs {
  PagedCache kc, vc;
  const int32_t* table;
  const int32_t* past;
  const int32_t* kept;         // [n_req, max_kept]
  const int32_t* n_kept;       // [n_req]
  int32_t* lens_out;           // [n_req]
  int n_req, max_pages, max_kept, hkv, d, page_log2, n_pages;
  int* status;
};

struct TreeAttnArgs {
  const __nv_bfloat16* q;
  __nv_bfloat16* o;
  float* lse;                  // [hq, rows] or null
  int64_t q_sh, q_sn, o_sh, o_sn;
  PagedCache kc, vc;
  const int32_t* table;        // [n_req, max_pages]
  const int32_t* seq_lens;     // [n_req]
  const int32_t* row_start;    // [n_req + 1]
  const uint32_t* bits;        // [rows, words] or null
  int hq, hkv, group, d, rows, n_req, max_pages, page_log2, n_pages, words;
  float scale_log2;
  int* status;
};

cudaError_t launch_page_tables(const PageTablesArgs& a, cudaStream_t s);
cudaError_t launch_qk_norm_rope(RopeArgs& a, cudaStream_t s);
cudaError_t launch_cache_keep(const KeepArgs& a, cudaStream_t s);
size_t tree_attn_workspace_bytes(int n_sm);
cudaError_t launch_tree_attn(const TreeAttnArgs& a, void* ws, int n_sm, cudaStream_t s);
cudaError_t launch_tree_attn_simt(const TreeAttnArgs& a, cudaStream_t s);

}  // namespace sp
