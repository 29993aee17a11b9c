// Host side of the decode-side calls: argument validation and launches.
#include <math.h>
#include <string.h>

#include <algorithm>

#include "ctx.cuh"
#include "q4.cuh"

namespace {

using namespace sp;

// A bf16 view whose size-1 dimensions may carry any stride (they are never stepped).
int check_view(const sp_tensor* t) {
  if (!t || !t->data) return SP_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(t->data) & 15) != 0) return SP_ERR_INVALID_ARG;
  for (int x = 0; x < 4; ++x)
    if (t->shape[x] <= 0 || t->shape[x] > INT32_MAX) return SP_ERR_INVALID_ARG;
  if (t->shape[3] > 1 && t->stride[3] != 1) return SP_ERR_INVALID_ARG;
  for (int x = 0; x < 3; ++x)
    if (t->shape[x] > 1 && (t->stride[x] < t->shape[3] || t->stride[x] % 8 != 0)) return SP_ERR_INVALID_ARG;
  return SP_OK;
}
bool same_shape(const sp_tensor* a, const sp_tensor* b) { return memcmp(a->shape, b->shape, sizeof(a->shape)) == 0; }
int64_t step(const sp_tensor* t, int x) { return t->shape[x] > 1 ? t->stride[x] : 0; }

int log2_of_page(int64_t page) {          // -1: not a supported page size
  for (int l = 4; l <= 8; ++l)
    if (page == (int64_t)1 << l) return l;
  return -1;
}

struct CacheShape {
  int pages, hkv, d, page_log2;
};
int check_cache(const sp_tensor* k, const sp_tensor* v, CacheShape* c) {
  int rc;
  if ((rc = check_view(k)) || (rc = check_view(v))) return rc;
  if (!same_shape(k, v)) return SP_ERR_INVALID_ARG;
  c->page_log2 = log2_of_page(k->shape[2]);
  if (c->page_log2 < 0 || (k->shape[3] != 64 && k->shape[3] != 128) || k->shape[1] > kMaxHeads) return SP_ERR_UNSUPPORTED;
  if (k->shape[0] > (INT32_MAX >> c->page_log2)) return SP_ERR_UNSUPPORTED;    // slots are 32-bit
  c->pages = (int)k->shape[0]; c->hkv = (int)k->shape[1]; c->d = (int)k->shape[3];
  return SP_OK;
}
PagedCache cache_of(const sp_tensor* t) {
  return PagedCache{static_cast<__nv_bfloat16*>(t->data), step(t, 0), step(t, 1), step(t, 2)};
}

// An int32 array of a call; `out`: the call writes it (in and out included).
struct Array {
  const void* p;
  int64_t n;
  bool out;
};
// Whether something written shares memory with another array of the call.  The blocks of a launch run in any order, so an
// output in place of an input would be read by some of them.
template <int N>
bool overlapping(const Array (&x)[N]) {
  for (int i = 0; i < N; ++i)
    for (int j = 0; j < i; ++j) {
      if ((!x[i].out && !x[j].out) || x[i].n == 0 || x[j].n == 0) continue;
      const uintptr_t a = reinterpret_cast<uintptr_t>(x[i].p), b = reinterpret_cast<uintptr_t>(x[j].p);
      if (a && b && a < b + 4 * (uintptr_t)x[j].n && b < a + 4 * (uintptr_t)x[i].n) return true;
    }
  return false;
}

// inv_freq / (2 pi) modulo one turn, in units of 2^-64, rounded down; 0 <= inv_freq < 2^30.  The double's 53 bits times 192 bits
// of 1 / (2 pi): the whole turns that drop out take none of the fraction's bits with them.
uint64_t turns_per_position(double inv_freq) {
  static const uint64_t kInvTwoPi[3] = {0x36d8a5664f10e410ull, 0x7f09d5f47d4d3770ull, 0x28be60db9391054aull};   // 2^-192 .. 2^-1
  int e;
  const double m = frexp(inv_freq, &e);
  const uint64_t bits = (uint64_t)ldexp(m, 53);          // inv_freq = bits * 2^(e - 53)
  uint64_t p[4] = {0, 0, 0, 0};                          // bits / (2 pi) * 2^192
  for (int i = 0; i < 3; ++i) {
    const unsigned __int128 x = (unsigned __int128)bits * kInvTwoPi[i] + p[i];
    p[i] = (uint64_t)x;
    p[i + 1] = (uint64_t)(x >> 64);
  }
  const int down = 128 + 53 - e, word = down / 64, off = down % 64;       // e <= 30: word >= 2
  if (word > 3) return 0;
  return p[word] >> off | (word < 3 && off > 0 ? p[word + 1] << (64 - off) : 0);
}

// What sp_qk_norm_rope and its form for a 4-bit cache have in common: everything but the cache.  `elsewhere`: k and v have a
// destination besides k_out, v_out.
int rope_args(const sp_ctx* ctx, const sp_tensor* q, const sp_tensor* k, const sp_tensor* v, const void* q_weight, const void* k_weight, float eps,
              const double* inv_freq, int n_freq, int interleaved, const int32_t* positions, const sp_tensor* q_out, const sp_tensor* k_out,
              const sp_tensor* v_out, bool elsewhere, RopeArgs* out) {
  if (!ctx || !positions || n_freq < 0 || (n_freq > 0 && !inv_freq)) return SP_ERR_INVALID_ARG;
  int rc;
  if ((rc = check_view(q)) || (rc = check_view(k)) || (rc = check_view(v)) || (rc = check_view(q_out))) return rc;
  if (!same_shape(q, q_out) || !same_shape(k, v)) return SP_ERR_INVALID_ARG;
  if (q->shape[0] != 1 || k->shape[0] != 1) return SP_ERR_UNSUPPORTED;
  if (q->shape[2] != k->shape[2] || q->shape[3] != k->shape[3]) return SP_ERR_INVALID_ARG;
  const int64_t d = q->shape[3];
  if ((d != 64 && d != 128) || q->shape[1] > kMaxHeads || k->shape[1] > kMaxHeads) return SP_ERR_UNSUPPORTED;
  if (2 * (int64_t)n_freq > d || n_freq % 8 != 0) return SP_ERR_UNSUPPORTED;
  if ((q_weight != nullptr) != (k_weight != nullptr)) return SP_ERR_INVALID_ARG;
  if (((reinterpret_cast<uintptr_t>(q_weight) | reinterpret_cast<uintptr_t>(k_weight)) & 15) != 0) return SP_ERR_INVALID_ARG;
  if (q_weight && !(eps >= 0.f && eps < INFINITY)) return SP_ERR_INVALID_ARG;
  if ((k_out != nullptr) != (v_out != nullptr)) return SP_ERR_INVALID_ARG;
  if (!k_out && !elsewhere) return SP_ERR_INVALID_ARG;
  if (k_out) {
    if ((rc = check_view(k_out)) || (rc = check_view(v_out))) return rc;
    if (!same_shape(k, k_out) || !same_shape(v, v_out)) return SP_ERR_INVALID_ARG;
  }
  RopeArgs& a = *out;
  memset(&a, 0, sizeof(a));
  for (int i = 0; i < n_freq; ++i) {
    if (!(inv_freq[i] >= 0.0 && inv_freq[i] < 1e9)) return SP_ERR_INVALID_ARG;
    a.phase[i] = turns_per_position(inv_freq[i]);
  }
  a.q = static_cast<const __nv_bfloat16*>(q->data);
  a.k = static_cast<const __nv_bfloat16*>(k->data);
  a.v = static_cast<const __nv_bfloat16*>(v->data);
  a.q_out = static_cast<__nv_bfloat16*>(q_out->data);
  a.q_sh = step(q, 1); a.q_sn = step(q, 2); a.k_sh = step(k, 1); a.k_sn = step(k, 2); a.v_sh = step(v, 1); a.v_sn = step(v, 2);
  a.qo_sh = step(q_out, 1); a.qo_sn = step(q_out, 2);
  if (k_out) {
    a.k_out = static_cast<__nv_bfloat16*>(k_out->data);
    a.v_out = static_cast<__nv_bfloat16*>(v_out->data);
    a.ko_sh = step(k_out, 1); a.ko_sn = step(k_out, 2); a.vo_sh = step(v_out, 1); a.vo_sn = step(v_out, 2);
  }
  a.q_weight = static_cast<const __nv_bfloat16*>(q_weight);
  a.k_weight = static_cast<const __nv_bfloat16*>(k_weight);
  a.positions = positions;
  a.hq = (int)q->shape[1]; a.hkv = (int)k->shape[1]; a.tokens = (int)q->shape[2]; a.d = (int)d;
  a.rot = 2 * n_freq; a.interleaved = interleaved != 0; a.eps = eps; a.status = ctx->status;
  return SP_OK;
}

// The 4-bit cache of a call.
struct Q4Shape {
  int pages, hkv, d, page_log2;
};
int check_q4(const sp_q4_cache* c, Q4Shape* s) {
  if (!c || !c->data || (reinterpret_cast<uintptr_t>(c->data) & 15) != 0) return SP_ERR_INVALID_ARG;
  for (const int64_t n : {c->pages, c->heads, c->page, c->head_dim})
    if (n <= 0 || n > INT32_MAX) return SP_ERR_INVALID_ARG;
  s->page_log2 = log2_of_page(c->page);
  if (s->page_log2 < 0 || (c->head_dim != 64 && c->head_dim != 128) || c->heads > kMaxHeads) return SP_ERR_UNSUPPORTED;
  const int64_t bytes = c->page / 16 * (17 * c->head_dim);
  if (c->pages > 1 && (c->stride_page < bytes || c->stride_page % 16 != 0)) return SP_ERR_INVALID_ARG;
  if (c->heads > 1 && (c->stride_head < bytes || c->stride_head % 16 != 0)) return SP_ERR_INVALID_ARG;
  if (c->pages > (INT32_MAX >> s->page_log2)) return SP_ERR_UNSUPPORTED;       // slots are 32-bit
  s->pages = (int)c->pages; s->hkv = (int)c->heads; s->d = (int)c->head_dim;
  return SP_OK;
}
Q4Cache q4_of(const sp_q4_cache* c) {
  return Q4Cache{static_cast<uint8_t*>(c->data), c->pages > 1 ? c->stride_page : 0, c->heads > 1 ? c->stride_head : 0};
}

// While this lives, this thread may allocate and synchronise although another stream is being captured in a mode that forbids it (to
// this thread, or to all): such a call would fail, and end that capture.  What is done meanwhile has nothing to do with the capture.
struct BesideCaptures {
  cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;
  BesideCaptures() { cudaThreadExchangeStreamCaptureMode(&mode); }
  ~BesideCaptures() { cudaThreadExchangeStreamCaptureMode(&mode); }
};

// The workspace of sp_tree_attn and sp_tree_attn_q4, with the context's device current.
int reserve_split(sp_ctx* ctx) {
  if (ctx->split_ws) return SP_OK;
  const BesideCaptures beside;
  int n_sm = 0;
  if (cudaDeviceGetAttribute(&n_sm, cudaDevAttrMultiProcessorCount, ctx->device) != cudaSuccess) return SP_ERR_CUDA;
  void* p = nullptr;
  const size_t parts = (std::max(tree_attn_workspace_bytes(n_sm), tree_attn_q4_workspace_bytes(n_sm)) + 15) / 16 * 16;
  if (cudaMalloc(&p, parts + n_sm * sizeof(int)) != cudaSuccess) { cudaGetLastError(); return SP_ERR_WORKSPACE; }
  ctx->n_sm = n_sm;
  ctx->arrived = reinterpret_cast<int*>(static_cast<char*>(p) + parts);
  if (reset_arrived(ctx) != cudaSuccess) { cudaGetLastError(); cudaFree(p); ctx->arrived = nullptr; return SP_ERR_CUDA; }
  ctx->split_ws = p;
  return SP_OK;
}

// ... for a call on this stream: an allocation inside a stream capture would spoil the capture.
int need_split(sp_ctx* ctx, cudaStream_t s) {
  if (ctx->split_ws) return SP_OK;
  cudaStreamCaptureStatus capturing = cudaStreamCaptureStatusNone;
  if (cudaStreamIsCapturing(s, &capturing) != cudaSuccess) { cudaGetLastError(); return SP_ERR_WORKSPACE; }
  if (capturing != cudaStreamCaptureStatusNone) return SP_ERR_WORKSPACE;
  return reserve_split(ctx);
}

}  // namespace

// On a stream of its own: the default one, and synchronising the device, would spoil a capture that is under way on another stream.
cudaError_t sp::reset_arrived(sp_ctx* ctx) {
  if (!ctx->arrived) return cudaSuccess;
  const BesideCaptures beside;
  cudaStream_t s = nullptr;
  cudaError_t e = cudaStreamCreateWithFlags(&s, cudaStreamNonBlocking);
  if (e != cudaSuccess) return e;
  e = cudaMemsetAsync(ctx->arrived, 0, ctx->n_sm * sizeof(int), s);
  const cudaError_t done = cudaStreamSynchronize(s);
  cudaStreamDestroy(s);
  return e != cudaSuccess ? e : done;
}

extern "C" {

int sp_ctx_reserve_decode(sp_ctx* ctx) {
  if (!ctx) return SP_ERR_INVALID_ARG;
  DeviceGuard g(ctx->device);
  if (!g.ok) return SP_ERR_CUDA;
  return reserve_split(ctx);
}

int sp_internal_split_counters(sp_ctx* ctx, int32_t* counters, int* n, int write) {
  if (!ctx || !counters || !n || *n < 0) return SP_ERR_INVALID_ARG;
  if (!ctx->split_ws) return SP_ERR_WORKSPACE;
  DeviceGuard g(ctx->device);
  if (!g.ok) return SP_ERR_CUDA;
  const size_t bytes = std::min(*n, ctx->n_sm) * sizeof(int);
  const cudaError_t e = write ? cudaMemcpy(ctx->arrived, counters, bytes, cudaMemcpyHostToDevice) : cudaMemcpy(counters, ctx->arrived, bytes, cudaMemcpyDeviceToHost);
  *n = ctx->n_sm;
  return e == cudaSuccess ? SP_OK : SP_ERR_CUDA;
}

int sp_page_tables(sp_ctx* ctx, const int32_t* past_lens, const int32_t* new_lens, int n_req, int page,
                   const int32_t* free_pages, int n_free, int32_t* block_table, int max_pages, const int32_t* parents,
                   int32_t* seq_lens, int32_t* row_start, int32_t* positions, int32_t* slots, uint32_t* tree_mask,
                   int mask_words, int n_rows, int32_t* info, void* stream) {
  if (!ctx || n_req < 0 || n_free < 0 || n_rows < 0) return SP_ERR_INVALID_ARG;
  const int pl = log2_of_page(page);
  if (pl < 0 || n_req > kMaxRequests || max_pages > (INT32_MAX >> pl)) return SP_ERR_UNSUPPORTED;
  if (n_req == 0) return SP_OK;            // before the arrays are looked at: without elements they may have no address
  if (!past_lens || !new_lens || !block_table || !seq_lens || !row_start || !info || max_pages <= 0) return SP_ERR_INVALID_ARG;
  if ((n_free > 0 && !free_pages) || (n_rows > 0 && (!positions || !slots))) return SP_ERR_INVALID_ARG;
  if ((parents != nullptr) != (tree_mask != nullptr)) return SP_ERR_INVALID_ARG;
  if (tree_mask && (mask_words < 1 || mask_words > kMaxMaskWords)) return SP_ERR_UNSUPPORTED;
  DeviceGuard g(ctx->device);
  if (!g.ok) return SP_ERR_CUDA;
  const Array arrays[] = {{past_lens, n_req, false}, {new_lens, n_req, false}, {free_pages, n_free, false},
                          {parents, n_rows, false}, {block_table, (int64_t)n_req * max_pages, true},
                          {seq_lens, n_req, true}, {row_start, (int64_t)n_req + 1, true}, {positions, n_rows, true},
                          {slots, n_rows, true}, {tree_mask, (int64_t)n_rows * mask_words, true}, {info, 4, true}};
  if (overlapping(arrays)) return SP_ERR_INVALID_ARG;
  PageTablesArgs a{past_lens, new_lens, free_pages, parents, block_table, seq_lens, row_start, positions, slots,
                   tree_mask, info, n_req, n_free, max_pages, pl, n_rows, tree_mask ? mask_words : 0, ctx->status};
  if (launch_page_tables(a, static_cast<cudaStream_t>(stream)) != cudaSuccess) return SP_ERR_CUDA;
  ctx->launches += 1;
  return SP_OK;
}

int sp_qk_norm_rope(sp_ctx* ctx, const sp_tensor* q, const sp_tensor* k, const sp_tensor* v, const void* q_weight,
                    const void* k_weight, float eps, const double* inv_freq, int n_freq, int interleaved,
                    const int32_t* positions, const sp_tensor* q_out, const sp_tensor* k_out, const sp_tensor* v_out,
                    const sp_tensor* k_cache, const sp_tensor* v_cache, const int32_t* slots, void* stream) {
  RopeArgs a;
  int rc = rope_args(ctx, q, k, v, q_weight, k_weight, eps, inv_freq, n_freq, interleaved, positions, q_out, k_out, v_out, k_cache != nullptr, &a);
  if (rc) return rc;
  if ((k_cache != nullptr) != (v_cache != nullptr)) return SP_ERR_INVALID_ARG;
  if (k_cache) {
    CacheShape c;
    if (!slots) return SP_ERR_INVALID_ARG;
    if ((rc = check_cache(k_cache, v_cache, &c))) return rc;
    if (c.hkv != a.hkv || c.d != a.d) return SP_ERR_INVALID_ARG;
    a.kc = cache_of(k_cache);
    a.vc = cache_of(v_cache);
    a.page_log2 = c.page_log2;
    a.n_slots = c.pages << c.page_log2;
    a.slots = slots;
  }
  DeviceGuard g(ctx->device);
  if (!g.ok) return SP_ERR_CUDA;
  if (launch_qk_norm_rope(a, static_cast<cudaStream_t>(stream)) != cudaSuccess) return SP_ERR_CUDA;
  ctx->launches += 1;
  return SP_OK;
}

int sp_tree_attn(sp_ctx* ctx, const sp_tensor* q, const sp_tensor* k_cache, const sp_tensor* v_cache,
                 const int32_t* block_table, int max_pages, const int32_t* seq_lens, const int32_t* row_start, int n_req,
                 const uint32_t* tree_mask, int mask_words, const sp_tensor* out, float* lse_out, void* stream) {
  if (!ctx || n_req < 0) return SP_ERR_INVALID_ARG;
  if (n_req == 0 && q && q->shape[2] == 0) return SP_OK;      // nobody, no rows: tensors without elements
  int rc;
  CacheShape c;
  if ((rc = check_view(q)) || (rc = check_view(out))) return rc;
  if ((rc = check_cache(k_cache, v_cache, &c))) return rc;
  if (!same_shape(q, out) || q->shape[3] != c.d) return SP_ERR_INVALID_ARG;
  if (q->shape[0] != 1 || q->shape[1] > kMaxHeads || q->shape[1] % c.hkv != 0) return SP_ERR_UNSUPPORTED;
  if (q->shape[2] * (q->shape[1] / c.hkv) > INT32_MAX) return SP_ERR_UNSUPPORTED;
  if (n_req > kMaxRequests || max_pages > (INT32_MAX >> c.page_log2)) return SP_ERR_UNSUPPORTED;
  if (tree_mask && (mask_words < 1 || mask_words > kMaxMaskWords)) return SP_ERR_UNSUPPORTED;
  CacheSteps steps;
  if (!cache_steps(cache_of(k_cache), c.hkv, c.pages, &steps) || !cache_steps(cache_of(v_cache), c.hkv, c.pages, &steps)) return SP_ERR_UNSUPPORTED;
  if (n_req == 0) return SP_OK;            // as in sp_page_tables
  if (!block_table || !seq_lens || !row_start || max_pages <= 0) return SP_ERR_INVALID_ARG;
  DeviceGuard g(ctx->device);
  if (!g.ok) return SP_ERR_CUDA;
  if (q->data == out->data) return SP_ERR_INVALID_ARG;         // in place: a run may be walked twice
  TreeAttnArgs a;
  memset(&a, 0, sizeof(a));
  a.q = static_cast<const __nv_bfloat16*>(q->data);
  a.o = static_cast<__nv_bfloat16*>(out->data);
  a.lse = lse_out;
  a.q_sh = step(q, 1); a.q_sn = step(q, 2); a.o_sh = step(out, 1); a.o_sn = step(out, 2);
  a.kc = cache_of(k_cache);
  a.vc = cache_of(v_cache);
  a.table = block_table; a.seq_lens = seq_lens; a.row_start = row_start;
  a.bits = tree_mask; a.words = tree_mask ? mask_words : 0;
  a.hq = (int)q->shape[1]; a.hkv = c.hkv; a.group = a.hq / a.hkv; a.d = c.d; a.rows = (int)q->shape[2];
  a.n_req = n_req; a.max_pages = max_pages; a.page_log2 = c.page_log2; a.n_pages = c.pages;
  a.scale_log2 = (float)(1.4426950408889634 / sqrt((double)c.d));
  a.status = ctx->status;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (ctx->kernel == 1) {
    if (launch_tree_attn_simt(a, s) != cudaSuccess) return SP_ERR_CUDA;
    ctx->launches += 1;
    return SP_OK;
  }
  if ((rc = need_split(ctx, s))) return rc;
  if (launch_tree_attn(a, ctx->split_ws, ctx->n_sm, s) != cudaSuccess) return SP_ERR_CUDA;
  ctx->launches += 2;
  return SP_OK;
}

int sp_cache_keep(sp_ctx* ctx, const sp_tensor* k_cache, const sp_tensor* v_cache, const int32_t* block_table, int max_pages,
                  const int32_t* past_lens, int n_req, const int32_t* kept, const int32_t* n_kept, int max_kept,
                  int32_t* lens_out, void* stream) {
  if (!ctx || n_req < 0) return SP_ERR_INVALID_ARG;
  int rc;
  CacheShape c;
  if ((rc = check_cache(k_cache, v_cache, &c))) return rc;
  if (n_req > kMaxRequests || max_pages > (INT32_MAX >> c.page_log2)) return SP_ERR_UNSUPPORTED;
  if (n_req == 0) return SP_OK;            // as in sp_page_tables
  if (!block_table || !past_lens || !n_kept || !lens_out || max_pages <= 0) return SP_ERR_INVALID_ARG;
  if (kept ? max_kept <= 0 : max_kept != 0) return SP_ERR_INVALID_ARG;     // no column: a list without elements
  DeviceGuard g(ctx->device);
  if (!g.ok) return SP_ERR_CUDA;
  const Array arrays[] = {{block_table, (int64_t)n_req * max_pages, false}, {past_lens, n_req, false},
                          {kept, (int64_t)n_req * max_kept, false}, {n_kept, n_req, false}, {lens_out, n_req, true}};
  if (overlapping(arrays)) return SP_ERR_INVALID_ARG;
  KeepArgs a{cache_of(k_cache), cache_of(v_cache), block_table, past_lens, kept, n_kept, lens_out, n_req, max_pages, max_kept,
             c.hkv, c.d, c.page_log2, c.pages, ctx->status};
  if (launch_cache_keep(a, static_cast<cudaStream_t>(stream)) != cudaSuccess) return SP_ERR_CUDA;
  ctx->launches += 1;
  return SP_OK;
}

// ---------------------------------------------------------------- the cache held in 4 bits

int sp_q4_page_bytes(int page, int head_dim, int64_t* bytes) {
  if (!bytes) return SP_ERR_INVALID_ARG;
  if (log2_of_page(page) < 0 || (head_dim != 64 && head_dim != 128)) return SP_ERR_UNSUPPORTED;
  *bytes = (int64_t)page / 16 * (17 * head_dim);
  return SP_OK;
}

int sp_qk_norm_rope_q4(sp_ctx* ctx, const sp_tensor* q, const sp_tensor* k, const sp_tensor* v, const void* q_weight,
                       const void* k_weight, float eps, const double* inv_freq, int n_freq, int interleaved,
                       const int32_t* positions, const sp_tensor* q_out, const sp_tensor* k_out, const sp_tensor* v_out,
                       const sp_q4_cache* cache, const int32_t* slots, void* stream) {
  RopeArgs a;
  Q4Shape c;
  int rc = rope_args(ctx, q, k, v, q_weight, k_weight, eps, inv_freq, n_freq, interleaved, positions, q_out, k_out, v_out, true, &a);
  if (rc) return rc;
  if (!slots) return SP_ERR_INVALID_ARG;
  if ((rc = check_q4(cache, &c))) return rc;
  if (c.hkv != a.hkv || c.d != a.d) return SP_ERR_INVALID_ARG;
  const Q4Cache to = q4_of(cache);
  a.q4 = to.data; a.q4_s_page = to.s_page; a.q4_s_head = to.s_head;
  a.page_log2 = c.page_log2;
  a.n_slots = c.pages << c.page_log2;
  a.slots = slots;
  DeviceGuard g(ctx->device);
  if (!g.ok) return SP_ERR_CUDA;
  if (launch_qk_norm_rope_q4(a, static_cast<cudaStream_t>(stream)) != cudaSuccess) return SP_ERR_CUDA;
  ctx->launches += 1;
  return SP_OK;
}

int sp_tree_attn_q4(sp_ctx* ctx, const sp_tensor* q, const sp_q4_cache* cache, const int32_t* block_table, int max_pages,
                    const int32_t* seq_lens, const int32_t* row_start, int n_req, const uint32_t* tree_mask, int mask_words,
                    const sp_tensor* out, float* lse_out, void* stream) {
  if (!ctx || n_req < 0) return SP_ERR_INVALID_ARG;
  if (n_req == 0 && q && q->shape[2] == 0) return SP_OK;      // nobody, no rows: tensors without elements
  int rc;
  Q4Shape c;
  if ((rc = check_view(q)) || (rc = check_view(out))) return rc;
  if ((rc = check_q4(cache, &c))) return rc;
  if (!same_shape(q, out) || q->shape[3] != c.d) return SP_ERR_INVALID_ARG;
  if (q->shape[0] != 1 || q->shape[1] > kMaxHeads || q->shape[1] % c.hkv != 0) return SP_ERR_UNSUPPORTED;
  if (q->shape[2] * (q->shape[1] / c.hkv) > INT32_MAX) return SP_ERR_UNSUPPORTED;
  if (n_req > kMaxRequests || max_pages > (INT32_MAX >> c.page_log2)) return SP_ERR_UNSUPPORTED;
  if (tree_mask && (mask_words < 1 || mask_words > kMaxMaskWords)) return SP_ERR_UNSUPPORTED;
  if (n_req == 0) return SP_OK;            // as in sp_page_tables
  if (!block_table || !seq_lens || !row_start || max_pages <= 0) return SP_ERR_INVALID_ARG;
  if (q->data == out->data) return SP_ERR_INVALID_ARG;
  DeviceGuard g(ctx->device);
  if (!g.ok) return SP_ERR_CUDA;
  TreeAttnArgs a;
  memset(&a, 0, sizeof(a));
  a.q = static_cast<const __nv_bfloat16*>(q->data);
  a.o = static_cast<__nv_bfloat16*>(out->data);
  a.lse = lse_out;
  a.q_sh = step(q, 1); a.q_sn = step(q, 2); a.o_sh = step(out, 1); a.o_sn = step(out, 2);
  a.table = block_table; a.seq_lens = seq_lens; a.row_start = row_start;
  a.bits = tree_mask; a.words = tree_mask ? mask_words : 0;
  a.hq = (int)q->shape[1]; a.hkv = c.hkv; a.group = a.hq / a.hkv; a.d = c.d; a.rows = (int)q->shape[2];
  a.n_req = n_req; a.max_pages = max_pages; a.page_log2 = c.page_log2; a.n_pages = c.pages;
  a.scale_log2 = (float)(1.4426950408889634 / sqrt((double)c.d));
  a.status = ctx->status;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (ctx->kernel == 1) {
    if (launch_tree_attn_q4_simt(a, q4_of(cache), s) != cudaSuccess) return SP_ERR_CUDA;
    ctx->launches += 1;
    return SP_OK;
  }
  if ((rc = need_split(ctx, s))) return rc;
  int launched = 0;
  if (launch_tree_attn_q4(a, q4_of(cache), ctx->split_ws, ctx->arrived, ctx->n_sm, s, &launched) != cudaSuccess) return SP_ERR_CUDA;
  ctx->launches += launched;
  return SP_OK;
}

int sp_cache_keep_q4(sp_ctx* ctx, const sp_q4_cache* cache, const int32_t* block_table, int max_pages, const int32_t* past_lens, int n_req,
                     const int32_t* kept, const int32_t* n_kept, int max_kept, int32_t* lens_out, void* stream) {
  if (!ctx || n_req < 0) return SP_ERR_INVALID_ARG;
  int rc;
  Q4Shape c;
  if ((rc = check_q4(cache, &c))) return rc;
  if (n_req > kMaxRequests || max_pages > (INT32_MAX >> c.page_log2)) return SP_ERR_UNSUPPORTED;
  if (n_req == 0) return SP_OK;            // as in sp_page_tables
  if (!block_table || !past_lens || !n_kept || !lens_out || max_pages <= 0) return SP_ERR_INVALID_ARG;
  if (kept ? max_kept <= 0 : max_kept != 0) return SP_ERR_INVALID_ARG;     // no column: a list without elements
  const Array arrays[] = {{block_table, (int64_t)n_req * max_pages, false}, {past_lens, n_req, false},
                          {kept, (int64_t)n_req * max_kept, false}, {n_kept, n_req, false}, {lens_out, n_req, true}};
  if (overlapping(arrays)) return SP_ERR_INVALID_ARG;
  DeviceGuard g(ctx->device);
  if (!g.ok) return SP_ERR_CUDA;
  const KeepQ4Args a{q4_of(cache), block_table, past_lens, kept, n_kept, lens_out, n_req, max_pages, max_kept,
                     c.hkv, c.d, c.page_log2, c.pages, ctx->status};
  if (launch_cache_keep_q4(a, static_cast<cudaStream_t>(stream)) != cudaSuccess) return SP_ERR_CUDA;
  ctx->launches += 1;
  return SP_OK;
}

int sp_cache_read_q4(sp_ctx* ctx, const sp_q4_cache* cache, const int32_t* block_table, int max_pages, const int32_t* seq_lens,
                     const int32_t* row_start, int n_req, const sp_tensor* k_out, const sp_tensor* v_out, void* stream) {
  if (!ctx || n_req < 0) return SP_ERR_INVALID_ARG;
  if (n_req == 0 && k_out && k_out->shape[2] == 0) return SP_OK;
  int rc;
  Q4Shape c;
  if ((rc = check_view(k_out)) || (rc = check_view(v_out))) return rc;
  if ((rc = check_q4(cache, &c))) return rc;
  if (!same_shape(k_out, v_out) || k_out->shape[1] != c.hkv || k_out->shape[3] != c.d || k_out->data == v_out->data) return SP_ERR_INVALID_ARG;
  if (k_out->shape[0] != 1) return SP_ERR_UNSUPPORTED;
  if (n_req > kMaxRequests || max_pages > (INT32_MAX >> c.page_log2)) return SP_ERR_UNSUPPORTED;
  if (n_req == 0) return SP_OK;            // as in sp_page_tables
  if (!block_table || !seq_lens || !row_start || max_pages <= 0) return SP_ERR_INVALID_ARG;
  DeviceGuard g(ctx->device);
  if (!g.ok) return SP_ERR_CUDA;
  ReadQ4Args a;
  memset(&a, 0, sizeof(a));
  a.c = q4_of(cache);
  a.table = block_table; a.seq_lens = seq_lens; a.row_start = row_start;
  a.k = static_cast<__nv_bfloat16*>(k_out->data);
  a.v = static_cast<__nv_bfloat16*>(v_out->data);
  a.k_sh = step(k_out, 1); a.k_sn = step(k_out, 2); a.v_sh = step(v_out, 1); a.v_sn = step(v_out, 2);
  a.n_req = n_req; a.max_pages = max_pages; a.rows = (int)k_out->shape[2]; a.hkv = c.hkv; a.d = c.d;
  a.page_log2 = c.page_log2; a.n_pages = c.pages; a.status = ctx->status;
  if (launch_cache_read_q4(a, static_cast<cudaStream_t>(stream)) != cudaSuccess) return SP_ERR_CUDA;
  ctx->launches += 1;
  return SP_OK;
}

}  // extern "C"
