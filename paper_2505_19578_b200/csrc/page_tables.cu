// Page tables, slot maps and tree visibility from request lengths (one launch), and the compaction of accepted tokens
// in the cache.  The paper has no counterpart: it decodes densely over a contiguous cache.
//
// page_tables_kernel.  With page size P, request b holds h_b = ceil(past_b / P) pages and needs
// n_b = ceil((past_b + new_b) / P) - h_b more; it takes free_pages[N_b ..], N_b = sum of n over the requests before it.
// Row t of the packed batch belongs to the request with row_start[b] <= t < row_start[b + 1] (row_start = prefix sum of
// new); its place in the sequence is p = past_b + (t - row_start[b]), its slot table[b][p / P] * P + p % P.
// Every CTA repeats the two prefix sums over the requests (a few kB from L2, one block-wide scan) instead of waiting for
// one that does it: the slots of newly taken pages follow from the sums and the free list, so no CTA reads what another
// writes, and one launch is enough.  The work is a few hundred kB at most; latency bounds it.
#include <limits.h>

#include "decode.cuh"

namespace sp {
namespace {

constexpr int kTableThreads = 256;

struct Sums {
  long long rows, pages;
};
__device__ __forceinline__ Sums operator+(Sums a, Sums b) { return {a.rows + b.rows, a.pages + b.pages}; }

// last index b in [0, n] with start[b] <= x, start ascending from 0
__device__ __forceinline__ int last_not_above(const int32_t* start, int n, int x) {
  int lo = 0, hi = n;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (start[mid] <= x) lo = mid; else hi = mid - 1;
  }
  return lo;
}

__global__ void __launch_bounds__(kTableThreads) page_tables_kernel(const __grid_constant__ PageTablesArgs a) {
  extern __shared__ int32_t sm[];
  int32_t* row0 = sm;                       // [n_req + 1] first row of each request, then the end
  int32_t* take0 = sm + a.n_req + 1;        // [n_req + 1] first position in the free list, then the end
  __shared__ Sums warp_sum[kTableThreads / 32];
  __shared__ int s_failed, s_longest;
  let_next_start();
  wait_for_previous();
  if (decode_poisoned(a.status)) return;

  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int page = 1 << a.page_log2;
  const long long room = (long long)a.max_pages << a.page_log2;        // tokens a table row can hold
  if (tid == 0) { s_failed = 0; s_longest = 0; }
  __syncthreads();

  auto lens = [&](int b, int* past, int* fresh) {
    *past = max(a.past[b], 0);
    *fresh = max(a.fresh[b], 0);
  };
  auto pages = [&](long long tokens) { return (int)((min(tokens, room) + page - 1) >> a.page_log2); };

  // prefix sums: each thread a run of requests, then across the block
  const int per = (a.n_req + kTableThreads - 1) / kTableThreads;
  const int b0 = min(tid * per, a.n_req), b1 = min(b0 + per, a.n_req);
  Sums mine{0, 0};
  int failed = 0, longest = 0;
  for (int b = b0; b < b1; ++b) {
    int p, f;
    lens(b, &p, &f);
    mine.rows += f;
    mine.pages += pages((long long)p + f) - pages(p);
    const long long total = (long long)p + f;
    longest = (int)max((long long)longest, min(total, (long long)INT_MAX));
    failed += a.past[b] < 0 || a.fresh[b] < 0 || total > room || (a.bits && f > 32 * a.words);
  }
  Sums incl = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const Sums up{__shfl_up_sync(0xffffffffu, incl.rows, o), __shfl_up_sync(0xffffffffu, incl.pages, o)};
    if (lane >= o) incl = incl + up;
  }
  if (lane == 31) warp_sum[warp] = incl;
  __syncthreads();
  Sums before{incl.rows - mine.rows, incl.pages - mine.pages};
  for (int w = 0; w < warp; ++w) before = before + warp_sum[w];
  for (int b = b0; b < b1; ++b) {
    int p, f;
    lens(b, &p, &f);
    row0[b] = (int)min(before.rows, (long long)INT_MAX);
    take0[b] = (int)min(before.pages, (long long)INT_MAX);
    const int need = pages((long long)p + f) - pages(p);
    before.rows += f;
    before.pages += need;
    failed += need > 0 && before.pages > a.n_free && !(a.past[b] < 0 || a.fresh[b] < 0 || (long long)p + f > room || (a.bits && f > 32 * a.words));
    if (blockIdx.x == 0) a.seq_lens[b] = (int)min((long long)p + f, (long long)INT_MAX);
    if (b == a.n_req - 1) {
      row0[a.n_req] = (int)min(before.rows, (long long)INT_MAX);
      take0[a.n_req] = (int)min(before.pages, (long long)INT_MAX);
    }
  }
  if (blockIdx.x == 0) {
    if (failed) atomicAdd(&s_failed, failed);          // whole numbers: the order does not matter
    atomicMax(&s_longest, longest);
  }
  __syncthreads();
  const int n_rows = row0[a.n_req], n_take = take0[a.n_req];
  if (blockIdx.x == 0) {
    for (int b = tid; b <= a.n_req; b += kTableThreads) a.row_start[b] = row0[b];
    if (tid == 0) {
      a.info[0] = n_rows;
      a.info[1] = min(n_take, a.n_free);
      a.info[2] = s_failed;
      a.info[3] = s_longest;
    }
  }

  const long long step = (long long)gridDim.x * kTableThreads, at = (long long)blockIdx.x * kTableThreads + tid;
  // newly taken pages into the tables
  for (long long i = at; i < n_take; i += step) {
    const int b = last_not_above(take0, a.n_req - 1, (int)i);
    const int col = pages(max(a.past[b], 0)) + (int)i - take0[b];
    a.table[(size_t)b * a.max_pages + col] = i < a.n_free ? a.free_pages[i] : -1;
  }
  // slots, positions and visibility of the rows
  const int words = a.bits ? a.words : 1;
  for (long long i = at; i < (long long)min(n_rows, a.rows) * words; i += step) {
    const int t = (int)(i / words), w = (int)(i - (long long)t * words);
    const int b = last_not_above(row0, a.n_req - 1, t);
    const int j = t - row0[b];
    const int past = max(a.past[b], 0);
    int depth = j;
    if (a.parents) {
      // up the tree: a parent is an earlier token of the request; anything else hangs off the last cached token
      uint32_t seen = 0;
      depth = -1;
      for (int x = j; x >= 0;) {
        if ((x >> 5) == w) seen |= 1u << (x & 31);
        ++depth;
        const int up = a.parents[t - j + x];
        x = up < x ? up : -1;
      }
      a.bits[i] = seen;
    }
    if (w == 0) {
      const long long p = (long long)past + j;
      const int held = pages(past);
      const long long c = p >> a.page_log2;
      long long id = -1;
      if (c < held) id = a.table[(size_t)b * a.max_pages + c];
      else if (c < a.max_pages) {
        const long long take = take0[b] + (c - held);
        if (take < a.n_free) id = a.free_pages[take];
      }
      const long long slot = (id << a.page_log2) + (p & (page - 1));
      a.slots[t] = id < 0 || slot > INT_MAX ? -1 : (int)slot;
      a.positions[t] = (int)min((long long)past + depth, (long long)INT_MAX);
    }
  }
}

// cache_keep_kernel: kept[b][0] < kept[b][1] < ... are the accepted tokens of request b among its new ones; the key and
// value at past_b + kept[b][i] move to past_b + i.  In place: a thread owns 16 bytes of every token of one head, and
// kept[b][i] >= i, so a destination is never a source that is still to be read.  All latency: the places of up to 64 moves
// are looked up by as many threads at once, then a thread has 16 loads in flight before its first store (a run of them
// may overlap its own destinations, hence loads first).
constexpr int kKeepThreads = 128, kKeepRun = 16, kKeepChunk = 64;

__global__ void __launch_bounds__(kKeepThreads) cache_keep_kernel(const __grid_constant__ KeepArgs a) {
  __shared__ int2 s_from[kKeepChunk], s_to[kKeepChunk];      // page, token in the page; page < 0: nothing to move
  let_next_start();
  wait_for_previous();
  if (decode_poisoned(a.status)) return;
  const int b = blockIdx.x;
  const int past = a.past[b];
  const int n = min(max(a.n_kept[b], 0), a.max_kept);
  if (blockIdx.y == 0 && threadIdx.x == 0) a.lens_out[b] = past + n;
  const int pieces = a.d / 8;
  const int x = blockIdx.y * kKeepThreads + threadIdx.x;
  const bool mine = x < 2 * a.hkv * pieces;
  const int piece = x % pieces, head = (x / pieces) % a.hkv;
  const PagedCache& c = x < a.hkv * pieces ? a.kc : a.vc;
  __nv_bfloat16* base = c.data + head * c.s_head + piece * 8;
  const int32_t* row = a.table + (size_t)b * a.max_pages;
  auto place = [&](long long p) -> int2 {            // page -1: not a place of this request's pages
    const long long col = p >> a.page_log2;
    int id = -1;
    if (p >= 0 && col < a.max_pages) id = row[col];
    if (id >= a.n_pages) id = -1;
    return make_int2(max(id, -1), (int)(p & ((1 << a.page_log2) - 1)));
  };
  for (int i0 = 0; i0 < n; i0 += kKeepChunk) {
    const int i = i0 + threadIdx.x;
    if (i0 > 0) __syncthreads();
    if (threadIdx.x < kKeepChunk && i < n) {
      const int kept = a.kept[(size_t)b * a.max_kept + i];
      int2 from = place((long long)past + kept), to = place((long long)past + i);
      if (kept < 0 || from.x < 0 || to.x < 0) {
        if (kept != i) report_range(a.status, kWhereKeepPage);
        from.x = -1;
      }
      if (kept == i) from.x = -1;
      s_from[threadIdx.x] = from;
      s_to[threadIdx.x] = to;
    }
    __syncthreads();
    if (!mine) continue;
    const int here = min(kKeepChunk, n - i0);
    for (int j0 = 0; j0 < here; j0 += kKeepRun) {
      uint4 val[kKeepRun];
#pragma unroll
      for (int u = 0; u < kKeepRun; ++u) {
        val[u] = make_uint4(0, 0, 0, 0);
        if (j0 + u < here) {
          const int2 from = s_from[j0 + u];
          if (from.x >= 0) val[u] = *reinterpret_cast<const uint4*>(base + from.x * c.s_page + from.y * c.s_tok);
        }
      }
#pragma unroll
      for (int u = 0; u < kKeepRun; ++u)
        if (j0 + u < here && s_from[j0 + u].x >= 0) {
          const int2 to = s_to[j0 + u];
          *reinterpret_cast<uint4*>(base + to.x * c.s_page + to.y * c.s_tok) = val[u];
        }
    }
  }
}

}  // namespace

cudaError_t launch_page_tables(const PageTablesArgs& a, cudaStream_t s) {
  const long long items = (long long)a.rows * (a.bits ? a.words : 1);
  const long long want = (items > a.n_free ? items : a.n_free) / kTableThreads;
  const int grid = (int)(want < 1 ? 1 : want > 148 ? 148 : want);
  const int smem = 2 * (a.n_req + 1) * (int)sizeof(int32_t);
  return launch_dependent(page_tables_kernel, dim3(grid), dim3(kTableThreads), smem, s, a);
}

cudaError_t launch_cache_keep(const KeepArgs& a, cudaStream_t s) {
  const int columns = 2 * a.hkv * a.d / 8;
  return launch_dependent(cache_keep_kernel, dim3(a.n_req, (columns + kKeepThreads - 1) / kKeepThreads), dim3(kKeepThreads), 0, s, a);
}

}  // namespace sp
