// Moving tokens inside a 4-bit paged cache, and reading them back as bf16.  The paper has no counterpart.
#include "q4.cuh"

namespace sp {
namespace {

// The place of token p of a request: page -1 where its table row, the cache or the request has none.
struct Place {
  int page, in;                    // token in the page
};
__device__ __forceinline__ Place place_of(const int32_t* row, long long p, int max_pages, int page_log2, int n_pages) {
  const long long col = p >> page_log2;
  int id = -1;
  if (p >= 0 && col < max_pages) id = row[col];
  if (id >= n_pages) id = -1;
  return {max(id, -1), (int)(p & ((1 << page_log2) - 1))};
}

// Compaction after verification, as for a bf16 cache: kept[b][0] < kept[b][1] < ... are the accepted tokens of request b among
// its new ones; their codes and scales move from past_b + kept[b][i] to past_b + i.  In place: a thread owns the same part
// of every token of one head (16 bytes of codes, or one scale), and kept[b][i] >= i, so a destination is never a source that
// is still to be read.  All latency: the places of up to 64 moves are looked up side by side, then a thread has 16 loads in
// flight before its first store.  8 heads of 128 elements, one request that keeps 5 of 16: 2.9 us, as long as a graph node that does
// nothing; 256 requests that keep 12 of 64: 6.5 (6.7 MB read and written: 1).
constexpr int kKeepThreads = 128, kKeepRun = 16, kKeepChunk = 64;

template <int D>
__global__ void __launch_bounds__(kKeepThreads) cache_keep_q4_kernel(const __grid_constant__ KeepQ4Args a) {
  using B = Block<D>;
  constexpr int PIECES = D / 16, UNITS = PIECES + 2 * B::GROUPS;     // 16-byte pieces of K and V; scales
  __shared__ Place s_from[kKeepChunk], s_to[kKeepChunk];             // page < 0: nothing to move
  let_next_start();
  wait_for_previous();
  if (decode_poisoned(a.status)) return;
  const int b = blockIdx.x;
  const int past = a.past[b];
  const int n = min(max(a.n_kept[b], 0), a.max_kept);
  if (blockIdx.y == 0 && threadIdx.x == 0) a.lens_out[b] = past + n;
  const int x = blockIdx.y * kKeepThreads + threadIdx.x;
  const int head = x / UNITS, unit = x % UNITS;
  const bool mine = head < a.hkv, piece = unit < PIECES;
  uint8_t* base = a.c.data + head * a.c.s_head;
  auto at = [&](const Place& p) {
    const int i = p.in & 15;
    int in;
    if (unit < PIECES / 2) in = B::k_word(i, unit * 4);
    else if (piece) in = B::v_word(i, (unit - PIECES / 2) * 4);
    else if (unit < PIECES + B::GROUPS) in = B::k_scale(i, unit - PIECES);
    else in = B::v_scale(i, unit - PIECES - B::GROUPS);
    return base + p.page * a.c.s_page + (p.in >> 4) * B::BYTES + in;
  };
  const int32_t* row = a.table + (size_t)b * a.max_pages;
  for (int i0 = 0; i0 < n; i0 += kKeepChunk) {
    const int i = i0 + threadIdx.x;
    if (i0 > 0) __syncthreads();
    if (threadIdx.x < kKeepChunk && i < n) {
      const int kept = a.kept[(size_t)b * a.max_kept + i];
      Place from = place_of(row, (long long)past + kept, a.max_pages, a.page_log2, a.n_pages);
      const Place to = place_of(row, (long long)past + i, a.max_pages, a.page_log2, a.n_pages);
      if (kept < 0 || from.page < 0 || to.page < 0) {
        if (kept != i) report_range(a.status, kWhereKeepPageQ4);
        from.page = -1;
      }
      if (kept == i) from.page = -1;
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
        if (j0 + u < here && s_from[j0 + u].page >= 0) {
          const uint8_t* src = at(s_from[j0 + u]);
          if (piece) val[u] = *reinterpret_cast<const uint4*>(src);
          else val[u].x = *src;
        }
      }
#pragma unroll
      for (int u = 0; u < kKeepRun; ++u)
        if (j0 + u < here && s_from[j0 + u].page >= 0) {
          uint8_t* dst = at(s_to[j0 + u]);
          if (piece) *reinterpret_cast<uint4*>(dst) = val[u];
          else *dst = (uint8_t)val[u].x;
        }
    }
  }
}

// Cached tokens as bf16 rows.  Bound by what is written (4 D bytes a token and head; 17 D / 16 are read).  A warp takes 16
// rows of the output, looks up their places (a lane a row), and walks its heads: D / 8 lanes a row, each a word of K and of
// V, so that a row is written in one run of 16-byte stores.  Eight documents of 3000 to 131000 tokens, 4 heads of 128 elements:
// 137 us, 90 % of the copy rate; 5001 tokens of 8 heads 6.7 us.
constexpr int kReadThreads = 256;

template <int D>
__global__ void __launch_bounds__(kReadThreads) cache_read_q4_kernel(const __grid_constant__ ReadQ4Args a) {
  using B = Block<D>;
  constexpr int WORDS = D / 8, PER = 32 / WORDS, STEPS = 16 / PER;   // words of a row, rows at a time, times
  const int lane = threadIdx.x & 31, word = lane % WORDS, sub = lane / WORDS;
  const int splits = (a.hkv + a.heads_per_warp - 1) / a.heads_per_warp;
  const long long unit = (long long)blockIdx.x * (kReadThreads / 32) + (threadIdx.x >> 5);
  const long long row0 = unit / splits * 16;
  const int head0 = (int)(unit % splits) * a.heads_per_warp, head1 = min(head0 + a.heads_per_warp, a.hkv);
  let_next_start();
  wait_for_previous();
  if (decode_poisoned(a.status) || row0 >= a.rows) return;
  // lane i (and i + 16): the place of row i
  const long long t = row0 + (lane & 15);
  int lo = 0, hi = a.n_req;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.row_start[mid] <= t) lo = mid; else hi = mid - 1;
  }
  long long offset = -1;                           // of the token's block, head 0; < 0: nothing to read
  int in = 0;
  if (lo < a.n_req && t < a.rows && a.row_start[lo] <= t) {          // else behind the last request: left as it was
    const int first = a.row_start[lo], n = a.row_start[lo + 1] - first;
    const Place p = place_of(a.table + (size_t)lo * a.max_pages, (long long)a.seq_lens[lo] - n + (t - first), a.max_pages, a.page_log2, a.n_pages);
    if (p.page < 0) report_range(a.status, kWhereReadPageQ4);
    else offset = p.page * a.c.s_page + (p.in >> 4) * B::BYTES;
    in = p.in & 15;
  }
  for (int h = head0; h < head1; ++h) {
    const uint8_t* base = a.c.data + h * a.c.s_head;
#pragma unroll 2
    for (int j0 = 0; j0 < STEPS; j0 += 4) {
      uint32_t kw[4], vw[4], ks[4], vs[4];
      bool live[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int r = (j0 + u) * PER + sub;
        const long long off = __shfl_sync(0xffffffffu, offset, r);
        const int i = __shfl_sync(0xffffffffu, in, r);
        live[u] = off >= 0;
        kw[u] = vw[u] = ks[u] = vs[u] = 0;
        if (live[u]) {
          const uint8_t* blk = base + off;
          kw[u] = *reinterpret_cast<const uint32_t*>(blk + B::k_word(i, word));
          vw[u] = *reinterpret_cast<const uint32_t*>(blk + B::v_word(i, word));
          ks[u] = blk[B::k_scale(i, word >> 2)];
          vs[u] = blk[B::v_scale(i, word >> 2)];
        }
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (!live[u]) continue;
        const long long r = row0 + (j0 + u) * PER + sub;
        auto put = [&](__nv_bfloat16* dst, uint32_t w, uint32_t byte) {
          // two codes at a time: 128 + c as bf16, then (128 + c) s - 136 s, which is (c - 8) s exactly
          const uint32_t sb = (byte << 4 | byte << 20) + 0x35803580u;
          const __nv_bfloat162 s = *reinterpret_cast<const __nv_bfloat162*>(&sb);
          const __nv_bfloat162 off = __hmul2(s, __floats2bfloat162_rn(-136.f, -136.f));
          uint32_t y[4];
#pragma unroll
          for (int p = 0; p < 4; ++p) {
            const uint32_t c = (w >> (4 * p) & 0x000f000fu) | 0x43004300u;
            const __nv_bfloat162 z = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&c), s, off);
            y[p] = *reinterpret_cast<const uint32_t*>(&z);
          }
          *reinterpret_cast<uint4*>(dst + word * 8) = make_uint4(y[0], y[1], y[2], y[3]);
        };
        put(a.k + h * a.k_sh + r * a.k_sn, kw[u], ks[u]);
        put(a.v + h * a.v_sh + r * a.v_sn, vw[u], vs[u]);
      }
    }
  }
}

template <int D>
cudaError_t launch_keep(const KeepQ4Args& a, cudaStream_t s) {
  const int units = a.hkv * (D / 16 + 2 * Block<D>::GROUPS);
  return launch_dependent(cache_keep_q4_kernel<D>, dim3(a.n_req, (units + kKeepThreads - 1) / kKeepThreads), dim3(kKeepThreads), 0, s, a);
}
template <int D>
cudaError_t launch_read(ReadQ4Args& a, cudaStream_t s) {
  // a warp takes all heads of its rows (which look up their places once) unless there are too few warps then
  const long long chunks = ((long long)a.rows + 15) / 16;
  const long long want = (148ll * 16 + chunks - 1) / chunks;         // warps per chunk that fill the device
  const int splits = (int)(want < a.hkv ? want : a.hkv);
  a.heads_per_warp = (a.hkv + splits - 1) / splits;
  const long long warps = chunks * ((a.hkv + a.heads_per_warp - 1) / a.heads_per_warp);
  return launch_dependent(cache_read_q4_kernel<D>, dim3((unsigned)((warps + kReadThreads / 32 - 1) / (kReadThreads / 32))), dim3(kReadThreads), 0, s, a);
}

}  // namespace

cudaError_t launch_cache_keep_q4(const KeepQ4Args& a, cudaStream_t s) { return a.d == 128 ? launch_keep<128>(a, s) : launch_keep<64>(a, s); }
cudaError_t launch_cache_read_q4(ReadQ4Args& a, cudaStream_t s) { return a.d == 128 ? launch_read<128>(a, s) : launch_read<64>(a, s); }

}  // namespace sp
