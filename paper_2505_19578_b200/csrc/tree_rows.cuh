// What the attention kernels over a paged cache share: the rows and keys of a request, which keys a row sees, and the join
// of units whose keys were cut over several CTAs.  Internal to the library.
#pragma once

#include "decode.cuh"
#include "tc_ptx.cuh"

namespace sp {
namespace {

using namespace tc;

constexpr float kNoMax = -1e30f;                 // reference maximum before any visible key: finite, below any logit

struct Meta {       // what the join kernel needs of a unit that begins in this CTA and goes on in later ones
  int last;         // CTA that has the unit's last tile; < 0: there is no such unit
  int start, r0, rows, g, pad[3];
};

struct Parts {
  float* part;      // [cta][2][ROWS][D] unnormalised sums: part 0 of a unit begun by an earlier CTA, part 1 of one begun here
  float2* ml;       // [cta][2][ROWS] reference, weight
  Meta* meta;       // [cta]
};

struct Request {
  int start, n, len, past, kt;                     // first row, rows (tokens), keys, keys that every row sees, tiles of keys
};
template <int TILE>
__device__ __forceinline__ Request request_of(const TreeAttnArgs& a, int b) {
  Request q;
  const int s0 = a.row_start[b], s1 = a.row_start[b + 1], seq = a.seq_lens[b];
  q.start = min(max(s0, 0), a.rows);
  q.n = s0 < 0 ? 0 : max(min(s1, a.rows) - q.start, 0);
  q.len = min(max(seq, 0), a.max_pages << a.page_log2);
  q.past = seq - (s1 - s0);
  q.kt = max((int)(((uint32_t)q.len + (TILE - 1)) / TILE), 1);     // (lengths go up to 2^31 - 16)
  return q;
}
__device__ __forceinline__ long long divide(long long x, long long y) {       // both are small as a rule
  return ((x | y) >> 32) == 0 ? (long long)((uint32_t)x / (uint32_t)y) : x / y;
}

__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Which of the 32 keys from k0 on a row sees: bit i = key k0 + i.
// u: len, past and start of its request.
template <typename U>
__device__ __forceinline__ uint32_t seen32(const TreeAttnArgs& a, const U& u, int token, int k0) {
  const int left = u.len - k0;                                       // keys of the sequence from here on
  uint32_t live = left >= 32 ? 0xffffffffu : left <= 0 ? 0u : (1u << left) - 1u;
  const int x0 = k0 - u.past;                                        // index of key k0 among the new tokens
  if (x0 + 31 < 0) return live;
  if (!a.bits) {
    const int upto = token - x0;                                     // keys 0 .. upto of these are seen
    return live & (upto >= 31 ? 0xffffffffu : upto < 0 ? 0u : (2u << upto) - 1u);
  }
  const uint32_t* row = a.bits + (size_t)(u.start + token) * a.words;
  const int w0 = x0 >> 5;                                            // floor: keys before the new tokens are words of ones
  auto word = [&](int w) { return w < 0 ? 0xffffffffu : w < a.words ? row[w] : 0u; };
  return live & __funnelshift_r(word(w0), word(w0 + 1), (uint32_t)x0 & 31u);
}

// Joins the parts of the cut units, in the order of the keys: the part of the CTA in which a unit begins, then those of
// the CTAs after it.  A warp reads a row's part at once (its 32 lanes the columns).  The work is a few MB from L2 at most
// and all latency, so it is spread as widely as it goes: every block lists the cut units (one per CTA of the first kernel
// at most) and takes every gridDim.x-th run of rows; as long as the device has warps to spare, 2, 4 or 8 of them share
// the parts of a row.
constexpr int kJoinWarps = 8, kJoinBlocksPerSm = 4;

template <int D, int ROWS>
__global__ void __launch_bounds__(kJoinWarps * 32, kJoinBlocksPerSm) tree_attn_join_kernel(const __grid_constant__ TreeAttnArgs a, const Parts work, int n_cta) {
  constexpr int E = D / 32;
  __shared__ float s_m[kJoinWarps], s_l[kJoinWarps], s_o[kJoinWarps][D];
  __shared__ int s_sum[kJoinWarps], s_owner, s_first;
  let_next_start();
  wait_for_previous();
  if (decode_poisoned(a.status)) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // rows of the unit that begins in CTA i and goes on in later ones; thread t looks after CTAs per * t ...
  const int per = (n_cta + kJoinWarps * 32 - 1) / (kJoinWarps * 32);
  auto rows_of = [&](int i) { return i < n_cta && work.meta[i].last >= 0 ? work.meta[i].rows : 0; };
  auto block_scan = [&](int mine, int* total) {      // sum over the threads before this one
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int up = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += up;
    }
    __syncthreads();
    if (lane == 31) s_sum[warp] = incl;
    __syncthreads();
    int before = incl - mine;
    *total = 0;
    for (int w = 0; w < kJoinWarps; ++w) {
      if (w < warp) before += s_sum[w];
      *total += s_sum[w];
    }
    return before;
  };
  int mine = 0, rows = 0;
  for (int i = threadIdx.x * per; i < (threadIdx.x + 1) * per; ++i) mine += rows_of(i);
  block_scan(mine, &rows);
  if (rows == 0) return;
  const int spare = (int)gridDim.x * kJoinWarps / rows;
  const int share = spare >= 8 ? 8 : spare >= 4 ? 4 : spare >= 2 ? 2 : 1, here = kJoinWarps / share;   // warps of a row, rows of a block
  mine = 0;
  for (int i = threadIdx.x * per; i < (threadIdx.x + 1) * per; ++i) mine += (rows_of(i) + here - 1) / here;
  int runs;
  const int before = block_scan(mine, &runs);
  for (int run = blockIdx.x; run < runs; run += gridDim.x) {
    __syncthreads();
    if (before <= run && run < before + mine) {
      int at = before;
      for (int i = threadIdx.x * per;; ++i) {
        const int n = (rows_of(i) + here - 1) / here;
        if (run < at + n) { s_owner = i; s_first = (run - at) * here; break; }
        at += n;
      }
    }
    __syncthreads();
    const int owner = s_owner, r = s_first + warp / share, turn = warp % share;
    const Meta m = work.meta[owner];
    const int parts = m.last - owner + 1;
    float mx = kNoMax, l = 0.f, o[E];
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = 0.f;
    if (r < m.rows) {
      constexpr int RUN = 4;                         // parts in flight
      for (int p0 = turn; p0 < parts; p0 += RUN * share) {
        float2 ml[RUN];
        float y[RUN][E];
#pragma unroll
        for (int i = 0; i < RUN; ++i) {
          const int p = p0 + i * share;
          ml[i] = make_float2(kNoMax, 0.f);
          if (p < parts) {
            const size_t slot = ((size_t)(owner + p) * 2 + (p == 0 ? 1 : 0)) * ROWS + r;
            ml[i] = work.ml[slot];
            if (E == 4) *reinterpret_cast<float4*>(y[i]) = *reinterpret_cast<const float4*>(work.part + slot * D + lane * 4);
            else *reinterpret_cast<float2*>(y[i]) = *reinterpret_cast<const float2*>(work.part + slot * D + lane * 2);
          }
        }
#pragma unroll
        for (int i = 0; i < RUN; ++i) {
          if (ml[i].y == 0.f) continue;              // no part, or nothing visible in it
          const float top = fmaxf(mx, ml[i].x), f_old = exp2f(mx - top), f = exp2f(ml[i].x - top);
          l = l * f_old + ml[i].y * f;
#pragma unroll
          for (int e = 0; e < E; ++e) o[e] = o[e] * f_old + y[i][e] * f;
          mx = top;
        }
      }
    }
    if (share > 1) {
      if (lane == 0) { s_m[warp] = mx; s_l[warp] = l; }
#pragma unroll
      for (int e = 0; e < E; ++e) s_o[warp][lane * E + e] = o[e];
      __syncthreads();
    }
    if (turn == 0 && r < m.rows) {
      for (int w = warp + 1; w < warp + share; ++w) {
        if (s_l[w] == 0.f) continue;
        const float top = fmaxf(mx, s_m[w]), f_old = exp2f(mx - top), f = exp2f(s_m[w] - top);
        l = l * f_old + s_l[w] * f;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = o[e] * f_old + s_o[w][lane * E + e] * f;
        mx = top;
      }
      const int abs_row = m.r0 + r, token = abs_row / a.group, head = m.g * a.group + abs_row % a.group;
      const float inv = l != 0.f ? 1.f / l : 0.f;
      __nv_bfloat16* dst = a.o + head * a.o_sh + (m.start + token) * a.o_sn + lane * E;
      uint32_t w[E / 2];
#pragma unroll
      for (int e = 0; e < E; e += 2) w[e / 2] = pack_bf16(o[e] * inv, o[e + 1] * inv);
      if (E == 4) *reinterpret_cast<uint2*>(dst) = make_uint2(w[0], w[E / 2 - 1]);
      else *reinterpret_cast<uint32_t*>(dst) = w[0];
      if (a.lse && lane == 0)
        a.lse[(size_t)head * a.rows + m.start + token] = l != 0.f ? (mx + log2f(l)) * 0.6931471805599453f : -CUDART_INF_F;
    }
  }
}

}  // namespace
}  // namespace sp
