// Attention of a few new tokens per request over a paged cache held in 4 bits (q4.cuh has the format), split along the keys.
//
//   out_r = sum_c p_rc v_c / sum_c p_rc,  p_rc = 2^(scale q_r.k_c - m_r) over the visible keys c.
//
// The rows of a unit are the new tokens of one request times the query heads that share a KV head (row = token * group +
// head), 8 NT at most.  Work is counted in steps, one for each block of 16 keys of a unit and kOwnSteps for the unit itself;
// the steps of all units stand in one line, which is cut into one equal run per WARP.  A warp is on its own: it copies its
// blocks into a ring of its own in shared memory (one bulk copy of 17 D bytes each, several ahead), turns codes into bf16
// fragments in registers and multiplies them by mma.sync m16n8k16.  Nothing is exchanged between warps until the runs are
// done; then the warps of a CTA add up what they have of the same unit, and a second kernel joins what CTAs have.
//
// Keys are the rows of A:  S^T = K Q^T (16 keys x 8 rows), O^T += V^T P^T (D x 8 rows), so that 8 rows fill an instruction;
// with the rows as A's, 16 would, and a single token of a group of 4 leave three quarters empty.  S^T's fragment becomes
// P^T's by one 8x8 transpose a half (movmatrix).  The order of the contraction's index is free as long as both operands have
// it: lane 4 g + q takes elements q D / 4 .. (q + 1) D / 4 - 1 of its keys, which are neighbours in the cache (and in q).
//
// Codes to bf16, two at a time: 0x4300 | c is 128 + c; times s, minus 136 s: (c - 8) s, exactly, one rounding that rounds
// nothing.  A shift, a mask-or and an FMA for two elements; V, whose pairs are of two tokens, one byte-permute more for 16.
//
// What bounds it: the cache's bytes, 2176 a block of 128-element heads: 94 cycles of an SM's share of the measured HBM rate,
// in which its schedulers issue 376 instructions.
#include <limits.h>

#include "q4.cuh"
#include "tree_rows.cuh"

namespace sp {
namespace {

constexpr int kKeys = 16;                        // keys of a block
constexpr int kOwnSteps = 4;                     // steps of a unit besides those of its blocks
constexpr int kLeastSteps = 8;                   // of a run, while there are warps to spare

template <int D, int NT>
struct Plan {
  static constexpr int ROWS = 8 * NT;
  static constexpr int WARPS = NT == 1 ? 16 : NT == 2 ? 12 : 8;
  static constexpr bool MERGE = NT <= 2;         // the CTA's warps add up their parts of a unit in shared memory
  static constexpr int BYTES = Block<D>::BYTES;
  static constexpr int RING = (NT == 4 ? 7 : 4) * (D == 128 ? 1 : 2);
  static constexpr int WORDS = D / 32;           // words of codes that a lane takes of a key
  static constexpr int STRIDE = D + 4;           // of a part's rows, floats
  static constexpr int RING_OFF = 0, RING_BYTES = WARPS * RING * BYTES;
  static constexpr int PART_OFF = RING_OFF + RING_BYTES, PART_BYTES = MERGE ? ROWS * STRIDE * 4 : 0;      // a warp's part of a unit that an earlier run began
  static constexpr int Q_OFF = PART_OFF + WARPS * PART_BYTES, Q_BYTES = MERGE ? 0 : NT * WORDS * 512;     // a warp's queries, in fragments
  static constexpr int ML_OFF = Q_OFF + WARPS * Q_BYTES;                                                  // float2 [WARPS][2][ROWS]
  static constexpr int INFO_OFF = ML_OFF + (MERGE ? WARPS * 2 * ROWS * 8 : 0);                            // PartInfo [WARPS][2]
  static constexpr int BAR_OFF = INFO_OFF + WARPS * 2 * 32;
  static constexpr int SCAN_OFF = BAR_OFF + WARPS * RING * 8;                                             // int64 [2][WARPS], int64 [WARPS], int [WARPS]
  static constexpr int FLAG_OFF = SCAN_OFF + WARPS * (3 * 8 + 4);
  static constexpr int TOTAL = FLAG_OFF + 16;
  static_assert(!MERGE || RING * BYTES >= ROWS * STRIDE * 4, "a drained ring holds a part");
  static_assert(TOTAL <= 232448 && BYTES % 16 == 0 && RING_BYTES % 16 == 0, "");
};

struct PartInfo {  // of a warp's part 0 (of a unit that an earlier run began) or 1 (of one that goes on in a later run)
  int rows;        // 0: there is none
  int ends;        // the unit's last block is in it
  int start, r0, g, pad[3];
};
static_assert(sizeof(PartInfo) == 32, "");

// Blocks of a unit that a run has.
struct Piece {
  int start, r0, rows, g, b, len, past;
  int kt0, n, kt_all;
};
// A place in a run.
struct Walk {
  long long rem, left;             // steps of request b before it, steps of the run behind it
  int b;
  Request q;
};
template <int ROWS>
__device__ __forceinline__ int passes(const TreeAttnArgs& a, const Request& q) { return (int)(((uint32_t)(q.n * a.group) + ROWS - 1) / ROWS); }
template <int ROWS>
__device__ __forceinline__ long long units_of(const TreeAttnArgs& a, const Request& q) { return (long long)a.hkv * passes<ROWS>(a, q); }

template <int ROWS>
__device__ __forceinline__ bool next_piece(const TreeAttnArgs& a, Walk& w, Piece& u) {
  while (w.left > 0) {
    while (w.rem >= units_of<ROWS>(a, w.q) * (w.q.kt + kOwnSteps) && w.b + 1 < a.n_req) { w.rem = 0; w.q = request_of<kKeys>(a, ++w.b); }
    if (w.rem >= units_of<ROWS>(a, w.q) * (w.q.kt + kOwnSteps)) return false;      // not reached while the lengths stand still
    const int all = w.q.kt + kOwnSteps, n_pass = passes<ROWS>(a, w.q);
    const int nth = (int)divide(w.rem, all), in = (int)(w.rem - (long long)nth * all);
    const int take = (int)min((long long)(all - in), w.left);
    w.left -= take;
    w.rem += take;
    u.kt0 = max(in - kOwnSteps, 0);
    u.n = max(in + take - kOwnSteps, 0) - u.kt0;
    if (u.n == 0) continue;                        // only of the unit's own steps: its blocks are the next run's
    u.kt_all = w.q.kt;
    u.g = n_pass == 1 ? nth : nth / n_pass;
    u.b = w.b;
    u.start = w.q.start;
    u.r0 = (nth - u.g * n_pass) * ROWS;
    u.rows = min(w.q.n * a.group - u.r0, ROWS);
    u.len = w.q.len;
    u.past = w.q.past;
    return true;
  }
  return false;
}

__device__ __forceinline__ void bulk_copy(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t permute(uint32_t a, uint32_t b, uint32_t sel) { return __byte_perm(a, b, sel); }
struct Scale2 {                    // two scales as bf16, and -136 times them
  __nv_bfloat162 s, off;
};
__device__ __forceinline__ Scale2 scale2(uint32_t bytes) {         // in bits 0 .. 7 and 16 .. 23
  const uint32_t w = (bytes << 4) + 0x35803580u;
  Scale2 r;
  r.s = *reinterpret_cast<const __nv_bfloat162*>(&w);
  r.off = __hmul2(r.s, __floats2bfloat162_rn(-136.f, -136.f));     // 17 * 8 times four significant bits: exact
  return r;
}
__device__ __forceinline__ uint32_t values(uint32_t codes, int p, const Scale2& s) {     // codes in bits 4 p .. and 16 + 4 p ..
  const uint32_t w = (codes >> (4 * p) & 0x000f000fu) | 0x43004300u;
  const __nv_bfloat162 y = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&w), s.s, s.off);
  return *reinterpret_cast<const uint32_t*>(&y);
}

template <int D, int NT>
__global__ void __launch_bounds__(Plan<D, NT>::WARPS * 32, 1) tree_attn_q4_kernel(const __grid_constant__ TreeAttnArgs a, const Q4Cache cache, const Parts work) {
  using P = Plan<D, NT>;
  using B = Block<D>;
  constexpr int WARPS = P::WARPS, ROWS = P::ROWS, THREADS = WARPS * 32, WORDS = P::WORDS;
  extern __shared__ __align__(128) uint8_t smem[];
  const uint32_t base = smem_u32(smem);
  float2* part_ml = reinterpret_cast<float2*>(smem + P::ML_OFF);
  PartInfo* infos = reinterpret_cast<PartInfo*>(smem + P::INFO_OFF);
  long long* scan = reinterpret_cast<long long*>(smem + P::SCAN_OFF);
  long long* start_rem = scan + 2 * WARPS;
  int* start_b = reinterpret_cast<int*>(start_rem + WARPS);
  volatile int* abort_flag = reinterpret_cast<int*>(smem + P::FLAG_OFF);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  const int cta = blockIdx.x;
  const Abort ab{abort_flag, a.status};
  auto bar = [&](int slot) { return base + P::BAR_OFF + (warp * P::RING + slot) * 8; };

  let_next_start();
  if (lane < P::RING) mbar_init(bar(lane), 1);
  if (lane < 2) infos[warp * 2 + lane].rows = 0;
  if (threadIdx.x == 0) *abort_flag = 0;
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  wait_for_previous();
  const bool idle = decode_poisoned(a.status);

  // ---- where the warps' runs begin
  const int per = (a.n_req + THREADS - 1) / THREADS;
  const int b_lo = min((int)threadIdx.x * per, a.n_req), b_hi = min(b_lo + per, a.n_req);
  long long mine = 0;
  for (int b = b_lo; b < b_hi; ++b) {
    const Request r = request_of<kKeys>(a, b);
    mine += units_of<ROWS>(a, r) * (r.kt + kOwnSteps);
  }
  long long incl = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long up = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += up;
  }
  if (lane == 31) scan[warp] = incl;
  __syncthreads();
  long long before = incl - mine, total = 0;
#pragma unroll
  for (int w = 0; w < WARPS; ++w) {
    if (w < warp) before += scan[w];
    total += scan[w];
  }
  // as many warps of each CTA as have kLeastSteps to do (a part costs its join)
  const long long want = divide(total, (long long)gridDim.x * kLeastSteps);
  const int warps = (int)max(1ll, min((long long)WARPS, want)), n_runs = gridDim.x * warps;
  const long long quota = divide(total, n_runs), extra = total - quota * n_runs;      // the first `extra` runs are one step longer
  auto run_begin = [&](int r) { return r * quota + min((long long)r, extra); };
  for (int i = 0; i < warps; ++i) {
    const long long w = run_begin(cta * warps + i);
    if (before <= w && w < before + mine) {
      long long step = before;
      for (int b = b_lo; b < b_hi; ++b) {
        const Request r = request_of<kKeys>(a, b);
        const long long n = units_of<ROWS>(a, r) * (r.kt + kOwnSteps);
        if (w < step + n) { start_b[i] = b; start_rem[i] = w - step; break; }
        step += n;
      }
    }
  }
  // units that go on in later CTAs (in later runs, where the warps' parts are joined one by one): none yet
  const int run = cta * warps + warp;
  if (P::MERGE) {
    if (threadIdx.x == 0) work.meta[cta].last = -1;
  } else {
    if (lane == 0 && warp < warps) work.meta[run].last = -1;
    for (int i = n_runs + cta * THREADS + threadIdx.x; i < (int)gridDim.x * WARPS; i += gridDim.x * THREADS) work.meta[i].last = -1;
  }
  __syncthreads();

  const long long w0 = run_begin(run), steps = warp < warps && !idle ? run_begin(run + 1) - w0 : 0;
  bool ok = true;
  if (steps > 0) {
    const uint32_t ring = base + P::RING_OFF + warp * (P::RING * P::BYTES);
    const uint8_t* ring_at = smem + P::RING_OFF + warp * (P::RING * P::BYTES);
    Walk walk{start_rem[warp], steps, start_b[warp], {}};
    walk.q = request_of<kKeys>(a, walk.b);

    // ---- fetching: a walk of its own, RING blocks ahead.  A lane holds the page of one of 32 blocks, and of the 32 after them.
    Walk ahead = walk;
    const int32_t* f_row = nullptr;
    const uint8_t* f_base = nullptr;
    int f_kt = 0, f_end = 0, f_len = 0, f_win = 0, id_now = -1, id_next = -1, f_slot = 0, pending = 0;
    bool f_more = true;
    auto lookup = [&](int kt) {                    // of block kt + lane
      const long long key = (long long)(kt + lane) * kKeys;
      return kt + lane < f_end && key < f_len ? f_row[key >> a.page_log2] : -1;
    };
    auto fetch = [&] {                             // whole warp; the next block into slot f_slot, if there is one
      if (f_kt == f_end) {
        Piece u;
        f_more = f_more && next_piece<ROWS>(a, ahead, u);
        if (!f_more) return;
        f_row = a.table + (size_t)u.b * a.max_pages;
        f_base = cache.data + u.g * cache.s_head;
        f_kt = f_win = u.kt0; f_end = u.kt0 + u.n; f_len = u.len;
        id_now = lookup(f_win);
        id_next = lookup(f_win + 32);
      } else if (f_kt - f_win == 32) {
        f_win = f_kt;
        id_now = id_next;
        id_next = lookup(f_win + 32);
      }
      const int id = __shfl_sync(0xffffffffu, id_now, f_kt - f_win), key = f_kt * kKeys;
      if (lane == 0) {
        if (key < f_len && id >= 0 && id < a.n_pages) {
          mbar_expect_tx(bar(f_slot), P::BYTES);
          bulk_copy(ring + f_slot * P::BYTES, f_base + id * cache.s_page + ((key & ((1 << a.page_log2) - 1)) >> 4) * P::BYTES, P::BYTES, bar(f_slot));
        } else {
          // no such page, or no key at all: whatever lies in the slot is finite
          if (key < f_len) report_range(a.status, kWhereTreePageQ4);
          mbar_arrive(bar(f_slot));
        }
      }
      ++f_kt;
      ++pending;
      if (++f_slot == P::RING) f_slot = 0;
    };
#pragma unroll 1
    for (int i = 0; i < P::RING; ++i) fetch();

    Piece u;
    int slot = 0;
    uint32_t phase = 0;
    while (ok && next_piece<ROWS>(a, walk, u)) {
      if (lane == 0 && u.kt0 == 0 && a.seq_lens[u.b] > u.len) report_range(a.status, kWhereTreePageQ4);   // longer than its table row
      // ---- queries: of row nt * 8 + g elements q D / 4 ..
      uint4 qf[P::MERGE ? NT : 1][WORDS];
      uint8_t* q_at = smem + P::Q_OFF + warp * P::Q_BYTES + lane * 16;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const int row = nt * 8 + g, abs_row = u.r0 + row;
        const __nv_bfloat16* src = a.q + (int64_t)(u.g * a.group + abs_row % a.group) * a.q_sh + (int64_t)(u.start + abs_row / a.group) * a.q_sn + q * (D / 4);
#pragma unroll
        for (int w = 0; w < WORDS; ++w) {
          uint4 x = make_uint4(0, 0, 0, 0);
          if (row < u.rows) x = *reinterpret_cast<const uint4*>(src + w * 8);
          if (P::MERGE) qf[P::MERGE ? nt : 0][w] = x;
          else *reinterpret_cast<uint4*>(q_at + (nt * WORDS + w) * 512) = x;
        }
      }
      float o[NT][D / 16][4], m[NT][2], l[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int t = 0; t < D / 16; ++t) o[nt][t][0] = o[nt][t][1] = o[nt][t][2] = o[nt][t][3] = 0.f;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          m[nt][i] = nt * 8 + 2 * q + i < u.rows ? kNoMax : -kNoMax;         // no row: all weights zero
          l[nt][i] = 0.f;
        }
      }
      const int no_mask = min(u.past, u.len), tiles = (u.rows + 7) / 8;
#pragma unroll 1
      for (int t = 0; t < u.n; ++t) {
        const int k0 = (u.kt0 + t) * kKeys;
        ok = __all_sync(0xffffffffu, mbar_wait(bar(slot), phase, ab, 100));
        if (!ok) break;
        const uint8_t* blk = ring_at + slot * P::BYTES;
        // ---- S^T = K Q^T
        uint32_t kw[2][WORDS];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint8_t* row = blk + B::k_word(g + 8 * h, q * WORDS);
          if constexpr (WORDS == 4) {
            const uint4 x = *reinterpret_cast<const uint4*>(row);
            kw[h][0] = x.x; kw[h][1] = x.y; kw[h][2] = x.z; kw[h][3] = x.w;
          } else {
            const uint2 x = *reinterpret_cast<const uint2*>(row);
            kw[h][0] = x.x; kw[h][1] = x.y;
          }
        }
        const uint32_t kb = *reinterpret_cast<const uint16_t*>(blk + B::k_scale(g, q * WORDS / 4));
        const Scale2 ks[2] = {scale2(permute(kb, 0u, 0x4040u)), scale2(permute(kb, 0u, 0x4141u))};
        float s[NT][4], s2[NT][4];                 // two sums: the products of one chain are dependent
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[nt][i] = s2[nt][i] = 0.f;
#pragma unroll
        for (int w = 0; w < WORDS; ++w) {
          const uint32_t f0[4] = {values(kw[0][w], 0, ks[0]), values(kw[1][w], 0, ks[1]), values(kw[0][w], 1, ks[0]), values(kw[1][w], 1, ks[1])};
          const uint32_t f1[4] = {values(kw[0][w], 2, ks[0]), values(kw[1][w], 2, ks[1]), values(kw[0][w], 3, ks[0]), values(kw[1][w], 3, ks[1])};
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            if (NT > 1 && nt >= tiles) break;
            const uint4 x = P::MERGE ? qf[P::MERGE ? nt : 0][w] : *reinterpret_cast<const uint4*>(q_at + (nt * WORDS + w) * 512);
            mma16816(s[nt], f0, x.x, x.y);
            mma16816(s2[nt], f1, x.z, x.w);
          }
        }
        // ---- softmax: lane has keys g, g + 8 and rows 2 q, 2 q + 1 of each tile
        const bool special = k0 + kKeys > no_mask;
        uint32_t p[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          if (NT > 1 && nt >= tiles) break;
#pragma unroll
          for (int i = 0; i < 4; ++i) s[nt][i] = (s[nt][i] + s2[nt][i]) * a.scale_log2;
          if (special) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const int row = nt * 8 + 2 * q + i;
              const uint32_t seen = row < u.rows ? seen32(a, u, (u.r0 + row) / a.group, k0) : 0u;
              if (!(seen >> g & 1)) s[nt][i] = -CUDART_INF_F;
              if (!(seen >> (g + 8) & 1)) s[nt][2 + i] = -CUDART_INF_F;
            }
          }
          const float x0 = fmaxf(s[nt][0], s[nt][2]), x1 = fmaxf(s[nt][1], s[nt][3]);
          if (__any_sync(0xffffffffu, x0 > m[nt][0] + 8.f || x1 > m[nt][1] + 8.f)) {
            // the rows' maxima over the lanes that have them; references are whole numbers, so nothing is rounded again
            float t0 = x0, t1 = x1;
#pragma unroll
            for (int e = 4; e < 32; e <<= 1) {
              t0 = fmaxf(t0, __shfl_xor_sync(0xffffffffu, t0, e));
              t1 = fmaxf(t1, __shfl_xor_sync(0xffffffffu, t1, e));
            }
            const float n0 = t0 > m[nt][0] + 8.f ? ceilf(t0) : m[nt][0], n1 = t1 > m[nt][1] + 8.f ? ceilf(t1) : m[nt][1];
            const float f0 = ex2_approx(m[nt][0] - n0), f1 = ex2_approx(m[nt][1] - n1);
            l[nt][0] *= f0;
            l[nt][1] *= f1;
            m[nt][0] = n0;
            m[nt][1] = n1;
#pragma unroll
            for (int i = 0; i < D / 16; ++i) { o[nt][i][0] *= f0; o[nt][i][1] *= f1; o[nt][i][2] *= f0; o[nt][i][3] *= f1; }
          }
          s[nt][0] = ex2_approx(s[nt][0] - m[nt][0]);
          s[nt][1] = ex2_approx(s[nt][1] - m[nt][1]);
          s[nt][2] = ex2_approx(s[nt][2] - m[nt][0]);
          s[nt][3] = ex2_approx(s[nt][3] - m[nt][1]);
          l[nt][0] += s[nt][0] + s[nt][2];
          l[nt][1] += s[nt][1] + s[nt][3];
          p[nt][0] = transpose8(cvt_bf16x2(s[nt][0], s[nt][1]));
          p[nt][1] = transpose8(cvt_bf16x2(s[nt][2], s[nt][3]));
        }
        // ---- O^T += V^T P^T: lane has tokens 2 q, 2 q + 1 and 2 q + 8, 2 q + 9, elements g D / 8 ..
        const uint32_t vb = *reinterpret_cast<const uint32_t*>(blk + B::v_scale(2 * q, g * (D / 8) / 32));
        const Scale2 v01 = scale2(vb & 0x00ff00ffu), v23 = scale2(vb >> 8 & 0x00ff00ffu);
        uint32_t vw[4][D / 64];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint8_t* row = blk + B::v_word(2 * q + (i & 1) + 8 * (i >> 1), g * (D / 64));
          if constexpr (D == 128) {
            const uint2 x = *reinterpret_cast<const uint2*>(row);
            vw[i][0] = x.x; vw[i][D / 64 - 1] = x.y;
          } else {
            vw[i][0] = *reinterpret_cast<const uint32_t*>(row);
          }
        }
#pragma unroll
        for (int w = 0; w < D / 64; ++w) {
          const uint32_t even01 = permute(vw[0][w], vw[1][w], 0x5410u), odd01 = permute(vw[0][w], vw[1][w], 0x7632u);
          const uint32_t even23 = permute(vw[2][w], vw[3][w], 0x5410u), odd23 = permute(vw[2][w], vw[3][w], 0x7632u);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t f[4] = {values(even01, e, v01), values(odd01, e, v01), values(even23, e, v23), values(odd23, e, v23)};
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              if (NT > 1 && nt >= tiles) break;
              mma16816(o[nt][w * 4 + e], f, p[nt][0], p[nt][1]);
            }
          }
        }
        __syncwarp();                              // all have read the block
        --pending;
        fetch();
        if (++slot == P::RING) { slot = 0; phase ^= 1; }
      }
      if (!ok) break;

      // ---- the unit's rows: results, or a part
      const bool whole = u.kt0 == 0 && u.n == u.kt_all;
      const int which = u.kt0 > 0 ? 0 : 1;
      float* part = P::MERGE ? reinterpret_cast<float*>(which == 0 ? smem + P::PART_OFF + warp * P::PART_BYTES : smem + P::RING_OFF + warp * (P::RING * P::BYTES)) : nullptr;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        if (NT > 1 && nt >= tiles) break;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float sum = l[nt][i];
#pragma unroll
          for (int e = 4; e < 32; e <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, e);
          const int row = nt * 8 + 2 * q + i, abs_row = u.r0 + row;
          if (row >= u.rows) continue;
          if (whole) {
            const int token = abs_row / a.group, head = u.g * a.group + abs_row % a.group;
            const float inv = sum != 0.f ? 1.f / sum : 0.f;
            uint4* dst = reinterpret_cast<uint4*>(a.o + head * a.o_sh + (int64_t)(u.start + token) * a.o_sn + g * (D / 8));
#pragma unroll
            for (int w = 0; w < D / 64; ++w)
              dst[w] = make_uint4(pack_bf16(o[nt][w * 4][i] * inv, o[nt][w * 4][2 + i] * inv), pack_bf16(o[nt][w * 4 + 1][i] * inv, o[nt][w * 4 + 1][2 + i] * inv),
                                  pack_bf16(o[nt][w * 4 + 2][i] * inv, o[nt][w * 4 + 2][2 + i] * inv), pack_bf16(o[nt][w * 4 + 3][i] * inv, o[nt][w * 4 + 3][2 + i] * inv));
            if (a.lse && g == 0)
              a.lse[(size_t)head * a.rows + u.start + token] = sum != 0.f ? (m[nt][i] + log2f(sum)) * 0.6931471805599453f : -CUDART_INF_F;
          } else {
            const size_t at = ((size_t)run * 2 + which) * ROWS + row;
            float4* dst = reinterpret_cast<float4*>((P::MERGE ? part + row * P::STRIDE : work.part + at * D) + g * (D / 8));
#pragma unroll
            for (int w = 0; w < D / 32; ++w)
              dst[w] = make_float4(o[nt][2 * w][i], o[nt][2 * w][2 + i], o[nt][2 * w + 1][i], o[nt][2 * w + 1][2 + i]);
            if (g == 0) (P::MERGE ? part_ml[(warp * 2 + which) * ROWS + row] : work.ml[at]) = make_float2(m[nt][i], sum);
          }
        }
      }
      if (!whole && lane == 0) {
        if (P::MERGE) infos[warp * 2 + which] = PartInfo{u.rows, u.kt0 + u.n == u.kt_all, u.start, u.r0, u.g, {0, 0, 0}};
        if (which == 1) {
          // the run that has the unit's last step: this one's end is the unit's step kOwnSteps + n
          const long long z = w0 + steps - 1 + (u.kt_all - u.n), cut = extra * (quota + 1);
          const int last = (int)(z < cut ? divide(z, quota + 1) : extra + divide(z - cut, quota));
          const int here = P::MERGE ? cta : run, to = P::MERGE ? last / warps : last;
          if (to > here) work.meta[here] = Meta{to, u.start, u.r0, u.rows, u.g, {0, 0, 0}};
        }
      }
      __syncwarp();
    }
    if (*abort_flag) {
      // let the copies already in flight land before the CTA gives its shared memory back
      const long long t0 = clock64();
      for (int i = slot; i < slot + pending; ++i)
        while (!mbar_try_wait(bar(i % P::RING), i < P::RING ? phase : phase ^ 1) && clock64() - t0 < kWaitCycles / 8) {}
    }
  }
  if (!P::MERGE) return;

  // ---- the CTA's parts, in the order of the keys: warp 0's part 0, its part 1 or warp 1's part 0, ...
  __syncthreads();
  if (*abort_flag || idle) return;
  int task = 0;
  for (int i = 0; i < 2 * warps; ++i) {
    if (infos[i].rows == 0 || !((i & 1) || i == 0)) continue;          // not the first of its unit here
    const PartInfo u = infos[i];
    int end = (i | 1) + 1;                                             // parts of the unit: i, then `end` - 2, .. - the part 0 of the warps after it
    bool ends = u.ends;
    while (!ends && end < 2 * warps && infos[end].rows != 0) { ends = infos[end].ends; end += 2; }
    const bool whole = (i & 1) && ends;
    for (int row = 0; row < u.rows; ++row) {
      if (task++ % WARPS != warp) continue;
      float top = kNoMax, sum = 0.f, y[WORDS];
#pragma unroll
      for (int e = 0; e < WORDS; ++e) y[e] = 0.f;
      for (int j = i; j < end; j = (j | 1) + 1) top = fmaxf(top, part_ml[j * ROWS + row].x);
      for (int j = i; j < end; j = (j | 1) + 1) {
        const float2 ml = part_ml[j * ROWS + row];
        const float f = ex2_approx(ml.x - top);
        const float* part = reinterpret_cast<const float*>((j & 1) == 0 ? smem + P::PART_OFF + (j >> 1) * P::PART_BYTES : smem + P::RING_OFF + (j >> 1) * (P::RING * P::BYTES)) +
                            row * P::STRIDE;
        sum += ml.y * f;
#pragma unroll
        for (int e = 0; e < WORDS; ++e) y[e] += part[lane * WORDS + e] * f;
      }
      const int abs_row = u.r0 + row, token = abs_row / a.group, head = u.g * a.group + abs_row % a.group;
      if (whole) {
        const float inv = sum != 0.f ? 1.f / sum : 0.f;
        uint32_t* dst = reinterpret_cast<uint32_t*>(a.o + head * a.o_sh + (int64_t)(u.start + token) * a.o_sn + lane * WORDS);
#pragma unroll
        for (int e = 0; e < WORDS; e += 2) dst[e / 2] = pack_bf16(y[e] * inv, y[e + 1] * inv);
        if (a.lse && lane == 0) a.lse[(size_t)head * a.rows + u.start + token] = sum != 0.f ? (top + log2f(sum)) * 0.6931471805599453f : -CUDART_INF_F;
      } else {
        const size_t at = ((size_t)cta * 2 + (i & 1)) * ROWS + row;
#pragma unroll
        for (int e = 0; e < WORDS; ++e) work.part[at * D + lane * WORDS + e] = y[e];
        if (lane == 0) work.ml[at] = make_float2(top, sum);
      }
    }
  }
}

template <int D, int NT>
cudaError_t launch(const TreeAttnArgs& a, const Q4Cache& c, void* ws, int n_sm, cudaStream_t s) {
  using P = Plan<D, NT>;
  const int parts = P::MERGE ? n_sm : n_sm * P::WARPS;
  Parts w;
  w.part = static_cast<float*>(ws);
  w.ml = reinterpret_cast<float2*>(w.part + (size_t)parts * 2 * P::ROWS * D);
  w.meta = reinterpret_cast<Meta*>(w.ml + (size_t)parts * 2 * P::ROWS);
  cudaError_t e = cudaFuncSetAttribute(tree_attn_q4_kernel<D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, P::TOTAL);
  if (e != cudaSuccess) return e;
  e = launch_dependent(tree_attn_q4_kernel<D, NT>, dim3(n_sm), dim3(P::WARPS * 32), P::TOTAL, s, a, c, w);
  if (e != cudaSuccess) return e;
  return launch_dependent(tree_attn_join_kernel<D, P::ROWS>, dim3(n_sm * kJoinBlocksPerSm), dim3(kJoinWarps * 32), 0, s, a, w, parts);
}

template <int D>
cudaError_t launch_rows(const TreeAttnArgs& a, const Q4Cache& c, void* ws, int n_sm, cudaStream_t s) {
  // rows of a request if all have as many; requests of more rows are several units, which is right for any lengths
  const long long rows = ((long long)a.rows + a.n_req - 1) / a.n_req * a.group;
  return rows <= 8 ? launch<D, 1>(a, c, ws, n_sm, s) : rows <= 16 ? launch<D, 2>(a, c, ws, n_sm, s) : launch<D, 4>(a, c, ws, n_sm, s);
}

template <int D, int NT>
constexpr size_t workspace_per_sm() {
  using P = Plan<D, NT>;
  return (P::MERGE ? 1 : P::WARPS) * (2 * P::ROWS * (D * sizeof(float) + sizeof(float2)) + sizeof(Meta));
}

}  // namespace

size_t tree_attn_q4_workspace_bytes(int n_sm) {
  size_t most = workspace_per_sm<128, 4>();
  for (const size_t x : {workspace_per_sm<128, 1>(), workspace_per_sm<128, 2>(), workspace_per_sm<64, 4>()}) most = x > most ? x : most;
  return most * n_sm;
}

cudaError_t launch_tree_attn_q4(const TreeAttnArgs& a, const Q4Cache& c, void* ws, int n_sm, cudaStream_t s) {
  return a.d == 128 ? launch_rows<128>(a, c, ws, n_sm, s) : launch_rows<64>(a, c, ws, n_sm, s);
}

}  // namespace sp
