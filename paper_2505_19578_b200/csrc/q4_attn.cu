// Attention of a few new tokens per request over a paged cache held in 4 bits (q4.cuh has the format), split along the keys.
//
//   out_r = sum_c p_rc v_c / sum_c p_rc,  p_rc = 2^(scale q_r.k_c - m_r) over the visible keys c.
//
// The rows of a unit are the new tokens of one request times the query heads that share a KV head (row = token * group +
// head), 8 NT at most.  Work is counted in steps, one for each 32 keys of a unit and kOwnSteps for the unit itself; the steps
// of all units stand in one line, which is cut into one equal run per WARP.  A warp is on its own: its blocks of codes come
// into a ring of its own in shared memory (a producer warp, a lane for each of the others, issues the bulk copies of 17 D
// bytes a block), it turns codes into bf16 fragments in registers and multiplies them by mma.sync m16n8k16.  Nothing is
// exchanged between warps until the runs are done; then the warps of a CTA add up what they have of the same unit, and of a
// unit that several CTAs have, the CTA that comes last adds up theirs, in the order of the keys.
//
// Keys are the rows of A:  S^T = K Q^T (16 keys x 8 rows), O^T += V^T P^T (D x 8 rows), so that 8 rows fill an instruction;
// with the rows as A's, 16 would, and a single token of a group of 4 leave three quarters empty.  S^T's fragment becomes
// P^T's by one 8x8 transpose a half (movmatrix).  The order of the contraction's index is free as long as both operands have
// it: lane 4 g + q takes elements q D / 4 .. (q + 1) D / 4 - 1 of its keys, which are neighbours in the cache (and in q).
//
// Codes to bf16, two at a time: 0x4300 | c is 128 + c; times s, minus 136 s: (c - 8) s, exactly, one rounding that rounds
// nothing.  A shift, a mask-or and an FMA for two elements; V, whose pairs are of two tokens, one byte-permute more for 16.
//
// What bounds it: the cache's bytes are 2176 a block of 128-element heads, 94 cycles of an SM's share of the measured HBM rate.
// A block takes 330 instructions of a warp, 170 of them on the integer pipe, which takes two cycles for each: 85 cycles of
// the SM's four.  Measured 170 cycles (131000 keys, 8 KV heads, a token of 4 rows each: 45 us, 6 of them before the first and
// 3 behind the last block; without turning codes into values 38).  Dequantisation is 112 of the integer instructions.  What was
// tried against it: shifts as high products (slower: 47 us), fp16 instead of bf16 values (fewer masks, twice the multiply-adds, no
// gain in a loop of nothing else), 15 warps of 128 registers (48), 7 (49).  Before that, steps of two blocks instead of one
// brought 64 -> 59, the producer and the addition by the last CTA (instead of copies by each warp and a second kernel) 53 -> 45.
#include <limits.h>

#include "q4.cuh"
#include "tree_rows.cuh"

namespace sp {
namespace {

// Steps of a unit besides those of its keys, and least steps of a run while there are warps to spare.  (With 1, 2, 4, 6: 256 chats
// 82.4, 78.4, 78.0, 79.5 us; 32 chats 24.8, 24.6, 23.2, 23.1; 2000 keys of 8 small heads 13.5, 12.3, 10.6, 10.6.  Runs of 1, 2, 4, 8 steps
// and more, with 2 of a unit's own: 8 chats 17.6, 15.9, 16.1, 22.3.)
constexpr int kOwnSteps = 4;
constexpr int kLeastSteps = 4;

template <int D, int NT>
struct Plan {
  static constexpr int ROWS = 8 * NT;
  static constexpr int WARPS = 11, THREADS = (WARPS + 1) * 32;                    // that multiply; the producer is one more (168 registers each)
  static constexpr int BLOCKS = 2, KEYS = 16 * BLOCKS;                            // of a step
  static constexpr int BLOCK = Block<D>::BYTES, BYTES = BLOCKS * BLOCK;
  static constexpr int RING = (NT == 1 ? 3 : 2) * (D == 128 ? 1 : 2);             // steps
  static constexpr int WORDS = D / 32;           // words of codes that a lane takes of a key
  static constexpr int STRIDE = D + 4;           // of a part's rows, floats
  static constexpr int RING_OFF = 0, RING_BYTES = WARPS * RING * BYTES;
  static constexpr int PART_OFF = RING_OFF + RING_BYTES, PART_BYTES = ROWS * STRIDE * 4;      // a warp's part of a unit that an earlier run began
  static constexpr int ML_OFF = PART_OFF + WARPS * PART_BYTES;                                // float2 [WARPS][2][ROWS]
  static constexpr int INFO_OFF = ML_OFF + WARPS * 2 * ROWS * 8;                              // PartInfo [WARPS][2]
  static constexpr int BAR_OFF = INFO_OFF + WARPS * 2 * 32;                                   // full, free [WARPS][RING]
  static constexpr int SCAN_OFF = BAR_OFF + 2 * WARPS * RING * 8;                             // int64 [WARPS + 1], int64 [WARPS], int [WARPS]
  static constexpr int STATE_OFF = SCAN_OFF + (2 * WARPS + 2) * 8 + (WARPS + 1) / 2 * 8;      // WarpState [WARPS]
  static constexpr int FLAG_OFF = STATE_OFF + WARPS * 80;
  static constexpr int TOTAL = FLAG_OFF + 16;
  static_assert(RING * BYTES >= ROWS * STRIDE * 4, "a drained ring holds a part");
  static_assert(TOTAL <= 232448 && BYTES % 16 == 0 && RING_BYTES % 16 == 0 && STATE_OFF % 8 == 0, "");
};

struct PartInfo {  // of a warp's part 0 (of a unit that an earlier run began) or 1 (of one that goes on in a later run)
  int rows;        // 0: there is none
  int ends;        // the unit's last block is in it
  int start, r0, g;
  int first, last; // CTAs that have the unit's first and last blocks
  int pad;
};
static_assert(sizeof(PartInfo) == 32, "");

// What CTAs have of units that several of them share.
struct CtaParts {
  float* part;     // [cta][2][ROWS][D] unnormalised sums: part 0 of a unit begun by an earlier CTA, part 1 of one begun here
  float2* ml;      // [cta][2][ROWS] reference, weight
  int* arrived;    // [cta] CTAs that are done with the unit that begins here and goes on later; zero between calls
};

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
// What a warp needs between the pieces of its run only: kept in shared memory, registers are short.
struct WarpState {
  Walk walk;
  Piece piece;
};
static_assert(sizeof(WarpState) == 80, "");
template <int ROWS>
__device__ __forceinline__ int passes(const TreeAttnArgs& a, const Request& q) { return (int)(((uint32_t)(q.n * a.group) + ROWS - 1) / ROWS); }
template <int ROWS>
__device__ __forceinline__ long long units_of(const TreeAttnArgs& a, const Request& q) { return (long long)a.hkv * passes<ROWS>(a, q); }

template <int ROWS, int KEYS>
__device__ __forceinline__ bool walk_on(const TreeAttnArgs& a, Walk& w, Piece& u) {
  while (w.left > 0) {
    while (w.rem >= units_of<ROWS>(a, w.q) * (w.q.kt + kOwnSteps) && w.b + 1 < a.n_req) { w.rem = 0; w.q = request_of<KEYS>(a, ++w.b); }
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

// Whole warp: the walk's next piece; both in shared memory.
template <int ROWS, int KEYS>
__device__ __noinline__ bool next_piece(const TreeAttnArgs& a, Walk& walk, Piece& piece) {
  Walk w = walk;
  Piece u;
  __syncwarp();
  const bool more = walk_on<ROWS, KEYS>(a, w, u);
  if ((threadIdx.x & 31) == 0) {
    walk = w;
    piece = u;
  }
  __syncwarp();
  return more;
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
  uint32_t w;                      // (left to the compiler, the mask and the or are two instructions: 13 instead of 7 a word)
  asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(w) : "r"(codes >> (4 * p)), "r"(0x000f000fu), "r"(0x43004300u));
  const __nv_bfloat162 y = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&w), s.s, s.off);
  return *reinterpret_cast<const uint32_t*>(&y);
}

// The producer, a whole warp: lane w issues the copies of warp w's run, if it has one, RING steps ahead of the products.
template <int D, int NT>
__device__ __noinline__ void produce(const TreeAttnArgs& a, const Q4Cache& cache, uint32_t base, const Abort& ab, Walk walk, int w) {
  using P = Plan<D, NT>;
  auto full = [&](int slot) { return base + P::BAR_OFF + (w * P::RING + slot) * 16; };
  const uint32_t ring = base + P::RING_OFF + w * (P::RING * P::BYTES);
  const bool one_copy = (1 << a.page_log2) >= P::KEYS;                 // a step's blocks lie together
  Piece u;
  u.kt0 = u.n = 0;
  int kt = 0, issued = 0, slot = 0, id0 = -1, id1 = -1, idle = 0;
  uint32_t lap = 0;
  long long since = 0;
  bool more = true, ready = false;                                     // ready: ids of step kt are on their way
  const int32_t* row = nullptr;
  const uint8_t* head = nullptr;
  while (more) {
    if (!ready) {
      if (kt == u.kt0 + u.n) {
        more = walk_on<P::ROWS, P::KEYS>(a, walk, u);
        if (!more) break;
        kt = u.kt0;
        row = a.table + (size_t)u.b * a.max_pages;
        head = cache.data + u.g * cache.s_head;
      }
      const long long key = (long long)kt * P::KEYS;
      id0 = key < u.len ? row[key >> a.page_log2] : -1;
      id1 = key + 16 < u.len ? row[(key + 16) >> a.page_log2] : -1;
      ready = true;
    }
    if (lap > 0 && !mbar_test(full(slot) + 8, (lap - 1) & 1)) {
      if (*ab.flag) break;
      if ((++idle & 63) == 0) {
        const int code = *reinterpret_cast<volatile int*>(ab.status);
        if (code != 0 && code != (int)SP_ERR_RANGE) { *ab.flag = 1; break; }
        const long long now = clock64();
        if (since == 0) since = now;
        else if (now - since > kWaitCycles) {
          *ab.flag = 1;
          report_timeout(ab.status, 101);
          break;
        }
      }
      __nanosleep(100);
      continue;
    }
    idle = 0;
    since = 0;
    // no such page, or no key at all: nothing is copied, whatever lies in the slot is finite
    const int key = kt * P::KEYS, in = key & ((1 << a.page_log2) - 1);
    const bool have0 = key < u.len && id0 >= 0 && id0 < a.n_pages, have1 = key + 16 < u.len && id1 >= 0 && id1 < a.n_pages;
    if ((key < u.len && !have0) || (key + 16 < u.len && !have1)) report_range(a.status, kWhereTreePageQ4);
    const uint32_t dst = ring + slot * P::BYTES;
    mbar_expect_tx(full(slot), (have0 + have1) * P::BLOCK);
    const uint8_t* src0 = head + id0 * cache.s_page + (in >> 4) * P::BLOCK;
    if (one_copy) {
      if (have0) bulk_copy(dst, src0, (have0 + have1) * P::BLOCK, full(slot));
    } else {
      if (have0) bulk_copy(dst, src0, P::BLOCK, full(slot));
      if (have1) bulk_copy(dst + P::BLOCK, head + id1 * cache.s_page + (((in + 16) & ((1 << a.page_log2) - 1)) >> 4) * P::BLOCK, P::BLOCK, full(slot));
    }
    ready = false;
    ++kt;
    ++issued;
    if (++slot == P::RING) { slot = 0; ++lap; }
  }
  // The copies that are still in flight land before the CTA can give its shared memory back: also those of a run that was issued to its
  // end, whose warp may give up, or stop with others, before it has waited for them.  (Behind all lanes' runs: a lane that polls
  // holds up the others.)
  __syncwarp();
  const long long t0 = clock64();
  for (int i = max(issued - P::RING, 0); i < issued; ++i)
    while (!mbar_test(full(i % P::RING), (i / P::RING) & 1) && clock64() - t0 < kWaitCycles / 8) __nanosleep(500);
}

template <int D, int NT>
__global__ void __launch_bounds__(Plan<D, NT>::THREADS, 1) tree_attn_q4_kernel(const __grid_constant__ TreeAttnArgs a, const __grid_constant__ Q4Cache cache,
                                                                              const CtaParts work) {
  using P = Plan<D, NT>;
  using B = Block<D>;
  constexpr int WARPS = P::WARPS, ROWS = P::ROWS, THREADS = P::THREADS, WORDS = P::WORDS;
  extern __shared__ __align__(128) uint8_t smem[];
  const uint32_t base = smem_u32(smem);
  float2* part_ml = reinterpret_cast<float2*>(smem + P::ML_OFF);
  PartInfo* infos = reinterpret_cast<PartInfo*>(smem + P::INFO_OFF);
  long long* scan = reinterpret_cast<long long*>(smem + P::SCAN_OFF);
  long long* start_rem = scan + WARPS + 1;
  int* start_b = reinterpret_cast<int*>(start_rem + WARPS + 1);
  volatile int* abort_flag = reinterpret_cast<int*>(smem + P::FLAG_OFF);
  volatile int* last_flags = abort_flag + 1;      // [2]: this CTA is the last of the unit of its part 0, 1
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  const int cta = blockIdx.x;
  const Abort ab{abort_flag, a.status};
  auto bar = [&](int slot) { return base + P::BAR_OFF + (warp * P::RING + slot) * 16; };       // full; + 8: free

  let_next_start();
  if (warp < WARPS) {
    if (lane < 2 * P::RING) mbar_init(base + P::BAR_OFF + (warp * 2 * P::RING + lane) * 8, 1);
    if (lane < 2) infos[warp * 2 + lane].rows = 0;
  }
  if (threadIdx.x == 0) *abort_flag = last_flags[0] = last_flags[1] = 0;
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  wait_for_previous();
  const bool poisoned = decode_poisoned(a.status);

  // ---- where the warps' runs begin
  const int per = (a.n_req + THREADS - 1) / THREADS;
  const int b_lo = min((int)threadIdx.x * per, a.n_req), b_hi = min(b_lo + per, a.n_req);
  long long mine = 0;
  for (int b = b_lo; b < b_hi; ++b) {
    const Request r = request_of<P::KEYS>(a, b);
    mine += units_of<ROWS>(a, r) * (r.kt + kOwnSteps);
  }
  long long incl = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long up = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += up;
  }
  if (lane == 31) scan[warp] = incl;
  const bool idle = __syncthreads_or(poisoned) != 0;                   // all or none: there are barriers and votes ahead
  long long before = incl - mine, total = 0;
#pragma unroll
  for (int w = 0; w <= WARPS; ++w) {
    if (w < warp) before += scan[w];
    total += scan[w];
  }
  // as many warps of each CTA as have kLeastSteps to do (a part costs its addition)
  const long long want = divide(total, (long long)gridDim.x * kLeastSteps);
  const int warps = (int)max(1ll, min((long long)WARPS, want)), n_runs = gridDim.x * warps;
  const long long quota = divide(total, n_runs), extra = total - quota * n_runs;      // the first `extra` runs are one step longer
  auto run_begin = [&](int r) { return r * quota + min((long long)r, extra); };
  auto cta_of = [&](long long z) {                 // that has step z
    const long long cut = extra * (quota + 1);
    return (int)(z < cut ? divide(z, quota + 1) : extra + divide(z - cut, quota)) / warps;
  };
  for (int i = 0; i < warps; ++i) {
    const long long w = run_begin(cta * warps + i);
    if (before <= w && w < before + mine) {
      long long step = before;
      for (int b = b_lo; b < b_hi; ++b) {
        const Request r = request_of<P::KEYS>(a, b);
        const long long n = units_of<ROWS>(a, r) * (r.kt + kOwnSteps);
        if (w < step + n) { start_b[i] = b; start_rem[i] = w - step; break; }
        step += n;
      }
    }
  }
  __syncthreads();

  const int mine_w = warp == WARPS ? lane : warp;                      // the run that a warp, or a lane of the producer, looks after
  const long long w0 = run_begin(cta * warps + mine_w), steps = mine_w < warps && !idle ? run_begin(cta * warps + mine_w + 1) - w0 : 0;
  bool ok = true;
  if (warp == WARPS) {
    produce<D, NT>(a, cache, base, ab, steps > 0 ? Walk{start_rem[lane], steps, start_b[lane], request_of<P::KEYS>(a, start_b[lane])} : Walk{}, lane);
    __syncwarp();
  } else if (steps > 0) {
    const int ring_at = P::RING_OFF + warp * (P::RING * P::BYTES);
    WarpState& st = reinterpret_cast<WarpState*>(smem + P::STATE_OFF)[warp];
    if (lane == 0) st.walk = Walk{start_rem[warp], steps, start_b[warp], request_of<P::KEYS>(a, start_b[warp])};
    __syncwarp();
    // this lane's part of a block: bytes from its begin
    const int k_at = B::k_word(g, q * WORDS), ks_at = B::k_scale(g, q * WORDS / 4), v_at = B::v_word(2 * q, g * (D / 64)), vs_at = B::v_scale(2 * q, g * (D / 8) / 32);
    constexpr int V1 = B::v_word(1, 0) - B::v_word(0, 0), V2 = B::v_word(8, 0) - B::v_word(0, 0);      // from token 2 q to 2 q + 1, 2 q + 8
    int slot = 0;
    uint32_t phase = 0;
    while (ok && next_piece<ROWS, P::KEYS>(a, st.walk, st.piece)) {
      const Piece& u = st.piece;
      if (lane == 0 && u.kt0 == 0 && a.seq_lens[u.b] > u.len) report_range(a.status, kWhereTreePageQ4);   // longer than its table row
      // ---- queries: of row nt * 8 + g elements q D / 4 ..
      uint4 qf[NT][WORDS];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const int row = nt * 8 + g, abs_row = u.r0 + row;
        const __nv_bfloat16* src = a.q + (int64_t)(u.g * a.group + abs_row % a.group) * a.q_sh + (int64_t)(u.start + abs_row / a.group) * a.q_sn + q * (D / 4);
#pragma unroll
        for (int w = 0; w < WORDS; ++w) {
          qf[nt][w] = make_uint4(0, 0, 0, 0);
          if (row < u.rows) qf[nt][w] = *reinterpret_cast<const uint4*>(src + w * 8);
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
      for (int k0 = u.kt0 * P::KEYS, left = u.n; left > 0; k0 += P::KEYS, --left) {
        if (!__all_sync(0xffffffffu, mbar_try_wait(bar(slot), phase))) {
          ok = __all_sync(0xffffffffu, mbar_wait_slow(bar(slot), phase, ab.flag, ab.status, 100, kWaitCycles));
          if (!ok) break;
        }
        const int step_at = ring_at + slot * P::BYTES;
        // ---- S^T = K Q^T
        float s[P::BLOCKS][NT][4];
#pragma unroll
        for (int h = 0; h < P::BLOCKS; ++h) {
          const uint8_t* blk = smem + step_at + h * P::BLOCK;
          uint32_t kw[2][WORDS];
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const uint8_t* row = blk + k_at + x * B::k_word(8, 0);
            if constexpr (WORDS == 4) {
              const uint4 y = *reinterpret_cast<const uint4*>(row);
              kw[x][0] = y.x; kw[x][1] = y.y; kw[x][2] = y.z; kw[x][3] = y.w;
            } else {
              const uint2 y = *reinterpret_cast<const uint2*>(row);
              kw[x][0] = y.x; kw[x][1] = y.y;
            }
          }
          const uint32_t kb = *reinterpret_cast<const uint16_t*>(blk + ks_at);
          const Scale2 ks[2] = {scale2(permute(kb, 0u, 0x4040u)), scale2(permute(kb, 0u, 0x4141u))};
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[h][nt][i] = 0.f;
#pragma unroll
          for (int w = 0; w < WORDS; ++w) {
            const uint32_t f0[4] = {values(kw[0][w], 0, ks[0]), values(kw[1][w], 0, ks[1]), values(kw[0][w], 1, ks[0]), values(kw[1][w], 1, ks[1])};
            const uint32_t f1[4] = {values(kw[0][w], 2, ks[0]), values(kw[1][w], 2, ks[1]), values(kw[0][w], 3, ks[0]), values(kw[1][w], 3, ks[1])};
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              if (NT > 1 && nt >= tiles) break;
              mma16816(s[h][nt], f0, qf[nt][w].x, qf[nt][w].y);
              mma16816(s[h][nt], f1, qf[nt][w].z, qf[nt][w].w);
            }
          }
        }
        // ---- softmax: lane has keys g, g + 8 of each block and rows 2 q, 2 q + 1 of each tile
        if (no_mask - k0 < P::KEYS) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            if (NT > 1 && nt >= tiles) break;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const int row = nt * 8 + 2 * q + i;
              const uint32_t seen = row < u.rows ? seen32(a, u, (u.r0 + row) / a.group, k0) >> g : 0u;
#pragma unroll
              for (int h = 0; h < P::BLOCKS; ++h) {
                if (!(seen >> (16 * h) & 1)) s[h][nt][i] = -CUDART_INF_F;
                if (!(seen >> (16 * h + 8) & 1)) s[h][nt][2 + i] = -CUDART_INF_F;
              }
            }
          }
        }
        uint32_t p[P::BLOCKS][NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          if (NT > 1 && nt >= tiles) break;
          float y[P::BLOCKS][4], top = -CUDART_INF_F;
          auto weigh = [&] {
#pragma unroll
            for (int h = 0; h < P::BLOCKS; ++h)
#pragma unroll
              for (int i = 0; i < 4; ++i) y[h][i] = fmaf(s[h][nt][i], a.scale_log2, -m[nt][i & 1]);
          };
          weigh();
#pragma unroll
          for (int h = 0; h < P::BLOCKS; ++h) top = max3(max3(top, y[h][0], y[h][1]), y[h][2], y[h][3]);
          if (__any_sync(0xffffffffu, top > 8.f)) {
            // a row's logits are 2^8 above its reference: the rows' maxima over the lanes that have them; references are whole
            // numbers, so nothing is rounded again
            float x[2], f[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              x[i] = fmaxf(s[0][nt][i], s[0][nt][2 + i]);
              if (P::BLOCKS > 1) x[i] = max3(x[i], s[P::BLOCKS - 1][nt][i], s[P::BLOCKS - 1][nt][2 + i]);
#pragma unroll
              for (int e = 4; e < 32; e <<= 1) x[i] = fmaxf(x[i], __shfl_xor_sync(0xffffffffu, x[i], e));
              x[i] *= a.scale_log2;
              const float now = x[i] > m[nt][i] + 8.f ? ceilf(x[i]) : m[nt][i];
              f[i] = ex2_approx(m[nt][i] - now);
              l[nt][i] *= f[i];
              m[nt][i] = now;
            }
#pragma unroll
            for (int t2 = 0; t2 < D / 16; ++t2) { o[nt][t2][0] *= f[0]; o[nt][t2][1] *= f[1]; o[nt][t2][2] *= f[0]; o[nt][t2][3] *= f[1]; }
            weigh();
          }
#pragma unroll
          for (int h = 0; h < P::BLOCKS; ++h) {
#pragma unroll
            for (int i = 0; i < 4; ++i) y[h][i] = ex2_approx(y[h][i]);
            l[nt][0] += y[h][0] + y[h][2];
            l[nt][1] += y[h][1] + y[h][3];
            p[h][nt][0] = transpose8(cvt_bf16x2(y[h][0], y[h][1]));
            p[h][nt][1] = transpose8(cvt_bf16x2(y[h][2], y[h][3]));
          }
        }
        // ---- O^T += V^T P^T: lane has tokens 2 q, 2 q + 1 and 2 q + 8, 2 q + 9 of a block, elements g D / 8 ..
#pragma unroll
        for (int h = 0; h < P::BLOCKS; ++h) {
          const uint8_t* blk = smem + step_at + h * P::BLOCK;
          const uint32_t vb = *reinterpret_cast<const uint32_t*>(blk + vs_at);
          const Scale2 v01 = scale2(vb & 0x00ff00ffu), v23 = scale2(vb >> 8 & 0x00ff00ffu);
          uint32_t vw[4][D / 64];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint8_t* row = blk + v_at + (i & 1) * V1 + (i >> 1) * V2;
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
                mma16816(o[nt][w * 4 + e], f, p[h][nt][0], p[h][nt][1]);
              }
            }
          }
        }
        __syncwarp();                              // all have read the step's keys
        if (lane == 0) mbar_arrive(bar(slot) + 8);
        if (++slot == P::RING) { slot = 0; phase ^= 1; }
      }
      if (!ok) break;

      // ---- the piece's rows: results, or a part
      const bool whole = u.kt0 == 0 && u.n == u.kt_all;
      const int which = u.kt0 > 0 ? 0 : 1;
      float* part = reinterpret_cast<float*>(which == 0 ? smem + P::PART_OFF + warp * P::PART_BYTES : smem + ring_at);
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
            float4* dst = reinterpret_cast<float4*>(part + row * P::STRIDE + g * (D / 8));
#pragma unroll
            for (int w = 0; w < D / 32; ++w)
              dst[w] = make_float4(o[nt][2 * w][i], o[nt][2 * w][2 + i], o[nt][2 * w + 1][i], o[nt][2 * w + 1][2 + i]);
            if (g == 0) part_ml[(warp * 2 + which) * ROWS + row] = make_float2(m[nt][i], sum);
          }
        }
      }
      if (!whole && lane == 0) {
        const long long end = w0 + steps - st.walk.left;                // the step behind the piece's last
        infos[warp * 2 + which] = PartInfo{u.rows, u.kt0 + u.n == u.kt_all, u.start, u.r0, u.g, cta_of(end - u.n - u.kt0), cta_of(end - 1 + u.kt_all - u.kt0 - u.n), 0};
      }
      __syncwarp();
    }
  }

  // ---- the CTA's parts, in the order of the keys: warp 0's part 0, its part 1 or warp 1's part 0, ...
  __syncthreads();
  if (*abort_flag || idle) return;
  // a row's result, or nothing seen
  auto result = [&](const PartInfo& u, int row, float top, float sum, const float (&y)[WORDS]) {
    const int abs_row = u.r0 + row, token = abs_row / a.group, head = u.g * a.group + abs_row % a.group;
    const float inv = sum != 0.f ? 1.f / sum : 0.f;
    uint32_t* dst = reinterpret_cast<uint32_t*>(a.o + head * a.o_sh + (int64_t)(u.start + token) * a.o_sn + lane * WORDS);
#pragma unroll
    for (int e = 0; e < WORDS; e += 2) dst[e / 2] = pack_bf16(y[e] * inv, y[e + 1] * inv);
    if (a.lse && lane == 0) a.lse[(size_t)head * a.rows + u.start + token] = sum != 0.f ? (top + log2f(sum)) * 0.6931471805599453f : -CUDART_INF_F;
  };
  int task = 0, shared_part[2] = {-1, -1};         // the parts that this CTA leaves: indices into infos
  for (int i = 0; i < 2 * warps; ++i) {
    if (infos[i].rows == 0 || !((i & 1) || i == 0)) continue;          // not the first of its unit here
    const PartInfo u = infos[i];
    int end = (i | 1) + 1;                                             // parts of the unit: i, then the part 0 of the warps after it, up to `end`
    bool ends = u.ends;
    while (!ends && end < 2 * warps && infos[end].rows != 0) { ends = infos[end].ends; end += 2; }
    const bool whole = (i & 1) && ends;
    if (!whole) shared_part[i & 1] = i;
    for (int row = 0; row < u.rows; ++row) {
      if (task++ % (WARPS + 1) != warp) continue;
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
      if (whole) {
        result(u, row, top, sum, y);
      } else {
        const size_t at = ((size_t)cta * 2 + (i & 1)) * ROWS + row;
#pragma unroll
        for (int e = 0; e < WORDS; ++e) work.part[at * D + lane * WORDS + e] = y[e];
        if (lane == 0) work.ml[at] = make_float2(top, sum);
      }
    }
  }
  if (shared_part[0] < 0 && shared_part[1] < 0) return;

  // ---- units that several CTAs have: the last to arrive adds up their parts
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int x = 0; x < 2; ++x) {
      if (shared_part[x] < 0) continue;
      const PartInfo u = infos[shared_part[x]];
      if (atomicAdd(work.arrived + u.first, 1) == u.last - u.first) {
        work.arrived[u.first] = 0;                 // nobody else comes; for the next call
        last_flags[x] = 1;
      }
    }
    __threadfence();
  }
  __syncthreads();
  float* sums = reinterpret_cast<float*>(smem + P::RING_OFF);          // [warp][STRIDE]
  float2* sums_ml = reinterpret_cast<float2*>(smem + P::ML_OFF);
  for (int x = 0; x < 2; ++x) {
    if (!last_flags[x]) continue;
    const PartInfo u = infos[shared_part[x]];
    const int parts = u.last - u.first + 1;
    int share = 1;                                 // warps for a row
    while (2 * share * u.rows <= WARPS && 2 * share < parts) share *= 2;
    for (int row0 = 0; row0 < u.rows; row0 += WARPS / share) {
      const int row = row0 + warp / share, turn = warp % share;
      const bool live = warp < WARPS / share * share && row < u.rows;
      float top = kNoMax, sum = 0.f, y[WORDS];
#pragma unroll
      for (int e = 0; e < WORDS; ++e) y[e] = 0.f;
      if (live) {
        constexpr int RUN = 8;                     // parts in flight
        for (int p0 = turn; p0 < parts; p0 += RUN * share) {
          float2 ml[RUN];
          float z[RUN][WORDS];
#pragma unroll
          for (int i = 0; i < RUN; ++i) {
            const int p = p0 + i * share;
            ml[i] = make_float2(kNoMax, 0.f);
#pragma unroll
            for (int e = 0; e < WORDS; ++e) z[i][e] = 0.f;
            if (p < parts) {
              const size_t at = ((size_t)(u.first + p) * 2 + (p == 0 ? 1 : 0)) * ROWS + row;
              ml[i] = __ldcg(work.ml + at);
              if constexpr (WORDS == 4) {
                const float4 t = __ldcg(reinterpret_cast<const float4*>(work.part + at * D) + lane);
                z[i][0] = t.x; z[i][1] = t.y; z[i][2] = t.z; z[i][3] = t.w;
              } else {
                const float2 t = __ldcg(reinterpret_cast<const float2*>(work.part + at * D) + lane);
                z[i][0] = t.x; z[i][1] = t.y;
              }
            }
          }
#pragma unroll
          for (int i = 0; i < RUN; ++i) {
            const float now = fmaxf(top, ml[i].x), f_old = ex2_approx(top - now), f = ex2_approx(ml[i].x - now);
            sum = sum * f_old + ml[i].y * f;
#pragma unroll
            for (int e = 0; e < WORDS; ++e) y[e] = y[e] * f_old + z[i][e] * f;
            top = now;
          }
        }
      }
      if (share > 1) {
        __syncthreads();                           // the last rows' sums have been read
        if (live) {
#pragma unroll
          for (int e = 0; e < WORDS; ++e) sums[warp * P::STRIDE + lane * WORDS + e] = y[e];
          if (lane == 0) sums_ml[warp] = make_float2(top, sum);
        }
        __syncthreads();
        if (live && turn == 0) {
          for (int w = warp + 1; w < warp + share; ++w) {
            const float2 ml = sums_ml[w];
            const float now = fmaxf(top, ml.x), f_old = ex2_approx(top - now), f = ex2_approx(ml.x - now);
            sum = sum * f_old + ml.y * f;
#pragma unroll
            for (int e = 0; e < WORDS; ++e) y[e] = y[e] * f_old + sums[w * P::STRIDE + lane * WORDS + e] * f;
            top = now;
          }
        }
      }
      if (live && turn == 0) result(u, row, top, sum, y);
    }
    __syncthreads();
  }
}

template <int D, int NT>
cudaError_t launch(const TreeAttnArgs& a, const Q4Cache& c, void* ws, int* arrived, int n_sm, cudaStream_t s) {
  using P = Plan<D, NT>;
  CtaParts w;
  w.part = static_cast<float*>(ws);
  w.ml = reinterpret_cast<float2*>(w.part + (size_t)n_sm * 2 * P::ROWS * D);
  w.arrived = arrived;
  const cudaError_t e = cudaFuncSetAttribute(tree_attn_q4_kernel<D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, P::TOTAL);
  if (e != cudaSuccess) return e;
  return launch_dependent(tree_attn_q4_kernel<D, NT>, dim3(n_sm), dim3(P::THREADS), P::TOTAL, s, a, c, w);
}

template <int D>
cudaError_t launch_rows(const TreeAttnArgs& a, const Q4Cache& c, void* ws, int* arrived, int n_sm, cudaStream_t s, int* launched) {
  // Rows of a request if all have as many.  More than 24 make tiles of 128 for the tensor cores' own memory; up to 24 are two
  // units of 16 at most, which read the cache twice, from L2 the second time, but cost less for each unit (so, and with the
  // tiles: 256 chats with 20 rows each 191 and 253 us, with 24 rows 206 and 252, with 32 rows 242 and 253, with 48 rows as three units 316
  // and 264; 32 chats with 32 rows 55 and 49; 32 ragged requests with 21 rows 196 and 174, with 28 rows 199 and 174; over 131000
  // keys 20 rows 116 and 101, 32 rows 120 and 102, 48 rows 164 and 107.  In one unit of up to 32 rows, of the registers of seven warps: 24 rows in
  // chats 273, 28 ragged 252, 32 rows over 131000 keys 160).  Requests of more rows than a form's units have are several units, which is
  // right for any lengths.
  const long long rows = ((long long)a.rows + a.n_req - 1) / a.n_req * a.group;
  *launched = rows <= 24 ? 1 : 2;
  return rows <= 8 ? launch<D, 1>(a, c, ws, arrived, n_sm, s) : rows <= 24 ? launch<D, 2>(a, c, ws, arrived, n_sm, s) : launch_tree_attn_q4_tall(a, c, ws, n_sm, s);
}

}  // namespace

size_t tree_attn_q4_workspace_bytes(int n_sm) { return (size_t)n_sm * 2 * 16 * (128 * sizeof(float) + sizeof(float2)); }

cudaError_t launch_tree_attn_q4(const TreeAttnArgs& a, const Q4Cache& c, void* ws, int* arrived, int n_sm, cudaStream_t s, int* launched) {
  return a.d == 128 ? launch_rows<128>(a, c, ws, arrived, n_sm, s, launched) : launch_rows<64>(a, c, ws, arrived, n_sm, s, launched);
}

}  // namespace sp
