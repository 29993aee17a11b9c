// Attention of a few new tokens per request (one, a chain, a tree of drafted ones) over the paged cache: tcgen05 / TMEM /
// TMA, split along the keys.
//
//   out_r = sum_c p_rc v_c / sum_c p_rc,  p_rc = 2^(scale q_r.k_c - m_r) over the visible keys c.
//
// The rows of a unit are the new tokens of one request times the query heads that share a KV head (row = token * group +
// head), so that every key and value is read once for all of them.  Work is counted in steps: one for each key tile of 128
// of a unit (request, KV head, rows), and some for the unit itself: two if it is narrow, four otherwise (see below).  The
// steps of all units stand in one line, which is cut into one equal run per SM wherever that falls; a unit that is cut
// leaves partial results (unnormalised sums, references, weights) that a second kernel joins in the order of the keys.  All
// lengths are read on the device: a prefix sum over the requests tells each CTA where its run begins.  (With too few steps
// for the unit itself the CTAs with many short requests finish late, with too many those with long ones.  256 chats of 60 to
// 4000 tokens and a new one each: 243, 200, 171, 173, 180, 194 us for 0, 1, 2, 3, 4, 6 steps; with trees of 8: 306, 255, 227,
// 219, 236 us for 1, 2, 3, 4, 6.)
//
// What bounds it: the cache's bytes.  A tile is 64 KB (head_dim 128), 2700 cycles of an SM's share of the measured HBM
// rate; its matrix products take 1020 cycles of the tensor core for up to 128 rows (it takes 128 rows at a time, however
// few are in use) and 1400 of the thread that issues them; its exponentials take 8 cycles per row of the SM's
// special-function units.  Everything else is a matter of keeping these from waiting for one another.
//
//   warps 0-7       softmax and epilogue, two groups of four: thread = TMEM lane = row
//   warp 8          producer: page ids from the table, TMA loads of K and V pages into a ring of tile slots, in the order
//                   in which the products need them, K `lead` tiles ahead of V
//   warps 9, 11     issuers (one thread each; warp 11 in wide units only): S = Q K^T and O += P V
//   warp 10         loader: walks the run, publishes units, gathers their Q rows into shared memory
//
// Three modes, by the largest number of rows that any request has (wide only where it saves enough tiles, see the kernel):
//
// Wide (more than 128): units have up to 256 rows, the groups are their halves and walk the same tiles 64 keys at a time,
// each with its O and two S of 64 columns in TMEM (all there is), so that the next S is computed during the softmax of this
// one.  The reference maximum moves, to a whole number, when the row maximum has grown by more than 2^8; O in TMEM is then
// rescaled (exactly).  The tensor core's operands bound it: 128 rows of Q for 64 keys are 6 KB of shared memory for each
// product of 48 cycles, 2500 cycles a tile in all, and the two groups' chains do not fill the gaps: 4000 a tile.  (With one
// S of 128 columns each: 5 % slower.  Two CTAs, a half each, on the same tiles: 208 us instead of 160 for 128K keys, L2 does
// not serve both at the rate of HBM.)  The prefill's paired kernel takes 3500 for tiles of this shape at
// head_dim 128, with one issuer, constant descriptors and hand-overs by named barriers: not tried here.
//
// Tall (17 to 128): one O, three S in turn, and the groups take the tiles in turn.  S of the next tiles is computed while
// both groups are in their softmax, so nothing waits for anything but the bytes.  One O means one reference for both
// groups: it is taken from the unit's first tile (2^24 above the row's maximum there) and stays, which fp32 and bf16, with
// 2^126 below and 2^127 above, have room for; no maximum is looked for in the other tiles.  If a row's weight comes out
// above 2^56 or below 2^-40 all the same (logits that climb 55 nats above the first tile's), the CTA walks its run once
// more, as wide.
//
// Narrow (at most 16, single tokens as a rule): 128-row products are the wrong tool, and a softmax with a row in a lane
// leaves most lanes empty.  The eight softmax warps are on their own: each takes 16 keys of every tile, S (16 rows x 16
// keys) and O (16 rows x head) in registers by mma.sync m16n8k16, K and V by ldmatrix from the same ring; their sums are
// added up at the unit's end.  16 mma.sync for each product and warp are a few hundred cycles of the 2700 that the tile's
// bytes take.  (256 x 950 tokens: 164 us so, 208 us by tcgen05 with the rows in the lanes, 236 us by tcgen05 with the keys
// in the lanes: MMAs of 16 columns are issued no faster than those of 128.)
//
// Masks.  Only tiles that hold a key at or behind the first new token need one.  There the row's visibility bits are
// shifted into place 32 keys at a time.  A masked probability is zero, but zero times a NaN in V is not: in those tiles
// the values behind the sequence are set to zero in shared memory, and non-finite values of new tokens too; if there were
// any, each row adds those that it sees at the end (from the cache: they are what the sum comes to anyway).
//
// Rounding: products bf16 x bf16 in fp32, softmax statistics and O in fp32, P rounded to bf16 for the second product (the
// sum of weights is taken before that rounding), the result once.  References are whole numbers, so that a change of
// reference is a change of exponents.
//
// Every wait is bounded as in the other tensor-core kernels: a wait that runs out raises the abort flag and the status
// word, and all roles fall through to the common end.
#include <limits.h>

#include "decode.cuh"
#include "tc_ptx.cuh"

namespace sp {
namespace {

using namespace tc;

constexpr int kTile = 128;                       // keys of a tile
constexpr int kUnitRows = 256;
constexpr int kThreads = 384, kWarps = kThreads / 32;
constexpr int kProducer = 8, kIssuer = 9, kLoader = 10, kIssuer1 = 11;
constexpr int kUnitRing = 4;
constexpr int kNarrowSteps = 2, kTallSteps = 4;  // steps of a unit besides those of its tiles (narrow; tall and wide); measured at head_dim 128
constexpr int kNarrowRows = 16;
constexpr float kNoMax = -1e30f;                 // reference maximum before any visible key: finite, below any logit
constexpr float kTallMargin = 24.f;              // tall: the reference above the first tile's maximum,
constexpr float kTallMost = 72057594037927936.f, kTallLeast = 9.094947017729282e-13f;      // and the weights that it serves: 2^56, 2^-40

template <int D>
struct Plan {
  // Rows in shared memory: groups of eight; a group is 1024 bytes for each 64 columns, 128-byte swizzled.  (A page's columns
  // then come by one TMA instruction, however many rows it has.  With all rows of 64 columns together it takes one for
  // each, and at 75 cycles each the producer was late for pages of 16: 215 instead of 175 us.)
  static constexpr int BOX = 1024, GROUP = D / 64 * BOX;
  static constexpr int QHALF = 128 / 8 * GROUP, SLOT = kTile / 8 * GROUP;
  static constexpr int SLOTS = D == 128 ? 5 : 10;
  static constexpr int RING_OFF = 2 * QHALF;
  static constexpr int MISC_OFF = RING_OFF + SLOTS * SLOT;
  // narrow: one slot more, in the second half of the Q area; two sets of 16 Q rows and the sums' exchange in the first
  static constexpr int NSLOTS = SLOTS + 1, NRING_OFF = RING_OFF - SLOT;
  static constexpr int NQ_BYTES = kNarrowRows / 8 * GROUP, SUM_OFF = 2 * NQ_BYTES;
  static constexpr int SUM_ROWS = 4, SUM_STRIDE = D + 8;                  // rows exchanged at a time; 8 columns more against bank conflicts
  static_assert(SLOT == QHALF && SUM_OFF + 8 * SUM_ROWS * SUM_STRIDE * 4 <= QHALF, "");
  // full and free: tiles; S, P: tall per buffer, wide [group][buffer], and PV likewise; REF, OFULL, OFREE: tall
  static constexpr int BAR_FULL = 0, BAR_FREE = BAR_FULL + NSLOTS, BAR_S = BAR_FREE + NSLOTS, BAR_P = BAR_S + 4, BAR_PV = BAR_P + 4, BAR_REF = BAR_PV + 4,
                       BAR_OFULL = BAR_REF + 1, BAR_OFREE = BAR_OFULL + 1, BAR_QFULL = BAR_OFREE + 1, BAR_QFREE = BAR_QFULL + 2,
                       BAR_UNIT = BAR_QFREE + 2, BAR_UFREE = BAR_UNIT + kUnitRing, BARS = BAR_UFREE + kUnitRing;
  static constexpr int UNIT_OFF = MISC_OFF + 2 * BARS * 8, UNIT_BYTES = 48;                  // a second set of barriers: for a run walked again
  static constexpr int SCAN_OFF = (UNIT_OFF + kUnitRing * UNIT_BYTES + 15) / 16 * 16;        // int64 [2][kWarps]
  static constexpr int RUN_OFF = SCAN_OFF + 2 * kWarps * 8;                           // int64 [3], int [4]
  static constexpr int TAG_OFF = RUN_OFF + 3 * 8 + 4 * 4;                             // int [8]
  static constexpr int EX_OFF = (TAG_OFF + 8 * 4 + 15) / 16 * 16;                     // narrow: float2 [8][16]; tall: float [2][128]
  static constexpr int REF_OFF = EX_OFF + 1024;                                       // tall: float [128]
  static constexpr int TOTAL = REF_OFF + 512;
  // TMEM columns: S 128 each; O: wide behind two S, tall behind three
  static constexpr int S_COL = 0, O_COL = 256, O_STEP = D, TALL_O_COL = 384;
};

struct Unit {
  int n_tiles;      // key tiles of this CTA's part; 0: no more units
  int kt0;          // first of them
  int kt_all;       // key tiles of the whole unit
  int start;        // first row of the request
  int r0, rows;     // first of the unit's rows (token * group + head) inside the request, and their number
  int g, b;
  int len, past;
  int pad[2];
};
static_assert(sizeof(Unit) == 48, "");

struct Meta {       // what the join kernel needs of a unit that begins in this CTA and goes on in later ones
  int last;         // CTA that has the unit's last tile; < 0: there is no such unit
  int start, r0, rows, g, pad[3];
};

struct Work {
  float* part;      // [cta][2][256][D] unnormalised sums: part 0 of a unit begun by an earlier CTA, part 1 of one begun here
  float2* ml;       // [cta][2][256] reference, weight
  Meta* meta;       // [cta]
  CacheSteps k, v;  // of the tensor maps
};

struct Request {
  int start, n, len, past, kt;
};
__device__ __forceinline__ Request request(const TreeAttnArgs& a, int b) {
  Request q;
  const int s0 = a.row_start[b], s1 = a.row_start[b + 1], seq = a.seq_lens[b];
  q.start = min(max(s0, 0), a.rows);
  q.n = s0 < 0 ? 0 : max(min(s1, a.rows) - q.start, 0);
  q.len = min(max(seq, 0), a.max_pages << a.page_log2);
  q.past = seq - (s1 - s0);
  q.kt = max((q.len + kTile - 1) / kTile, 1);
  return q;
}
// units of the request per KV head, of 128 or 256 rows (n * group fits 32 bits: the host has checked)
__device__ __forceinline__ int passes(const TreeAttnArgs& a, const Request& q, int rows) { return (int)(((uint32_t)(q.n * a.group) + rows - 1) >> (rows == 128 ? 7 : 8)); }
__device__ __forceinline__ long long units_of(const TreeAttnArgs& a, const Request& q, int rows) { return (long long)a.hkv * passes(a, q, rows); }
__device__ __forceinline__ long long divide(long long x, long long y) {       // both are small as a rule
  return ((x | y) >> 32) == 0 ? (long long)((uint32_t)x / (uint32_t)y) : x / y;
}

__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
// Three barriers polled at once (bit i: phase of barrier i over): the round trips overlap.
__device__ __forceinline__ uint32_t mbar_test3(uint32_t b0, uint32_t par0, uint32_t b1, uint32_t par1, uint32_t b2, uint32_t par2) {
  uint32_t r0, r1, r2;
  asm volatile(
      "{\n\t.reg .pred p, q, r;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%3], %4;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 q, [%5], %6;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 r, [%7], %8;\n\t"
      "selp.u32 %0, 1, 0, p;\n\tselp.u32 %1, 2, 0, q;\n\tselp.u32 %2, 4, 0, r;\n\t}"
      : "=r"(r0), "=r"(r1), "=r"(r2)
      : "r"(b0), "r"(par0), "r"(b1), "r"(par1), "r"(b2), "r"(par2)
      : "memory");
  return r0 | r1 | r2;
}
__device__ __forceinline__ uint32_t mbar_test2(uint32_t b0, uint32_t par0, uint32_t b1, uint32_t par1) {
  uint32_t r0, r1;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%2], %3;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 q, [%4], %5;\n\t"
      "selp.u32 %0, 1, 0, p;\n\tselp.u32 %1, 2, 0, q;\n\t}"
      : "=r"(r0), "=r"(r1)
      : "r"(b0), "r"(par0), "r"(b1), "r"(par1)
      : "memory");
  return r0 | r1;
}
__device__ __forceinline__ void tma_load_5d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1, int c2, int c3, int c4) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, %7}], [%2];"
      ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(c4)
      : "memory");
}
// Products with operand descriptors given by their low words (address and leading offset); the high word is the same for
// all operands here (the bytes between 8-row groups, 128-byte swizzle).
template <int D>
constexpr uint32_t kDescHigh = ((uint32_t)Plan<D>::GROUP >> 4) | (1u << 14) | (2u << 29);
template <int D>
__device__ __forceinline__ void mma_ss_lo(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t accum) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
      "mov.b64 da, {%1, %5};\n\tmov.b64 db, {%2, %5};\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accum), "n"(kDescHigh<D>)
      : "memory");
}
template <int D>
__device__ __forceinline__ void mma_ts_lo(uint32_t d_tmem, uint32_t a_tmem, uint32_t b_lo, uint32_t idesc, uint32_t accum) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 db;\n\t"
      "mov.b64 db, {%2, %5};\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "r"(b_lo), "r"(idesc), "r"(accum), "n"(kDescHigh<D>)
      : "memory");
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
// Four 8x8 blocks of 16-bit elements from shared memory (lanes 8 i .. 8 i + 7: the rows of block i), as they are or
// transposed, and D += A B of 16x16 by 16x8 fragments, bf16 in, fp32 out.
__device__ __forceinline__ void ldmatrix4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4t(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ bool nonfinite2(uint32_t w) { return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u; }

// Which of the 32 keys from k0 on a row sees: bit i = key k0 + i.
__device__ __forceinline__ uint32_t seen32(const TreeAttnArgs& a, const Unit& u, int token, int k0) {
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

// The non-finite values of new tokens that a row sees, added to columns lo .. hi - 1 of what its thread has just written
// (they were left out of the products): bf16 results, or fp32 partial sums.
template <typename T>
__device__ __noinline__ void add_nonfinite(const TreeAttnArgs& a, const Unit& u, int token, T* out, int lo, int hi) {
  const int k_from = max(u.kt0 * kTile, u.past), k_to = min((u.kt0 + u.n_tiles) * kTile, u.len);
  for (int key = k_from; key < k_to; ++key) {
    const int id = a.table[(size_t)u.b * a.max_pages + (key >> a.page_log2)];
    if (id < 0 || id >= a.n_pages || !(seen32(a, u, token, key) & 1)) continue;
    const __nv_bfloat16* v = a.vc.data + id * a.vc.s_page + u.g * a.vc.s_head + (key & ((1 << a.page_log2) - 1)) * a.vc.s_tok;
    for (int c = lo; c < hi; ++c) {
      const float x = __bfloat162float(v[c]);
      if (!isfinite(x)) out[c] = static_cast<T>(static_cast<float>(out[c]) + x);
    }
  }
}

// Rare path of the softmax: the row's reference maximum has moved, so O of the earlier tiles (when there are any) and
// the P chunks of this tile that are already stored are brought to the new one.  alpha is a power of two (references are
// whole numbers), so nothing is rounded again.  What is read here may just have been stored (P of the chunk before, O by
// the call before), and a load does not wait for earlier stores by itself.  Called by whole warps.
template <int D>
__device__ __noinline__ void rescale_tmem(uint32_t t_o, uint32_t t_s, float alpha, int stored, bool with_o) {
  tmem_wait_st();
  if (with_o) {
#pragma unroll 1
    for (int c = 0; c < D / 32; ++c) {
      uint32_t o[32];
      tmem_ld32(t_o + c * 32, o);
#pragma unroll
      for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
      tmem_st32(t_o + c * 32, o);
    }
  }
#pragma unroll 1
  for (int c = 0; c < stored; ++c) {
    uint32_t p[16];
    tmem_ld16(t_s + c * 16, p);
#pragma unroll
    for (int e = 0; e < 16; ++e) p[e] = cvt_bf16x2(__uint_as_float(p[e] << 16) * alpha, __uint_as_float(p[e] & 0xffff0000u) * alpha);
    tmem_st16(t_s + c * 16, p);
  }
}

// The logits of the keys that a row does not see are set to -infinity in TMEM before the common path reads them.  Called
// by whole warps; a row that is not the unit's (token < 0) sees nothing.  Whether the row sees any of the tile's keys.
__device__ __noinline__ bool mask_tmem(const TreeAttnArgs& a, const Unit& u, int token, int k0, int keys, uint32_t t_s) {
  uint32_t any = 0;
#pragma unroll 1
  for (int c = 0; c < keys / 32; ++c) {
    const uint32_t seen = token >= 0 ? seen32(a, u, token, k0 + c * 32) : 0u;
    any |= seen;
    if (__all_sync(0xffffffffu, seen == 0xffffffffu)) continue;
    uint32_t s[32];
    tmem_ld32(t_s + c * 32, s);
#pragma unroll
    for (int e = 0; e < 32; ++e) s[e] = (seen >> e) & 1 ? s[e] : 0xff800000u;
    tmem_st32(t_s + c * 32, s);
  }
  tmem_wait_st();
  return any != 0;
}

// Values behind the sequence become zero in a V tile, and so do non-finite ones of new tokens (reported: see
// add_nonfinite).  Rows lo .. hi - 1 of the tile, one after the other, the warp's lanes across the columns.  v: this lane's
// first word of row 0.  Rolled loops: the code runs once a unit and is fetched anew each time; unrolled by eight rows it
// took 2000 cycles for sixteen.
template <int D>
__device__ __noinline__ void clean_values(uint32_t* v, int lo, int hi, int first_behind, volatile int* tags, int mark) {
  constexpr int BOXES = D / 64, BOX_WORDS = 1024 / 4, GROUP_WORDS = BOXES * BOX_WORDS;
  auto at = [&](int r, int b) { return v + (r >> 3) * GROUP_WORDS + b * BOX_WORDS + (r & 7) * 32; };
  int r = lo;
#pragma unroll 1
  for (; r < min(hi, first_behind); ++r) {
    uint32_t w[BOXES];
    bool met = false;
#pragma unroll
    for (int b = 0; b < BOXES; ++b) {
      w[b] = *at(r, b);
      met |= nonfinite2(w[b]);
    }
    if (met) {
      tags[mark % 8] = mark;
      __threadfence_block();
#pragma unroll
      for (int b = 0; b < BOXES; ++b) {
        uint32_t x = w[b];
        if ((x & 0x7f80u) == 0x7f80u) x &= 0xffff0000u;
        if ((x & 0x7f800000u) == 0x7f800000u) x &= 0xffffu;
        *at(r, b) = x;
      }
    }
  }
#pragma unroll 2
  for (r = max(lo, first_behind); r < hi; ++r)
#pragma unroll
    for (int b = 0; b < BOXES; ++b) *at(r, b) = 0u;
}

// Columns lo .. hi - 1 of a row from TMEM, scaled by f: the result, or a part for the join.  Rolled, out of the hot loop.
// Called by whole warps; what is not `live` is not written.  Whether all of the row's values were finite.
__device__ __noinline__ bool write_columns(uint32_t t_o, int lo, int hi, float f, bool live, __nv_bfloat16* out, float* part) {
  bool finite = true;
#pragma unroll 1
  for (int c = lo; c < hi; c += 32) {
    uint32_t y[32];
    tmem_ld32(t_o + c, y);
    if (!live) continue;
#pragma unroll
    for (int i = 0; i < 32; ++i) finite &= (y[i] & 0x7f800000u) != 0x7f800000u;
    auto val = [&](int i) { return __uint_as_float(y[i]) * f; };
    if (part == nullptr) {
      uint4* dst = reinterpret_cast<uint4*>(out + c);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        dst[i] = make_uint4(pack_bf16(val(8 * i), val(8 * i + 1)), pack_bf16(val(8 * i + 2), val(8 * i + 3)), pack_bf16(val(8 * i + 4), val(8 * i + 5)),
                            pack_bf16(val(8 * i + 6), val(8 * i + 7)));
    } else {
      float4* dst = reinterpret_cast<float4*>(part + c);
#pragma unroll
      for (int i = 0; i < 8; ++i) dst[i] = make_float4(val(4 * i), val(4 * i + 1), val(4 * i + 2), val(4 * i + 3));
    }
  }
  return finite;
}

// Where a unit's row goes: its result, or its part if the unit was cut.
struct Place {
  int token, head;
  __nv_bfloat16* out;
  size_t slot;
  bool whole;
};
__device__ __forceinline__ Place place_of(const TreeAttnArgs& a, const Unit& u, int row) {
  Place p;
  const int abs_row = u.r0 + row;
  p.token = abs_row / a.group;
  p.head = u.g * a.group + abs_row % a.group;
  p.out = a.o + p.head * a.o_sh + (u.start + p.token) * a.o_sn;
  p.whole = u.kt0 == 0 && u.n_tiles == u.kt_all;
  p.slot = ((size_t)blockIdx.x * 2 + (u.kt0 > 0 ? 0 : 1)) * kUnitRows + row;
  return p;
}
__device__ __forceinline__ void write_weight(const TreeAttnArgs& a, const Work& work, const Unit& u, const Place& p, float m, float l) {
  if (!p.whole) work.ml[p.slot] = make_float2(m, l);
  else if (a.lse) a.lse[(size_t)p.head * a.rows + u.start + p.token] = l != 0.f ? (m + log2f(l)) * 0.6931471805599453f : -CUDART_INF_F;
}

// Tall: the reference of this thread's row, from the S of the unit's first tile.  Called by whole warps.
__device__ __noinline__ float first_reference(uint32_t t_s, float scale, bool live) {
  float top = -CUDART_INF_F;
#pragma unroll 1
  for (int c = 0; c < kTile; c += 32) {
    uint32_t s[32];
    tmem_ld32(t_s + c, s);
#pragma unroll
    for (int e = 0; e < 32; ++e) top = fmaxf(top, __uint_as_float(s[e]));
  }
  top *= scale;
  // nothing seen here: 0, and the weights tell at the end whether that served
  return !live ? -kNoMax : top > -CUDART_INF_F && top < CUDART_INF_F ? ceilf(top) + kTallMargin : 0.f;
}

// Requests of at most 16 rows: products and softmax in the registers of the eight warps, one call for the whole run.
// (A function of its own, so that the registers of the other modes' loops are not allotted around it.)
template <int D>
__device__ __noinline__ void narrow_warps(const TreeAttnArgs& a, const Work& work, uint8_t* smem, const Abort& ab) {
  using P = Plan<D>;
  const uint32_t base = smem_u32(smem);
  auto bar = [&](int which) { return base + P::MISC_OFF + which * 8; };
  Unit* units = reinterpret_cast<Unit*>(smem + P::UNIT_OFF);
  volatile int* bad_tag = reinterpret_cast<int*>(smem + P::TAG_OFF);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // Fragments of mma.sync m16n8k16: lane = (row g = lane / 4, and g + 8; columns 2 q, 2 q + 1, q = lane % 4).
  const int g = lane >> 2, q = lane & 3;
  float2* ex = reinterpret_cast<float2*>(smem + P::EX_OFF);          // [warp][row] reference, weight
  float* sums = reinterpret_cast<float*>(smem + P::SUM_OFF);         // [warp][row % 4][SUM_STRIDE]
  // ldmatrix addresses of this lane: a row of the four 8x8 blocks, whose 16-byte pieces are swizzled by the row
  const int k_row = warp * 16 + (lane & 7) + ((lane >> 4) << 3), k_piece = (lane >> 3) & 1;   // K: keys 0-7, 8-15 by piece, piece + 1
  const int v_row = warp * 16 + (lane & 15), v_piece = lane >> 4;                            // V (and Q): rows 0-7, 8-15, then the next piece
  const uint32_t ring = base + P::NRING_OFF;
  auto at = [](uint32_t tile, int row, int piece) {
    return tile + (row >> 3) * P::GROUP + (piece >> 3) * P::BOX + (row & 7) * 128 + (((piece ^ row) & 7) << 4);
  };
  const float scale = a.scale_log2;
  uint32_t slot = 0, phase = 0;                     // of the next tile in the ring
  bool ok = true;
  for (int seq = 0;; ++seq) {
    const int e = seq % kUnitRing;
    ok = __all_sync(0xffffffffu, ok && mbar_wait(bar(P::BAR_UNIT + e), (seq / kUnitRing) & 1, ab, 70));
    // the eight warps go on together or stop together: none is left at the barriers below
    if (!bar_and(1, 256, ok)) break;
    const Unit& u = units[e];
    const int n_tiles = u.n_tiles;
    if (n_tiles == 0) break;
    const int rows = u.rows, no_mask = min(u.past, u.len);
    uint32_t qf[D / 16][4];
    ok = __all_sync(0xffffffffu, mbar_wait(bar(P::BAR_QFULL + (seq & 1)), (seq >> 1) & 1, ab, 71));
    if (ok) {
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk)
        ldmatrix4(at(base + (seq & 1) * P::NQ_BYTES, lane & 15, 2 * kk + v_piece), qf[kk]);
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(bar(P::BAR_QFREE + (seq & 1)));
    float o[D / 8][4];
#pragma unroll
    for (int n = 0; n < D / 8; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;
    float m0 = g < rows ? kNoMax : -kNoMax, m1 = g + 8 < rows ? kNoMax : -kNoMax, l0 = 0.f, l1 = 0.f;   // no row: all weights zero
    for (int t = 0; t < n_tiles && ok; ++t) {
      const int k0 = (u.kt0 + t) * kTile;
      ok = __all_sync(0xffffffffu, mbar_wait(bar(P::BAR_FULL + slot), phase, ab, 72));
      if (!ok) break;
      float s[2][4] = {};
      {
        const uint32_t tile = ring + slot * P::SLOT;
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
          uint32_t b[4];
          ldmatrix4(at(tile, k_row, 2 * kk + k_piece), b);
          mma16816(s[0], qf[kk], b[0], b[1]);
          mma16816(s[1], qf[kk], b[2], b[3]);
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(P::BAR_FREE + slot));
      if (++slot == P::NSLOTS) { slot = 0; phase ^= 1; }
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[n][i] *= scale;
      const bool special = k0 + kTile > no_mask;
      if (special) {
        const int key = k0 + warp * 16;
        const uint32_t seen0 = g < rows ? seen32(a, u, g / a.group, key) : 0u, seen1 = g + 8 < rows ? seen32(a, u, (g + 8) / a.group, key) : 0u;
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            if (!((seen0 >> (n * 8 + 2 * q + i)) & 1)) s[n][i] = -CUDART_INF_F;
            if (!((seen1 >> (n * 8 + 2 * q + i)) & 1)) s[n][2 + i] = -CUDART_INF_F;
          }
      }
      const float x0 = fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[1][0], s[1][1])), x1 = fmaxf(fmaxf(s[0][2], s[0][3]), fmaxf(s[1][2], s[1][3]));
      if (__any_sync(0xffffffffu, x0 > m0 + 8.f || x1 > m1 + 8.f)) {
        // the row's maximum over its four lanes; references are whole numbers, as above
        float t0 = fmaxf(x0, __shfl_xor_sync(0xffffffffu, x0, 1)), t1 = fmaxf(x1, __shfl_xor_sync(0xffffffffu, x1, 1));
        t0 = fmaxf(t0, __shfl_xor_sync(0xffffffffu, t0, 2));
        t1 = fmaxf(t1, __shfl_xor_sync(0xffffffffu, t1, 2));
        const float n0 = t0 > m0 + 8.f ? ceilf(t0) : m0, n1 = t1 > m1 + 8.f ? ceilf(t1) : m1;
        const float f0 = ex2_approx(m0 - n0), f1 = ex2_approx(m1 - n1);
        l0 *= f0;
        l1 *= f1;
        m0 = n0;
        m1 = n1;
#pragma unroll
        for (int n = 0; n < D / 8; ++n) { o[n][0] *= f0; o[n][1] *= f0; o[n][2] *= f1; o[n][3] *= f1; }
      }
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        s[n][0] = ex2_approx(s[n][0] - m0);
        s[n][1] = ex2_approx(s[n][1] - m0);
        s[n][2] = ex2_approx(s[n][2] - m1);
        s[n][3] = ex2_approx(s[n][3] - m1);
        l0 += s[n][0] + s[n][1];
        l1 += s[n][2] + s[n][3];
      }
      const uint32_t pf[4] = {cvt_bf16x2(s[0][0], s[0][1]), cvt_bf16x2(s[0][2], s[0][3]), cvt_bf16x2(s[1][0], s[1][1]), cvt_bf16x2(s[1][2], s[1][3])};
      ok = __all_sync(0xffffffffu, mbar_wait(bar(P::BAR_FULL + slot), phase, ab, 73));
      if (!ok) break;
      if (special) {
        // values behind the sequence count as zero, and so do non-finite ones of new tokens (see add_nonfinite)
        const int lo = max(no_mask - k0, warp * 16);
        if (lo < warp * 16 + 16) {
          clean_values<D>(reinterpret_cast<uint32_t*>(smem + P::NRING_OFF + slot * P::SLOT) + lane, lo, warp * 16 + 16, u.len - k0, bad_tag, seq + 1);
          fence_async_smem();
        }
        __syncwarp();
      }
      {
        const uint32_t tile = ring + slot * P::SLOT;
#pragma unroll
        for (int n = 0; n < D / 8; n += 2) {
          uint32_t b[4];
          ldmatrix4t(at(tile, v_row, n + v_piece), b);
          mma16816(o[n], pf, b[0], b[1]);
          mma16816(o[n + 1], pf, b[2], b[3]);
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(P::BAR_FREE + slot));
      if (++slot == P::NSLOTS) { slot = 0; phase ^= 1; }
    }
    // the row's weight over its four lanes, then the eight warps' references and weights
    l0 += __shfl_xor_sync(0xffffffffu, l0, 1);
    l1 += __shfl_xor_sync(0xffffffffu, l1, 1);
    l0 += __shfl_xor_sync(0xffffffffu, l0, 2);
    l1 += __shfl_xor_sync(0xffffffffu, l1, 2);
    if (q == 0) {
      ex[warp * kNarrowRows + g] = make_float2(m0, l0);
      ex[warp * kNarrowRows + g + 8] = make_float2(m1, l1);
    }
    if (!bar_and(1, 256, ok)) break;
    float top0 = kNoMax, top1 = kNoMax;
#pragma unroll
    for (int w = 0; w < 8; ++w) {
      top0 = fmaxf(top0, ex[w * kNarrowRows + g].x);
      top1 = fmaxf(top1, ex[w * kNarrowRows + g + 8].x);
    }
    const float f0 = ex2_approx(m0 - top0), f1 = ex2_approx(m1 - top1);
    // four rows at a time: each warp its sums, then each thread two columns (one) of a row from the eight warps
#pragma unroll 1
    for (int r0 = 0; r0 < rows; r0 += P::SUM_ROWS) {
      if (r0 > 0) bar_sync(1, 256);
      const int in = g - (r0 & 7);                  // this lane's row among them
      if (in >= 0 && in < P::SUM_ROWS) {
        float* mine_at = sums + (warp * P::SUM_ROWS + in) * P::SUM_STRIDE + 2 * q;
        if (r0 < 8) {
#pragma unroll
          for (int n = 0; n < D / 8; ++n) *reinterpret_cast<float2*>(mine_at + n * 8) = make_float2(o[n][0] * f0, o[n][1] * f0);
        } else {
#pragma unroll
          for (int n = 0; n < D / 8; ++n) *reinterpret_cast<float2*>(mine_at + n * 8) = make_float2(o[n][2] * f1, o[n][3] * f1);
        }
      }
      bar_sync(1, 256);
      constexpr int PER = P::SUM_ROWS * D / 256;    // columns of a thread
      const int sub = threadIdx.x >> 6, row = r0 + sub, col = (threadIdx.x & 63) * PER;
      if (row < rows) {
        float top = kNoMax, all = 0.f, y[PER] = {};
#pragma unroll
        for (int w = 0; w < 8; ++w) top = fmaxf(top, ex[w * kNarrowRows + row].x);
#pragma unroll 4
        for (int w = 0; w < 8; ++w) {
          all += ex[w * kNarrowRows + row].y * ex2_approx(ex[w * kNarrowRows + row].x - top);
#pragma unroll
          for (int i = 0; i < PER; ++i) y[i] += sums[(w * P::SUM_ROWS + sub) * P::SUM_STRIDE + col + i];
        }
        const Place p = place_of(a, u, row);
        const float inv = all != 0.f ? 1.f / all : 0.f;
        if (!p.whole) {
#pragma unroll
          for (int i = 0; i < PER; ++i) work.part[p.slot * D + col + i] = y[i];
        } else if constexpr (PER == 2) {
          *reinterpret_cast<uint32_t*>(p.out + col) = pack_bf16(y[0] * inv, y[1] * inv);
        } else {
          p.out[col] = __float2bfloat16(y[0] * inv);
        }
        if ((threadIdx.x & 63) == 0) write_weight(a, work, u, p, top, all);
      }
    }
    if (bad_tag[(seq + 1) % 8] == seq + 1) {
      bar_sync(1, 256);                             // the rows are written
      if (threadIdx.x < rows) {
        const Place p = place_of(a, u, threadIdx.x);
        if (p.whole) add_nonfinite(a, u, p.token, p.out, 0, D);
        else add_nonfinite(a, u, p.token, work.part + p.slot * D, 0, D);
      }
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(bar(P::BAR_UFREE + e));
  }
}

// Positions in the ring, a CTA's tile j of n, K `lead` tiles ahead of V: K j + max(0, j - lead), V behind the K of tile j + lead
// (lead 2: K0 K1 K2 V0 K3 V1 ... K(n-1) V(n-3) V(n-2) V(n-1)).
constexpr uint32_t kWideLead = 1, kTallLead = 2;
__device__ __forceinline__ uint32_t k_pos(uint32_t j, uint32_t lead) { return j + (j > lead ? j - lead : 0u); }
__device__ __forceinline__ uint32_t v_pos(uint32_t j, uint32_t n, uint32_t lead) { return min(2 * j + 1 + lead, n + j); }

// P of 32 logits: exponentials, bf16 pairs; their sum.
__device__ __forceinline__ float weights(const uint32_t (&s)[32], float scale, float m, uint32_t (&p)[16]) {
  auto val = [&](int e) { return __uint_as_float(s[e]); };
  const float2 sc2 = make_float2(scale, scale), nm2 = make_float2(-m, -m);
  float2 sum01 = make_float2(0.f, 0.f), sum23 = make_float2(0.f, 0.f);
#pragma unroll
  for (int e = 0; e < 32; e += 4) {
    float2 x01 = __ffma2_rn(make_float2(val(e), val(e + 1)), sc2, nm2);
    float2 x23 = __ffma2_rn(make_float2(val(e + 2), val(e + 3)), sc2, nm2);
    x01.x = ex2_approx(x01.x);
    x01.y = ex2_approx(x01.y);
    x23.x = ex2_approx(x23.x);
    x23.y = ex2_approx(x23.y);
    sum01 = __fadd2_rn(sum01, x01);
    sum23 = __fadd2_rn(sum23, x23);
    p[e / 2] = cvt_bf16x2(x01.x, x01.y);
    p[e / 2 + 1] = cvt_bf16x2(x23.x, x23.y);
  }
  return (sum01.x + sum01.y) + (sum23.x + sum23.y);
}

// The issuer of the tall mode: one thread.  (The long loops are functions of their own: in one body each pays for the others' registers, 10 us
// of 180 for 128K keys and a tree of 64.)
template <int D>
__device__ __noinline__ void issue_tall(const TreeAttnArgs& a, uint8_t* smem, const Abort& ab, uint32_t tmem, uint32_t n_tiles_cta) {
  using P = Plan<D>;
  const uint32_t base = smem_u32(smem);
  auto bar = [&](int which) { return base + P::MISC_OFF + which * 8; };
  Unit* units = reinterpret_cast<Unit*>(smem + P::UNIT_OFF);
  volatile int* abort_flag = reinterpret_cast<int*>(smem + P::RUN_OFF + 3 * 8) + 1;
  constexpr uint32_t idesc_qk = instr_desc(128, kTile, 0, 0), idesc_pv = instr_desc(128, D, 0, 1);
  const uint32_t d_q = (uint32_t)smem_desc(base, 16, P::GROUP), d_k = (uint32_t)smem_desc(base + P::RING_OFF, 16, P::GROUP),
                 d_v = (uint32_t)smem_desc(base + P::RING_OFF, P::BOX, P::GROUP);
  // One thread does all of this, and every instruction of its loops delays the tiles: 32-bit counters, no arrays that are
  // indexed at run time.  Tiles are seen to arrive in the order of the ring: a barrier's parity tells which phase is
  // over only to one who has seen the phase before it.
  uint32_t arrived = 0, a_slot = 0, a_phase = 0, polls = 0;
  long long idle_since = 0;
  auto arrival = [&] {
    ++arrived;
    if (++a_slot == P::SLOTS) { a_slot = 0; a_phase ^= 1; }
  };
  auto stalled = [&](bool moved) {                 // true: give up
    if (moved) {
      idle_since = 0;
      polls = 0;
      return false;
    }
    if ((++polls & 63u) != 0u) return false;
    if (*abort_flag) return true;
    if ((polls & 4095u) != 0u) return false;
    const long long now = clock64();
    if (idle_since == 0) idle_since = now;
    else if (now - idle_since > kWaitCycles) {
      *abort_flag = 1;
      report_timeout(a.status, 60);
      return true;
    }
    return false;
  };
  auto issue_qk = [&](uint32_t col, uint32_t half, uint32_t slot) {
    const uint32_t dq = d_q + half * (P::QHALF >> 4), dk = d_k + slot * (P::SLOT >> 4);
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk)
      mma_ss_lo<D>(tmem + P::S_COL + col, dq + (kk >> 2) * (P::BOX >> 4) + (kk & 3) * 2, dk + (kk >> 2) * (P::BOX >> 4) + (kk & 3) * 2, idesc_qk, kk > 0);
  };
  auto issue_pv = [&](uint32_t o_col, uint32_t col, uint32_t slot, bool first) {
    const uint32_t dv = d_v + slot * (P::SLOT >> 4);
#pragma unroll
    for (int kk = 0; kk < kTile / 16; ++kk)
      mma_ts_lo<D>(tmem + o_col, tmem + P::S_COL + col + kk * 8, dv + kk * (2 * P::GROUP >> 4), idesc_pv, kk > 0 || !first);
  };
  // Tall.  S of tile i in buffer i % 3, computed up to three tiles ahead of its product with V.
  uint32_t n_qk = 0, n_pv = 0, q_buf = 0, p_buf = 0, p_phase = 0;
  uint32_t k_slot = 0, v_slot = v_pos(0, n_tiles_cta, kTallLead) % P::SLOTS, k_at = 0, v_at = v_pos(0, n_tiles_cta, kTallLead);
  uint32_t left = 0, seq = 0, pv_unit = 0;
  uint32_t first = 0, last = 0;                  // bit b: the tile in buffer b opens / ends its unit's sum
  bool q_here = false, fresh = false;
  while (n_pv != n_tiles_cta) {
    bool moved = false;
    // a poll is a round trip to shared memory, 200 cycles and more while the tensor core streams from it
    const uint32_t polled = mbar_test3(bar(P::BAR_P + p_buf), p_phase, bar(P::BAR_OFREE), (pv_unit + 1) & 1, bar(P::BAR_FULL + a_slot), a_phase);
    if ((polled & 4) && arrived != 2 * n_tiles_cta) {
      arrival();
      moved = true;
    }
    const bool opens = (first >> p_buf) & 1;
    if (n_qk != n_pv && v_at < arrived && (polled & 1) && (!opens || pv_unit == 0 || (polled & 2))) {
      // (the first product of a unit overwrites O: the groups have read the last unit's)
      tc_fence_after();
      issue_pv(P::TALL_O_COL, p_buf * 128, v_slot, opens);
      mma_commit(bar(P::BAR_FREE + v_slot));
      if ((last >> p_buf) & 1) {
        mma_commit(bar(P::BAR_OFULL));
        ++pv_unit;
      }
      ++n_pv;
      const uint32_t to = v_pos(n_pv, n_tiles_cta, kTallLead);
      v_slot += to - v_at;
      v_at = to;
      if (v_slot >= P::SLOTS) v_slot -= P::SLOTS;
      if (++p_buf == 3) { p_buf = 0; p_phase ^= 1; }
      moved = true;
    }
    if (n_qk != n_tiles_cta && n_qk - n_pv < 3) {
      if (left == 0) {
        const uint32_t e = seq % kUnitRing;
        if (mbar_test(bar(P::BAR_UNIT + e), (seq / kUnitRing) & 1)) {
          left = units[e].n_tiles;
          mbar_arrive(bar(P::BAR_UFREE + e));
          ++seq;
          q_here = false;
          fresh = true;
        }
      }
      if (left != 0 && k_at < arrived) {
        const uint32_t half = (seq - 1) & 1;
        if (!q_here) q_here = mbar_test(bar(P::BAR_QFULL + half), ((seq - 1) >> 1) & 1);
        if (q_here) {
          tc_fence_after();
          issue_qk(q_buf * 128, half, k_slot);
          mma_commit(bar(P::BAR_S + q_buf));
          mma_commit(bar(P::BAR_FREE + k_slot));
          --left;
          if (left == 0) mma_commit(bar(P::BAR_QFREE + half));
          const uint32_t bit = 1u << q_buf;
          first = fresh ? first | bit : first & ~bit;
          last = left == 0 ? last | bit : last & ~bit;
          fresh = false;
          ++n_qk;
          const uint32_t to = k_pos(n_qk, kTallLead);
          k_slot += to - k_at;
          k_at = to;
          if (k_slot >= P::SLOTS) k_slot -= P::SLOTS;
          if (++q_buf == 3) q_buf = 0;
          moved = true;
        }
      }
    }
    if (stalled(moved)) break;
  }
}

// The issuer of a wide unit's group x (there are two such threads).  Keys come 64 at a time here: S of 128 rows is 64 columns,
// and each group has two of them, so that the next S is computed during the softmax of this one.
template <int D>
__device__ __noinline__ void issue_wide(const TreeAttnArgs& a, uint8_t* smem, uint32_t bars, const Abort& ab, uint32_t tmem, uint32_t n_tiles_cta, uint32_t x) {
  using P = Plan<D>;
  const uint32_t base = smem_u32(smem);
  auto bar = [&](int which) { return bars + which * 8; };
  Unit* units = reinterpret_cast<Unit*>(smem + P::UNIT_OFF);
  volatile int* abort_flag = reinterpret_cast<int*>(smem + P::RUN_OFF + 3 * 8) + 1;
  constexpr uint32_t idesc_qk = instr_desc(128, kTile / 2, 0, 0), idesc_pv = instr_desc(128, D, 0, 1);
  const uint32_t d_q = (uint32_t)smem_desc(base, 16, P::GROUP), d_k = (uint32_t)smem_desc(base + P::RING_OFF, 16, P::GROUP),
                 d_v = (uint32_t)smem_desc(base + P::RING_OFF, P::BOX, P::GROUP);
  uint32_t arrived = 0, a_slot = 0, a_phase = 0, polls = 0;
  long long idle_since = 0;
  auto arrival = [&] {
    ++arrived;
    if (++a_slot == P::SLOTS) { a_slot = 0; a_phase ^= 1; }
  };
  auto stalled = [&](bool moved) {                 // true: give up
    if (moved) {
      idle_since = 0;
      polls = 0;
      return false;
    }
    if ((++polls & 63u) != 0u) return false;
    if (*abort_flag) return true;
    if ((polls & 4095u) != 0u) return false;
    const long long now = clock64();
    if (idle_since == 0) idle_since = now;
    else if (now - idle_since > kWaitCycles) {
      *abort_flag = 1;
      report_timeout(a.status, 60);
      return true;
    }
    return false;
  };
  const uint32_t s_col = P::S_COL + x * 128, o_col = P::O_COL + x * P::O_STEP, n = 2 * n_tiles_cta, lead = kWideLead;
  const uint32_t dq = d_q + x * (P::QHALF >> 4);
  constexpr uint32_t half = kTile / 2 / 8 * P::GROUP >> 4;          // from the first 64 keys of a tile to the others
  uint32_t n_qk = 0, n_pv = 0, left = 0, seq = 0;      // products issued; halves left of the unit; units taken
  uint32_t k_at = 0, k_slot = 0, v_at = v_pos(0, n_tiles_cta, lead), v_slot = v_at % P::SLOTS;
  uint32_t first = 0;                                  // bit b: what is in buffer b opens its unit's sum
  bool q_here = false, fresh = false;
  auto advance = [&](uint32_t& at, uint32_t& slot, uint32_t to) {
    slot += to - at;
    at = to;
    if (slot >= P::SLOTS) slot -= P::SLOTS;
  };
  while (n_pv != n) {
    bool moved = false;
    const uint32_t polled = mbar_test2(bar(P::BAR_P + 2 * x + (n_pv & 1)), (n_pv >> 1) & 1, bar(P::BAR_FULL + a_slot), a_phase);
    if ((polled & 2) && arrived != n) {
      arrival();
      moved = true;
    }
    if (n_qk != n_pv && v_at < arrived && (polled & 1)) {
      const uint32_t b = n_pv & 1, dv = d_v + v_slot * (P::SLOT >> 4) + b * half;
      const bool opens = (first >> b) & 1;
      tc_fence_after();
#pragma unroll
      for (int kk = 0; kk < kTile / 32; ++kk)
        mma_ts_lo<D>(tmem + o_col, tmem + s_col + b * 64 + kk * 8, dv + kk * (2 * P::GROUP >> 4), idesc_pv, kk > 0 || !opens);
      mma_commit(bar(P::BAR_PV + 2 * x + b));
      if (b == 1) {
        mma_commit(bar(P::BAR_FREE + v_slot));
        advance(v_at, v_slot, v_pos((n_pv + 1) >> 1, n_tiles_cta, lead));
      }
      ++n_pv;
      moved = true;
    }
    if (n_qk != n && n_qk - n_pv < 2) {
      if (left == 0) {
        const uint32_t e = seq % kUnitRing;
        if (mbar_test(bar(P::BAR_UNIT + e), (seq / kUnitRing) & 1)) {
          left = 2 * units[e].n_tiles;
          mbar_arrive(bar(P::BAR_UFREE + e));
          ++seq;
          q_here = false;
          fresh = true;
        }
      }
      if (left != 0 && k_at < arrived) {
        if (!q_here) q_here = mbar_test(bar(P::BAR_QFULL + x), (seq - 1) & 1);
        if (q_here) {
          const uint32_t b = n_qk & 1, dk = d_k + k_slot * (P::SLOT >> 4) + b * half;
          tc_fence_after();
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk)
            mma_ss_lo<D>(tmem + s_col + b * 64, dq + (kk >> 2) * (P::BOX >> 4) + (kk & 3) * 2, dk + (kk >> 2) * (P::BOX >> 4) + (kk & 3) * 2, idesc_qk, kk > 0);
          mma_commit(bar(P::BAR_S + 2 * x + b));
          if (--left == 0) mma_commit(bar(P::BAR_QFREE + x));
          if (b == 1) {
            mma_commit(bar(P::BAR_FREE + k_slot));
            advance(k_at, k_slot, k_pos((n_qk + 1) >> 1, lead));
          }
          first = fresh ? first | 1u << b : first & ~(1u << b);
          fresh = false;
          ++n_qk;
          moved = true;
        }
      }
    }
    if (stalled(moved)) break;
  }
}

// Softmax and epilogue, wide: a group for each half of the rows.
template <int D>
__device__ __noinline__ void softmax_wide(const TreeAttnArgs& a, const Work& work, uint8_t* smem, uint32_t bars, const Abort& ab, uint32_t tmem, uint32_t n_tiles_cta) {
  using P = Plan<D>;
  const uint32_t base = smem_u32(smem);
  auto bar = [&](int which) { return bars + which * 8; };
  Unit* units = reinterpret_cast<Unit*>(smem + P::UNIT_OFF);
  volatile int* abort_flag = reinterpret_cast<int*>(smem + P::RUN_OFF + 3 * 8) + 1;
  volatile int* bad_tag = reinterpret_cast<int*>(smem + P::TAG_OFF);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int x = warp >> 2;                          // group
  const int row = threadIdx.x & 127;                // TMEM lane, row of the group
  const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16);
  const float scale = a.scale_log2;
  // The V of a tile with masked keys: what lies behind the sequence counts as zero, and so do non-finite values of new
  // tokens (see add_nonfinite).  V comes after K, hence not before the softmax.  S of the tile was there, so every tile up
  // to its K has arrived, the one before V in V's slot among them: the barrier's parity can be told.
  auto clean = [&](uint32_t j, const Unit& u, int k0, int half, int no_mask, int seq) {
    const uint32_t p = v_pos(j, n_tiles_cta, kWideLead), s = p % P::SLOTS;
    const bool here = __all_sync(0xffffffffu, mbar_wait(bar(P::BAR_FULL + s), (p / P::SLOTS) & 1, ab, 32));
    // each warp of the group 16 keys
    const int from = half * 64 + (warp & 3) * 16, lo = max(no_mask - k0, from);
    if (here && lo < from + 16)
      clean_values<D>(reinterpret_cast<uint32_t*>(smem + P::RING_OFF + s * P::SLOT) + lane, lo, from + 16, u.len - k0, bad_tag, seq + 1);
    fence_async_smem();
    return here;
  };
  bool ok = true;
  uint32_t done = 0;                                // tiles of earlier units
  const uint32_t t_o = lanes + P::O_COL + x * P::O_STEP;
  for (int seq = 0; ok; ++seq) {
    const int e = seq % kUnitRing;
    ok = __all_sync(0xffffffffu, mbar_wait(bar(P::BAR_UNIT + e), (seq / kUnitRing) & 1, ab, 30));
    if (!ok) break;
    const Unit& u = units[e];                     // stays in shared memory until the unit is done: registers are short
    const int n_tiles = u.n_tiles;
    if (n_tiles == 0) break;
    const int my_row = x * 128 + row;
    const bool warp_live = x * 128 + (warp & 3) * 32 < u.rows, live = my_row < u.rows;
    const int token = (u.r0 + my_row) / a.group;
    const int kt0 = u.kt0, no_mask = min(u.past, u.len);      // keys before it are seen by every row
    float m_ref = live ? kNoMax : -kNoMax, l = 0.f;           // lanes without a row: all weights zero
    for (int t = 0; t < 2 * n_tiles && ok; ++t) {
      const int k0 = (kt0 + (t >> 1)) * kTile, half = t & 1;      // half a tile in buffer `half`
      const uint32_t t_s = lanes + P::S_COL + x * 128 + half * 64, phase = (done + (t >> 1)) & 1;
      const bool special = k0 + half * 64 + 64 > no_mask;
      ok = __all_sync(0xffffffffu, mbar_wait(bar(P::BAR_S + 2 * x + half), phase, ab, 31));
      if (!ok) break;
      tc_fence_after();
      if (warp_live) {
        // Two chunks of 32 logits, the next one's load in flight, each a step of the running softmax
        if (special) mask_tmem(a, u, live ? token : -1, k0 + half * 64, 64, t_s);
        uint32_t s[2][32];
        float sum = 0.f;
        tmem_ld32_async(t_s, s[0]);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          tmem_ld_wait();
          reg_fence32(s[c & 1]);
          const uint32_t* y = s[c & 1];
          auto val = [&](int i) { return __uint_as_float(y[i]); };
          float m0 = max3(val(0), val(1), val(2)), m1 = max3(val(3), val(4), val(5)), m2 = max3(val(6), val(7), val(8)),
                m3 = max3(val(9), val(10), val(11));
#pragma unroll
          for (int i = 12; i < 28; i += 8) {
            m0 = max3(m0, val(i), val(i + 1));
            m1 = max3(m1, val(i + 2), val(i + 3));
            m2 = max3(m2, val(i + 4), val(i + 5));
            m3 = max3(m3, val(i + 6), val(i + 7));
          }
          m0 = max3(m0, val(28), val(29));
          m1 = max3(m1, val(30), val(31));
          const float mx = fmaxf(fmaxf(m0, m1), fmaxf(m2, m3)) * scale;
          const bool grown = mx > m_ref + 8.f;              // never in lanes without a row
          if (__any_sync(0xffffffffu, grown)) {
            const float m_new = grown ? ceilf(mx) : m_ref;
            const float alpha = ex2_approx(m_ref - m_new);
            // nothing of this P has been handed over; the product of the P before it has to be in O (those before that are:
            // their buffer is this S's, and the barrier's parity can be told)
            if (t > 0) {
              ok = __all_sync(0xffffffffu, mbar_wait(bar(P::BAR_PV + 2 * x + (half ^ 1)), half ? phase : phase ^ 1, ab, 35));
              tc_fence_after();
            }
            rescale_tmem<D>(t_o, t_s, alpha, c, t > 0);
            l *= alpha;
            sum *= alpha;
            m_ref = m_new;
          }
          // not before the call above: its registers must not be moved while the load is under way
          if (c < 1) tmem_ld32_async(t_s + 32, s[1]);
          uint32_t p[16];
          sum += weights(s[c & 1], scale, m_ref, p);
          tmem_st16(t_s + c * 16, p);
        }
        l += sum;
        tmem_wait_st();
      }
      if (special && ok) ok = clean(done + (t >> 1), u, k0, half, no_mask, seq);
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(P::BAR_P + 2 * x + half));
    }
    if (ok) ok = __all_sync(0xffffffffu, mbar_wait(bar(P::BAR_PV + 2 * x + 1), (done + n_tiles - 1) & 1, ab, 33));
    if (ok && warp_live) {
      tc_fence_after();
      const Place p = place_of(a, u, my_row);
      float* part = p.whole ? nullptr : work.part + p.slot * D;
      write_columns(t_o, 0, D, !p.whole ? 1.f : l != 0.f ? 1.f / l : 0.f, live, p.out, part);
      if (live) {
        if (bad_tag[(seq + 1) % 8] == seq + 1) {
          if (p.whole) add_nonfinite(a, u, p.token, p.out, 0, D);
          else add_nonfinite(a, u, p.token, part, 0, D);
        }
        write_weight(a, work, u, p, m_ref, l);
      }
      __syncwarp();
      tc_fence_before();                          // O has left TMEM: before the P after which the next product overwrites it
    }
    done += n_tiles;
    __syncwarp();
    if (lane == 0) mbar_arrive(bar(P::BAR_UFREE + e));
  }
}

// Softmax and epilogue, tall: the groups take the tiles in turn.
template <int D>
__device__ __noinline__ void softmax_tall(const TreeAttnArgs& a, const Work& work, uint8_t* smem, const Abort& ab, uint32_t tmem, uint32_t n_tiles_cta) {
  using P = Plan<D>;
  const uint32_t base = smem_u32(smem);
  auto bar = [&](int which) { return base + P::MISC_OFF + which * 8; };
  Unit* units = reinterpret_cast<Unit*>(smem + P::UNIT_OFF);
  volatile int* abort_flag = reinterpret_cast<int*>(smem + P::RUN_OFF + 3 * 8) + 1;
  volatile int* bad_tag = reinterpret_cast<int*>(smem + P::TAG_OFF);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int x = warp >> 2;                          // group
  const int row = threadIdx.x & 127;                // TMEM lane, row of the group
  const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16);
  const float scale = a.scale_log2;
  volatile int* redo = abort_flag + 2;
  // The V of a tile with masked keys: what lies behind the sequence counts as zero, and so do non-finite values of new
  // tokens (see add_nonfinite).  V comes after K, hence not before the softmax.  S of the tile was there, so every tile up
  // to its K has arrived, the one before V in V's slot among them: the barrier's parity can be told.
  auto clean = [&](uint32_t j, const Unit& u, int k0, int no_mask, int seq) {
    const uint32_t p = v_pos(j, n_tiles_cta, kTallLead), s = p % P::SLOTS;
    const bool here = __all_sync(0xffffffffu, mbar_wait(bar(P::BAR_FULL + s), (p / P::SLOTS) & 1, ab, 32));
    // each warp of the group 32 keys
    const int lo = max(no_mask - k0, (warp & 3) * 32);
    if (here && lo < (warp & 3) * 32 + 32)
      clean_values<D>(reinterpret_cast<uint32_t*>(smem + P::RING_OFF + s * P::SLOT) + lane, lo, (warp & 3) * 32 + 32, u.len - k0, bad_tag, seq + 1);
    fence_async_smem();
    return here;
  };
  bool ok = true;
  uint32_t done = 0;                                // tiles of earlier units
  const uint32_t t_o = lanes + P::TALL_O_COL;
  float* ex = reinterpret_cast<float*>(smem + P::EX_OFF);            // [group][row] weight, -1: nothing seen
  float* refs = reinterpret_cast<float*>(smem + P::REF_OFF);         // [row]
  for (int seq = 0;; ++seq) {
    const int e = seq % kUnitRing;
    ok = __all_sync(0xffffffffu, ok && mbar_wait(bar(P::BAR_UNIT + e), (seq / kUnitRing) & 1, ab, 30));
    // the eight warps go on together or stop together: none is left at the barriers below
    if (!bar_and(1, 256, ok)) break;
    const Unit& u = units[e];
    const int n_tiles = u.n_tiles;
    if (n_tiles == 0) break;
    const bool warp_live = (warp & 3) * 32 < u.rows, live = row < u.rows;
    const int token = (u.r0 + row) / a.group;
    const int kt0 = u.kt0, no_mask = min(u.past, u.len);
    const int t0 = (int)((done + x) & 1);         // the CTA's tiles in turn: tile i is of group i & 1, in buffer i % 3
    float m_ref = -kNoMax, l = 0.f;
    bool have_ref = false, saw = false;
    for (int t = t0; t < n_tiles && ok; t += 2) {
      const uint32_t i = done + t, buf = i % 3;
      const uint32_t t_s = lanes + P::S_COL + buf * 128;
      const int k0 = (kt0 + t) * kTile;
      const bool special = k0 + kTile > no_mask;
      ok = __all_sync(0xffffffffu, mbar_wait(bar(P::BAR_S + buf), (i / 3) & 1, ab, 31));
      if (!ok) break;
      tc_fence_after();
      if (warp_live) saw |= special ? mask_tmem(a, u, live ? token : -1, k0, kTile, t_s) : true;
      if (t == 0) {
        if (warp_live) refs[row] = first_reference(t_s, scale, live);
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(P::BAR_REF));
      }
      if (!have_ref) {
        ok = __all_sync(0xffffffffu, mbar_wait(bar(P::BAR_REF), seq & 1, ab, 34));
        if (!ok) break;
        m_ref = live ? refs[row] : -kNoMax;
        have_ref = true;
      }
      if (warp_live) {
        uint32_t s[2][32];
        tmem_ld32_async(t_s, s[0]);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          tmem_ld_wait();
          reg_fence32(s[c & 1]);
          if (c < 3) tmem_ld32_async(t_s + (c + 1) * 32, s[(c + 1) & 1]);
          uint32_t p[16];
          l += weights(s[c & 1], scale, m_ref, p);
          tmem_st16(t_s + c * 16, p);
        }
        tmem_wait_st();
      }
      if (special) ok = clean(i, u, k0, no_mask, seq);
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(P::BAR_P + buf));
    }
    if (ok && !have_ref) {                        // a unit of one tile, the other group's
      ok = __all_sync(0xffffffffu, mbar_wait(bar(P::BAR_REF), seq & 1, ab, 34));
      if (ok) m_ref = live ? refs[row] : -kNoMax;
    }
    if (ok) ok = __all_sync(0xffffffffu, mbar_wait(bar(P::BAR_OFULL), seq & 1, ab, 33));
    ex[x * 128 + row] = saw ? l : -1.f;
    if (!bar_and(1, 256, ok)) break;
    tc_fence_after();
    if (warp_live) {
      const float l0 = ex[row], l1 = ex[128 + row];
      const bool seen = l0 != -1.f || l1 != -1.f;
      l = (l0 == -1.f ? 0.f : l0) + (l1 == -1.f ? 0.f : l1);
      const Place p = place_of(a, u, row);
      float* part = p.whole ? nullptr : work.part + p.slot * D;
      const int lo = x * (D / 2);                 // each group half of the columns
      const bool finite = write_columns(t_o, lo, lo + D / 2, !p.whole ? 1.f : l != 0.f ? 1.f / l : 0.f, live, p.out, part);
      if (live) {
        if (seen && (l > kTallMost || l < kTallLeast || (l > 256.f && !finite))) *redo = 1;
        if (bad_tag[(seq + 1) % 8] == seq + 1) {
          if (p.whole) add_nonfinite(a, u, p.token, p.out, lo, lo + D / 2);
          else add_nonfinite(a, u, p.token, part, lo, lo + D / 2);
        }
        if (x == 0) write_weight(a, work, u, p, l != 0.f ? m_ref : kNoMax, l);
      }
      __syncwarp();
    }
    tc_fence_before();
    __syncwarp();
    if (lane == 0) {
      mbar_arrive(bar(P::BAR_OFREE));
      mbar_arrive(bar(P::BAR_UFREE + e));
    }
    done += n_tiles;
  }
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
tree_attn_kernel(const __grid_constant__ TreeAttnArgs a, const __grid_constant__ Work work, const __grid_constant__ CUtensorMap tm_k,
                 const __grid_constant__ CUtensorMap tm_v) {
  using P = Plan<D>;
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t base = smem_u32(smem);
  uint32_t bars = base + P::MISC_OFF;
  auto bar = [&](int which) { return bars + which * 8; };
  Unit* units = reinterpret_cast<Unit*>(smem + P::UNIT_OFF);
  long long* scan = reinterpret_cast<long long*>(smem + P::SCAN_OFF);
  long long* start_rem = reinterpret_cast<long long*>(smem + P::RUN_OFF);      // steps of the request before the run
  long long* tiles_at = start_rem + 1;             // tiles before the run's begin and end
  int* words = reinterpret_cast<int*>(smem + P::RUN_OFF + 3 * 8);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(words);
  volatile int* abort_flag = words + 1;
  int* start_b = words + 2;                        // request in which the run begins
  volatile int* redo = words + 3;                  // tall: the references did not serve
  // number, from 1, of a unit in which a non-finite value was met, at that number modulo 8 (the groups of wide units are two
  // units apart at most)
  volatile int* bad_tag = reinterpret_cast<int*>(smem + P::TAG_OFF);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int cta = blockIdx.x, n_cta = gridDim.x;
  const Abort ab{abort_flag, a.status};

  let_next_start();
  const bool misplaced = (base & 1023u) != 0;      // the tiles' swizzle needs the window's alignment
  if (warp == kProducer && lane < 2) asm volatile("prefetch.tensormap [%0];" ::"l"(lane == 0 ? &tm_k : &tm_v) : "memory");
  if (threadIdx.x == 0) {
    *abort_flag = *redo = 0;
    for (int i = 0; i < 8; ++i) bad_tag[i] = 0;
  }
  wait_for_previous();
  const bool poisoned = decode_poisoned(a.status);

  // ---- where the run begins
  const int per = (a.n_req + kThreads - 1) / kThreads;
  const int b_lo = min((int)threadIdx.x * per, a.n_req), b_hi = min(b_lo + per, a.n_req);
  int unit_rows = kUnitRows;
  long long mine_t = 0, mine_u = 0, more_t = 0;    // tiles, units; tiles in addition with units of 128 rows
  bool many = false, some = false;
  for (int b = b_lo; b < b_hi; ++b) {
    const Request q = request(a, b);
    const long long n = units_of(a, q, unit_rows);
    mine_u += n;
    mine_t += n * q.kt;
    more_t += (units_of(a, q, 128) - n) * q.kt;
    many |= q.n * a.group > 128;
    some |= q.n * a.group > kNarrowRows;
  }
  long long incl_t, incl_u;
  auto sums = [&] {                                // over the threads before and this one; over the warps, in `scan`
    incl_t = mine_t;
    incl_u = mine_u;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long up_t = __shfl_up_sync(0xffffffffu, incl_t, o), up_u = __shfl_up_sync(0xffffffffu, incl_u, o);
      if (lane >= o) { incl_t += up_t; incl_u += up_u; }
    }
    if (lane == 31) { scan[warp] = incl_t; scan[kWarps + warp] = incl_u; }
  };
  sums();
  if (threadIdx.x == 0 && misplaced && atomicCAS(a.status, 0, (int)SP_ERR_UNSUPPORTED) == 0) a.status[1] = 90;
  bool wide = __syncthreads_or(many) != 0;
  const bool narrow = __syncthreads_or(some) == 0;
  if (wide) {
    // Units of 256 rows take half as many tiles again of the time of those of 128 (2.5 and 1.6 us a tile): tall, if cutting
    // them adds no more than that half (one chunk of a prompt among many single tokens, or 257 to 384 rows each: a request of
    // 256 rows among 255 of one token 251 us so, 317 as wide; one of 1024 rows 297 and 487).
    long long tiles = 0;
    for (int w = 0; w < kWarps; ++w) tiles += scan[w];
    __syncthreads();
    for (int o = 16; o > 0; o >>= 1) more_t += __shfl_down_sync(0xffffffffu, more_t, o);
    if (lane == 0) scan[warp] = more_t;
    __syncthreads();
    long long more = 0;
    for (int w = 0; w < kWarps; ++w) more += scan[w];
    __syncthreads();
    wide = 2 * more > tiles;
    if (!wide) {
      unit_rows = 128;
      mine_t = mine_u = 0;
      for (int b = b_lo; b < b_hi; ++b) {
        const Request q = request(a, b);
        mine_u += units_of(a, q, unit_rows);
        mine_t += units_of(a, q, unit_rows) * q.kt;
      }
    }
    sums();
    __syncthreads();
  }
  if (!narrow) {
    if (warp == kIssuer) tmem_alloc(smem_u32(tmem_slot), 512);
    // rows of the Q area that no unit fills stay zero: products of whatever lay there would cost power, and with it clock
    for (int i = threadIdx.x; i < 2 * P::QHALF / 16; i += kThreads) reinterpret_cast<uint4*>(smem)[i] = make_uint4(0, 0, 0, 0);
    fence_async_smem();
  }
  const int own = narrow ? kNarrowSteps : kTallSteps;         // a unit's steps besides its tiles'
  long long before_t = incl_t - mine_t, before_u = incl_u - mine_u, total_t = 0, total = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) { before_t += scan[w]; before_u += scan[kWarps + w]; }
    total_t += scan[w];
    total += scan[w] + own * scan[kWarps + w];
  }
  const long long quota = divide(total, n_cta), extra = total - quota * n_cta;      // the first `extra` runs are one step longer
  auto run_begin = [&](int w) { return w * quota + min((long long)w, extra); };
  for (int end = 0; end < 2; ++end) {
    const long long w = run_begin(cta + end);
    long long step = before_t + own * before_u, tile = before_t;
    if (w >= total) {
      if (threadIdx.x == 0) tiles_at[end] = total_t;
    } else if (step <= w && w < step + mine_t + own * mine_u) {
      for (int b = b_lo; b < b_hi; ++b) {
        const Request q = request(a, b);
        const long long n = units_of(a, q, unit_rows);
        if (w < step + n * (q.kt + own)) {
          const long long rem = w - step, nth = divide(rem, q.kt + own), in = rem - nth * (q.kt + own);
          tiles_at[end] = tile + nth * q.kt + max(in - own, 0ll);
          if (end == 0) { *start_b = b; *start_rem = rem; }
          break;
        }
        step += n * (q.kt + own);
        tile += n * q.kt;
      }
    }
  }
  auto init_barriers = [&](uint32_t bars, bool wide) {
    auto bar = [&](int which) { return bars + which * 8; };
    for (int s = 0; s < P::NSLOTS; ++s) mbar_init(bar(P::BAR_FULL + s), 1);
    for (int i = 0; i < 4; ++i) {
      mbar_init(bar(P::BAR_S + i), 1);
      mbar_init(bar(P::BAR_P + i), 4);
      mbar_init(bar(P::BAR_PV + i), 1);
    }
    mbar_init(bar(P::BAR_REF), 4);
    mbar_init(bar(P::BAR_OFULL), 1);
    mbar_init(bar(P::BAR_OFREE), 8);
    // who lets a tile go: the issuer once, or (wide) for each group, or the eight warps; likewise the queries, which come
    // from 32 lanes' copies when narrow; a unit is read by the eight warps, the producer and the issuers, if it has work
    for (int s = 0; s < P::NSLOTS; ++s) mbar_init(bar(P::BAR_FREE + s), narrow ? 8 : wide ? 2 : 1);
    for (int x = 0; x < 2; ++x) {
      mbar_init(bar(P::BAR_QFULL + x), narrow ? 32 : 1);
      mbar_init(bar(P::BAR_QFREE + x), narrow ? 8 : 1);
    }
    for (int e = 0; e < kUnitRing; ++e) {
      mbar_init(bar(P::BAR_UNIT + e), 1);
      mbar_init(bar(P::BAR_UFREE + e), narrow ? 9 : wide ? 11 : 10);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  };
  if (threadIdx.x == 0) init_barriers(bars, wide);
  if (threadIdx.x == 32 && !wide && !narrow) init_barriers(bars + P::BARS * 8, true);
  tc_fence_before();
  const bool idle = __syncthreads_or(poisoned || misplaced) != 0;
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const uint32_t n_tiles_cta = idle ? 0u : (uint32_t)(tiles_at[1] - tiles_at[0]);

  for (;;) {
    const uint32_t lead = narrow ? 0u : wide ? kWideLead : kTallLead;
    if (warp == kLoader) {
      // ------------------------------------------------------------ units and their queries
      bool ok = true;
      int seq = 0;
      if (lane == 0) work.meta[cta].last = -1;
      if (n_tiles_cta > 0) {
        int b = *start_b;
        long long rem = *start_rem, w = run_begin(cta);
        const long long w1 = run_begin(cta + 1);
        Request q = request(a, b);
        while (w < w1 && ok) {
          while (rem >= units_of(a, q, unit_rows) * (q.kt + own) && b + 1 < a.n_req) { rem = 0; q = request(a, ++b); }
          if (rem >= units_of(a, q, unit_rows) * (q.kt + own)) break;       // not reached while the lengths stand still
          Unit u;
          const int n_pass = passes(a, q, unit_rows), all_rows = q.n * a.group;
          const int nth = (int)divide(rem, q.kt + own), in = (int)(rem - (long long)nth * (q.kt + own));       // step of the unit: tile `in - own`
          const int take = (int)min((long long)(q.kt + own - in), w1 - w);
          w += take;
          rem += take;
          u.kt0 = max(in - own, 0);
          u.kt_all = q.kt;
          u.n_tiles = max(in + take - own, 0) - u.kt0;
          if (u.n_tiles == 0) continue;                // only the unit's own step: its tiles are the next CTA's
          u.g = n_pass == 1 ? nth : nth / n_pass;
          u.b = b;
          u.start = q.start;
          u.r0 = (nth - u.g * n_pass) * unit_rows;
          u.rows = min(all_rows - u.r0, unit_rows);
          u.len = q.len;
          u.past = q.past;
          const int e = seq % kUnitRing;
          if (seq >= kUnitRing) ok = __all_sync(0xffffffffu, mbar_wait(bar(P::BAR_UFREE + e), (seq / kUnitRing - 1) & 1, ab, 40));
          if (!ok) break;
          if (lane == 0) {
            units[e] = u;
            mbar_arrive(bar(P::BAR_UNIT + e));
            if (u.kt0 == 0 && u.n_tiles < u.kt_all) {
              const long long z = w - take - in + own - 1 + u.kt_all, cut = extra * (quota + 1);     // the step of the unit's last tile
              Meta m{(int)(z < cut ? divide(z, quota + 1) : extra + divide(z - cut, quota)), u.start, u.r0, u.rows, u.g, {0, 0, 0}};
              work.meta[cta] = m;
            }
            if (a.seq_lens[b] > q.len) report_range(a.status, kWhereTreePage);   // longer than its table row
          }
          // its queries: rows of 128-byte boxes, 16-byte pieces swizzled as the MMA descriptors say.  A lane keeps its
          // piece of every (32 / pieces)-th row, whose token and head advance without division (one division a piece:
          // 13000 cycles for 128 rows).  Narrow and tall: two sets of rows in turn; wide: one of two halves.
          const int first = wide ? 0 : seq & 1, lap = wide ? seq : seq >> 1, halves = wide ? 2 : 1;
          constexpr int PIECES = D / 8, STEP = 32 / PIECES;
          const int piece = lane % PIECES;
          int r = lane / PIECES, hg = (u.r0 + r) % a.group;
          const __nv_bfloat16* src = a.q + (int64_t)(u.g * a.group + hg) * a.q_sh + (int64_t)(u.start + (u.r0 + r) / a.group) * a.q_sn + piece * 8;
          const int64_t down = STEP * a.q_sh, wrap = a.q_sn - a.group * a.q_sh;
          for (int i = 0; i < halves && ok; ++i) {
            const int set = first + i, end = min(u.rows, (i + 1) * 128);
            if (lap > 0) ok = __all_sync(0xffffffffu, mbar_wait(bar(P::BAR_QFREE + set), (lap - 1) & 1, ab, 41));
            if (!ok) break;
            const uint32_t box = base + set * (narrow ? P::NQ_BYTES : P::QHALF) + (piece >> 3) * P::BOX;
#pragma unroll 2
            for (; r < end; r += STEP) {
              cp_async16(box + ((r & 127) >> 3) * P::GROUP + (r & 7) * 128 + (((piece ^ r) & 7) << 4), src);
              src += down;
              hg += STEP;
              while (hg >= a.group) { hg -= a.group; src += wrap; }
            }
            if (narrow) {                              // read by ldmatrix: the copies' arrival is enough, and nobody waits for it here
              asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar(P::BAR_QFULL + set)) : "memory");
            } else {
              asm volatile("cp.async.wait_all;" ::: "memory");
              fence_async_smem();
              __syncwarp();
              if (lane == 0) mbar_arrive(bar(P::BAR_QFULL + set));
            }
          }
          ++seq;
        }
      }
      // no more units
      const int e = seq % kUnitRing;
      if (ok && seq >= kUnitRing) ok = __all_sync(0xffffffffu, mbar_wait(bar(P::BAR_UFREE + e), (seq / kUnitRing - 1) & 1, ab, 40));
      if (ok && lane == 0) {
        units[e].n_tiles = 0;
        mbar_arrive(bar(P::BAR_UNIT + e));
      }
    } else if (warp == kProducer) {
      // ------------------------------------------------------------ K and V tiles
      bool ok = true;
      const uint32_t ring = base + (narrow ? P::NRING_OFF : P::RING_OFF), slots = narrow ? P::NSLOTS : P::SLOTS;
      uint32_t s = 0, lap = 0;                         // next slot of the ring, times round
      const int page = 1 << a.page_log2;
      const int per_tile = max(kTile >> a.page_log2, 1), rows = min(page, kTile);
      struct Tile {                                    // this lane's page of a tile
        int id, off, g;
        bool live;
      };
      auto load = [&](const Tile& tile, const CUtensorMap& map, const CacheSteps& steps) {
        if (ok && lap > 0) ok = __all_sync(0xffffffffu, mbar_wait(bar(P::BAR_FREE + s), (lap - 1) & 1, ab, 51));
        if (!ok) return;
        const int n_live = __popc(__ballot_sync(0xffffffffu, tile.live));
        if (lane == 0) mbar_expect_tx(bar(P::BAR_FULL + s), n_live * rows * D * 2);
        __syncwarp();
        if (tile.live) {
          // (an id outside the cache: outside the tensor map, the load fills in zeros)
          const int at = tile.id < 0 ? steps.extent : tile.id * steps.page + tile.g * steps.head;
          tma_load_5d(ring + s * P::SLOT + lane * (rows / 8 * P::GROUP), &map, bar(P::BAR_FULL + s), 0, 0, 0, tile.off >> 3, at);
        }
        __syncwarp();
        if (++s == slots) { s = 0; ++lap; }
      };
      int seq = 0, kt = 0, kt_end = 0, len = 0, g = 0, b = 0, id = 0;      // id: this lane's page of tile kt
      // lane p looks up page p of the tile, a tile ahead
      auto lookup = [&] {
        const int key = kt * kTile + lane * page;
        return lane < per_tile && key < len ? a.table[(size_t)b * a.max_pages + (key >> a.page_log2)] : -1;
      };
      Tile now{0, 0, 0, false}, last1 = now, last2 = now;      // the tile, and the ones before it
      for (uint32_t j = 0; j < n_tiles_cta && ok; ++j) {
        if (kt == kt_end) {
          const int e = seq % kUnitRing;
          ok = __all_sync(0xffffffffu, mbar_wait(bar(P::BAR_UNIT + e), (seq / kUnitRing) & 1, ab, 50));
          if (!ok) break;
          const Unit& u = units[e];
          kt = u.kt0; kt_end = u.kt0 + u.n_tiles; len = u.len; g = u.g; b = u.b;
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(P::BAR_UFREE + e));
          ++seq;
          id = lookup();
        }
        const int key = kt * kTile + lane * page;
        last2 = last1;
        last1 = now;
        now = Tile{id, key & (page - 1), g, lane < per_tile && key < len};
        if (now.live && (id < 0 || id >= a.n_pages)) {
          report_range(a.status, kWhereTreePage);
          now.id = -1;
        }
        ++kt;
        if (kt < kt_end) id = lookup();
        load(now, tm_k, work.k);
        if (j >= lead) load(lead == 0 ? now : lead == 1 ? last1 : last2, tm_v, work.v);
      }
      if (n_tiles_cta > 1 && lead > 1) load(last1, tm_v, work.v);
      if (n_tiles_cta > 0 && lead > 0) load(now, tm_v, work.v);
      if (*abort_flag && lane == 0) {
        // let the copies already in flight land before the CTA gives its shared memory back
        const long long t0 = clock64();
        for (uint32_t i = 0; i < slots; ++i) {
          const uint32_t laps = lap + (i < s);          // loads that this slot has been given
          while (laps > 0 && !mbar_test(bar(P::BAR_FULL + i), (laps - 1) & 1) && clock64() - t0 < kWaitCycles / 8) {}
        }
      }
    } else if (warp == kIssuer || warp == kIssuer1) {
      if (lane == 0 && wide) issue_wide<D>(a, smem, bars, ab, tmem, n_tiles_cta, warp == kIssuer1);
      else if (lane == 0 && !narrow && warp == kIssuer) issue_tall<D>(a, smem, ab, tmem, n_tiles_cta);
      __syncwarp();
    } else if (narrow) {
      narrow_warps<D>(a, work, smem, ab);
    } else if (wide) {
      softmax_wide<D>(a, work, smem, bars, ab, tmem, n_tiles_cta);
    } else {
      softmax_tall<D>(a, work, smem, ab, tmem, n_tiles_cta);
    }

    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (wide || *redo == 0 || *abort_flag) break;
    // Tall, and a reference did not serve: the run once more, wide, with barriers of its own (some of the first walk's end in
    // odd phases).  All products of the first walk are in O, which has been read.
    if (threadIdx.x < 8) bad_tag[threadIdx.x] = 0;
    bars += P::BARS * 8;
    wide = true;
    __syncthreads();
  }
  if (warp == kIssuer && !narrow) {
    tmem_dealloc(tmem, 512);
  }
}

// Joins the parts of the cut units, in the order of the keys: the part of the CTA in which a unit begins, then those of
// the CTAs after it.  A warp reads a row's part at once (its 32 lanes the columns).  The work is a few MB from L2 at most
// and all latency, so it is spread as widely as it goes: every block lists the cut units (one per CTA of the first kernel
// at most) and takes every gridDim.x-th run of rows; as long as the device has warps to spare, 2, 4 or 8 of them share
// the parts of a row.
constexpr int kJoinWarps = 8, kJoinBlocksPerSm = 4;

template <int D>
__global__ void __launch_bounds__(kJoinWarps * 32, kJoinBlocksPerSm) tree_attn_join_kernel(const __grid_constant__ TreeAttnArgs a, const Work work, int n_cta) {
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
            const size_t slot = ((size_t)(owner + p) * 2 + (p == 0 ? 1 : 0)) * kUnitRows + r;
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

// ------------------------------------------------------------------ host side

// [pages, heads, page, D] cache -> tensor map of 64 columns, 8 rows, D / 64, the page's groups of 8 rows, and heads and pages
// together; a box is all of a page (of 128 of its rows), 128-byte swizzle.
bool make_cache_map(CUtensorMap* m, const PagedCache& c, int d, int page, const CacheSteps& steps) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[5] = {64, 8, (cuuint64_t)d / 64, (cuuint64_t)page / 8, (cuuint64_t)steps.extent};
  cuuint64_t strides[4] = {(cuuint64_t)c.s_tok * 2, 128, (cuuint64_t)c.s_tok * 16, (cuuint64_t)steps.unit * 2};
  cuuint32_t box[5] = {64, 8, (cuuint32_t)d / 64, (cuuint32_t)(page < kTile ? page : kTile) / 8, 1};
  cuuint32_t estr[5] = {1, 1, 1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, c.data, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D>
cudaError_t launch(const TreeAttnArgs& a, void* ws, int n_cta, cudaStream_t s) {
  CUtensorMap tk, tv;
  Work w;
  if (!cache_steps(a.kc, a.hkv, a.n_pages, &w.k) || !cache_steps(a.vc, a.hkv, a.n_pages, &w.v)) return cudaErrorInvalidValue;
  if (!make_cache_map(&tk, a.kc, D, 1 << a.page_log2, w.k) || !make_cache_map(&tv, a.vc, D, 1 << a.page_log2, w.v)) return cudaErrorInvalidValue;
  const size_t slots = (size_t)n_cta * 2 * kUnitRows;
  w.part = static_cast<float*>(ws);
  w.ml = reinterpret_cast<float2*>(w.part + slots * 128);
  w.meta = reinterpret_cast<Meta*>(w.ml + slots);
  constexpr int smem = Plan<D>::TOTAL > 120 * 1024 ? Plan<D>::TOTAL : 120 * 1024;      // one CTA per SM (it takes all of TMEM)
  static_assert(smem <= 232448, "");
  cudaError_t e = cudaFuncSetAttribute(tree_attn_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  e = launch_dependent(tree_attn_kernel<D>, dim3(n_cta), dim3(kThreads), smem, s, a, w, tk, tv);
  if (e != cudaSuccess) return e;
  return launch_dependent(tree_attn_join_kernel<D>, dim3(n_cta * kJoinBlocksPerSm), dim3(kJoinWarps * 32), 0, s, a, w, n_cta);
}

}  // namespace

size_t tree_attn_workspace_bytes(int n_sm) {
  return (size_t)n_sm * (2 * kUnitRows * (128 * sizeof(float) + sizeof(float2)) + sizeof(Meta));
}

cudaError_t launch_tree_attn(const TreeAttnArgs& a, void* ws, int n_sm, cudaStream_t s) {
  return a.d == 128 ? launch<128>(a, ws, n_sm, s) : launch<64>(a, ws, n_sm, s);
}

}  // namespace sp
