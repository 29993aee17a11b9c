// Attention of a few new tokens per request (one, a chain, a tree of drafted ones) over the paged cache: tcgen05 / TMEM /
// TMA, split along the keys.
//
//   out_r = sum_c p_rc v_c / sum_c p_rc,  p_rc = 2^(scale q_r.k_c - m_r) over the visible keys c.
//
// The rows of a unit are the new tokens of one request times the query heads that share a KV head (row = token * group +
// head), so that every key and value is read once for all of them.  Work is counted in steps: one for the unit (request,
// KV head, rows) and one for each of its key tiles of 128.  The steps of all units stand in one line, which is cut into one
// equal run per worker wherever that falls; a unit that is cut leaves partial results (unnormalised sums, reference maxima,
// weights) that a second kernel joins in the order of the keys.  All lengths are read on the device: a prefix sum over the
// requests tells each worker where its run begins.  (Without the step for the unit itself, workers with many short requests
// finish late: XXX.)
//
// What bounds it: the cache's bytes.  A tile is 64 KB (head_dim 128), 2700 cycles of an SM's share of the measured HBM
// rate; its matrix products take 1020 cycles for up to 128 rows (the tensor core takes 128 rows at a time, however few
// are in use), 2040 for 256.  With 256 rows its 32768 exponentials (2048 cycles of the SM's special-function units) come
// close to the bytes.
//
// Two streams per CTA, each with its own Q, its own S and O columns in TMEM, its own four softmax warps and its own
// loader, share the tensor core and the ring of K and V tiles, so that one stream's softmax, waits and epilogues overlap
// the other's products.  If no request has more than 128 rows the streams are workers of their own, with a run of tiles
// each (a unit's beginning and end then cost one stream a wait, not the SM).  Otherwise ("wide") a CTA is a worker, units
// have up to 256 rows, and the streams are the two halves of them and walk the same tiles.
//
// With at most 16 rows in every request (single tokens as a rule) the tensor core's 128-row products are the wrong tool:
// a tile costs the issuing thread 16 of them, 1400 cycles, and the softmax 128 exponentials in a row by one warp of four.
// Then ("narrow") the eight softmax warps are on their own: each takes 16 keys of every tile, S (16 rows x 16 keys) and
// O (16 rows x head) in registers by mma.sync m16n8k16, K and V by ldmatrix from the same ring, no hand-over between K
// and V; their sums are added up at the unit's end.  16 mma.sync for each product and warp are a few hundred cycles of
// the 2700 that the tile's bytes take.  (256 chats of 60 to 4000 tokens: 253 us by tcgen05 with the rows in the lanes, 291 us
// by tcgen05 with the keys in the lanes, XXX us so.)
//
//   warps 0-3, 4-7  softmax and epilogue of stream 0 / 1: thread = TMEM lane = row
//   warp 8          producer: page ids from the table, TMA loads of K and V pages into a ring of tile slots, in the order
//                   in which the products need them: K0 K1 V0 K2 V1 ... (a V tile that arrived with its K would hold a
//                   slot for the whole softmax); with separate runs the streams' tiles in turn
//   warp 9          issuer (one thread): S = Q K^T and O += P V of whichever stream is ready
//   warps 10, 11    loader of stream 0 / 1: walks the run, publishes units, gathers their Q rows into shared memory
//
// Masks.  Only tiles that hold a key at or behind the first new token need one.  There the row's visibility bits are
// shifted into place 32 keys at a time.  A masked probability is zero, but zero times a NaN in V is not: in those tiles
// the values behind the sequence are set to zero in shared memory, and non-finite values of new tokens too; if there were
// any, each row adds those that it sees at the end (from the cache: they are what the sum comes to anyway).
//
// Rounding: products bf16 x bf16 in fp32, softmax statistics and O in fp32, P rounded to bf16 for the second product (the
// sum of weights is taken before that rounding), the result once.  The reference maximum moves only when the row maximum
// has grown by more than 2^8 (P stays below 2^8, exact scaling otherwise).
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
constexpr int kThreads = 384;
constexpr int kProducer = 8, kIssuer = 9, kLoader = 10;
constexpr int kUnitRing = 4;
constexpr int kNarrowRows = 16;
constexpr float kNoMax = -1e30f;                 // reference maximum before any visible key: finite, below any logit

template <int D>
struct Plan {
  static constexpr int NBOX = D / 64;                       // 64-column (128-byte) boxes
  static constexpr int QBOX = 128 * 128, QHALF = NBOX * QBOX;
  static constexpr int KBOX = kTile * 128, SLOT = NBOX * KBOX;
  static constexpr int SLOTS = D == 128 ? 5 : 10;
  static constexpr int RING_OFF = 2 * QHALF;
  static constexpr int MISC_OFF = RING_OFF + SLOTS * SLOT;
  // narrow: one slot more, in the second half of the Q area; two sets of 16 Q rows and the sums' exchange in the first
  static constexpr int NSLOTS = SLOTS + 1, NRING_OFF = RING_OFF - SLOT;
  static constexpr int NQ_BYTES = NBOX * kNarrowRows * 128, SUM_OFF = 2 * NQ_BYTES;
  static constexpr int SUM_ROWS = 4, SUM_STRIDE = D + 8;                  // rows exchanged at a time; 8 columns more against bank conflicts
  static_assert(SLOT == QHALF && SUM_OFF + 8 * SUM_ROWS * SUM_STRIDE * 4 <= QHALF, "");
  static constexpr int BAR_FULL = 0, BAR_FREE = BAR_FULL + NSLOTS, BAR_S = BAR_FREE + NSLOTS, BAR_P = BAR_S + 2, BAR_PV = BAR_P + 2,
                       BAR_QFULL = BAR_PV + 2, BAR_QFREE = BAR_QFULL + 2, BAR_UNIT = BAR_QFREE + 2, BAR_UFREE = BAR_UNIT + 2 * kUnitRing,
                       BARS = BAR_UFREE + 2 * kUnitRing;
  static constexpr int UNIT_OFF = MISC_OFF + BARS * 8, UNIT_BYTES = 48;               // [stream][kUnitRing]
  static constexpr int SCAN_OFF = (UNIT_OFF + 2 * kUnitRing * UNIT_BYTES + 15) / 16 * 16;    // int64 [24]
  static constexpr int RUN_OFF = SCAN_OFF + 24 * 8;                                   // int64 [6], int [4]
  static constexpr int TAG_OFF = RUN_OFF + 6 * 8 + 4 * 4;                             // int [16]
  static constexpr int EX_OFF = TAG_OFF + 16 * 4;                                     // narrow: float2 [8][16]
  static constexpr int TOTAL = EX_OFF + 8 * kNarrowRows * 8;
  static constexpr int S_COL = 0, O_COL = 256, O_STEP = D;  // S: 128 columns a stream; O: D columns a stream
};

struct Unit {       // of one stream
  int n_tiles;      // key tiles of this worker's part; 0: no more units
  int kt0;          // first of them
  int kt_all;       // key tiles of the whole unit
  int start;        // first row of the request
  int r0, rows;     // first of the stream's rows (token * group + head) inside the request, and their number
  int g, b;
  int len, past;
  int pad[2];
};
static_assert(sizeof(Unit) == 48, "");

struct Meta {       // what the join kernel needs of a unit that begins in this worker and goes on in later ones
  int last;         // worker that has the unit's last tile; < 0: there is no such unit
  int start, r0, rows, g, wide, pad[2];
};

// Worker w is stream w / n_cta of CTA w % n_cta (wide: CTA w), so that few tiles spread over the SMs first.
struct Work {
  float* part;      // [cta][2][256][D] unnormalised sums (stream 1: rows 128 on): part 0 of a unit begun by an earlier
                    // worker, part 1 of one begun here
  float2* ml;       // [cta][2][256] reference maximum, weight
  Meta* meta;       // [worker]
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
// units of the request per KV head (n * group fits 32 bits: the host has checked)
__device__ __forceinline__ int passes(const TreeAttnArgs& a, const Request& q) { return (q.n * a.group + kUnitRows - 1) / kUnitRows; }
__device__ __forceinline__ long long units_of(const TreeAttnArgs& a, const Request& q) { return (long long)a.hkv * passes(a, q); }
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
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1, int c2, int c3) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
      ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3)
      : "memory");
}
// Products with operand descriptors given by their low words (address and leading offset); the high word is the same for
// all tiles here (1024 bytes between 8-row groups, 128-byte swizzle).
constexpr uint32_t kDescHigh = (1024u >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ void mma_ss_lo(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t accum) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
      "mov.b64 da, {%1, %5};\n\tmov.b64 db, {%2, %5};\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accum), "n"(kDescHigh)
      : "memory");
}
__device__ __forceinline__ void mma_ts_lo(uint32_t d_tmem, uint32_t a_tmem, uint32_t b_lo, uint32_t idesc, uint32_t accum) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 db;\n\t"
      "mov.b64 db, {%2, %5};\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "r"(b_lo), "r"(idesc), "r"(accum), "n"(kDescHigh)
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

// The non-finite values of new tokens that a row sees, added to the d columns that its thread has just written (they were
// left out of the products): bf16 results, or fp32 partial sums.
template <typename T>
__device__ __noinline__ void add_nonfinite(const TreeAttnArgs& a, const Unit& u, int token, T* out, int d) {
  const int k_from = max(u.kt0 * kTile, u.past), k_to = min((u.kt0 + u.n_tiles) * kTile, u.len);
  for (int key = k_from; key < k_to; ++key) {
    const int id = a.table[(size_t)u.b * a.max_pages + (key >> a.page_log2)];
    if (id < 0 || id >= a.n_pages || !(seen32(a, u, token, key) & 1)) continue;
    const __nv_bfloat16* v = a.vc.data + id * a.vc.s_page + u.g * a.vc.s_head + (key & ((1 << a.page_log2) - 1)) * a.vc.s_tok;
    for (int c = 0; c < d; ++c) {
      const float x = __bfloat162float(v[c]);
      if (!isfinite(x)) out[c] = static_cast<T>(static_cast<float>(out[c]) + x);
    }
  }
}

// Rare path of the softmax: the row's reference maximum has moved, so O of the earlier tiles (when there are any) and
// the P chunks of this tile that are already stored are brought to the new one.  alpha is a power of two (references are
// whole numbers), so nothing is rounded again.  Called by whole warps.
template <int D>
__device__ __noinline__ void rescale_tmem(uint32_t t_o, uint32_t t_s, float alpha, int stored, bool with_o) {
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
// by whole warps; a row that is not the unit's (token < 0) sees nothing.
__device__ __noinline__ void mask_tmem(const TreeAttnArgs& a, const Unit& u, int token, int k0, uint32_t t_s) {
#pragma unroll 1
  for (int c = 0; c < kTile / 32; ++c) {
    const uint32_t seen = token >= 0 ? seen32(a, u, token, k0 + c * 32) : 0u;
    if (__all_sync(0xffffffffu, seen == 0xffffffffu)) continue;
    uint32_t s[32];
    tmem_ld32(t_s + c * 32, s);
#pragma unroll
    for (int e = 0; e < 32; ++e) s[e] = (seen >> e) & 1 ? s[e] : 0xff800000u;
    tmem_st32(t_s + c * 32, s);
  }
  tmem_wait_st();
}

// Values behind the sequence become zero in a V tile, and so do non-finite ones of new tokens (reported: see
// add_nonfinite).  Rows lo .. hi - 1 of the tile, one after the other, the warp's lanes across the columns.  v: this lane's
// first word of row 0.  Rolled loops: the code runs once a unit and is fetched anew each time; unrolled by eight rows it
// took 2000 cycles for sixteen.
template <int D>
__device__ __noinline__ void clean_values(uint32_t* v, int lo, int hi, int first_behind, volatile int* tags, int tag_lo, int tag_hi, int mark) {
  constexpr int BOXES = D / 64, BOX_WORDS = kTile * 128 / 4;
  int r = lo;
#pragma unroll 1
  for (; r < min(hi, first_behind); ++r) {
    uint32_t w[BOXES];
    bool met = false;
#pragma unroll
    for (int b = 0; b < BOXES; ++b) {
      w[b] = v[b * BOX_WORDS + r * 32];
      met |= nonfinite2(w[b]);
    }
    if (met) {
      for (int x = tag_lo; x <= tag_hi; ++x) tags[x * 8 + mark % 8] = mark;
      __threadfence_block();
#pragma unroll
      for (int b = 0; b < BOXES; ++b) {
        uint32_t x = w[b];
        if ((x & 0x7f80u) == 0x7f80u) x &= 0xffff0000u;
        if ((x & 0x7f800000u) == 0x7f800000u) x &= 0xffffu;
        v[b * BOX_WORDS + r * 32] = x;
      }
    }
  }
#pragma unroll 2
  for (r = max(lo, first_behind); r < hi; ++r)
#pragma unroll
    for (int b = 0; b < BOXES; ++b) v[b * BOX_WORDS + r * 32] = 0u;
}

// Epilogue of a stream's unit, out of the hot loop: the rows' results, or their part for the join.  Called by whole warps.
template <int D>
__device__ __noinline__ void write_rows(const TreeAttnArgs& a, const Work& work, const Unit& u, int x, int row, int token, int head, uint32_t t_o,
                                        float m_ref, float l, bool repair) {
  const bool live = row < u.rows, whole = u.kt0 == 0 && u.n_tiles == u.kt_all;
  const float f = !whole ? 1.f : l != 0.f ? 1.f / l : 0.f;
  const size_t slot = ((size_t)blockIdx.x * 2 + (u.kt0 > 0 ? 0 : 1)) * kUnitRows + x * 128 + row;
  __nv_bfloat16* out = a.o + head * a.o_sh + (u.start + token) * a.o_sn;
  float* part = work.part + slot * D;
#pragma unroll 1
  for (int c = 0; c < D / 32; ++c) {
    uint32_t y[32];
    tmem_ld32(t_o + c * 32, y);
    if (!live) continue;
    auto val = [&](int i) { return __uint_as_float(y[i]) * f; };
    if (whole) {
      uint4* dst = reinterpret_cast<uint4*>(out + c * 32);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        dst[i] = make_uint4(pack_bf16(val(8 * i), val(8 * i + 1)), pack_bf16(val(8 * i + 2), val(8 * i + 3)), pack_bf16(val(8 * i + 4), val(8 * i + 5)),
                            pack_bf16(val(8 * i + 6), val(8 * i + 7)));
    } else {
      float4* dst = reinterpret_cast<float4*>(part + c * 32);
#pragma unroll
      for (int i = 0; i < 8; ++i) dst[i] = make_float4(val(4 * i), val(4 * i + 1), val(4 * i + 2), val(4 * i + 3));
    }
  }
  if (live) {
    if (repair) {
      if (whole) add_nonfinite(a, u, token, out, D);
      else add_nonfinite(a, u, token, part, D);
    }
    if (!whole) work.ml[slot] = make_float2(m_ref, l);
    else if (a.lse) a.lse[(size_t)head * a.rows + u.start + token] = l != 0.f ? (m_ref + log2f(l)) * 0.6931471805599453f : -CUDART_INF_F;
  }
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
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, cta = blockIdx.x;
  // Fragments of mma.sync m16n8k16: lane = (row g = lane / 4, and g + 8; columns 2 q, 2 q + 1, q = lane % 4).
  const int g = lane >> 2, q = lane & 3;
  float2* ex = reinterpret_cast<float2*>(smem + P::EX_OFF);          // [warp][row] reference, weight
  float* sums = reinterpret_cast<float*>(smem + P::SUM_OFF);         // [warp][row % 4][SUM_STRIDE]
  // ldmatrix addresses of this lane: a row of the four 8x8 blocks, whose 16-byte pieces are swizzled by the row
  const int k_row = warp * 16 + (lane & 7) + ((lane >> 4) << 3), k_piece = (lane >> 3) & 1;   // K: keys 0-7, 8-15 by piece, piece + 1
  const int v_row = warp * 16 + (lane & 15), v_piece = lane >> 4;                            // V (and Q): rows 0-7, 8-15, then the next piece
  const uint32_t ring = base + P::NRING_OFF;
  auto at = [](uint32_t tile, int box, int row, int piece) {
    return tile + (piece >> 3) * box + row * 128 + (((piece & 7) ^ (row & 7)) << 4);
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
        ldmatrix4(at(base + (seq & 1) * P::NQ_BYTES, kNarrowRows * 128, lane & 15, 2 * kk + v_piece), qf[kk]);
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
          ldmatrix4(at(tile, P::KBOX, k_row, 2 * kk + k_piece), b);
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
          clean_values<D>(reinterpret_cast<uint32_t*>(smem + P::NRING_OFF + slot * P::SLOT) + lane, lo, warp * 16 + 16, u.len - k0, bad_tag, 0, 0, seq + 1);
          fence_async_smem();
        }
        __syncwarp();
      }
      {
        const uint32_t tile = ring + slot * P::SLOT;
#pragma unroll
        for (int n = 0; n < D / 8; n += 2) {
          uint32_t b[4];
          ldmatrix4t(at(tile, P::KBOX, v_row, n + v_piece), b);
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
    const bool whole = u.kt0 == 0 && n_tiles == u.kt_all;
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
        const int token = row / a.group, head = u.g * a.group + row % a.group;
        const size_t part = ((size_t)cta * 2 + (u.kt0 > 0 ? 0 : 1)) * kUnitRows + row;
        __nv_bfloat16* out = a.o + head * a.o_sh + (u.start + token) * a.o_sn;
        const float inv = all != 0.f ? 1.f / all : 0.f;
        if (!whole) {
#pragma unroll
          for (int i = 0; i < PER; ++i) work.part[part * D + col + i] = y[i];
        } else if constexpr (PER == 2) {
          *reinterpret_cast<uint32_t*>(out + col) = pack_bf16(y[0] * inv, y[1] * inv);
        } else {
          out[col] = __float2bfloat16(y[0] * inv);
        }
        if ((threadIdx.x & 63) == 0) {
          if (!whole) work.ml[part] = make_float2(top, all);
          else if (a.lse) a.lse[(size_t)head * a.rows + u.start + token] = all != 0.f ? (top + log2f(all)) * 0.6931471805599453f : -CUDART_INF_F;
        }
      }
    }
    if (bad_tag[(seq + 1) % 8] == seq + 1) {
      bar_sync(1, 256);                             // the rows are written
      if (threadIdx.x < rows) {
        const int row = threadIdx.x, token = row / a.group, head = u.g * a.group + row % a.group;
        if (whole) add_nonfinite(a, u, token, a.o + head * a.o_sh + (u.start + token) * a.o_sn, D);
        else add_nonfinite(a, u, token, work.part + (((size_t)cta * 2 + (u.kt0 > 0 ? 0 : 1)) * kUnitRows + row) * D, D);
      }
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(bar(P::BAR_UFREE + e));
  }
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
tree_attn_kernel(const __grid_constant__ TreeAttnArgs a, const __grid_constant__ Work work, const __grid_constant__ CUtensorMap tm_k,
                 const __grid_constant__ CUtensorMap tm_v) {
  using P = Plan<D>;
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t base = smem_u32(smem);
  auto bar = [&](int which) { return base + P::MISC_OFF + which * 8; };
  Unit* units = reinterpret_cast<Unit*>(smem + P::UNIT_OFF);
  long long* scan = reinterpret_cast<long long*>(smem + P::SCAN_OFF);
  long long* start_rem = reinterpret_cast<long long*>(smem + P::RUN_OFF);      // [stream] steps of the request before the run
  long long* tiles_at = start_rem + 2;             // [stream][2] tiles before the run's begin and end
  int* words = reinterpret_cast<int*>(smem + P::RUN_OFF + 6 * 8);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(words);
  volatile int* abort_flag = words + 1;
  int* start_b = words + 2;                        // [stream] request in which the run begins
  // [stream][8]: number, from 1, of a unit in which a non-finite value was met, at that number modulo 8 (the streams of
  // wide units write each other's and are two units apart at most)
  volatile int* bad_tag = reinterpret_cast<int*>(smem + P::TAG_OFF);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int cta = blockIdx.x, n_cta = gridDim.x;
  const Abort ab{abort_flag, a.status};

  let_next_start();
  const bool misplaced = (base & 1023u) != 0;      // the tiles' swizzle needs the window's alignment
  if (warp == kProducer && lane < 2) asm volatile("prefetch.tensormap [%0];" ::"l"(lane == 0 ? &tm_k : &tm_v) : "memory");
  if (threadIdx.x == 0) {
    for (int s = 0; s < P::NSLOTS; ++s) mbar_init(bar(P::BAR_FULL + s), 1);
    for (int x = 0; x < 2; ++x) {
      mbar_init(bar(P::BAR_S + x), 1);
      mbar_init(bar(P::BAR_P + x), 4);
      mbar_init(bar(P::BAR_PV + x), 1);
    }
    *abort_flag = 0;
    for (int i = 0; i < 16; ++i) bad_tag[i] = 0;
  }
  wait_for_previous();
  const bool poisoned = decode_poisoned(a.status);

  // ---- where the runs begin
  const int per = (a.n_req + kThreads - 1) / kThreads;
  const int b_lo = min((int)threadIdx.x * per, a.n_req), b_hi = min(b_lo + per, a.n_req);
  long long mine_t = 0, mine_u = 0;                // tiles, units
  bool many = false, some = false;
  for (int b = b_lo; b < b_hi; ++b) {
    const Request q = request(a, b);
    const long long n = units_of(a, q);
    mine_u += n;
    mine_t += n * q.kt;
    many |= q.n * a.group > 128;
    some |= q.n * a.group > kNarrowRows;
  }
  long long incl_t = mine_t, incl_u = mine_u;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long up_t = __shfl_up_sync(0xffffffffu, incl_t, o), up_u = __shfl_up_sync(0xffffffffu, incl_u, o);
    if (lane >= o) { incl_t += up_t; incl_u += up_u; }
  }
  if (lane == 31) { scan[warp] = incl_t; scan[12 + warp] = incl_u; }
  if (threadIdx.x == 0 && misplaced && atomicCAS(a.status, 0, (int)SP_ERR_UNSUPPORTED) == 0) a.status[1] = 90;
  const bool wide = __syncthreads_or(many) != 0, narrow = __syncthreads_or(some) == 0;
  const bool by_cta = wide || narrow;              // a CTA is a worker
  if (!narrow) {
    if (warp == kIssuer) tmem_alloc(smem_u32(tmem_slot), 512);
    // rows of the Q area that no unit fills stay zero: products of whatever lay there would cost power, and with it clock
    for (int i = threadIdx.x; i < 2 * P::QHALF / 16; i += kThreads) reinterpret_cast<uint4*>(smem)[i] = make_uint4(0, 0, 0, 0);
    fence_async_smem();
  }
  long long before_t = incl_t - mine_t, before_u = incl_u - mine_u, total_t = 0, total = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) {
    if (w < warp) { before_t += scan[w]; before_u += scan[12 + w]; }
    total_t += scan[w];
    total += scan[w] + scan[12 + w];
  }
  const int workers = by_cta ? n_cta : 2 * n_cta;
  const long long quota = divide(total, workers), extra = total - quota * workers;      // the first `extra` runs are one step longer
  auto run_begin = [&](int w) { return w * quota + min((long long)w, extra); };
  for (int i = 0; i < (by_cta ? 2 : 4); ++i) {
    const int x = i >> 1, end = i & 1;
    const long long w = run_begin((by_cta ? cta : x * n_cta + cta) + end);
    long long step = before_t + before_u, tile = before_t;
    if (w >= total) {
      if (threadIdx.x == 0) tiles_at[i] = total_t;
    } else if (step <= w && w < step + mine_t + mine_u) {
      for (int b = b_lo; b < b_hi; ++b) {
        const Request q = request(a, b);
        const long long n = units_of(a, q);
        if (w < step + n * (q.kt + 1)) {
          const long long rem = w - step, nth = divide(rem, q.kt + 1), in = rem - nth * (q.kt + 1);
          tiles_at[i] = tile + nth * q.kt + max(in - 1, 0ll);
          if (!end) { start_b[x] = b; start_rem[x] = rem; }
          break;
        }
        step += n * (q.kt + 1);
        tile += n * q.kt;
      }
    }
  }
  if (threadIdx.x == 0) {
    // who lets a tile go: the stream's issuer, both streams', or the eight warps; likewise the queries
    for (int s = 0; s < P::NSLOTS; ++s) mbar_init(bar(P::BAR_FREE + s), narrow ? 8 : wide ? 2 : 1);
    for (int x = 0; x < 2; ++x) {
      mbar_init(bar(P::BAR_QFULL + x), narrow ? 32 : 1);
      mbar_init(bar(P::BAR_QFREE + x), narrow ? 8 : 1);
    }
    // a unit is read by four softmax warps, the issuer and the producer (wide: in ring 0 only), or by eight warps and the producer
    for (int e = 0; e < 2 * kUnitRing; ++e) {
      mbar_init(bar(P::BAR_UNIT + e), 1);
      mbar_init(bar(P::BAR_UFREE + e), narrow ? 9 : 4 + 1 + (wide && e >= kUnitRing ? 0 : 1));
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  tc_fence_before();
  const bool idle = __syncthreads_or(poisoned || misplaced) != 0;
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  // tiles of the streams' runs, and of the CTA.  Job j of the CTA is a tile of one stream, the streams in turn as long as both
  // have some; wide: a tile of both.
  uint32_t n_run[2];
#pragma unroll
  for (int x = 0; x < 2; ++x) n_run[x] = idle || (narrow && x == 1) ? 0u : (uint32_t)(tiles_at[by_cta ? 1 : 2 * x + 1] - tiles_at[by_cta ? 0 : 2 * x]);
  const uint32_t n_steps = wide ? n_run[0] : n_run[0] + n_run[1], in_turn = min(n_run[0], n_run[1]);
  auto job_of = [&](int x, uint32_t i) { return wide ? i : i < in_turn ? 2 * i + x : in_turn + i; };
  // ring positions of the K and V tiles of job j: K0 K1 V0 K2 V1 ... K(n-1) V(n-2) V(n-1); narrow: K0 V0 K1 V1 ...
  auto k_pos = [&](uint32_t j) { return j == 0 ? 0u : 2 * j - 1; };
  auto v_pos = [&](uint32_t j) { return j + 1 == n_steps ? 2 * j + 1 : 2 * j + 2; };

  if (warp >= kLoader) {
    // ------------------------------------------------------------ units of stream x and their queries
    const int x = warp - kLoader, me = by_cta ? cta : x * n_cta + cta;
    bool ok = true;
    int seq = 0;
    if (lane == 0) work.meta[x * n_cta + cta].last = -1;
    if (n_run[x] > 0) {
      int b = start_b[by_cta ? 0 : x];
      long long rem = start_rem[by_cta ? 0 : x], w = run_begin(me);
      const long long w1 = run_begin(me + 1);
      Request q = request(a, b);
      while (w < w1 && ok) {
        while (rem >= units_of(a, q) * (q.kt + 1) && b + 1 < a.n_req) { rem = 0; q = request(a, ++b); }
        if (rem >= units_of(a, q) * (q.kt + 1)) break;       // not reached while the lengths stand still
        Unit u;
        const int n_pass = passes(a, q), all_rows = q.n * a.group;
        const int nth = (int)divide(rem, q.kt + 1), in = (int)(rem - (long long)nth * (q.kt + 1));       // step of the unit: tile `in - 1`
        const int take = (int)min((long long)(q.kt + 1 - in), w1 - w);
        w += take;
        rem += take;
        u.kt0 = max(in - 1, 0);
        u.kt_all = q.kt;
        u.n_tiles = in + take - 1 - u.kt0;
        if (u.n_tiles == 0) continue;                // only the unit's own step: its tiles are the next worker's
        u.g = n_pass == 1 ? nth : nth / n_pass;
        u.b = b;
        u.start = q.start;
        u.r0 = (nth - u.g * n_pass) * kUnitRows + (wide ? x * 128 : 0);
        u.rows = min(128, max(all_rows - u.r0, 0));
        u.len = q.len;
        u.past = q.past;
        const int e = x * kUnitRing + seq % kUnitRing;
        if (seq >= kUnitRing) ok = __all_sync(0xffffffffu, mbar_wait(bar(P::BAR_UFREE + e), (seq / kUnitRing - 1) & 1, ab, 40));
        if (!ok) break;
        if (lane == 0) {
          units[e] = u;
          mbar_arrive(bar(P::BAR_UNIT + e));
          if (u.kt0 == 0 && u.n_tiles < u.kt_all && !(wide && x == 1)) {
            const long long z = w - take - in + u.kt_all, cut = extra * (quota + 1);     // the step of the unit's last tile
            Meta m{(int)(z < cut ? divide(z, quota + 1) : extra + divide(z - cut, quota)), u.start, u.r0,
                   wide ? min(all_rows - u.r0, kUnitRows) : u.rows, u.g, wide, {0, 0}};
            work.meta[me] = m;
          }
          if (a.seq_lens[b] > q.len) report_range(a.status, kWhereTreePage);   // longer than its table row
        }
        // its queries: rows of 128-byte boxes, 16-byte pieces swizzled as the MMA descriptors say.  A lane keeps its
        // piece of every (32 / pieces)-th row, whose token and head advance without division.
        // (narrow: two sets of rows in turn)
        const int set = narrow ? seq & 1 : x, lap = narrow ? seq >> 1 : seq;
        if (lap > 0) ok = __all_sync(0xffffffffu, mbar_wait(bar(P::BAR_QFREE + set), (lap - 1) & 1, ab, 41));
        if (!ok) break;
        {
          constexpr int PIECES = D / 8, STEP = 32 / PIECES;
          const int piece = lane % PIECES;
          int r = lane / PIECES, hg = (u.r0 + r) % a.group;
          const __nv_bfloat16* src = a.q + (int64_t)(u.g * a.group + hg) * a.q_sh + (int64_t)(u.start + (u.r0 + r) / a.group) * a.q_sn + piece * 8;
          const int64_t down = STEP * a.q_sh, wrap = a.q_sn - a.group * a.q_sh;
          const uint32_t box = narrow ? base + set * P::NQ_BYTES + (piece >> 3) * (kNarrowRows * 128) : base + x * P::QHALF + (piece >> 3) * P::QBOX;
#pragma unroll 2
          for (; r < u.rows; r += STEP) {
            cp_async16(box + r * 128 + (((piece & 7) ^ (r & 7)) << 4), src);
            src += down;
            hg += STEP;
            while (hg >= a.group) { hg -= a.group; src += wrap; }
          }
        }
        if (narrow) {                                // read by ldmatrix: the copies' arrival is enough, and nobody waits for it here
          asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar(P::BAR_QFULL + set)) : "memory");
        } else {
          asm volatile("cp.async.wait_all;" ::: "memory");
          fence_async_smem();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(P::BAR_QFULL + set));
        }
        ++seq;
      }
    }
    // no more units
    const int e = x * kUnitRing + seq % kUnitRing;
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
    } last{0, 0, 0, false};
    auto load = [&](const Tile& tile, const CUtensorMap& map) {
      if (ok && lap > 0) ok = __all_sync(0xffffffffu, mbar_wait(bar(P::BAR_FREE + s), (lap - 1) & 1, ab, 51));
      if (!ok) return;
      const int n_live = __popc(__ballot_sync(0xffffffffu, tile.live));
      if (lane == 0) mbar_expect_tx(bar(P::BAR_FULL + s), n_live * rows * D * 2);
      __syncwarp();
      if (tile.live) {
        const uint32_t dst = ring + s * P::SLOT + lane * rows * 128;
#pragma unroll
        for (int x = 0; x < P::NBOX; ++x) tma_load_4d(dst + x * P::KBOX, &map, bar(P::BAR_FULL + s), x * 64, tile.off, tile.g, tile.id);
      }
      __syncwarp();
      if (++s == slots) { s = 0; ++lap; }
    };
    // where each stream's walk stands (wide: stream 0's serves both)
    struct Walk {
      int seq, kt, kt_end, len, g, b, id;            // id: this lane's page of tile kt
    } walk[2];
    walk[0].seq = walk[1].seq = 0;
    walk[0].kt = walk[0].kt_end = walk[1].kt = walk[1].kt_end = 0;
    // lane p looks up page p of the tile, a tile ahead
    auto lookup = [&](const Walk& k, int kt) {
      const int key = kt * kTile + lane * page;
      return lane < per_tile && key < k.len ? a.table[(size_t)k.b * a.max_pages + (key >> a.page_log2)] : -1;
    };
    auto step = [&](Walk& k, int x) -> Tile {
      if (k.kt == k.kt_end) {
        const int e = x * kUnitRing + k.seq % kUnitRing;
        ok = ok && __all_sync(0xffffffffu, mbar_wait(bar(P::BAR_UNIT + e), (k.seq / kUnitRing) & 1, ab, 50));
        if (!ok) return Tile{0, 0, 0, false};
        const Unit& u = units[e];
        k.kt = u.kt0; k.kt_end = u.kt0 + u.n_tiles; k.len = u.len; k.g = u.g; k.b = u.b;
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(P::BAR_UFREE + e));
        ++k.seq;
        k.id = lookup(k, k.kt);
      }
      const int key = k.kt * kTile + lane * page;
      Tile tile{k.id, key & (page - 1), k.g, lane < per_tile && key < k.len};
      if (tile.live && (tile.id < 0 || tile.id >= a.n_pages)) {
        report_range(a.status, kWhereTreePage);
        tile.id = a.n_pages;                         // outside the tensor map: the load fills in zeros
      }
      ++k.kt;
      if (k.kt < k.kt_end) k.id = lookup(k, k.kt);
      return tile;
    };
    for (uint32_t j = 0; j < n_steps && ok; ++j) {
      const Tile now = by_cta || (j < 2 * in_turn ? (j & 1) == 0 : n_run[0] > n_run[1]) ? step(walk[0], 0) : step(walk[1], 1);
      load(now, tm_k);
      if (narrow) load(now, tm_v);
      else if (j > 0) load(last, tm_v);
      last = now;
    }
    if (n_steps > 0 && !narrow) load(last, tm_v);
    // the last entry of each ring that this warp reads says that there are no more units: nothing to take from it
    if (*abort_flag && lane == 0) {
      // let the copies already in flight land before the CTA gives its shared memory back
      const long long t0 = clock64();
      for (uint32_t i = 0; i < slots; ++i) {
        const uint32_t laps = lap + (i < s);          // loads that this slot has been given
        while (laps > 0 && !mbar_test(bar(P::BAR_FULL + i), (laps - 1) & 1) && clock64() - t0 < kWaitCycles / 8) {}
      }
    }
  } else if (warp == kIssuer) {
    // ------------------------------------------------------------ products
    if (lane == 0 && !narrow) {
      constexpr uint32_t idesc_qk = instr_desc(128, kTile, 0, 0), idesc_pv = instr_desc(128, D, 0, 1);
      const uint32_t d_q = (uint32_t)smem_desc(base, 16, 1024), d_k = (uint32_t)smem_desc(base + P::RING_OFF, 16, 1024),
                     d_v = (uint32_t)smem_desc(base + P::RING_OFF, P::KBOX, 1024);
      // One thread does all of this, and every instruction of the loop delays both streams: 32-bit counters, everything
      // about a stream in registers (the loop over the streams is unrolled).  A stream's next S is computed when its last
      // P has gone into its product.
      struct Stream {
        uint32_t n_qk, n_pv;                         // products issued
        uint32_t left, seq;                          // tiles left in the unit, units taken
        uint32_t k_at, k_slot, v_at, v_slot;         // ring positions of the next K and V tile
        bool first, q_here;                          // the next O opens a sum; the unit's Q has been seen
      } st[2];
      auto advance = [&](uint32_t& at, uint32_t& slot, uint32_t to) {        // a stream's tiles are at most four apart
        slot += to - at;
        at = to;
        if (slot >= P::SLOTS) slot -= P::SLOTS;
      };
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        st[x].n_qk = st[x].n_pv = st[x].left = st[x].seq = 0;
        st[x].first = st[x].q_here = false;
        const uint32_t j = job_of(x, 0);
        st[x].k_at = k_pos(j); st[x].k_slot = st[x].k_at % P::SLOTS;
        st[x].v_at = v_pos(j); st[x].v_slot = st[x].v_at % P::SLOTS;
      }
      // Tiles are seen to arrive in the order of the ring, whichever stream they are for: a barrier's parity says which
      // phase is over only to one who has seen the phase before it, and a slot's phase before may be the other stream's.
      uint32_t arrived = 0, a_slot = 0, a_phase = 0;
      uint32_t polls = 0;
      long long idle_since = 0;
      while (st[0].n_pv != n_run[0] || st[1].n_pv != n_run[1]) {
        bool moved = false;
        // a poll is a round trip to shared memory, 200 cycles and more while the tensor core streams from it
        const uint32_t polled = mbar_test3(bar(P::BAR_P), st[0].n_pv & 1, bar(P::BAR_P + 1), st[1].n_pv & 1, bar(P::BAR_FULL + a_slot), a_phase);
        if ((polled & 4) && arrived != 2 * n_steps) {
          ++arrived;
          if (++a_slot == P::SLOTS) { a_slot = 0; a_phase ^= 1; }
          moved = true;
        }
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          Stream& t = st[x];
          if (t.n_qk != t.n_pv && t.v_at < arrived && ((polled >> x) & 1)) {
            tc_fence_after();
            const uint32_t dv = d_v + t.v_slot * (P::SLOT >> 4);
#pragma unroll
            for (int kk = 0; kk < kTile / 16; ++kk)
              mma_ts_lo(tmem + P::O_COL + x * P::O_STEP, tmem + P::S_COL + x * 128 + kk * 8, dv + kk * (16 * 128 >> 4), idesc_pv, kk > 0 || !t.first);
            mma_commit(bar(P::BAR_PV + x));
            mma_commit(bar(P::BAR_FREE + t.v_slot));
            ++t.n_pv;
            t.first = false;
            advance(t.v_at, t.v_slot, v_pos(job_of(x, t.n_pv)));
            moved = true;
          }
          if (t.n_qk == t.n_pv && t.n_qk != n_run[x]) {
            if (t.left == 0) {
              const uint32_t e = x * kUnitRing + t.seq % kUnitRing;
              if (mbar_test(bar(P::BAR_UNIT + e), (t.seq / kUnitRing) & 1)) {
                t.left = units[e].n_tiles;
                mbar_arrive(bar(P::BAR_UFREE + e));
                ++t.seq;
                t.q_here = false;
                t.first = true;
              }
            }
            if (t.left != 0 && t.k_at < arrived) {
              if (!t.q_here) t.q_here = mbar_test(bar(P::BAR_QFULL + x), (t.seq - 1) & 1);
              if (t.q_here) {
                tc_fence_after();
                const uint32_t dq = d_q + x * (P::QHALF >> 4), dk = d_k + t.k_slot * (P::SLOT >> 4);
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk)
                  mma_ss_lo(tmem + P::S_COL + x * 128, dq + (kk >> 2) * (P::QBOX >> 4) + (kk & 3) * 2, dk + (kk >> 2) * (P::KBOX >> 4) + (kk & 3) * 2,
                            idesc_qk, kk > 0);
                mma_commit(bar(P::BAR_S + x));
                mma_commit(bar(P::BAR_FREE + t.k_slot));
                if (--t.left == 0) mma_commit(bar(P::BAR_QFREE + x));
                ++t.n_qk;
                advance(t.k_at, t.k_slot, k_pos(job_of(x, t.n_qk)));
                moved = true;
              }
            }
          }
        }
        if (moved) {
          idle_since = 0;
          polls = 0;
        } else if ((++polls & 63u) == 0u) {
          if (*abort_flag) break;
          if ((polls & 4095u) == 0u) {
            const long long now = clock64();
            if (idle_since == 0) idle_since = now;
            else if (now - idle_since > kWaitCycles) {
              *abort_flag = 1;
              if (atomicCAS(a.status, 0, (int)SP_ERR_TIMEOUT) == 0) a.status[1] = 60;
              break;
            }
          }
        }
      }
    }
    __syncwarp();
  } else if (narrow) {
    narrow_warps<D>(a, work, smem, ab);
  } else {
    // ------------------------------------------------------------ softmax and epilogue
    const int x = warp >> 2;                          // stream
    const int row = threadIdx.x & 127;                // TMEM lane, row of the stream
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t t_s = tmem + lanes + P::S_COL + x * 128, t_o = tmem + lanes + P::O_COL + x * P::O_STEP;
    const float scale = a.scale_log2;
    bool ok = true;
    uint32_t n_jobs = 0;                              // of this stream so far
    for (int seq = 0; ok; ++seq) {
      const int e = x * kUnitRing + seq % kUnitRing;
      ok = __all_sync(0xffffffffu, mbar_wait(bar(P::BAR_UNIT + e), (seq / kUnitRing) & 1, ab, 30));
      if (!ok) break;
      const Unit& u = units[e];                       // stays in shared memory until the unit is done: registers are short
      const int n_tiles = u.n_tiles;
      if (n_tiles == 0) break;
      const bool warp_live = (warp & 3) * 32 < u.rows, live = row < u.rows;
      const int abs_row = u.r0 + row;
      const int token = abs_row / a.group, head = u.g * a.group + abs_row % a.group;
      const int kt0 = u.kt0, no_mask = min(u.past, u.len);      // keys before it are seen by every row
      float m_ref = live ? kNoMax : -kNoMax, l = 0.f;           // lanes without a row: all weights zero
      for (int t = 0; t < n_tiles && ok; ++t) {
        const int k0 = (kt0 + t) * kTile;
        const bool special = k0 + kTile > no_mask;
        ok = __all_sync(0xffffffffu, mbar_wait(bar(P::BAR_S + x), n_jobs & 1, ab, 31));
        if (!ok) break;
        tc_fence_after();
        if (warp_live) {
          // Four chunks of 32 logits, the next one's load in flight, each a step of the running softmax.  The reference
          // moves, to a whole number, when the row maximum has grown by more than 2^8.
          if (special) mask_tmem(a, u, live ? token : -1, k0, t_s);
          uint32_t s[2][32];
          float sum = 0.f;
          tmem_ld32_async(t_s, s[0]);
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            tmem_ld_wait();
            reg_fence32(s[c & 1]);
            const uint32_t* y = s[c & 1];
            auto val = [&](int e) { return __uint_as_float(y[e]); };
            float m0 = max3(val(0), val(1), val(2)), m1 = max3(val(3), val(4), val(5)), m2 = max3(val(6), val(7), val(8)),
                  m3 = max3(val(9), val(10), val(11));
#pragma unroll
            for (int e = 12; e < 28; e += 8) {
              m0 = max3(m0, val(e), val(e + 1));
              m1 = max3(m1, val(e + 2), val(e + 3));
              m2 = max3(m2, val(e + 4), val(e + 5));
              m3 = max3(m3, val(e + 6), val(e + 7));
            }
            m0 = max3(m0, val(28), val(29));
            m1 = max3(m1, val(30), val(31));
            const float mx = fmaxf(fmaxf(m0, m1), fmaxf(m2, m3)) * scale;
            const bool grown = mx > m_ref + 8.f;              // never in lanes without a row
            if (__any_sync(0xffffffffu, grown)) {
              const float m_new = grown ? ceilf(mx) : m_ref;
              const float alpha = ex2_approx(m_ref - m_new);
              // the stream's previous product came before this S, and nothing of this P has been handed over
              rescale_tmem<D>(t_o, t_s, alpha, c, t > 0);
              l *= alpha;
              sum *= alpha;
              m_ref = m_new;
            }
            // not before the call above: its registers must not be moved while the load is under way
            if (c < 3) tmem_ld32_async(t_s + (c + 1) * 32, s[(c + 1) & 1]);
            const float2 sc2 = make_float2(scale, scale), nm2 = make_float2(-m_ref, -m_ref);
            float2 sum01 = make_float2(0.f, 0.f), sum23 = make_float2(0.f, 0.f);
            uint32_t p[16];
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
            sum += (sum01.x + sum01.y) + (sum23.x + sum23.y);
            tmem_st16(t_s + c * 16, p);
          }
          l += sum;
          tmem_wait_st();
        }
        if (special) {
          // Values behind the sequence count as zero, and so do non-finite ones of new tokens (see add_nonfinite).  V comes
          // after K, hence not before the softmax.  S of the tile was there, so every tile up to its K has arrived, the one
          // before V in V's slot among them: the barrier's parity can be told.
          const uint32_t p = v_pos(job_of(x, n_jobs)), s = p % P::SLOTS;
          ok = __all_sync(0xffffffffu, mbar_wait(bar(P::BAR_FULL + s), (p / P::SLOTS) & 1, ab, 32));
          if (!ok) break;
          // each warp of the stream 32 keys
          const int r_lo = (warp & 3) * 32, lo = max(no_mask - k0, r_lo);
          if (lo < r_lo + 32) {
            uint32_t* v = reinterpret_cast<uint32_t*>(smem + P::RING_OFF + s * P::SLOT) + lane;
            // the tags before the zeros: in a wide unit both streams clean the same tile, and who finds zeros finds its tag
            clean_values<D>(v, lo, r_lo + 32, u.len - k0, bad_tag, wide ? 0 : x, wide ? 1 : x, seq + 1);
          }
          fence_async_smem();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(P::BAR_P + x));
        ++n_jobs;
      }
      if (ok) ok = __all_sync(0xffffffffu, mbar_wait(bar(P::BAR_PV + x), (n_jobs - 1) & 1, ab, 33));
      if (ok) {
        tc_fence_after();
        if (warp_live) {
          write_rows<D>(a, work, u, x, row, token, head, t_o, m_ref, l, bad_tag[x * 8 + (seq + 1) % 8] == seq + 1);
          __syncwarp();
        }
        tc_fence_before();                            // O has left TMEM: before the P after which the next product overwrites it
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(P::BAR_UFREE + e));
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == kIssuer && !narrow) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

// Joins the parts of the cut units, in the order of the keys: the part of the worker in which a unit begins, then those
// of the workers after it.  A warp reads a row's part at once (its 32 lanes the columns).  The work is a few MB from L2 at most
// and all latency, so it is spread as widely as it goes: every block lists the cut units (one per worker of the first
// kernel at most) and takes every gridDim.x-th run of rows; as long as the device has warps to spare, 2, 4 or 8 of them share
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
  // rows of the unit that begins in worker i and goes on in later ones; thread t looks after workers per * t ...
  const int per = (2 * n_cta + kJoinWarps * 32 - 1) / (kJoinWarps * 32);
  auto rows_of = [&](int i) { return i < 2 * n_cta && work.meta[i].last >= 0 ? work.meta[i].rows : 0; };
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
            const int w = owner + p, stream = w >= n_cta;          // wide: never
            const size_t slot = ((size_t)(w - stream * n_cta) * 2 + (p == 0 ? 1 : 0)) * kUnitRows + stream * 128 + r;
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

// [pages, heads, page, D] cache -> 4-D tensor map with a (64 columns x page rows, 128 at most) box, 128-byte swizzle.
bool make_cache_map(CUtensorMap* m, const PagedCache& c, int d, int page, int heads, int pages) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  // the stride of a size-1 dimension is never used, but the encoder wants a valid one
  const cuuint64_t any = (cuuint64_t)d * 2;
  cuuint64_t dims[4] = {(cuuint64_t)d, (cuuint64_t)page, (cuuint64_t)heads, (cuuint64_t)pages};
  cuuint64_t strides[3] = {(cuuint64_t)c.s_tok * 2, heads > 1 ? (cuuint64_t)c.s_head * 2 : any, pages > 1 ? (cuuint64_t)c.s_page * 2 : any};
  cuuint32_t box[4] = {64, (cuuint32_t)(page < kTile ? page : kTile), 1, 1};
  cuuint32_t estr[4] = {1, 1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, c.data, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D>
cudaError_t launch(const TreeAttnArgs& a, void* ws, int n_cta, cudaStream_t s) {
  CUtensorMap tk, tv;
  if (!make_cache_map(&tk, a.kc, D, 1 << a.page_log2, a.hkv, a.n_pages) || !make_cache_map(&tv, a.vc, D, 1 << a.page_log2, a.hkv, a.n_pages))
    return cudaErrorInvalidValue;
  Work w;
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
  return (size_t)n_sm * (2 * kUnitRows * (128 * sizeof(float) + sizeof(float2)) + 2 * sizeof(Meta));
}

cudaError_t launch_tree_attn(const TreeAttnArgs& a, void* ws, int n_sm, cudaStream_t s) {
  return a.d == 128 ? launch<128>(a, ws, n_sm, s) : launch<64>(a, ws, n_sm, s);
}

}  // namespace sp
