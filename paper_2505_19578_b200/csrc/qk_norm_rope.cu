// Norm of every query and key head, position rotation, and the move of q, k, v from the projection's rows into
// head-major tensors and/or the paged cache, in one pass over the data.  The paper has no counterpart (its models do
// this before the attention it describes).
//
//   y = x / sqrt(mean(x^2) + eps) * w       (each head on its own; left out without weights)
//   (a, b) -> (a cos - b sin, b cos + a sin)  for each rotated pair, angle = position * inv_freq
//
// Bound by memory: every element is read once and written once per destination.  A head is held by D / 16 lanes, each
// with two 8-element pieces chosen so that both members of every rotated pair sit in one lane: nothing is exchanged but
// the sum of squares.  The sines and cosines of a token's pairs are computed by the warp's lanes, two pairs each, handed
// round by shuffles and used for all the heads that the warp walks.
//
// Angles: the turns per position of each pair are a 64-bit fraction of a turn (rounded down: 2^-33 of a turn at a 31-bit
// position), so that position * frequency modulo one turn is one wrapping integer product; its top 32 bits (2^-32 cut off) go
// to sincospif as fp32 half turns (24 bits: 2^-26 of a turn).  Under 2^-25 of a turn in all, at any position; fp32 products would be off by
// 4e-3 rad at position 1e5.  Everything else is fp32, rounded once to bf16.
//
// The form for a cache held in 4 bits (q4.cuh has the format) stores keys and values as codes with a scale for each 32
// elements of a head: a = max |y|, s = a / 7 to four significant bits, code = y / s to the nearest, both ties to even.  An
// 8-element piece is a word of codes.  Keys are quantised from the fp32 values, not from their bf16 rounding.  The code is
// the one that exact arithmetic gives: where the fp32 value lies within its own error of a border between two codes or two
// scales, the warp computes the pass again in 64 bits (of the passes of four heads of 128 elements 1.4 %, 0.5 % without a
// norm, by the bounds below on normal values).  So the same token has the same codes
// whichever kernel stored it, and a border decides nothing by chance.
// That form is bound by instructions: a warp's pass over four heads of 128 elements is 250 for queries and 480 for keys and values (K with
// its borders more, V less), and the schedulers issue in 60 % of the cycles, four warps of long chains each.  131072 rows of 48 heads
// 711 us (2.8 GB: 431 at the copy rate), 16384 rows 98, 1000 rows of 36 heads 9.6, one row 2.4.
#include <math_constants.h>

#include "q4.cuh"

namespace sp {
namespace {

// Arithmetic on pairs of neighbouring elements, one instruction for both.  (With single ones a pass over four heads was 320
// instructions and the schedulers two thirds busy: 1000 rows of 36 heads 8.9 instead of 7.5 us, 16384 rows 67 instead of 60.)
__device__ __forceinline__ void unpack8(const uint4& u, float2 (&x)[4]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
}
__device__ __forceinline__ uint4 pack8(const float2 (&x)[4]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    __nv_bfloat162 h = __floats2bfloat162_rn(x[i].x, x[i].y);
    w[i] = *reinterpret_cast<uint32_t*>(&h);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }

// A pass of a warp: 32 / (D / 16) heads of one token, this lane two pieces of one of them.
struct Pass {
  int kind, head;                  // 0 q, 1 k, 2 v, -1 nothing for this lane
};
template <int D>
struct Lane {
  static constexpr int LPH = D / 16, HPW = 32 / LPH;      // lanes per head, heads per pass
  int l, hw, c0, c1;               // lane in the head, head in the pass, the two pieces
  int from0, from1;
  bool turn0, turn1;               // which of the pieces turn
  __device__ __forceinline__ Lane(const RopeArgs& a, int lane) {
    l = lane % LPH;
    hw = lane / LPH;
    // neighbouring lanes have neighbouring pieces: 2 l, 2 l + 1 would read and write every 32-byte sector twice
    const int turning = a.rot / 16;                // half: the first `turning` lanes have pairs (piece l, piece l + turning)
    const bool rest = !a.interleaved && l >= turning;
    c0 = rest ? l + turning : l;
    c1 = a.interleaved || rest ? l + LPH : l + turning;
    turn0 = a.interleaved ? c0 < 2 * turning : !rest;
    turn1 = a.interleaved ? c1 < 2 * turning : !rest;
    // the pairs of the lane's angles 0-3 and 4-7, four at a time: pair 4 i + e was computed by lane 2 i + e / 2
    from0 = 2 * (a.interleaved ? c0 : 2 * l);
    from1 = 2 * (a.interleaved ? c1 : 2 * l + 1);
  }
  __device__ __forceinline__ Pass pass(const RopeArgs& a, int p) const {
    const int pq = (a.hq + HPW - 1) / HPW, pkv = (a.hkv + HPW - 1) / HPW;
    const int kind = p < pq ? 0 : p < pq + pkv ? 1 : 2;
    const int head = (p - (kind == 0 ? 0 : kind == 1 ? pq : pq + pkv)) * HPW + hw;
    return {p < pq + 2 * pkv && head < (kind == 0 ? a.hq : a.hkv) ? kind : -1, head};
  }
  __device__ __forceinline__ const __nv_bfloat16* source(const RopeArgs& a, const Pass& p, int t) const {
    return p.kind == 0 ? a.q + p.head * a.q_sh + t * a.q_sn : p.kind == 1 ? a.k + p.head * a.k_sh + t * a.k_sn : a.v + p.head * a.v_sh + t * a.v_sn;
  }
};

// Turns per position of the two pairs whose sine and cosine this lane computes (pairs 2 lane, 2 lane + 1).
__device__ __forceinline__ void lane_phases(const RopeArgs& a, int lane, uint64_t (&f)[2]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) f[i] = 2 * lane + i < a.rot / 2 ? a.phase[2 * lane + i] : 0;
}
// Cosine and sine of the eight pairs of this lane's pieces (1 and 0 where nothing turns).  Whole warps.
template <int D>
__device__ __forceinline__ void angles(const uint64_t (&f)[2], int pos, const Lane<D>& ln, float (&cs)[8], float (&sn)[8]) {
  float c[2], s[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint64_t turns = f[i] * (uint64_t)(int64_t)pos;                      // modulo one turn
    sincospif((float)(int32_t)(uint32_t)(turns >> 32) * 4.656612873077393e-10f /* 2^-31: half turns */, &s[i], &c[i]);
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int from = ((e < 4 ? ln.from0 : ln.from1) + ((e & 3) >> 1)) & 31;
    const float ce = __shfl_sync(0xffffffffu, c[e & 1], from), se = __shfl_sync(0xffffffffu, s[e & 1], from);
    const bool turn = e < 4 ? ln.turn0 : ln.turn1;
    cs[e] = turn ? ce : 1.f;
    sn[e] = turn ? se : 0.f;
  }
}

// The largest of the lanes' v0 (piece c0) and v1 (piece c1) over the pieces of each piece's group of 32 elements.  Whole warps.
__device__ __forceinline__ double larger(double x, double y) { return fmax(x, y); }
__device__ __forceinline__ float larger(float x, float y) {            // a NaN if either is one
  float z;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(z) : "f"(x), "f"(y));
  return z;
}
template <int D, typename T>
__device__ __forceinline__ void group_max(const RopeArgs& a, const Lane<D>& ln, T& v0, T& v1) {
  constexpr uint32_t kAll = 0xffffffffu;
  if (a.interleaved || a.rot % 64 == 0) {          // a group's four pieces are those of four neighbouring lanes
#pragma unroll
    for (int o = 1; o <= 2; o <<= 1) {
      v0 = larger(v0, __shfl_xor_sync(kAll, v0, o));
      v1 = larger(v1, __shfl_xor_sync(kAll, v1, o));
    }
    return;
  }
  T m0 = 0, m1 = 0;
#pragma unroll 1
  for (int y = 0; y < D / 32; ++y) {
    T m = larger(ln.c0 >> 2 == y ? v0 : (T)0, ln.c1 >> 2 == y ? v1 : (T)0);
#pragma unroll
    for (int o = 1; o < Lane<D>::LPH; o <<= 1) m = larger(m, __shfl_xor_sync(kAll, m, o));
    if (ln.c0 >> 2 == y) m0 = m;
    if (ln.c1 >> 2 == y) m1 = m;
  }
  v0 = m0;
  v1 = m1;
}

struct Codes {                     // of a lane's two pieces: words of codes, and their groups' scale bytes
  uint32_t word0, word1, scale0, scale1;
};
__device__ __forceinline__ uint32_t clamp_scale(uint32_t bits) { return min(max(bits, kScaleLeast), kScaleMost); }
// x / y, where r is 1 / y to an ulp: exact where the quotient has an fp32 (ties between codes and scales do).
__device__ __forceinline__ float quotient(float x, float y, float r) {
  const float q = x * r;
  return fmaf(fmaf(-q, y, x), r, q);
}
// Scale of a group whose largest magnitude is a, as fp32 bits: a / 7 to three bits behind the leading one, ties to even.
__device__ __forceinline__ uint32_t seventh(float a) { return __float_as_uint(quotient(a, 7.f, 1.f / 7.f)); }
__device__ __forceinline__ uint32_t scale_bits(uint32_t u) { return clamp_scale((u + 0x7ffffu + (u >> 20 & 1u)) & 0xfff00000u); }
// An error of at most err > 0 in a could change the scale that u, a / 7, is rounded to.  The border in the middle of u's own
// interval is the one in question where the error is below a 128th of a; below 7 * 2^-20 * (1 + 1/16) there is none.
__device__ __forceinline__ bool near_border(uint32_t u, float a, float err) {
  const float border = __uint_as_float((u & 0xfff00000u) | 0x80000u);
  return (fabsf(__uint_as_float(u) - border) <= err * 0.143f || err * 128.f > a) && err > 0.f && a + err > 7e-6f;
}
__device__ __forceinline__ uint32_t scale_byte(uint32_t bits) { return (bits - kScaleLeast) >> 20; }

// Codes of eight elements of at most 7.5 s; `far`: the largest distance of one from its code's value.  Sums with 1.5 * 2^23 + 8
// round to whole numbers, ties to even, and leave the code in the low bits (rounding and conversion instructions run at a
// sixteenth of the rate).  Without EXACT the quotient is off by 2.4e-7 of itself, relative, which is less than the error that
// an element of a normed or rotated key is taken to have: whatever that could change is computed again.
template <bool EXACT>
__device__ __forceinline__ uint32_t piece_codes(const float2 (&v)[4], float s, float& far) {
  float inv;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(s));
  uint32_t pair[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float2 t = __fmul2_rn(v[i], both(inv));
    if (EXACT) t = __ffma2_rn(__ffma2_rn(t, both(-s), v[i]), both(inv), t);
    const float2 c = __fadd2_rn(t, both(12582920.f)), r = __ffma2_rn(__fadd2_rn(c, both(-12582920.f)), both(-s), v[i]);
    far = fmaxf(fmaxf(far, fabsf(r.x)), fabsf(r.y));
    pair[i] = __byte_perm(__float_as_uint(c.x), __float_as_uint(c.y), 0x5410);
  }
  return ((pair[3] * 16 + pair[2]) * 16 + pair[1]) * 16 + pair[0];
}

__device__ __forceinline__ double quotient(double x, double y, double r) {
  const double q = x * r;
  return fma(fma(-q, y, x), r, q);
}
// The codes of a pass of keys in 64 bits, from its inputs.  Out of line and rare, but a step of a few tokens waits for it: sines
// and cosines are shared by the warp's lanes as in fp32, and nothing is divided.  Whole warps.
template <int D>
__device__ __noinline__ Codes exact_codes(const RopeArgs& a, int pos, uint4 in0, uint4 in1) {
  constexpr uint32_t kAll = 0xffffffffu;
  const int lane = threadIdx.x & 31;
  const Lane<D> ln(a, lane);
  double y[2][8];
  {
    float2 x0[4], x1[4];
    unpack8(in0, x0);
    unpack8(in1, x1);
#pragma unroll
    for (int i = 0; i < 4; ++i) { y[0][2 * i] = x0[i].x; y[0][2 * i + 1] = x0[i].y; y[1][2 * i] = x1[i].x; y[1][2 * i + 1] = x1[i].y; }
  }
  if (a.k_weight) {
    double ss[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) ss[i] = fma(y[0][i], y[0][i], fma(y[0][4 + i], y[0][4 + i], fma(y[1][i], y[1][i], y[1][4 + i] * y[1][4 + i])));
    double sum = (ss[0] + ss[1]) + (ss[2] + ss[3]);
#pragma unroll
    for (int o = Lane<D>::LPH / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(kAll, sum, o);
    const double inv = rsqrt(sum * (1.0 / D) + (double)a.eps);
    float2 w0[4], w1[4];
    unpack8(__ldg(reinterpret_cast<const uint4*>(a.k_weight + ln.c0 * 8)), w0);
    unpack8(__ldg(reinterpret_cast<const uint4*>(a.k_weight + ln.c1 * 8)), w1);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      y[0][2 * i] *= inv * w0[i].x; y[0][2 * i + 1] *= inv * w0[i].y;
      y[1][2 * i] *= inv * w1[i].x; y[1][2 * i + 1] *= inv * w1[i].y;
    }
  }
  if (a.rot > 0) {
    double c[2], s[2];                             // of pairs 2 lane, 2 lane + 1
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint64_t f = 2 * lane + i < a.rot / 2 ? a.phase[2 * lane + i] : 0;
      sincospi((double)(int64_t)(f * (uint64_t)(int64_t)pos) * 1.0842021724855044e-19 /* 2^-63: half turns */, &s[i], &c[i]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int from = ((e < 4 ? ln.from0 : ln.from1) + ((e & 3) >> 1)) & 31;
      const double ce = __shfl_sync(kAll, c[e & 1], from), se = __shfl_sync(kAll, s[e & 1], from);
      if (!(e < 4 ? ln.turn0 : ln.turn1)) continue;
      double& u = a.interleaved ? y[e >> 2][2 * (e & 3)] : y[0][e];
      double& v = a.interleaved ? y[e >> 2][2 * (e & 3) + 1] : y[1][e];
      const double w = u * ce - v * se;
      v = v * ce + u * se;
      u = w;
    }
  }
  double m[2];
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    m[x] = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m[x] = fmax(m[x], fabs(y[x][i]));
  }
  group_max<D>(a, ln, m[0], m[1]);
  Codes out;
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    // the same rounding of a / 7 as scale_bits, on the bits of a double; clamped first, so that the result is one of fp32
    const double f = quotient(fmin(fmax(m[x], 7 * 9.5367431640625e-07), 7 * 3840.0), 7.0, 1.0 / 7);
    const unsigned long long u = (unsigned long long)__double_as_longlong(f), odd = u >> 49 & 1;
    const double s = __longlong_as_double((long long)((u + ((1ull << 48) - 1) + odd) & ~((1ull << 49) - 1))), r = 1.0 / s;
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const double z = y[x][i], t = rint(quotient(z == z ? fmin(fmax(z, -7 * s), 7 * s) : 0.0, s, r));
      w |= (uint32_t)(__double2int_rn(t) + 8) << (4 * (i >> 1) + 16 * (i & 1));
    }
    const uint32_t byte = scale_byte(clamp_scale(__float_as_uint((float)s)));
    if (x == 0) { out.word0 = w; out.scale0 = byte; } else { out.word1 = w; out.scale1 = byte; }
  }
  return out;
}

// Codes of a pass of keys (its pieces x, y in fp32, each off by `err` at most, any of the head by `top_err`) or values (0, 0).
// Whole warps.
template <int D>
__device__ __forceinline__ Codes codes_of(const RopeArgs& a, const Lane<D>& ln, bool is_v, bool normed, float err, float top_err, int pos, uint4 in0, uint4 in1,
                                          const float2 (&x)[4], const float2 (&y)[4]) {
  float a0 = 0.f, a1 = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    a0 = larger(larger(a0, fabsf(x[i].x)), fabsf(x[i].y));
    a1 = larger(larger(a1, fabsf(y[i].x)), fabsf(y[i].y));
  }
  group_max<D>(a, ln, a0, a1);
  constexpr float kMost = 7.f * 3840.f;            // 7 times the largest scale
  Codes c;
  bool unsure = !(top_err < 1e30f);
  if (__any_sync(0xffffffffu, !(a0 <= kMost && a1 <= kMost))) {
    // something is not finite, or beyond the largest scale: a NaN counts as zero, the rest as 7 times the scale at most
    float2 u[4], v[4];
    auto in_range = [&](float z) { return z == z ? fminf(fmaxf(z, -kMost), kMost) : 0.f; };
    a0 = a1 = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      u[i] = make_float2(in_range(x[i].x), in_range(x[i].y));
      v[i] = make_float2(in_range(y[i].x), in_range(y[i].y));
      a0 = fmaxf(fmaxf(a0, fabsf(u[i].x)), fabsf(u[i].y));
      a1 = fmaxf(fmaxf(a1, fabsf(v[i].x)), fabsf(v[i].y));
    }
    group_max<D>(a, ln, a0, a1);
    float far = 0.f;
    const uint32_t s0 = scale_bits(seventh(a0)), s1 = scale_bits(seventh(a1));
    c = {piece_codes<true>(u, __uint_as_float(s0), far), piece_codes<true>(v, __uint_as_float(s1), far), scale_byte(s0), scale_byte(s1)};
    unsure |= top_err > 0.f;
  } else {
    const uint32_t u0 = seventh(a0), u1 = seventh(a1), s0 = scale_bits(u0), s1 = scale_bits(u1);
    const float f0 = __uint_as_float(s0), f1 = __uint_as_float(s1);
    float far0 = 0.f, far1 = 0.f;
    c.scale0 = scale_byte(s0);
    c.scale1 = scale_byte(s1);
    if (is_v || !(normed || a.rot == D)) {         // elements that are as they came lie on borders between codes
      c.word0 = piece_codes<true>(x, f0, far0);
      c.word1 = piece_codes<true>(y, f1, far1);
    } else {
      c.word0 = piece_codes<false>(x, f0, far0);
      c.word1 = piece_codes<false>(y, f1, far1);
    }
    if (!is_v) {
      // a border between two codes or two scales within the error
      if (normed || ln.turn0) unsure |= far0 >= 0.5f * f0 - err;
      if (normed || ln.turn1) unsure |= far1 >= 0.5f * f1 - err;
      unsure |= near_border(u0, a0, top_err) || near_border(u1, a1, top_err);
    }
  }
  if (!is_v && __any_sync(0xffffffffu, unsure)) c = exact_codes<D>(a, pos, in0, in1);
  return c;
}

// Norm and rotation of one pass (q and k; v goes through as it is) and its stores.  Whole warps.  Q4: keys and values go into
// the 4-bit cache.
template <int D, bool Q4>
__device__ __forceinline__ void finish_pass(const RopeArgs& a, const Lane<D>& ln, const Pass& p, bool is_v, bool is_q, int t, int slot, int pos, uint4 in0, uint4 in1,
                                            const float (&cs)[8], const float (&sn)[8]) {
  Codes codes;
  float2 x[4], y[4];
  float err = 0.f, top_err = 0.f;
  if (!is_v || Q4) {                               // uniform over the warp, as is all that depends on the kind
    unpack8(in0, x);
    unpack8(in1, y);
  }
  if (!is_v) {
    bool odd = false;                              // the squares' sum left the range in which fp32 has it to the bound below
    const __nv_bfloat16* weight = is_q ? a.q_weight : a.k_weight;
    if (weight) {
      float2 sum = __fmul2_rn(x[0], x[0]);
#pragma unroll
      for (int i = 1; i < 4; ++i) sum = __ffma2_rn(x[i], x[i], sum);
#pragma unroll
      for (int i = 0; i < 4; ++i) sum = __ffma2_rn(y[i], y[i], sum);
      float ss = sum.x + sum.y;
#pragma unroll
      for (int o = Lane<D>::LPH / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
      if (Q4 && !is_q) odd = !(ss <= 1e38f) || (ss < 1e-30f && a.eps < 1e-20f);
      const float2 inv = both(rsqrtf(ss * (1.f / D) + a.eps));       // 2 ulp of fp32
      float2 wx[4], wy[4];
      unpack8(__ldg(reinterpret_cast<const uint4*>(weight + ln.c0 * 8)), wx);
      unpack8(__ldg(reinterpret_cast<const uint4*>(weight + ln.c1 * 8)), wy);
#pragma unroll
      for (int i = 0; i < 4; ++i) { x[i] = __fmul2_rn(x[i], __fmul2_rn(inv, wx[i])); y[i] = __fmul2_rn(y[i], __fmul2_rn(inv, wy[i])); }
    }
    if (Q4 && !is_q && (weight || a.rot > 0)) {
      // fp32: the angle is off by 2^-26 of a turn, 1e-7, sine and cosine by 1.2e-7 and the rotation's two roundings by as much,
      // 3.4e-7 of |a| + |b| for each pair; the norm by 8.4e-7, relative (16 roundings of the sum of squares, halved by the root: 4.8e-7,
      // its 2 ulp: 2.4e-7, and two products: 1.2e-7), 1.2e-6 with it.  Taken to be 6e-7 and 1.5e-6
      float pair = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 u = a.interleaved ? make_float2(fabsf(x[i].x) + fabsf(x[i].y), fabsf(y[i].x) + fabsf(y[i].y)) :
                                         make_float2(fabsf(x[i].x) + fabsf(y[i].x), fabsf(x[i].y) + fabsf(y[i].y));
        pair = fmaxf(fmaxf(pair, u.x), u.y);
      }
      err = top_err = pair * (weight ? 1.5e-6f : 6e-7f);
#pragma unroll
      for (int o = Lane<D>::LPH / 2; o > 0; o >>= 1) top_err = fmaxf(top_err, __shfl_xor_sync(0xffffffffu, top_err, o));
      if (odd) top_err = CUDART_INF_F;
    }
    if (ln.turn0 || ln.turn1) {
      if (a.interleaved) {
        auto turn = [](float2 v, float c, float s) { return __ffma2_rn(v, both(c), __fmul2_rn(make_float2(v.y, v.x), make_float2(-s, s))); };
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[i] = turn(x[i], cs[i], sn[i]); y[i] = turn(y[i], cs[4 + i], sn[4 + i]); }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 xa = x[i], xb = y[i], c = make_float2(cs[2 * i], cs[2 * i + 1]), s = make_float2(sn[2 * i], sn[2 * i + 1]);
          x[i] = __ffma2_rn(xa, c, __fmul2_rn(xb, make_float2(-s.x, -s.y)));
          y[i] = __ffma2_rn(xb, c, __fmul2_rn(xa, s));
        }
      }
    }
  }
  if (Q4 && !is_q) codes = codes_of<D>(a, ln, is_v, !is_v && a.k_weight != nullptr, err, top_err, pos, in0, in1, x, y);
  if (!is_v) {
    in0 = pack8(x);
    in1 = pack8(y);
  }
  if (p.kind < 0) return;
  auto put = [&](__nv_bfloat16* dst) {
    *reinterpret_cast<uint4*>(dst + ln.c0 * 8) = in0;
    *reinterpret_cast<uint4*>(dst + ln.c1 * 8) = in1;
  };
  if (p.kind == 0) {
    put(a.q_out + p.head * a.qo_sh + t * a.qo_sn);
    return;
  }
  const bool k = p.kind == 1;
  if (k ? a.k_out != nullptr : a.v_out != nullptr) put(k ? a.k_out + p.head * a.ko_sh + t * a.ko_sn : a.v_out + p.head * a.vo_sh + t * a.vo_sn);
  if (slot >= 0 && slot < a.n_slots) {             // a negative slot: a row that no request owns
    if (Q4) {
      using B = Block<D>;
      const int in = slot & ((1 << a.page_log2) - 1), i = in & 15;
      uint8_t* block = a.q4 + (int64_t)(slot >> a.page_log2) * a.q4_s_page + p.head * a.q4_s_head + (in >> 4) * B::BYTES;
      *reinterpret_cast<uint32_t*>(block + (k ? B::k_word(i, ln.c0) : B::v_word(i, ln.c0))) = codes.word0;
      *reinterpret_cast<uint32_t*>(block + (k ? B::k_word(i, ln.c1) : B::v_word(i, ln.c1))) = codes.word1;
      if ((ln.c0 & 3) == 0) block[k ? B::k_scale(i, ln.c0 >> 2) : B::v_scale(i, ln.c0 >> 2)] = (uint8_t)codes.scale0;
      if ((ln.c1 & 3) == 0) block[k ? B::k_scale(i, ln.c1 >> 2) : B::v_scale(i, ln.c1 >> 2)] = (uint8_t)codes.scale1;
      return;
    }
    const PagedCache& c = k ? a.kc : a.vc;
    put(c.data + (int64_t)(slot >> a.page_log2) * c.s_page + (slot & ((1 << a.page_log2) - 1)) * c.s_tok + p.head * c.s_head);
  }
}

// Few rows: as many warps per token as fill the device, each its share of the token's passes.
constexpr int kRopeThreads = 128;
template <bool Q4>
__device__ __forceinline__ bool cached(const RopeArgs& a) { return Q4 || a.kc.data != nullptr; }

template <int D, bool Q4>
__global__ void __launch_bounds__(kRopeThreads) qk_norm_rope_kernel(const __grid_constant__ RopeArgs a) {
  constexpr int RUN = 2;                           // passes whose loads are in flight together
  const int lane = threadIdx.x & 31;
  const long long unit = (long long)blockIdx.x * (kRopeThreads / 32) + (threadIdx.x >> 5);
  const int t = (int)(unit / a.splits), split = (int)(unit - (long long)t * a.splits);
  const Lane<D> ln(a, lane);
  uint64_t f[2];
  lane_phases(a, lane, f);
  let_next_start();
  wait_for_previous();
  if (decode_poisoned(a.status) || t >= a.tokens) return;
  const int pq = (a.hq + Lane<D>::HPW - 1) / Lane<D>::HPW, pkv = (a.hkv + Lane<D>::HPW - 1) / Lane<D>::HPW, passes = pq + 2 * pkv;
  const int pos = a.positions[t], slot = cached<Q4>(a) ? a.slots[t] : -1;
  if (slot >= a.n_slots && cached<Q4>(a) && lane == 0) report_range(a.status, Q4 ? (int)kWhereRopeSlotQ4 : (int)kWhereRopeSlot);
  float cs[8], sn[8];
  bool have = false;
  for (int p0 = split; p0 < passes; p0 += RUN * a.splits) {
    uint4 in0[RUN], in1[RUN];
    Pass pass[RUN];
#pragma unroll
    for (int u = 0; u < RUN; ++u) {
      pass[u] = ln.pass(a, p0 + u * a.splits);
      in0[u] = in1[u] = make_uint4(0, 0, 0, 0);
      if (pass[u].kind >= 0) {
        const __nv_bfloat16* src = ln.source(a, pass[u], t);
        in0[u] = __ldcs(reinterpret_cast<const uint4*>(src + ln.c0 * 8));
        in1[u] = __ldcs(reinterpret_cast<const uint4*>(src + ln.c1 * 8));
      }
    }
    if (!have) {                                   // with the first loads under way
      angles<D>(f, pos, ln, cs, sn);
      have = true;
    }
#pragma unroll
    for (int u = 0; u < RUN; ++u) {
      const int p = p0 + u * a.splits;
      if (p < passes) finish_pass<D, Q4>(a, ln, pass[u], p >= pq + pkv, p < pq, t, slot, pos, in0[u], in1[u], cs, sn);
    }
  }
}

// Many rows: one CTA per SM, each warp a share of the (token, three passes) items, which it fetches three items ahead into
// a ring of its own in shared memory (cp.async; a lane reads back only what it has copied, so nothing is synchronised).
// 16 warps have 144 KB under way then, which registers could not hold.  Four passes, two items ahead: 2 % faster for
// 131072 rows of 48 heads, 7 % slower for 1000 rows of 36, whose 9 passes do not divide.
constexpr int kStreamSms = 148, kStreamWarps = 16, kStreamStages = 4, kStreamRun = 3;
constexpr int kStreamItem = kStreamRun * 1024 + 32;        // bytes of an item: 32 lanes x two pieces a pass, position and slot

__device__ __forceinline__ void copy16(uint32_t dst, const void* src) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory"); }
__device__ __forceinline__ void copy4(uint32_t dst, const void* src) { asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory"); }

template <int D, bool Q4>
__global__ void __launch_bounds__(kStreamWarps * 32, 1) qk_norm_rope_stream_kernel(const __grid_constant__ RopeArgs a) {
  extern __shared__ __align__(16) uint8_t smem[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const Lane<D> ln(a, lane);
  uint64_t f[2];
  lane_phases(a, lane, f);
  const int pq = (a.hq + Lane<D>::HPW - 1) / Lane<D>::HPW, pkv = (a.hkv + Lane<D>::HPW - 1) / Lane<D>::HPW, passes = pq + 2 * pkv;
  const int per_token = (passes + kStreamRun - 1) / kStreamRun;
  // The warps' tokens (items, if there are fewer tokens than warps) in turn, so that what is read and written at a time lies
  // together (a run of tokens for each warp: 695 us instead of 640 for 131072 rows).
  const int n_warps = gridDim.x * kStreamWarps, me = warp * gridDim.x + blockIdx.x, span = a.tokens >= n_warps ? per_token : 1;
  // Passes that quantise take three times as long as the others.  Where a token's items would fall to the same SMs in every round,
  // the item that a warp takes is turned on from four warps to the next and from round to round, so that every scheduler has of each
  // (2000 rows of 48 heads: 18.1 instead of 22.1 us).
  const bool turned = Q4 && span == 1 && n_warps % per_token == 0;
  const int jump_t = span > 1 ? n_warps : n_warps / per_token, jump_b = span > 1 ? 1 - per_token : turned ? 1 : n_warps % per_token;
  struct At {                                      // an item
    int t, b;
  };
  auto next = [&](At& x) {
    if (span > 1 && x.b + 1 < per_token) { ++x.b; return; }
    x.t += jump_t;
    x.b += jump_b;
    if (x.b >= per_token) { x.b -= per_token; x.t += turned ? 0 : 1; }
  };
  uint8_t* mine = smem + warp * kStreamStages * kStreamItem;
  const uint32_t mine_at = (uint32_t)__cvta_generic_to_shared(mine);
  let_next_start();
  wait_for_previous();
  if (decode_poisoned(a.status)) return;

  At begin = span > 1 ? At{me, 0} : At{me / per_token, me % per_token};
  if (turned) begin.b = (begin.b + begin.t / max(4 * (int)gridDim.x / per_token, 1)) % per_token;
  At ahead = begin;                                // the item to fetch next
  int fstage = 0;
  auto fetch = [&] {
    if (ahead.t < a.tokens) {
      const uint32_t at = mine_at + fstage * kStreamItem;
#pragma unroll
      for (int u = 0; u < kStreamRun; ++u) {
        const Pass p = ln.pass(a, ahead.b * kStreamRun + u);
        if (p.kind >= 0) {
          const __nv_bfloat16* src = ln.source(a, p, ahead.t);
          copy16(at + u * 1024 + lane * 16, src + ln.c0 * 8);
          copy16(at + u * 1024 + 512 + lane * 16, src + ln.c1 * 8);
        }
      }
      if (lane == 0) copy4(at + kStreamRun * 1024, a.positions + ahead.t);
      if (lane == 1 && cached<Q4>(a)) copy4(at + kStreamRun * 1024 + 4, a.slots + ahead.t);
      next(ahead);
      if (++fstage == kStreamStages) fstage = 0;
    }
    asm volatile("cp.async.commit_group;" ::: "memory");       // an empty one at the end keeps the count
  };
#pragma unroll
  for (int i = 0; i + 1 < kStreamStages; ++i) fetch();
  int stage = 0, angle_of = -1;
  float cs[8], sn[8];
  for (At x = begin; x.t < a.tokens; next(x)) {
    const int t = x.t;
    fetch();
    asm volatile("cp.async.wait_group %0;" ::"n"(kStreamStages - 1) : "memory");
    __syncwarp();                                  // position and slot were copied by lanes 0 and 1
    const uint8_t* at = mine + stage * kStreamItem;
    const int pos = *reinterpret_cast<const int*>(at + kStreamRun * 1024);
    const int slot = cached<Q4>(a) ? *reinterpret_cast<const int*>(at + kStreamRun * 1024 + 4) : -1;
    if (angle_of != t) {
      angles<D>(f, pos, ln, cs, sn);
      angle_of = t;
      if (slot >= a.n_slots && cached<Q4>(a) && lane == 0) report_range(a.status, Q4 ? (int)kWhereRopeSlotQ4 : (int)kWhereRopeSlot);
    }
    const int p0 = x.b * kStreamRun;
    auto finish = [&](const Pass& p, bool is_v, bool is_q, int u) {
      finish_pass<D, Q4>(a, ln, p, is_v, is_q, t, slot, pos, *reinterpret_cast<const uint4*>(at + u * 1024 + lane * 16),
                         *reinterpret_cast<const uint4*>(at + u * 1024 + 512 + lane * 16), cs, sn);
    };
    if (!Q4) {
#pragma unroll
      for (int u = 0; u < kStreamRun; ++u)
        if (p0 + u < passes) finish(ln.pass(a, p0 + u), p0 + u >= pq + pkv, p0 + u < pq, u);
    } else {
      // code of its own for each kind, once: with the three passes of an item of queries side by side it outgrows the instruction
      // cache (131072 rows: 864 instead of 713 us)
      auto kind = [&](int k, int first, int heads, int u) {
        const int head = (p0 + u - first) * Lane<D>::HPW + ln.hw;
        finish(Pass{head < heads ? k : -1, head}, k == 2, k == 0, u);
      };
#pragma unroll 1
      for (int u = 0; u < kStreamRun && p0 + u < passes; ++u) {
        if (p0 + u < pq) kind(0, 0, a.hq, u);
        else if (p0 + u < pq + pkv) kind(1, pq, a.hkv, u);
        else kind(2, pq + pkv, a.hkv, u);
      }
    }
    __syncwarp();                                  // all have read position and slot before the stage is filled again
    if (++stage == kStreamStages) stage = 0;
  }
}

template <int D, bool Q4>
cudaError_t launch(RopeArgs& a, cudaStream_t s) {
  // From an item for every other of the device's warps on, the streaming kernel (36 heads, with it and with the other one:
  // 250 rows 4.8 and 4.2 us, 500 rows 5.5 and 7.0, 1000 rows 7.6 and 8.8; 131072 rows of 48 heads, head-major and cached: 662
  // and 688.  The 4-bit form, 36 heads: 300 rows 7.4 and 6.7, 500 rows 7.7 and 10.2, 1000 rows 9.7 and 11.0, 4000 rows 20.4 and 30.8;
  // 48 heads: 300 rows 7.7 and 6.9, 500 rows 8.2 and 9.4.  What follows can start earlier beside the other one: 1000 rows of 36
  // heads and their attention 56.6 and 57.2, and reading them back 16.7 and 15.9).
  const int passes = (a.hq + Lane<D>::HPW - 1) / Lane<D>::HPW + 2 * ((a.hkv + Lane<D>::HPW - 1) / Lane<D>::HPW);
  const long long items = (long long)a.tokens * ((passes + kStreamRun - 1) / kStreamRun);
  if (items >= kStreamSms * kStreamWarps / 2) {
    constexpr int smem = kStreamWarps * kStreamStages * kStreamItem;
    const cudaError_t e = cudaFuncSetAttribute(qk_norm_rope_stream_kernel<D, Q4>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    return launch_dependent(qk_norm_rope_stream_kernel<D, Q4>, dim3(kStreamSms), dim3(kStreamWarps * 32), smem, s, a);
  }
  // warps to fill the device; of the 4-bit form's (over 128 registers) 12 fit an SM, and more would come in a second wave (1000
  // rows of 36 heads, written and read back: 15.6 us so, 18.5 with 32)
  const long long splits = (148ll * (Q4 ? 12 : 32) + a.tokens - 1) / a.tokens;
  a.splits = (int)(splits > passes ? passes : splits);
  const long long warps = (long long)a.tokens * a.splits;
  return launch_dependent(qk_norm_rope_kernel<D, Q4>, dim3((unsigned)((warps + kRopeThreads / 32 - 1) / (kRopeThreads / 32))), dim3(kRopeThreads), 0, s, a);
}

}  // namespace

cudaError_t launch_qk_norm_rope(RopeArgs& a, cudaStream_t s) { return a.d == 128 ? launch<128, false>(a, s) : launch<64, false>(a, s); }
cudaError_t launch_qk_norm_rope_q4(RopeArgs& a, cudaStream_t s) { return a.d == 128 ? launch<128, true>(a, s) : launch<64, true>(a, s); }

}  // namespace sp
