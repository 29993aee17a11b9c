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
#include "decode.cuh"

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

// Norm and rotation of one pass (q and k; v goes through as it is) and its stores.  Whole warps.
template <int D>
__device__ __forceinline__ void finish_pass(const RopeArgs& a, const Lane<D>& ln, const Pass& p, bool is_v, bool is_q, int t, int slot, uint4 in0, uint4 in1,
                                            const float (&cs)[8], const float (&sn)[8]) {
  if (!is_v) {                                     // uniform over the warp
    float2 x[4], y[4];
    unpack8(in0, x);
    unpack8(in1, y);
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
      const float2 inv = both(rsqrtf(ss * (1.f / D) + a.eps));       // 2 ulp of fp32
      float2 wx[4], wy[4];
      unpack8(__ldg(reinterpret_cast<const uint4*>(weight + ln.c0 * 8)), wx);
      unpack8(__ldg(reinterpret_cast<const uint4*>(weight + ln.c1 * 8)), wy);
#pragma unroll
      for (int i = 0; i < 4; ++i) { x[i] = __fmul2_rn(x[i], __fmul2_rn(inv, wx[i])); y[i] = __fmul2_rn(y[i], __fmul2_rn(inv, wy[i])); }
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
    const PagedCache& c = k ? a.kc : a.vc;
    put(c.data + (int64_t)(slot >> a.page_log2) * c.s_page + (slot & ((1 << a.page_log2) - 1)) * c.s_tok + p.head * c.s_head);
  }
}

// Few rows: as many warps per token as fill the device, each its share of the token's passes.
constexpr int kRopeThreads = 128;

template <int D>
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
  const int pos = a.positions[t], slot = a.kc.data ? a.slots[t] : -1;
  if (slot >= a.n_slots && a.kc.data && lane == 0) report_range(a.status, kWhereRopeSlot);
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
      if (p < passes) finish_pass<D>(a, ln, pass[u], p >= pq + pkv, p < pq, t, slot, in0[u], in1[u], cs, sn);
    }
  }
}

// Many rows: one CTA per SM, each warp a share of the (token, three passes) items, which it fetches three items ahead into
// a ring of its own in shared memory (cp.async; a lane reads back only what it has copied, so nothing is synchronised).
// 16 warps have 144 KB under way then, which registers could not hold.  Four passes, two items ahead: 2 % faster for
// 131072 rows of 48 heads, 7 % slower for 1000 rows of 36, whose 9 passes do not divide.
constexpr int kStreamWarps = 16, kStreamStages = 4, kStreamRun = 3;
constexpr int kStreamItem = kStreamRun * 1024 + 32;        // bytes of an item: 32 lanes x two pieces a pass, position and slot

__device__ __forceinline__ void copy16(uint32_t dst, const void* src) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory"); }
__device__ __forceinline__ void copy4(uint32_t dst, const void* src) { asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory"); }

template <int D>
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
  const int jump_t = span > 1 ? n_warps : n_warps / per_token, jump_b = span > 1 ? 1 - per_token : n_warps % per_token;
  struct At {                                      // an item
    int t, b;
  };
  auto next = [&](At& x) {
    if (span > 1 && x.b + 1 < per_token) { ++x.b; return; }
    x.t += jump_t;
    x.b += jump_b;
    if (x.b >= per_token) { x.b -= per_token; ++x.t; }
  };
  uint8_t* mine = smem + warp * kStreamStages * kStreamItem;
  const uint32_t mine_at = (uint32_t)__cvta_generic_to_shared(mine);
  let_next_start();
  wait_for_previous();
  if (decode_poisoned(a.status)) return;

  const At begin = span > 1 ? At{me, 0} : At{me / per_token, me % per_token};
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
      if (lane == 1 && a.kc.data) copy4(at + kStreamRun * 1024 + 4, a.slots + ahead.t);
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
    const int slot = a.kc.data ? *reinterpret_cast<const int*>(at + kStreamRun * 1024 + 4) : -1;
    if (angle_of != t) {
      angles<D>(f, pos, ln, cs, sn);
      angle_of = t;
      if (slot >= a.n_slots && a.kc.data && lane == 0) report_range(a.status, kWhereRopeSlot);
    }
#pragma unroll
    for (int u = 0; u < kStreamRun; ++u) {
      const int p = x.b * kStreamRun + u;
      if (p < passes)
        finish_pass<D>(a, ln, ln.pass(a, p), p >= pq + pkv, p < pq, t, slot, *reinterpret_cast<const uint4*>(at + u * 1024 + lane * 16),
                       *reinterpret_cast<const uint4*>(at + u * 1024 + 512 + lane * 16), cs, sn);
    }
    __syncwarp();                                  // all have read position and slot before the stage is filled again
    if (++stage == kStreamStages) stage = 0;
  }
}

template <int D>
cudaError_t launch(RopeArgs& a, cudaStream_t s) {
  // From an item for every other of the device's warps on, the streaming kernel (36 heads, with it and with the other one:
  // 250 rows 4.8 and 4.2 us, 500 rows 5.5 and 7.0, 1000 rows 7.6 and 8.8; 131072 rows of 48 heads, head-major and cached: 662
  // and 688).
  const int passes = (a.hq + Lane<D>::HPW - 1) / Lane<D>::HPW + 2 * ((a.hkv + Lane<D>::HPW - 1) / Lane<D>::HPW);
  const long long items = (long long)a.tokens * ((passes + kStreamRun - 1) / kStreamRun);
  if (items >= 148 * kStreamWarps / 2) {
    constexpr int smem = kStreamWarps * kStreamStages * kStreamItem;
    const cudaError_t e = cudaFuncSetAttribute(qk_norm_rope_stream_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    return launch_dependent(qk_norm_rope_stream_kernel<D>, dim3(148), dim3(kStreamWarps * 32), smem, s, a);
  }
  const long long splits = (148ll * 32 + a.tokens - 1) / a.tokens;             // warps to fill the device
  a.splits = (int)(splits > passes ? passes : splits);
  const long long warps = (long long)a.tokens * a.splits;
  return launch_dependent(qk_norm_rope_kernel<D>, dim3((unsigned)((warps + kRopeThreads / 32 - 1) / (kRopeThreads / 32))), dim3(kRopeThreads), 0, s, a);
}

}  // namespace

cudaError_t launch_qk_norm_rope(RopeArgs& a, cudaStream_t s) { return a.d == 128 ? launch<128>(a, s) : launch<64>(a, s); }

}  // namespace sp
