// Norm of every query and key head, position rotation, and the move of q, k, v from the projection's rows into
// head-major tensors and/or the paged cache, in one pass over the data.  The paper has no counterpart (its models do
// this before the attention it describes).
//
//   y = x / sqrt(mean(x^2) + eps) * w       (each head on its own; left out without weights)
//   (a, b) -> (a cos - b sin, b cos + a sin)  for each rotated pair, angle = position * inv_freq
//
// Bound by memory: every element is read once and written once per destination.  A head is held by D / 16 lanes, each
// with two 8-element pieces chosen so that both members of every rotated pair sit in one lane: nothing is exchanged but
// the sum of squares.  The sine and cosine of a token's pairs are computed once per warp and serve all the heads that
// the warp walks.
//
// Angles: the turns per position of each pair are a 64-bit fraction of a turn, so that position * frequency modulo one
// turn is one wrapping integer product, exact at any position; its top 32 bits (2^-33 of a turn off at most) go to
// sincospif.  fp32 products would be off by 4e-3 rad at position 1e5.  Everything else is fp32, rounded once to bf16.
#include "decode.cuh"

namespace sp {
namespace {

constexpr int kRopeThreads = 128;
constexpr int kRopeRun = 4;        // passes whose loads are in flight together

__device__ __forceinline__ void unpack8(const uint4& u, float (&x)[8]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    w[i] = *reinterpret_cast<uint32_t*>(&h);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

template <int D>
__global__ void __launch_bounds__(kRopeThreads) qk_norm_rope_kernel(const __grid_constant__ RopeArgs a) {
  constexpr int LPH = D / 16;      // lanes per head
  constexpr int HPW = 32 / LPH;    // heads per pass of a warp
  let_next_start();
  wait_for_previous();
  if (decode_poisoned(a.status)) return;
  const int lane = threadIdx.x & 31;
  const long long unit = (long long)blockIdx.x * (kRopeThreads / 32) + (threadIdx.x >> 5);
  if (unit >= (long long)a.tokens * a.splits) return;
  const int t = (int)(unit / a.splits), split = (int)(unit - (long long)t * a.splits);
  const int l = lane % LPH, hw = lane / LPH;

  // this lane's two pieces and the first of their pairs
  const int turning = a.rot / 16;                // lanes of a head whose pieces turn
  const bool turn = l < turning;
  const int c0 = (a.interleaved || !turn) ? 2 * l : l;
  const int c1 = (a.interleaved || !turn) ? 2 * l + 1 : l + turning;
  float cs[8], sn[8];
  const int pos = a.positions[t];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    cs[e] = 1.f;
    sn[e] = 0.f;
    if (turn) {
      const uint64_t turns = a.phase[8 * l + e] * (uint64_t)(int64_t)pos;      // modulo one turn
      sincospif((float)(int32_t)(uint32_t)(turns >> 32) * 4.656612873077393e-10f /* 2^-31: half turns */, &sn[e], &cs[e]);
    }
  }
  int64_t cache_off_k = -1, cache_off_v = -1;
  if (a.kc.data) {
    const int slot = a.slots[t];
    if (slot >= a.n_slots) {
      report_range(a.status, kWhereRopeSlot);
    } else if (slot >= 0) {                      // a negative slot: a row that no request owns
      const int64_t page = slot >> a.page_log2, off = slot & ((1 << a.page_log2) - 1);
      cache_off_k = page * a.kc.s_page + off * a.kc.s_tok;
      cache_off_v = page * a.vc.s_page + off * a.vc.s_tok;
    }
  }

  const int pq = (a.hq + HPW - 1) / HPW, pkv = (a.hkv + HPW - 1) / HPW;
  const int passes = pq + 2 * pkv;
  for (int p0 = split; p0 < passes; p0 += kRopeRun * a.splits) {
    uint4 in0[kRopeRun], in1[kRopeRun];
    int kind[kRopeRun], head[kRopeRun];          // 0 q, 1 k, 2 v, -1 nothing
#pragma unroll
    for (int u = 0; u < kRopeRun; ++u) {
      const int p = p0 + u * a.splits;
      kind[u] = p < pq ? 0 : p < pq + pkv ? 1 : 2;
      head[u] = (p - (kind[u] == 0 ? 0 : kind[u] == 1 ? pq : pq + pkv)) * HPW + hw;
      if (p >= passes || head[u] >= (kind[u] == 0 ? a.hq : a.hkv)) kind[u] = -1;
      in0[u] = in1[u] = make_uint4(0, 0, 0, 0);
      if (kind[u] >= 0) {
        const __nv_bfloat16* src = kind[u] == 0 ? a.q + head[u] * a.q_sh + t * a.q_sn
                                 : kind[u] == 1 ? a.k + head[u] * a.k_sh + t * a.k_sn
                                                : a.v + head[u] * a.v_sh + t * a.v_sn;
        in0[u] = __ldcs(reinterpret_cast<const uint4*>(src + c0 * 8));
        in1[u] = __ldcs(reinterpret_cast<const uint4*>(src + c1 * 8));
      }
    }
#pragma unroll
    for (int u = 0; u < kRopeRun; ++u) {
      const int p = p0 + u * a.splits;
      if (p >= passes) break;                    // uniform over the warp
      if (p < pq + pkv) {
        float x[8], y[8];
        unpack8(in0[u], x);
        unpack8(in1[u], y);
        const __nv_bfloat16* weight = p < pq ? a.q_weight : a.k_weight;
        if (weight) {
          float ss = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) ss += x[e] * x[e] + y[e] * y[e];
#pragma unroll
          for (int o = LPH / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
          const float inv = 1.f / sqrtf(ss * (1.f / D) + a.eps);
          float wx[8], wy[8];
          unpack8(__ldg(reinterpret_cast<const uint4*>(weight + c0 * 8)), wx);
          unpack8(__ldg(reinterpret_cast<const uint4*>(weight + c1 * 8)), wy);
#pragma unroll
          for (int e = 0; e < 8; ++e) { x[e] *= inv * wx[e]; y[e] *= inv * wy[e]; }
        }
        if (turn) {
          if (a.interleaved) {
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
              const float xa = x[e], xb = x[e + 1], ya = y[e], yb = y[e + 1];
              const int i = e / 2, j = 4 + e / 2;
              x[e] = xa * cs[i] - xb * sn[i];
              x[e + 1] = xb * cs[i] + xa * sn[i];
              y[e] = ya * cs[j] - yb * sn[j];
              y[e + 1] = yb * cs[j] + ya * sn[j];
            }
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float xa = x[e], xb = y[e];
              x[e] = xa * cs[e] - xb * sn[e];
              y[e] = xb * cs[e] + xa * sn[e];
            }
          }
        }
        in0[u] = pack8(x);
        in1[u] = pack8(y);
      }
      if (kind[u] < 0) continue;
      auto put = [&](__nv_bfloat16* dst) {
        *reinterpret_cast<uint4*>(dst + c0 * 8) = in0[u];
        *reinterpret_cast<uint4*>(dst + c1 * 8) = in1[u];
      };
      if (kind[u] == 0) {
        put(a.q_out + head[u] * a.qo_sh + t * a.qo_sn);
      } else if (kind[u] == 1) {
        if (a.k_out) put(a.k_out + head[u] * a.ko_sh + t * a.ko_sn);
        if (cache_off_k >= 0) put(a.kc.data + cache_off_k + head[u] * a.kc.s_head);
      } else {
        if (a.v_out) put(a.v_out + head[u] * a.vo_sh + t * a.vo_sn);
        if (cache_off_v >= 0) put(a.vc.data + cache_off_v + head[u] * a.vc.s_head);
      }
    }
  }
}

}  // namespace

cudaError_t launch_qk_norm_rope(RopeArgs& a, cudaStream_t s) {
  // A warp walks all the heads of a token once there are tokens enough to fill the device (the sines are then computed
  // once per token); with few tokens the heads of a token are spread over as many warps as there are passes.
  const int hpw = 32 / (a.d / 16);
  const int passes = (a.hq + hpw - 1) / hpw + 2 * ((a.hkv + hpw - 1) / hpw);
  const long long full = 148ll * 32;             // warps
  long long splits = (full + a.tokens - 1) / a.tokens;
  a.splits = (int)(splits > passes ? passes : splits);
  const long long warps = (long long)a.tokens * a.splits;
  const unsigned grid = (unsigned)((warps + kRopeThreads / 32 - 1) / (kRopeThreads / 32));
  return launch_dependent(a.d == 128 ? qk_norm_rope_kernel<128> : qk_norm_rope_kernel<64>, dim3(grid), dim3(kRopeThreads), 0, s, a);
}

}  // namespace sp
