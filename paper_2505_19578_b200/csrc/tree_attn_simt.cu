// Attention of new tokens over a paged cache on CUDA cores: one CTA per (row, query head), its warps take the keys in
// turn, fp32 throughout, masked keys are not read at all.  Kept as the on-device cross-check of the tensor-core kernel
// (selected like the other CUDA-core kernel); no tuning.  The same over a bf16 cache and over one held in 4 bits.
#include <math_constants.h>

#include "q4.cuh"

namespace sp {
namespace {

constexpr int kWarps = 8;

// This lane's E elements, lane E .. lane E + E - 1, of the key and the value of a token.
template <int D>
struct Bf16Rows {
  PagedCache kc, vc;
  static constexpr int kWhere = kWhereTreePage;
  __device__ __forceinline__ void load(int id, int g, int off, int lane, float (&k)[D / 32], float (&v)[D / 32]) const {
    const __nv_bfloat16* kr = kc.data + id * kc.s_page + g * kc.s_head + off * kc.s_tok + lane * (D / 32);
    const __nv_bfloat16* vr = vc.data + id * vc.s_page + g * vc.s_head + off * vc.s_tok + lane * (D / 32);
#pragma unroll
    for (int e = 0; e < D / 32; ++e) { k[e] = __bfloat162float(kr[e]); v[e] = __bfloat162float(vr[e]); }
  }
};
template <int D>
struct Q4Rows {
  Q4Cache c;
  static constexpr int kWhere = kWhereTreePageQ4;
  __device__ __forceinline__ void load(int id, int g, int off, int lane, float (&k)[D / 32], float (&v)[D / 32]) const {
    using B = Block<D>;
    const uint8_t* block = c.data + id * c.s_page + g * c.s_head + (off >> 4) * B::BYTES;
    const int i = off & 15, x = lane * (D / 32), w = x >> 3;
    const uint32_t kw = *reinterpret_cast<const uint32_t*>(block + B::k_word(i, w)), vw = *reinterpret_cast<const uint32_t*>(block + B::v_word(i, w));
    const float ks = scale_value(block[B::k_scale(i, w >> 2)]), vs = scale_value(block[B::v_scale(i, w >> 2)]);
#pragma unroll
    for (int e = 0; e < D / 32; ++e) { k[e] = code_value(kw, (x & 7) + e) * ks; v[e] = code_value(vw, (x & 7) + e) * vs; }
  }
};

template <int D, typename Rows>
__global__ void __launch_bounds__(kWarps * 32) tree_attn_simt_kernel(const TreeAttnArgs a, const Rows cache) {
  constexpr int E = D / 32;                        // elements of a row per lane
  __shared__ float s_m[kWarps], s_l[kWarps], s_o[kWarps][D];
  if (decode_poisoned(a.status)) return;
  const int t = blockIdx.x, h = blockIdx.y;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // the request that owns row t
  int lo = 0, hi = a.n_req;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.row_start[mid] <= t) lo = mid; else hi = mid - 1;
  }
  const int b = lo;
  if (b >= a.n_req) return;                        // behind the last request: left as it was
  const int first = a.row_start[b], j = t - first, n = a.row_start[b + 1] - first;
  const int len = min(max(a.seq_lens[b], 0), a.max_pages << a.page_log2);
  if (j < 0) return;
  if (a.seq_lens[b] > len && threadIdx.x == 0) report_range(a.status, Rows::kWhere);   // longer than its table row
  const int past = a.seq_lens[b] - n;              // keys before it are visible to every row
  const int g = h / a.group;

  float q[E], o[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    q[e] = __bfloat162float(a.q[h * a.q_sh + t * a.q_sn + lane * E + e]);
    o[e] = 0.f;
  }
  float m = -CUDART_INF_F, l = 0.f;
  for (int key = warp; key < len; key += kWarps) {
    const int x = key - past;                      // index among the new tokens
    bool visible = x < 0;
    if (!visible) visible = a.bits ? x < 32 * a.words && ((a.bits[(size_t)t * a.words + (x >> 5)] >> (x & 31)) & 1) : x <= j;
    if (!visible) continue;
    const int id = a.table[(size_t)b * a.max_pages + (key >> a.page_log2)];
    if (id < 0 || id >= a.n_pages) {
      if (lane == 0) report_range(a.status, Rows::kWhere);
      continue;
    }
    const int off = key & ((1 << a.page_log2) - 1);
    float kr[E], vr[E];
    cache.load(id, g, off, lane, kr, vr);
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) s += q[e] * kr[e];
#pragma unroll
    for (int x2 = 16; x2 > 0; x2 >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x2);
    s *= a.scale_log2;
    if (s == -CUDART_INF_F) continue;              // weight 0
    const float m_new = fmaxf(m, s);
    const float alpha = m == -CUDART_INF_F ? 0.f : exp2f(m - m_new), p = exp2f(s - m_new);
    l = l * alpha + p;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = o[e] * alpha + p * vr[e];
    m = m_new;
  }
  if (lane == 0) { s_m[warp] = m; s_l[warp] = l; }
#pragma unroll
  for (int e = 0; e < E; ++e) s_o[warp][lane * E + e] = o[e];
  __syncthreads();
  float top = -CUDART_INF_F, total = 0.f;
  for (int w = 0; w < kWarps; ++w)
    if (s_l[w] != 0.f) top = fmaxf(top, s_m[w]);
  for (int w = 0; w < kWarps; ++w)
    if (s_l[w] != 0.f) total += s_l[w] * exp2f(s_m[w] - top);
  for (int c = threadIdx.x; c < D; c += kWarps * 32) {
    float acc = 0.f;
    for (int w = 0; w < kWarps; ++w)
      if (s_l[w] != 0.f) acc += s_o[w][c] * exp2f(s_m[w] - top);
    a.o[h * a.o_sh + t * a.o_sn + c] = __float2bfloat16(total != 0.f ? acc / total : 0.f);   // nothing visible: zeros
  }
  if (a.lse && threadIdx.x == 0)
    a.lse[(size_t)h * a.rows + t] = total != 0.f ? (top + log2f(total)) * 0.6931471805599453f : -CUDART_INF_F;
}

}  // namespace

cudaError_t launch_tree_attn_simt(const TreeAttnArgs& a, cudaStream_t s) {
  const dim3 grid(a.rows, a.hq);
  if (a.d == 128) tree_attn_simt_kernel<128><<<grid, kWarps * 32, 0, s>>>(a, Bf16Rows<128>{a.kc, a.vc});
  else tree_attn_simt_kernel<64><<<grid, kWarps * 32, 0, s>>>(a, Bf16Rows<64>{a.kc, a.vc});
  return cudaGetLastError();
}

cudaError_t launch_tree_attn_q4_simt(const TreeAttnArgs& a, const Q4Cache& c, cudaStream_t s) {
  const dim3 grid(a.rows, a.hq);
  if (a.d == 128) tree_attn_simt_kernel<128><<<grid, kWarps * 32, 0, s>>>(a, Q4Rows<128>{c});
  else tree_attn_simt_kernel<64><<<grid, kWarps * 32, 0, s>>>(a, Q4Rows<64>{c});
  return cudaGetLastError();
}

}  // namespace sp
