// The format of a paged cache held in 4 bits, and the internal declarations of the operators on it.
//
// A code c in 0 .. 15 stands for (c - 8) s with s = (1 + m / 8) 2^(e - 20), one byte (e << 3 | m) for 32 neighbouring
// elements of a token's head.  (c - 8) s has at most 4 + 4 significant bits, so a bf16 holds it exactly and the tensor
// cores multiply the values themselves.  Every bit pattern is a finite number: what lies in unused places of a page can be
// multiplied by zero.
//
// A block holds 16 tokens of one head, 17 D bytes, in the order in which the attention's lanes take it: for mma.sync
// m16n8k16 with the keys as the rows of A (K) or as its columns (V transposed), lane = 4 g + q,
//   K codes    [16][D / 2]          lane takes tokens g, g + 8, elements q D / 4 ..: one 16-byte (D = 64: 8-byte) load each
//   V codes    [D / 64][16][32]     lane takes tokens 2 q, 2 q + 1, 2 q + 8, 2 q + 9, elements g D / 8 ..; tokens in the order
//                                   0 2 4 6 1 3 5 7, 8 10 .., so that the four lanes of a load read four rows side by side
//   K scales   [8][D / 32][2]       lane's tokens g and g + 8 next to each other
//   V scales   [D / 32][4][4]       lane's tokens in the order 2 q, 2 q + 8, 2 q + 1, 2 q + 9
// In a 32-bit word of codes (8 elements) element 2 p has bits 4 p .. and element 2 p + 1 bits 16 + 4 p ..: a shift and a mask
// give a pair for the two halves of a register.  No byte is shared by two tokens, so tokens are written independently.
#pragma once

#include "decode.cuh"

namespace sp {

// Ids of device-side range failures (SP_ERR_RANGE in the status word) of the operators on a 4-bit cache.
enum { kWhereTreePageQ4 = 71, kWhereRopeSlotQ4 = 76, kWhereKeepPageQ4 = 81, kWhereReadPageQ4 = 86 };

constexpr uint32_t kScaleLeast = 0x35800000u, kScaleMost = 0x45700000u;      // 2^-20 and 1.875 * 2^11 as fp32

template <int D>
struct Block {                     // byte offsets inside a block
  static constexpr int BYTES = 17 * D, GROUPS = D / 32;
  static constexpr int V = 8 * D, KS = 16 * D, VS = KS + 16 * GROUPS;
  static __host__ __device__ constexpr int v_row(int i) { return (i & 8) | (i & 1) << 2 | (i & 7) >> 1; }
  // word w (elements 8 w .. 8 w + 7) of token i
  static __host__ __device__ constexpr int k_word(int i, int w) { return i * (D / 2) + w * 4; }
  static __host__ __device__ constexpr int v_word(int i, int w) { return V + (w >> 3) * 512 + v_row(i) * 32 + (w & 7) * 4; }
  // scale of group y (elements 32 y .. 32 y + 31) of token i
  static __host__ __device__ constexpr int k_scale(int i, int y) { return KS + (i & 7) * (2 * GROUPS) + 2 * y + (i >> 3); }
  static __host__ __device__ constexpr int v_scale(int i, int y) { return VS + 16 * y + ((i & 7) >> 1) * 4 + (i >> 3) + 2 * (i & 1); }
};

struct Q4Cache {                   // strides in bytes
  uint8_t* data;
  int64_t s_page, s_head;
};

__device__ __forceinline__ float scale_value(uint32_t byte) { return __uint_as_float((byte << 20) + kScaleLeast); }
// Element e (0 .. 7) of a word of codes.
__device__ __forceinline__ float code_value(uint32_t word, int e) { return (float)((int)(word >> (4 * (e >> 1) + 16 * (e & 1)) & 15u) - 8); }

struct KeepQ4Args {
  Q4Cache c;
  const int32_t* table;
  const int32_t* past;
  const int32_t* kept;             // [n_req, max_kept]
  const int32_t* n_kept;           // [n_req]
  int32_t* lens_out;               // [n_req]
  int n_req, max_pages, max_kept, hkv, d, page_log2, n_pages;
  int* status;
};

struct ReadQ4Args {
  Q4Cache c;
  const int32_t* table;            // [n_req, max_pages]
  const int32_t* seq_lens;         // [n_req]
  const int32_t* row_start;        // [n_req + 1]
  __nv_bfloat16* k;
  __nv_bfloat16* v;
  int64_t k_sh, k_sn, v_sh, v_sn;
  int n_req, max_pages, rows, hkv, d, page_log2, n_pages;
  int heads_per_warp;              // launcher
  int* status;
};

cudaError_t launch_qk_norm_rope_q4(RopeArgs& a, cudaStream_t s);
cudaError_t launch_cache_keep_q4(const KeepQ4Args& a, cudaStream_t s);
cudaError_t launch_cache_read_q4(ReadQ4Args& a, cudaStream_t s);
// a.kc and a.vc are not used.  arrived: [n_sm] zeros, and zeros again afterwards (not after a timeout).
size_t tree_attn_q4_workspace_bytes(int n_sm);
cudaError_t launch_tree_attn_q4(const TreeAttnArgs& a, const Q4Cache& c, void* ws, int* arrived, int n_sm, cudaStream_t s, int* launched);
cudaError_t launch_tree_attn_q4_tall(const TreeAttnArgs& a, const Q4Cache& c, void* ws, int n_sm, cudaStream_t s);      // ws as sp_tree_attn's
cudaError_t launch_tree_attn_q4_simt(const TreeAttnArgs& a, const Q4Cache& c, cudaStream_t s);

}  // namespace sp
