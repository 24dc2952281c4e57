// Internal declarations of the decode operators around the MoE layer: the
// host-side launchers of linear.hip, linear_pack.hip, kv_append.hip,
// attn_decode.hip, attn_prefix.hip, block_norm.hip and sample.hip.
#pragma once

#include "internal.h"

namespace d2moe {

// ---- 4-bit linear layers: blocks of 16 rows by 128 columns -------------------
constexpr int kLinRows = 16, kLinCols = 128;
inline int lin_row_blocks(const d2moe_linear* w) { return (w->rows - 1) / kLinRows + 1; }
inline int lin_col_blocks(const d2moe_linear* w) { return (w->cols - 1) / kLinCols + 1; }

hipError_t launch_linear_pack(const float* W, const d2moe_linear* out, hipStream_t s);
hipError_t launch_linear_pack_codes(const uint8_t* codes, const uint16_t* scales,
                                    const uint8_t* zeros, const d2moe_linear* out, hipStream_t s);
hipError_t launch_linear(const void* x, d2moe_dtype xd, int T, const d2moe_linear* w,
                         const float* bias, void* y, d2moe_dtype yd, hipStream_t s);

// ---- paged key-value cache -----------------------------------------------------
// n / d for 0 <= n < 2^31 as (n * mul) >> shift, by the round-up reciprocal:
// mul = floor(2^(31 + s) / d) + 1 with 2^s >= d is off by e <= d <= 2^s in
// 2^(31 + s), so that n e < 2^(31 + s).
struct FastDiv {
  uint32_t mul, d;
  int shift;
  __device__ uint32_t div(uint32_t n) const { return (uint32_t)(((uint64_t)n * mul) >> shift); }
};
inline FastDiv fast_div(int d) {
  int s = 0;
  while ((1ll << s) < d) ++s;
  return FastDiv{(uint32_t)((1ull << (31 + s)) / (uint64_t)d + 1), (uint32_t)d, 31 + s};
}

hipError_t launch_kv_append(const void* q, int64_t q_stride, int q_heads, const void* k,
                            const void* v, int64_t kv_stride, d2moe_dtype xd, int N,
                            const d2moe_kv_cache* c, const int32_t* table, int n_seqs,
                            int max_pages, const int32_t* positions, const int32_t* token_seq,
                            const float* cos, const float* sin, int n_rot, void* q_out,
                            hipStream_t s);

hipError_t launch_kv_append_norm(const void* q, int64_t q_stride, int q_heads, const void* k,
                                 const void* v, int64_t kv_stride, d2moe_dtype xd, int N,
                                 const d2moe_kv_cache* c, const int32_t* table, int n_seqs,
                                 int max_pages, const int32_t* positions, const int32_t* token_seq,
                                 const float* q_weight, const float* k_weight, float eps,
                                 const float* cos, const float* sin, int n_rot, int rot_dim,
                                 bool interleaved, void* q_out, hipStream_t s);

// scores are scaled in units of log2, scale * kLog2e
constexpr float kLog2e = 1.44269504088896340736f;
size_t attn_decode_workspace(int B, int q_heads, int n_heads, int dim, int max_len);
hipError_t launch_attn_decode(const void* q, int64_t q_stride, int B, int q_heads,
                              const d2moe_kv_cache* c, const int32_t* table, int max_pages,
                              const int32_t* lengths, int max_len, int window, float scale,
                              void* out, void* ws, hipStream_t s);

size_t attn_prefix_workspace(int B, int q_heads, int n_heads, int dim, int max_prefix,
                             int max_rest);
hipError_t launch_attn_prefix(const void* q, int64_t q_stride, int B, int q_heads,
                              const d2moe_kv_cache* c, const int32_t* table, int max_pages,
                              const int32_t* lengths, const int32_t* prefix_table,
                              int prefix_pages, const int32_t* prefix_lens, int max_prefix,
                              int max_rest, float scale, void* out, void* ws, hipStream_t s);

hipError_t launch_block_norm(float* x, float x_scale, const void* y, d2moe_dtype yd, float y_scale,
                             const float* post_w, const void* gate, d2moe_dtype gd,
                             int64_t gate_stride, const float* pre_w, int T, int d, float eps,
                             void* h, d2moe_dtype hd, hipStream_t s);

hipError_t launch_sample(const void* logits, d2moe_dtype dtype, int64_t stride, int B, int V,
                         const float* u, const float* temperature, const int32_t* top_k,
                         const float* top_p, const float* min_p, int32_t* tokens, float* probs,
                         hipStream_t s);

}  // namespace d2moe
