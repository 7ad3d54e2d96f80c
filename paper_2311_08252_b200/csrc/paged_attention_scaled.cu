// rest_paged_attention_scaled: the attention of rest_paged_attention over pages of e4m3 codes with a scale for every
// 16 rows of a head.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "common.cuh"
#include "paged_attention.cuh"
#include "rest.h"

rest_status rest::take_scaled_error_flags(uint32_t* h_flags) { return take_error_flags(h_flags); }

extern "C" rest_status rest_paged_attention_scaled(const void* d_q, const void* d_k_pages, const void* d_v_pages,
                                                   const int64_t* strides, const float* d_k_scales, const float* d_v_scales,
                                                   int32_t dtype, int32_t P, int32_t page, const int32_t* d_table,
                                                   int64_t table_stride, int32_t table_cols, const int32_t* d_kv_len,
                                                   const int32_t* d_n_nodes, const uint32_t* d_mask, int32_t B, int32_t H,
                                                   int32_t H_kv, int32_t N, int32_t D, int32_t window, int32_t sinks,
                                                   float scale, void* d_out, float* d_lse, void* d_ws, size_t ws_bytes,
                                                   void* stream) {
  return attend<true>(d_q, d_k_pages, d_v_pages, strides, d_k_scales, d_v_scales, dtype, P, page, d_table, table_stride,
                      table_cols, d_kv_len, d_n_nodes, d_mask, B, H, H_kv, N, D, window, sinks, scale, d_out, d_lse, d_ws,
                      ws_bytes, stream);
}
