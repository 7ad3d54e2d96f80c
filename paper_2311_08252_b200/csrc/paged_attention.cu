// rest_paged_attention: attention of draft rows (or single tokens) over a KV cache in pages, with
// an optional sliding window and first tokens that stay visible.
//
// The G = H / H_kv query heads of a KV head times the n nodes of a context give R = G n rows that
// all read the same keys, so the rows (node-major, r = i G + g) are packed into 128-row tiles of
// tcgen05.mma: S = Q K^T, then O += P V.
//
// Work.  The key tiles of all (context, KV head) units stand in one flat list, and every thread
// block takes an equal, contiguous share of it, by cost: uneven lengths, windows, one long context or
// hundreds of short ones all give the same even load in a single wave, and the shares follow from
// the lengths on the device alone.  A unit that a share's border cuts leaves partial rows
// (unnormalised O, maximum, sum) in the caller's scratch, which a second small kernel joins.  When R
// needs several row blocks of 256 rows, each has a list and blocks of its own (see plan).  With a
// window the tiles between the sinks and the earliest visible position are not in the list at all.
//
// Two kernel shapes, picked by R (rows per KV head):
//   R <= 128  one 128-row tile, two blocks per SM: bound by the K/V stream, so what counts is bytes
//             in flight (5 tiles of 16 KB a block) and a second block that fills the first one's gaps.
//   R > 128   two 128-row tiles that share each 64-key K/V tile (read once for 256 rows), one block
//             per SM: bound by the chain from S to P (exponentials half of it) and the tensor core.
// S has two buffers in TMEM for each row tile, so the tensor core runs a key tile ahead of the softmax
// warps and neither waits for the other's round trip (one 128-key buffer per row tile instead, which
// spends a fifth less tensor time, needed 5500 cycles per 128 keys and 256 rows).
// P is written back over S in TMEM and is the A operand of P V from there: no shared-memory round
// trip for it.
// O stays in TMEM and accumulates; its reference maximum is only raised when a tile exceeds it by
// 2^8, and only then is the O row rescaled.
//
// K and V tiles arrive by TMA, one box per page (or per 64-key slice of a larger page) and
// 64-element half of the head, in the 128-byte-swizzled operand layout; a page index that is out
// of range reads as zeros.  Every wait is bounded (see rest_device_error_flags).
//
// Precision: scores, maxima, sums and O in 32 bits; P is rounded to the cache's type for the
// tensor core (half a step, 2^-9 of each probability in bf16 - the output is rounded as much), the
// sum takes the unrounded values, so lse carries none of it.
//
// Measured (B200, join included; the copy rate is 6536 GB/s, the bf16 matrix rate 1669 TFLOP/s): calls back to back
// (the large ones then run into the board's power limit, at 1500 to 1700 of 1965 MHz; captured in a graph they take
// the same), and in brackets one at a time at the full clock with a cold L2.  64 nodes x 2048 keys, 32 KV
// heads, 24.4 us (latency); 61 ragged trees x 4096 keys, 32/8 heads, page 16, 277 us (252: 595 TFLOP/s); 16 trees of
// 128 nodes x 16384 keys, 40/8 heads, 800 us (674: 1030 TFLOP/s); 64 trees of 33 nodes, window 4096, 250 us (226: 4.9
// TB/s); 256 tokens, window 2048, D = 64, fp16, 240 us (211: 5.3 TB/s).  1 token x 2048 keys, 32/8 heads: 21 us a call, of
// which the GPU needs 15 (captured).  Of the fourth, with half the keys, a profile shows no pipe full (tensor core
// 46 %, exponentials 49 %, issue 37 %, DRAM 32 %): two softmax warps a scheduler, each with its chain of S
// out of TMEM, maximum, exponentials and P back, do not fill each other's waits.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "common.cuh"
#include "paged_attention.cuh"
#include "rest.h"

rest_status rest::take_paged_error_flags(uint32_t* h_flags) { return take_error_flags(h_flags); }

extern "C" size_t rest_paged_attention_workspace_bytes(int32_t B, int32_t H, int32_t H_kv, int32_t N, int32_t D) {
  if (B <= 0 || H <= 0 || H_kv <= 0 || N <= 0 || N > REST_MAX_N || (D != 64 && D != 128) || H % H_kv) return 0;
  // pages of codes take no more: as many rows, and at most as many blocks
  return workspace_bytes(plan(H, H_kv, N, false), D);
}

extern "C" rest_status rest_paged_attention(const void* d_q, const void* d_k_pages, const void* d_v_pages,
                                            const int64_t* strides, int32_t dtype, int32_t P, int32_t page,
                                            const int32_t* d_table, int64_t table_stride, int32_t table_cols,
                                            const int32_t* d_kv_len, const int32_t* d_n_nodes,
                                            const uint32_t* d_mask, int32_t B, int32_t H, int32_t H_kv, int32_t N,
                                            int32_t D, int32_t window, int32_t sinks, float scale, void* d_out,
                                            float* d_lse, void* d_ws, size_t ws_bytes, void* stream) {
  return attend<false>(d_q, d_k_pages, d_v_pages, strides, nullptr, nullptr, dtype, P, page, d_table, table_stride, table_cols,
                       d_kv_len, d_n_nodes, d_mask, B, H, H_kv, N, D, window, sinks, scale, d_out, d_lse, d_ws, ws_bytes, stream);
}
