// Rows and pages of a cache of e4m3 codes with a scale for every 16 rows of a head: the accepted path moved to the front
// (rest_paged_kv_commit_scaled), pages copied for a fork (rest_pages_copy_scaled).  Not in the paper, which never
// describes the cache.
//
// Rows that move from one block of 16 into another meet another scale.  The block that they move into is treated
// as if the values that they stand for had been appended: the smallest power of two that holds them, never less than
// before where the block has older rows, which are requantised when it grows.
//
// Both move bytes: the bound is HBM for many contexts or pages, and for one context the chain length -> table -> rows ->
// largest value -> rows.  Measured (B200, captured, back to back): 1 context, 8 or 32 heads, 3.6 us; 128 contexts, 32 heads, paths
// of up to 16 rows 8.7 us (a warp takes two heads one after another).  With the lengths in place a context has one block:
// 1 context, 8 heads, the same; 32 heads 4.1 us more and 128 contexts 3.6 us more (four heads a warp).  128 pages of 64 rows
// copied, 134 MB, 20.5 us (6.6 TB/s, a part of it from L2).
#include <cuda_runtime.h>
#include <stdint.h>

#include "common.cuh"
#include "e4m3.cuh"
#include "paged_pool.cuh"
#include "rest.h"

namespace {

using namespace rest_pool;
using namespace rest_e4m3;

constexpr int kMaxDepth = REST_MAX_M;
static_assert(kMaxDepth <= kBlockRows, "a path lies in two blocks of rows at most");

// A warp per head of K or V: it holds all rows of the path before it writes the first, so a row may be the
// source of one position and the target of another.
constexpr int kCommitThreads = 512;

template <int D>
__global__ void __launch_bounds__(kCommitThreads)
rest_paged_kv_commit_scaled_kernel(Pool c, float* k_scales, float* v_scales, const int32_t* kv_len,
                                   const int32_t* __restrict__ accept_nodes, const int32_t* __restrict__ accept_len,
                                   int H_kv, int N, int max_depth, int32_t* new_kv_len) {
  grid_wait();
  constexpr int kLanes = D / 16, kRows = 32 / kLanes, kSteps = kMaxDepth / kRows;
  __shared__ int64_t s_from[kMaxDepth], s_to[kMaxDepth], s_kept;      // vector offsets of rows in the pool
  __shared__ int64_t s_from_cell[kMaxDepth], s_to_cell[2];            // scales of head 0
  const int b = blockIdx.x;
  const int L = *reinterpret_cast<const volatile int32_t*>(kv_len + b);
  int len = accept_len[b];
  len = len < 0 ? 0 : (len > max_depth ? max_depth : len);
  const int cells = 1 << (c.page_log - 4);                            // of a head in a page
  auto cell_of = [&](int at) -> int64_t {                             // (the page exists)
    return (int64_t)c.table[b * c.table_stride + (at >> c.page_log)] * H_kv * cells + ((at & ((1 << c.page_log) - 1)) >> 4);
  };
  if (threadIdx.x < kMaxDepth) {
    const int i = threadIdx.x;
    int64_t from = -1, to = -1;
    if (i < len && L >= 0) {
      int nd = accept_nodes[(int64_t)b * max_depth + i];
      nd = nd < 0 ? 0 : (nd >= N ? N - 1 : nd);
      from = L > 0x7FFFFFFF - nd ? -1 : row_offset(c, b, L + nd);
      to = L > 0x7FFFFFFF - i ? -1 : row_offset(c, b, L + i);
      if (to < 0) from = -1;
      if (from >= 0) s_from_cell[i] = cell_of(L + nd);
      // the path's first row in a block says where the block's scale is (a block lies in one page)
      if (to >= 0 && (i == 0 || ((L + i) & 15) == 0)) s_to_cell[i == 0 ? 0 : 1] = cell_of(L + i);
    }
    s_from[i] = from;
    s_to[i] = to;
    if (i == 0) s_kept = to >= 0 && (L & 15) ? row_offset(c, b, L & ~15) : -1;
  }
  __syncthreads();
  const int lane = threadIdx.x & 31, sub = lane / kLanes, chunk = lane % kLanes;
  const int kept = L & 15, in_first = 16 - kept;                      // path positions from in_first on are in the second block
  const int warps = blockDim.x / 32;
  for (int u = (threadIdx.x >> 5) + blockIdx.y * warps; L >= 0 && len > 0 && u < 2 * H_kv; u += warps * gridDim.y) {
    const int h = u >> 1;
    uint4* base = ((u & 1) ? c.v : c.k) + h * c.s_head + chunk;
    float* scales = ((u & 1) ? v_scales : k_scales) + (int64_t)h * cells;
    uint4 x[kSteps];
    float scale[kSteps], most[2] = {0.f, 0.f};
    bool any[2] = {false, false};
#pragma unroll
    for (int k = 0; k < kSteps; ++k) {
      const int i = k * kRows + sub;
      scale[k] = 0.f;
      if (i < len && s_from[i] >= 0) {
        x[k] = base[s_from[i]];
        scale[k] = within_limits(scales[s_from_cell[i]]);
      }
    }
#pragma unroll
    for (int k = 0; k < kSteps; ++k) {
      const int i = k * kRows + sub;
      if (i < len && s_from[i] >= 0) {
        const float top = largest16(x[k]) * scale[k];
        if (i < in_first) { most[0] = fmaxf(most[0], top); any[0] = true; }
        else { most[1] = fmaxf(most[1], top); any[1] = true; }
      }
    }
    float s[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      any[t] = __any_sync(0xFFFFFFFFu, any[t]);
      s[t] = fitting_scale(warp_max(most[t]));
    }
    if (any[0] && s_kept >= 0) {
      const float old = within_limits(scales[s_to_cell[0]]);
      if (s[0] > old) {                                               // older rows: the scale grows
        const float ratio = old / s[0];
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
          const int r = k * kRows + sub;
          if (r < kept) {
            uint4* p = base + s_kept + r * c.s_row;
            *p = rescale16(*p, ratio);
          }
        }
      } else {
        s[0] = old;
      }
    }
    __syncwarp();                                                     // (all lanes have read the scales)
#pragma unroll
    for (int k = 0; k < kSteps; ++k) {
      const int i = k * kRows + sub;
      if (i < len && s_from[i] >= 0) {
        const float to = i < in_first ? s[0] : s[1];
        if (to != scale[k]) x[k] = rescale16(x[k], scale[k] / to);
        base[s_to[i]] = x[k];
      }
    }
#pragma unroll
    for (int t = 0; t < 2; ++t)
      if (any[t] && lane == t) scales[s_to_cell[t]] = s[t];
  }
  if (new_kv_len && threadIdx.x == 0 && blockIdx.y == 0) new_kv_len[b] = L + len;
}

// One block per 16 KB of one page of K or V; the first one of a page copies its scales as well.
constexpr int kCopyThreads = 256, kCopyVecs = 1024;

__global__ void __launch_bounds__(kCopyThreads)
rest_pages_copy_scaled_kernel(Pool c, float* k_scales, float* v_scales, const int32_t* __restrict__ src,
                              const int32_t* __restrict__ dst, int chunks, int vecs, int dv_log, int page_scales) {
  grid_wait();
  const int pair = blockIdx.x / chunks, chunk = blockIdx.x % chunks;
  const int a = src[pair], z = dst[pair];
  if (a < 0 || a >= c.P || z < 0 || z >= c.P || a == z) return;
  uint4* base = blockIdx.y ? c.v : c.k;
  int64_t at[4];
  uint4 x[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int e = chunk * kCopyVecs + j * kCopyThreads + threadIdx.x;
    const int row = (e >> dv_log) & ((1 << c.page_log) - 1), h = e >> (dv_log + c.page_log);
    at[j] = h * c.s_head + row * c.s_row + (e & ((1 << dv_log) - 1));
    if (e < vecs) x[j] = base[a * c.s_page + at[j]];
  }
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (chunk * kCopyVecs + j * kCopyThreads + (int)threadIdx.x < vecs) base[z * c.s_page + at[j]] = x[j];
  if (chunk == 0) {
    float* scales = blockIdx.y ? v_scales : k_scales;
    for (int e = threadIdx.x; e < page_scales; e += kCopyThreads)
      scales[(int64_t)z * page_scales + e] = scales[(int64_t)a * page_scales + e];
  }
}

}  // namespace

extern "C" rest_status rest_paged_kv_commit_scaled(void* d_k_pages, void* d_v_pages, const int64_t* page_strides,
                                                   float* d_k_scales, float* d_v_scales, int32_t P, int32_t page,
                                                   const int32_t* d_table, int64_t table_stride, int32_t table_cols,
                                                   const int32_t* d_kv_len, const int32_t* d_accept_nodes,
                                                   const int32_t* d_accept_len, int32_t B, int32_t H_kv, int32_t N, int32_t D,
                                                   int32_t max_depth, int32_t* d_new_kv_len, void* stream) {
  if (B < 0 || H_kv < 1 || N < 1 || max_depth < 1) return REST_INVALID_ARG;
  if (B == 0) return REST_OK;
  if (!d_kv_len || !d_accept_nodes || !d_accept_len || !d_k_scales || !d_v_scales ||
      !table_ok(d_table, table_stride, table_cols))
    return REST_INVALID_ARG;
  if (max_depth > kMaxDepth) return REST_UNSUPPORTED;
  Pool c;
  if (rest_status st = fill_pool(c, d_k_pages, d_v_pages, page_strides, d_table, table_stride, table_cols, P, H_kv, page, D, 16))
    return st;
  // Heads are shared out to blocks of 256 threads, four an SM (128 contexts, 32 heads and 128 pages copied behind them 32.4 us,
  // with two of 512 33.9); not when the new lengths go into the array that the old ones are read from: one of 512 then.
  const bool apart = d_new_kv_len != d_kv_len;
  const int threads = apart ? kCommitThreads / 2 : kCommitThreads, sms = rest::sm_count();
  const int rounds = (2 * H_kv + threads / 32 - 1) / (threads / 32);
  int parts = apart ? 4 * (sms > 0 ? sms : 148) / B : 1;
  parts = parts < 1 ? 1 : parts > rounds ? rounds : parts;
  REST_CUDA_TRY(launch(D == 128 ? rest_paged_kv_commit_scaled_kernel<128> : rest_paged_kv_commit_scaled_kernel<64>,
                       dim3((unsigned)B, (unsigned)parts), threads, 0, stream, c, d_k_scales, d_v_scales, d_kv_len,
                       d_accept_nodes, d_accept_len, (int)H_kv, (int)N, (int)max_depth, d_new_kv_len));
  return REST_OK;
}

extern "C" rest_status rest_pages_copy_scaled(void* d_k_pages, void* d_v_pages, const int64_t* page_strides,
                                              float* d_k_scales, float* d_v_scales, int32_t P, int32_t page, int32_t H_kv,
                                              int32_t D, const int32_t* d_src, const int32_t* d_dst, int32_t n, void* stream) {
  if (n < 0 || H_kv < 1) return REST_INVALID_ARG;
  if (n == 0) return REST_OK;
  if (!d_src || !d_dst || !d_k_scales || !d_v_scales) return REST_INVALID_ARG;
  Pool c;
  if (rest_status st = fill_pool(c, d_k_pages, d_v_pages, page_strides, nullptr, 0, 0, P, H_kv, page, D, 16)) return st;
  const int64_t vecs = (int64_t)H_kv * page * (D / 16), chunks = (vecs + kCopyVecs - 1) / kCopyVecs;
  if (vecs > (1 << 30) || chunks * n > 0x7FFFFFFFll) return REST_UNSUPPORTED;
  REST_CUDA_TRY(launch(rest_pages_copy_scaled_kernel, dim3((unsigned)(chunks * n), 2), kCopyThreads, 0, stream, c, d_k_scales,
                       d_v_scales, d_src, d_dst, (int)chunks, (int)vecs, log2_of(D / 16), (int)(H_kv * (page / 16))));
  return REST_OK;
}
