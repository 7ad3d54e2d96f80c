// What the kernels of a cache in pages share: the pool and its checks, launches that may start before
// the kernel ahead of them has ended.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "common.cuh"
#include "rest.h"

namespace rest_pool {

__device__ __forceinline__ void grid_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

template <typename... P, typename... A>
cudaError_t launch(void (*kernel)(P...), dim3 grid, int threads, size_t smem, void* stream, A... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = static_cast<cudaStream_t>(stream);
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, args...);
  if (e == cudaSuccess) rest::count_launch();
  return e;
}

inline bool page_ok(int page) { return page >= 16 && page <= 256 && (page & (page - 1)) == 0; }
inline int log2_of(int x) { int n = 0; while ((1 << n) < x) ++n; return n; }
inline bool stride_ok(const int64_t* s, int n, int per_vec = 8) {
  for (int i = 0; i < n; ++i)
    if (s[i] < 0 || (s[i] % per_vec) != 0) return false;
  return true;
}
inline bool aligned16(const void* a, const void* b) {
  return ((reinterpret_cast<uintptr_t>(a) | reinterpret_cast<uintptr_t>(b)) & 15) == 0;
}

// strides of the pool in 16-byte vectors: page, head, row
struct Pool {
  uint4 *k, *v;
  int64_t s_page, s_head, s_row;
  const int32_t* table;
  int64_t table_stride;
  int table_cols, P, page_log;
};

// vector offset of row `at` of context b, or -1 when the table has no such page
__device__ __forceinline__ int64_t row_offset(const Pool& c, int b, int at) {
  if (at < 0) return -1;
  const int col = at >> c.page_log;
  if (col >= c.table_cols) return -1;
  const int p = c.table[b * c.table_stride + col];
  if (p < 0 || p >= c.P) return -1;
  return p * c.s_page + (int64_t)(at & ((1 << c.page_log) - 1)) * c.s_row;
}

// elements of `per_vec` to a 16-byte vector
inline rest_status fill_pool(Pool& c, void* k, void* v, const int64_t* strides, const int32_t* table, int64_t table_stride,
                             int32_t table_cols, int32_t P, int32_t H_kv, int32_t page, int32_t D, int per_vec = 8) {
  if (!k || !v || !strides || P < 1) return REST_INVALID_ARG;
  if (!page_ok(page) || (D != 64 && D != 128) || H_kv > (1 << 20)) return REST_UNSUPPORTED;
  // a dimension that is stepped through advances by a row at least (strides that make rows of different pages,
  // heads or places share memory all the same are the caller's mistake)
  const int64_t extent[3] = {P, H_kv, page};
  for (int i = 0; i < 3; ++i)
    if (extent[i] > 1 && strides[i] < D) return REST_INVALID_ARG;
  if (!stride_ok(strides, 3, per_vec) || !aligned16(k, v)) return REST_INVALID_ARG;
  c.k = static_cast<uint4*>(k); c.v = static_cast<uint4*>(v);
  c.s_page = strides[0] / per_vec; c.s_head = strides[1] / per_vec; c.s_row = strides[2] / per_vec;
  c.table = table; c.table_stride = table_stride; c.table_cols = table_cols;
  c.P = P; c.page_log = log2_of(page);
  return REST_OK;
}

inline bool table_ok(const int32_t* table, int64_t stride, int32_t cols) { return table && cols >= 1 && stride >= cols; }

}  // namespace rest_pool
