// rest_paged_attention: attention of draft rows (or single tokens) over a KV cache in pages.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "common.cuh"
#include "rest.h"

namespace {

struct Args {
  const void *q, *k, *v;
  void* out;
  float* lse;
  const int32_t *table, *kv_len, *n_nodes;
  const uint32_t* mask;
  int64_t q_b, q_n, q_h, p_p, p_h, p_r, o_b, o_n, o_h, table_stride;
  int B, H, group, N, Wm, D, P, page_log, table_cols, window, sinks;
  float scale;
};

template <typename T> __device__ __forceinline__ float to_f(T x) { return (float)x; }

// depth of node i in its tree (its own position among its ancestors, 1-based) and "i sees node j"
__device__ __forceinline__ int node_depth(const Args& a, int b, int i) {
  if (!a.mask) return i + 1;
  const uint32_t* m = a.mask + ((int64_t)b * a.N + i) * a.Wm;
  int d = 0;
  for (int w = 0; w < a.Wm; ++w) d += __popc(m[w]);
  return d;
}

// One block per (node, head, context), four warps that take the keys in turn.
template <typename T>
__global__ void __launch_bounds__(128) rest_paged_attention_simple_kernel(Args a) {
  const int i = blockIdx.x, h = blockIdx.y, b = blockIdx.z, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int nn = a.n_nodes ? min(max(a.n_nodes[b], 0), a.N) : a.N;
  if (i >= nn) return;
  const int L = max(a.kv_len[b], 0), per = a.D / 32;
  const T* q = static_cast<const T*>(a.q) + b * a.q_b + i * a.q_n + h * a.q_h;
  float qv[4], o[4] = {0.f, 0.f, 0.f, 0.f}, m = -INFINITY, l = 0.f;
  for (int e = 0; e < per; ++e) qv[e] = to_f(q[lane * per + e]) * a.scale;
  const int depth = node_depth(a, b, i), pos = L + max(depth, 1) - 1;
  for (int key = warp; key < L + nn; key += 4) {
    int at = key;
    bool seen = true;
    if (key >= L) {
      const int j = key - L;
      seen = a.mask ? (a.mask[((int64_t)b * a.N + i) * a.Wm + (j >> 5)] >> (j & 31)) & 1u : j <= i;
      if (seen && a.window) at = L + node_depth(a, b, j) - 1;
    }
    if (a.window) seen = seen && (at < a.sinks || at > pos - a.window);
    const int col = key >> a.page_log;
    if (!seen || col >= a.table_cols) continue;
    const int p = a.table[b * a.table_stride + col];
    const bool there = p >= 0 && p < a.P;
    const int64_t off = p * a.p_p + (h / a.group) * a.p_h + (key & ((1 << a.page_log) - 1)) * a.p_r + lane * per;
    float s = 0.f, kv[4];
    for (int e = 0; e < per; ++e) s += there ? qv[e] * to_f(static_cast<const T*>(a.k)[off + e]) : 0.f;
    for (int e = 0; e < per; ++e) kv[e] = there ? to_f(static_cast<const T*>(a.v)[off + e]) : 0.f;
    for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
    const float mn = fmaxf(m, s), alpha = mn == -INFINITY ? 1.f : expf(m - mn), w = mn == -INFINITY ? 0.f : expf(s - mn);
    l = l * alpha + w;
    for (int e = 0; e < per; ++e) o[e] = o[e] * alpha + w * kv[e];
    m = mn;
  }
  __shared__ float s_m[4], s_l[4], s_o[4][128];
  if (lane == 0) { s_m[warp] = m; s_l[warp] = l; }
  for (int e = 0; e < per; ++e) s_o[warp][lane * per + e] = o[e];
  __syncthreads();
  const float top = fmaxf(fmaxf(s_m[0], s_m[1]), fmaxf(s_m[2], s_m[3]));
  float sum = 0.f, x = 0.f;
  for (int w = 0; w < 4; ++w) {
    const float c = s_m[w] == -INFINITY ? 0.f : expf(s_m[w] - top);
    sum += c * s_l[w];
    if (threadIdx.x < a.D && c != 0.f) x += c * s_o[w][threadIdx.x];
  }
  if (threadIdx.x < a.D)
    static_cast<T*>(a.out)[b * a.o_b + i * a.o_n + h * a.o_h + threadIdx.x] = (T)(sum == 0.f ? 0.f : x / sum);
  if (threadIdx.x == 0 && a.lse) a.lse[((int64_t)b * a.H + h) * a.N + i] = sum == 0.f ? -INFINITY : top + logf(sum);
}

}  // namespace

extern "C" size_t rest_paged_attention_workspace_bytes(int32_t B, int32_t H, int32_t H_kv, int32_t N, int32_t D) {
  if (B <= 0 || H <= 0 || H_kv <= 0 || N <= 0 || (D != 64 && D != 128) || H % H_kv) return 0;
  return 0;
}

extern "C" rest_status rest_paged_attention(const void* d_q, const void* d_k_pages, const void* d_v_pages,
                                            const int64_t* strides, int32_t dtype, int32_t P, int32_t page,
                                            const int32_t* d_table, int64_t table_stride, int32_t table_cols,
                                            const int32_t* d_kv_len, const int32_t* d_n_nodes,
                                            const uint32_t* d_mask, int32_t B, int32_t H, int32_t H_kv, int32_t N,
                                            int32_t D, int32_t window, int32_t sinks, float scale, void* d_out,
                                            float* d_lse, void* d_ws, size_t ws_bytes, void* stream) {
  if (B < 0 || H < 1 || H_kv < 1 || N < 1 || !strides || window < 0 || sinks < 0 || P < 1) return REST_INVALID_ARG;
  if (dtype != REST_BF16 && dtype != REST_FP16) return REST_INVALID_ARG;
  if (B == 0) return REST_OK;
  if (!d_q || !d_k_pages || !d_v_pages || !d_table || !d_kv_len || !d_out) return REST_INVALID_ARG;
  if (table_cols < 1 || table_stride < table_cols) return REST_INVALID_ARG;
  if (!(scale > 0.f) || !(scale < INFINITY)) return REST_INVALID_ARG;
  if ((D != 64 && D != 128) || N > REST_MAX_N || (H % H_kv) != 0) return REST_UNSUPPORTED;
  if (page < 16 || page > 256 || (page & (page - 1)) != 0 || (int64_t)table_cols * page > 0x7FFFFF00ll)
    return REST_UNSUPPORTED;
  const int64_t extent[9] = {B, N, H, P, H_kv, page, B, N, H};
  for (int i = 0; i < 9; ++i) {
    if (strides[i] < 0 || (strides[i] % 8) != 0) return REST_INVALID_ARG;
    if (extent[i] > 1 && strides[i] < D) return REST_INVALID_ARG;
  }
  if ((reinterpret_cast<uintptr_t>(d_q) | reinterpret_cast<uintptr_t>(d_k_pages) |
       reinterpret_cast<uintptr_t>(d_v_pages) | reinterpret_cast<uintptr_t>(d_out)) & 15)
    return REST_INVALID_ARG;
  (void)d_ws; (void)ws_bytes;
  Args a;
  a.q = d_q; a.k = d_k_pages; a.v = d_v_pages; a.out = d_out; a.lse = d_lse;
  a.table = d_table; a.kv_len = d_kv_len; a.n_nodes = d_n_nodes; a.mask = d_mask;
  a.q_b = strides[0]; a.q_n = strides[1]; a.q_h = strides[2];
  a.p_p = strides[3]; a.p_h = strides[4]; a.p_r = strides[5];
  a.o_b = strides[6]; a.o_n = strides[7]; a.o_h = strides[8];
  a.table_stride = table_stride;
  a.B = B; a.H = H; a.group = H / H_kv; a.N = N; a.Wm = (N + 31) / 32; a.D = D; a.P = P; a.table_cols = table_cols;
  a.window = window; a.sinks = sinks; a.scale = scale;
  a.page_log = 4;
  while ((1 << a.page_log) < page) ++a.page_log;
  if (H > 65535 || B > 65535) return REST_UNSUPPORTED;
  const dim3 grid((unsigned)N, (unsigned)H, (unsigned)B);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (dtype == REST_BF16) rest_paged_attention_simple_kernel<__nv_bfloat16><<<grid, 128, 0, st>>>(a);
  else rest_paged_attention_simple_kernel<__half><<<grid, 128, 0, st>>>(a);
  REST_CUDA_TRY(cudaGetLastError());
  rest::count_launch();
  return REST_OK;
}
