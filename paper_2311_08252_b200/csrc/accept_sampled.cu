// rest_accept_sampled: draft acceptance against the verifier's probabilities (Sec. 4.1 "Sampling
// strategies": temperature, nucleus).  One block per context walks from the root, row by row.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "common.cuh"
#include "rest.h"

namespace {

typedef unsigned long long u64;
constexpr int kThreads = 1024;
constexpr double kOne = 17592186044416.0;      // 2^44: the weight of a row's largest logit

struct Args {
  const void* logits;
  int64_t s_ctx, s_row;
  const int32_t *tokens, *parents, *n_nodes;
  const float *uniforms, *temperature, *top_p;
  int32_t *accept_len, *accept_nodes, *out_tokens;
  int V, N, max_depth;
};

template <typename T> __device__ __forceinline__ float load(const T* p, int v) { return (float)p[v] + 0.f; }

// order-preserving integer of a logit; NaN and -infinity are 0 (impossible)
__device__ __forceinline__ uint32_t key_of(float x) {
  if (!(x > -INFINITY)) return 0u;
  const uint32_t b = __float_as_uint(x);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

struct Row { float top; double inv_t; uint32_t cut_key; int cut_tie; bool greedy; };

// weight of logit x in 2^-44 of the largest, before the nucleus cut
__device__ __forceinline__ u64 weight(const Row& r, float x) {
  if (!(x > -INFINITY)) return 0ull;
  if (x == r.top) return (u64)kOne;
  if (r.greedy) return 0ull;
  return __double2ull_rn(exp(((double)x - (double)r.top) * r.inv_t) * kOne);
}
__device__ __forceinline__ bool kept(const Row& r, uint32_t key, int v) {
  return key > r.cut_key || (key == r.cut_key && v <= r.cut_tie);
}

__device__ u64 block_sum(u64 x, u64* s) {
  for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, d);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = x;
  __syncthreads();
  u64 t = 0;
  for (int w = 0; w < kThreads / 32; ++w) t += s[w];
  return t;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) rest_accept_sampled_kernel(Args a) {
  extern __shared__ uint32_t s_gone[];            // one bit per token: refused at the current node
  __shared__ u64 s_sum[kThreads / 32];
  __shared__ u64 s_left;
  __shared__ int s_child, s_n_rej, s_rej[REST_MAX_N], s_token;
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int nn = min(max(a.n_nodes[b], 0), a.N);
  const int32_t *tok = a.tokens + (int64_t)b * a.N, *par = a.parents + (int64_t)b * a.N;
  const float* uni = a.uniforms + (int64_t)b * (a.N + 1);
  const float temp = a.temperature[b], top_p = a.top_p[b];
  for (int d = tid; d < a.max_depth; d += kThreads) a.accept_nodes[(int64_t)b * a.max_depth + d] = -1;
  for (int d = tid; d <= a.max_depth; d += kThreads) a.out_tokens[(int64_t)b * (a.max_depth + 1) + d] = -1;
  for (int w = tid; w < (a.V + 31) / 32; w += kThreads) s_gone[w] = 0u;
  auto uniform = [&](int s) -> double { const float u = uni[s]; return u > 0.f ? (double)fminf(u, 0.99999994f) : 0.0; };
  int cur = -1;
  for (int len = 0;; ++len) {
    const T* row = static_cast<const T*>(a.logits) + b * a.s_ctx + (int64_t)(cur + 1) * a.s_row;
    Row r;
    r.greedy = !(temp > 0.f);
    r.inv_t = r.greedy ? 0.0 : 1.0 / (double)temp;
    // the largest logit
    uint32_t top = 0;
    for (int v = tid; v < a.V; v += kThreads) top = max(top, key_of(load(row, v)));
    top = __reduce_max_sync(0xFFFFFFFFu, top);
    __syncthreads();
    if (lane == 0) s_sum[warp] = top;
    __syncthreads();
    for (int w = 0; w < kThreads / 32; ++w) top = max(top, (uint32_t)s_sum[w]);
    r.top = top == 0 ? -INFINITY : __uint_as_float(top & 0x80000000u ? top & 0x7FFFFFFFu : ~top);
    r.cut_key = 0u; r.cut_tie = 0x7FFFFFFF;
    __syncthreads();
    // the whole mass, then the nucleus: the smallest key whose tokens and all above reach the target
    u64 mass = 0;
    for (int v = tid; v < a.V; v += kThreads) mass += weight(r, load(row, v));
    mass = block_sum(mass, s_sum);
    if (top != 0 && (r.greedy || top_p < 1.f)) {
      u64 target = 1;
      if (!r.greedy && top_p > 0.f) target = max((u64)1, (u64)ceil((double)top_p * (double)mass));
      uint32_t cut = 0;
      for (int bit = 31; bit >= 0; --bit) {
        const uint32_t at = cut | (1u << bit);
        u64 above = 0;
        for (int v = tid; v < a.V; v += kThreads) { const float x = load(row, v); if (key_of(x) >= at) above += weight(r, x); }
        if (block_sum(above, s_sum) >= target) cut = at;
      }
      u64 above = 0;
      for (int v = tid; v < a.V; v += kThreads) { const float x = load(row, v); if (key_of(x) > cut) above += weight(r, x); }
      above = block_sum(above, s_sum);
      const u64 each = weight(r, __uint_as_float(cut & 0x80000000u ? cut & 0x7FFFFFFFu : ~cut));
      const u64 ties = (target - above + each - 1) / each;             // tokens at the cut that stay, lowest first
      int lo = 0, hi = a.V;                                            // smallest `hi` with `ties` of them below it
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        u64 n = 0;
        for (int v = tid; v < mid; v += kThreads) n += key_of(load(row, v)) == cut;
        if (block_sum(n, s_sum) >= ties) hi = mid; else lo = mid;
      }
      r.cut_key = cut; r.cut_tie = hi - 1;
      mass = above + ties * each;
    }
    // children, in index order
    if (warp == 0) {
      int child = -1, n_rej = 0;
      u64 left = mass;
      for (int base = 0; base < nn && child < 0 && len < a.max_depth; base += 32) {
        const int i = base + lane;
        const bool is = i < nn && par[i] == cur;
        const int t = is ? tok[i] : -1;
        u64 w = 0;
        double u = 0.0;
        if (is && t >= 0 && t < a.V) {
          const float x = load(row, t);
          if (kept(r, key_of(x), t)) w = weight(r, x);
          u = uniform(i + 1);
          for (int j = 0; j < n_rej; ++j) if (s_rej[j] == t) w = 0;
        }
        unsigned todo = __ballot_sync(0xFFFFFFFFu, is && w != 0);
        while (todo) {
          const int l = __ffs(todo) - 1;
          todo &= todo - 1;
          const u64 wl = __shfl_sync(0xFFFFFFFFu, w, l);
          const double ul = __shfl_sync(0xFFFFFFFFu, u, l);
          const int tl = __shfl_sync(0xFFFFFFFFu, t, l);
          if (wl == 0) continue;
          if (ul * (double)left < (double)wl) { child = base + l; break; }
          left -= wl;
          if (lane == 0) s_rej[n_rej] = tl;
          __syncwarp();
          ++n_rej;
          if (t == tl) w = 0;
        }
      }
      if (lane == 0) { s_child = child; s_left = left; s_n_rej = n_rej; s_token = -1; }
    }
    __syncthreads();
    const int child = s_child;
    if (child >= 0) {
      if (tid == 0) {
        a.accept_nodes[(int64_t)b * a.max_depth + len] = child;
        a.out_tokens[(int64_t)b * (a.max_depth + 1) + len] = tok[child];
      }
      cur = child;
      __syncthreads();
      continue;
    }
    // the last token, from what the refused children leave
    for (int j = tid; j < s_n_rej; j += kThreads) atomicOr(&s_gone[s_rej[j] >> 5], 1u << (s_rej[j] & 31));
    __syncthreads();
    auto rest_weight = [&](int v) -> u64 {
      const float x = load(row, v);
      return kept(r, key_of(x), v) && !((s_gone[v >> 5] >> (v & 31)) & 1u) ? weight(r, x) : 0ull;
    };
    const int per = ((a.V + kThreads - 1) / kThreads) * 32, v0 = warp * per, v1 = min(a.V, v0 + per);
    u64 sum = 0;
    for (int v = v0 + lane; v < v1; v += 32) sum += rest_weight(v);
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
    if (lane == 0) s_sum[warp] = sum;
    __syncthreads();
    u64 before = 0;
    for (int w = 0; w < warp; ++w) before += s_sum[w];
    const double goal = uniform(0) * (double)s_left;
    if (sum != 0 && !((double)before > goal) && (double)(before + sum) > goal) {   // one warp
      for (int base = v0; base < v1; base += 32) {
        u64 inc = base + lane < v1 ? rest_weight(base + lane) : 0;
        for (int d = 1; d < 32; d <<= 1) { const u64 y = __shfl_up_sync(0xFFFFFFFFu, inc, d); if (lane >= d) inc += y; }
        const unsigned hit = __ballot_sync(0xFFFFFFFFu, (double)(before + inc) > goal);
        if (hit) { if (lane == 0) s_token = base + __ffs(hit) - 1; break; }
        before += __shfl_sync(0xFFFFFFFFu, inc, 31);
      }
    }
    __syncthreads();
    if (tid == 0) {
      a.out_tokens[(int64_t)b * (a.max_depth + 1) + len] = s_token;
      a.accept_len[b] = len;
    }
    return;
  }
}

}  // namespace

extern "C" rest_status rest_accept_sampled(const void* d_logits, int32_t dtype, int64_t ctx_stride, int64_t row_stride,
                                           int32_t V, const int32_t* d_tokens, const int32_t* d_parents,
                                           const int32_t* d_n_nodes, const float* d_uniforms,
                                           const float* d_temperature, const float* d_top_p, int32_t B, int32_t N,
                                           int32_t max_depth, int32_t* d_accept_len, int32_t* d_accept_nodes,
                                           int32_t* d_out_tokens, void* stream) {
  if (B < 0 || N < 1 || max_depth < 1 || V < 1 || ctx_stride < 0 || row_stride < 0) return REST_INVALID_ARG;
  if (dtype != REST_BF16 && dtype != REST_FP16 && dtype != REST_FP32) return REST_INVALID_ARG;
  if (B == 0) return REST_OK;
  if (!d_logits || !d_tokens || !d_parents || !d_n_nodes || !d_uniforms || !d_temperature || !d_top_p ||
      !d_accept_len || !d_accept_nodes || !d_out_tokens)
    return REST_INVALID_ARG;
  if (V > REST_MAX_VOCAB_SAMPLED || max_depth > REST_MAX_M || N > REST_MAX_N) return REST_UNSUPPORTED;
  Args a;
  a.logits = d_logits; a.s_ctx = ctx_stride; a.s_row = row_stride;
  a.tokens = d_tokens; a.parents = d_parents; a.n_nodes = d_n_nodes;
  a.uniforms = d_uniforms; a.temperature = d_temperature; a.top_p = d_top_p;
  a.accept_len = d_accept_len; a.accept_nodes = d_accept_nodes; a.out_tokens = d_out_tokens;
  a.V = V; a.N = N; a.max_depth = max_depth;
  const size_t smem = 4 * (((size_t)V + 31) / 32);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (dtype == REST_BF16) rest_accept_sampled_kernel<__nv_bfloat16><<<B, kThreads, smem, st>>>(a);
  else if (dtype == REST_FP16) rest_accept_sampled_kernel<__half><<<B, kThreads, smem, st>>>(a);
  else rest_accept_sampled_kernel<float><<<B, kThreads, smem, st>>>(a);
  REST_CUDA_TRY(cudaGetLastError());
  rest::count_launch();
  return REST_OK;
}
